// Attention with several heads, a bucket bias and dropout, and the rows' log-sum-exp: the forward pass of training, and (without
// dropout) that of serving.
//
//   s = scale * x_i . y_j + bias(j - i),  out_i = sum over the stored j of dropout(softmax(s)) h_j,  lse_i = log sum exp(s)
//
// A wavefront walks one item of the work list for one head, block by block (32 vectors of a window of V rows):
//   * the 32 rows of Y and of H are gathered row by row and put to LDS while the ones before are computed with;
//   * the scores of the V x 32 block come from the matrix cores, Y's rows as the left operand and the window's rows of X, held in
//     registers, as the right one: lane (j, g) gets the scores of window row j and vectors 8g .. 8g+7;
//   * bias and pattern are applied in fp32 in units of log2, the running maximum m (fp16: less 12) and sum l of the row are updated, the
//     probabilities that dropout keeps become two numbers of the element type, the rounded one and what the rounding left;
//   * both meet H's rows, read transposed from LDS, on the matrix cores; the accumulators are scaled by 2^(m_old - m_new).
//     (The second product costs 3 to 7 %.  Without it the rounding of P would be in out beside out's own, and through D = g . out, whose
//     parts cancel in sums over many entries, in the gradient of the bias: 1.5 times the error on a graph of 8 k rows.)
// At a window's end the tile is divided by l (1 / (1 - p) goes in with it) and stored; parts of a cut window leave fp32 tiles and
// (m, l), which k_merge_parts merges in slot order.  l counts what dropout takes out as well: the mask applies after the softmax.
// Heads are the slower grid dimension, so that one head's rows of Y and H share the L2s; query heads with the same keys are neighbours.
//
// Bounds, with 64 columns of both kinds, bias and dropout: on a lognormal graph of 262 k rows, two heads, the fabric (397 us; 2.7 GB fetched,
// 6.95 of the 7.5 TB/s that such rows reach, since every gathered row misses the L2s); on a sequence of 4096 with a window of 256, eight heads
// on two, vector instructions at 58 % of the issue slots, 429 a block of which the generator is 180 (41 us, 2.1 GFLOP); on an R-MAT graph of 65 k
// rows, 32 and 128 columns, the same at 49 % with two of three wavefronts a SIMD there on average (42 us); for one row of 1028 entries, eight heads,
// the chain item -> indices -> rows, 10 us.  Wavefronts hide that chain, so registers decide: four a SIMD where tiles of up to 64 columns let
// them, three up to KS * NT = 16, two above.  Addresses are worked out where they are used, because a spilled one's load waits behind the
// gathers (four with spills were slower than three without, lognormal graph 458 us and 420).
#include <type_traits>

#include "fs_common.h"
#include "fs_heads.h"

namespace {

// What a row's probabilities are held relative to, given its largest score so far: fp16 holds them times 2^12, since beside a sink those of
// thousands of entries would lie below its smallest number.  (Far from zero, where 12 less would be rounded, they are as they are.)
template <int DT>
__device__ __forceinline__ float reference_of(float top) { return DT == FS_F16 && fabsf(top) < 0x1p20f ? top - 12.f : top; }

template <int DT, int V, int KS, int NT>
__global__ void __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(KS <= 2 && NT <= 4 ? 4 : KS * NT <= 16 ? 3 : 2)))
k_heads_forward(fs_walk a, fs_operand X, fs_operand Y, fs_operand H, int share, int d, int N, float sl2, fs_bias_args bias, fs_drop_args drop,
                fs_operand out, float *__restrict__ lse, float *__restrict__ part, float *__restrict__ stats)
{
    using tile_y = fs_gathered<32 * KS>;
    using tile_h = fs_gathered<16 * NT>;
    __shared__ __attribute__((aligned(16))) unsigned char lds[tile_y::kBytes > tile_h::kBytes ? tile_y::kBytes : tile_h::kBytes];  // Y's rows, then H's
    __shared__ __attribute__((aligned(16))) int lds_cols[32];
    __shared__ fs_entries<V> entries;
    extern __shared__ __attribute__((aligned(16))) unsigned char dyn[];
    float *table = reinterpret_cast<float *>(dyn);
    uint8_t *lut = dyn + 4 * bias.n_buckets;

    const int lane = threadIdx.x, head = blockIdx.y;
    const int turn = __builtin_amdgcn_readfirstlane(fs_launch_turn<1>(blockIdx.x, a.slice, a.n_swz));
    if (turn >= a.n_items) return;
    const int4 it = a.items[turn];
    // while the item is on its way: what does not depend on it
    if (bias.n_buckets > 0) {
        fs_load_buckets(bias, lut, lane, 64);
        for (int i = lane; i < bias.n_buckets; i += 64) table[i] = fs_bias_log2(fs_widen<DT>(bias.table[head * bias.ld + i]));
    }
    const fs_key key = fs_drop_key(drop, head);
    const int nblk = it.y;
    if (nblk == 0) return;
    int slot = it.z;
    const int j = lane & 15, g = lane >> 4;
    const int4 my_desc = a.blk_desc[it.x + min(lane, nblk - 1)];
    auto block = [&](int i) -> BlockDesc { return fs_item_block(my_desc, i, nblk); };
    const unsigned char *Xb = X.p + head * X.head, *Yb = Y.p + head / share * Y.head, *Hb = H.p + head / share * H.head;
    const uint32_t y_colb = tile_y::column_bytes(lane, d), h_colb = tile_h::column_bytes(lane, N);

    int cols0 = fs_first_cols(a, it, lane);
    BlockDesc d0 = block(0), d1 = block(1);
    cols0 = fs_cut_cols(cols0, d0.kb, lane);
    int cols1 = fs_block_cols(a, d1, lane);
    uint32_t bits0 = fs_row_bits<V>(a, it.x, 0, nblk, lane);
    fs_frag xf[KS];
    fs_load_window<V>(xf, Xb, X.pitch, d, d0.w, a.M, lane);
    tile_y y;
    tile_h h;
    y.load(Yb, Y.pitch, y_colb, cols0, lane);
    h.load(Hb, H.pitch, h_colb, cols0, lane);

    const bool looks_up = bias.n_buckets > 0 || drop.state;

    fs_f4 acc[NT];
    fs_clear(acc);
    float m_run = -INFINITY, l_run = 0.f;  // the largest reference so far; this lane's share of the sum relative to it
    bool from_first = d0.first;
    int step = 0;
    auto block_step = [&](auto more_) {
        constexpr bool MORE = decltype(more_)::value;
        if (const int l = fs_lane_here(lane); l < 32) lds_cols[l] = cols0;
        const BlockDesc d2 = block(step + 2);
        int cols2 = 0;
        uint32_t bits1 = 0;
        if constexpr (MORE) {
            cols2 = fs_block_cols(a, d2, lane);
            bits1 = fs_row_bits<V>(a, it.x, step + 1, nblk, lane);
        }
        FS_WAVE_SYNC();
        if (looks_up) entries.template look_up<false>(entries.make_list(bits0, lane, drop.state), lane, d0.w * V, cols0, lds_cols, bias, table, lut, drop, key);
        y.put(lds, lane, d);
        if constexpr (MORE) y.load(Yb, Y.pitch, y_colb, cols1, lane);
        FS_WAVE_SYNC();
        fs_f4 sc[2];
#pragma unroll
        for (int t = 0; t < 2; t++) sc[t] = tile_y::template contract<DT>(lds, t, lane, xf);
        FS_WAVE_SYNC();
        h.put(lds, lane, N);
        if (MORE && d1.w != d0.w) fs_load_window<V>(xf, Xb, X.pitch, d, d1.w, a.M, lane);
        if constexpr (MORE) h.load(Hb, H.pitch, h_colb, cols1, lane);
        FS_WAVE_SYNC();
        const uint32_t m8 = bits0 >> (8 * g);
        float p[8], mx = -INFINITY;
        uint2 kept = make_uint2(~0u, ~0u);
        if (looks_up) {
            if (drop.state) kept = entries.kept_bytes(lane);
            entries.values(p, lane);
#pragma unroll
            for (int x = 0; x < 8; x++) p[x] = fmaf(sc[x >> 2][x & 3], sl2, p[x]);
        } else {
#pragma unroll
            for (int x = 0; x < 8; x++) p[x] = sc[x >> 2][x & 3] * sl2;
        }
#pragma unroll
        for (int x = 0; x < 8; x++) {
            p[x] = fs_choose(fs_bit_mask(m8, x), p[x], -INFINITY);
            mx = fmaxf(mx, p[x]);
        }
        const float m_new = fmaxf(m_run, reference_of<DT>(fs_row_max(mx)));
        const float m_use = m_new == -INFINITY ? 0.f : m_new;  // nothing seen so far
        const float corr = __builtin_amdgcn_exp2f(m_run - m_use);
        float ps = 0.f;
#pragma unroll
        for (int x = 0; x < 8; x++) {
            p[x] = __builtin_amdgcn_exp2f(p[x] - m_use);
            ps += p[x];
        }
        l_run = l_run * corr + ps;
        m_run = m_new;
#pragma unroll
        for (int x = 0; x < 8; x++) p[x] = __uint_as_float(fs_kept_mask(kept, x) & __float_as_uint(p[x]));
        const fs_frag hi = fs_round8<DT>(p), lo = fs_round8_rest<DT>(p, hi);
        if (d0.kb > 0) {
#pragma unroll
            for (int t = 0; t < NT; t++) {
                const fs_frag rows = tile_h::transposed(lds, t, lane);
                acc[t] = fs_mfma_16x16x32<DT>(rows, lo, fs_mfma_16x16x32<DT>(rows, hi, acc[t] * corr));
            }
        }
        FS_WAVE_SYNC();
        if (d0.last || !MORE) {
            const float l_tot = fs_row_sum(l_run);
            const int l = fs_lane_here(lane), j = l & 15, g = l >> 4, row = d0.w * V + j;
            if (d0.last && from_first) {
                fs_store_window<DT, V, 16 * NT>(lds, acc, l_tot == 0.f ? 0.f : drop.factor / l_tot, out.p + head * out.head, out.pitch, N, d0.w, a.M, lane);
                if (lse && g == 0 && j < V && row < a.M) lse[(int64_t)head * a.M + row] = fs_log_sum(m_run, l_tot);
            } else {
                fs_store_part<V>(part + (int64_t)head * a.n_slots * V * N, slot, N, acc, lane);
                if (g == 0 && j < V) {
                    float *st = stats + ((int64_t)head * a.n_slots + slot) * 2 * V;
                    st[j] = m_run;
                    st[V + j] = l_tot;
                }
                slot++;
            }
            fs_clear(acc);
            m_run = -INFINITY;
            l_run = 0.f;
        }
        if (d0.last) from_first = true;
        d0 = d1;
        d1 = d2;
        cols0 = cols1;
        cols1 = cols2;
        bits0 = bits1;
    };
    for (; step + 1 < nblk; step++) block_step(std::true_type{});
    block_step(std::false_type{});
}

// Merges the parts of one cut window, 32 columns a wavefront, for every head, in slot order.  The parts carry (maximum m, sum l) per
// row in units of log2, and with m* the largest m of a row
//   out = factor * sum_k 2^(m_k - m*) tile_k / sum_k 2^(m_k - m*) l_k,   lse = ln 2 * (m* + log2 of that sum).
// Lane (row r = lane % V, q = lane / V) first walks the parts q, q + 64/V, ...; tiles are read in their storage order, sixteen loads in
// flight, and the rounded rows leave through LDS.
template <int DT, int V>
__global__ void __launch_bounds__(64)
k_merge_parts(const int4 *__restrict__ split_windows, const float *__restrict__ part, const float *__restrict__ stats, int n_slots, int N,
            fs_operand out, float factor, int64_t M, float *__restrict__ lse)
{
    constexpr int CH = 32, KQ = 64 / V;
    __shared__ __attribute__((aligned(16))) uint16_t out_t[V][CH + 8];
    const int n_chunks = (N + CH - 1) / CH, head = blockIdx.y;
    const int4 sw = split_windows[blockIdx.x / n_chunks];
    const int w = sw.x, p0 = sw.y, cnt = sw.z;
    const int lane = threadIdx.x, r = lane % V, q = lane / V;
    const int c0 = (blockIdx.x % n_chunks) * CH, nc = min(CH, N - c0);
    const float *st = stats + ((int64_t)head * n_slots + p0) * 2 * V;
    float top = -INFINITY;
    for (int k = q; k < cnt; k += KQ) top = fmaxf(top, st[(int64_t)k * 2 * V + r]);
#pragma unroll
    for (int o = V; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    const float use = top == -INFINITY ? 0.f : top;
    float total = 0.f;
    for (int k = q; k < cnt; k += KQ) total += st[(int64_t)k * 2 * V + V + r] * __builtin_amdgcn_exp2f(st[(int64_t)k * 2 * V + r] - use);
#pragma unroll
    for (int o = V; o < 64; o <<= 1) total += __shfl_xor(total, o, 64);
    const float inv = total == 0.f ? 0.f : factor / total;
    if (lse && c0 == 0 && q == 0 && (int64_t)w * V + r < M) lse[(int64_t)head * M + (int64_t)w * V + r] = fs_log_sum(use, total);
    const int64_t tile4 = (int64_t)V * N / 4;
    const fs_f4 *src0 = reinterpret_cast<const fs_f4 *>(part) + ((int64_t)head * n_slots + p0) * tile4 + (c0 / 4) * V;
    for (int idx = lane; idx < (nc / 4) * V; idx += 64) {  // idx % V == r
        const int ct = idx / (4 * V), rem = idx - ct * 4 * V, g = rem / V, j = rem - g * V;
        const fs_f4 *src = src0 + idx;
        fs_f4 sum = fs_f4{0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < cnt; k += 16) {
            fs_f4 v[16];
            float wk[16];
#pragma unroll
            for (int u = 0; u < 16; u++) {
                const int kk = min(k + u, cnt - 1);
                v[u] = src[(int64_t)kk * tile4];
                wk[u] = st[(int64_t)kk * 2 * V + j];
            }
#pragma unroll
            for (int u = 0; u < 16; u++)
                if (k + u < cnt) sum += v[u] * __builtin_amdgcn_exp2f(wk[u] - use);
        }
        uint2 o;
        o.x = fs_pack2<DT>(sum[0] * inv, sum[1] * inv);
        o.y = fs_pack2<DT>(sum[2] * inv, sum[3] * inv);
        *reinterpret_cast<uint2 *>(&out_t[j][16 * ct + 4 * g]) = o;
    }
    __syncthreads();
    const int c8n = nc / 8;
    for (int t = lane; t < V * c8n; t += 64) {
        const int j = t / c8n, c8 = t - j * c8n;
        const int64_t row = (int64_t)w * V + j;
        if (row < M)
            __builtin_nontemporal_store(*reinterpret_cast<const fs_u4 *>(&out_t[j][8 * c8]),
                                        reinterpret_cast<fs_u4 *>(out.p + head * out.head + row * out.pitch + 2 * (c0 + 8 * c8)));
    }
}

__global__ void __launch_bounds__(256) k_zero_heads(fs_operand m, int64_t rows, int pieces, float *__restrict__ lse)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / pieces;
    if (row >= rows) return;
    const int c = (int)(i - row * pieces);
    *reinterpret_cast<fs_u4 *>(m.p + blockIdx.y * m.head + row * m.pitch + 16 * c) = fs_u4{0u, 0u, 0u, 0u};
    if (lse && c == 0) lse[blockIdx.y * rows + row] = -INFINITY;
}

struct call {
    int heads, share, d, N;
    float sl2;
    fs_operand X, Y, H, out;
    fs_bias_args bias;
    fs_drop_args drop;
    float *lse, *work;
    hipStream_t st;
};

template <int DT, int V, int KS, int NT>
fs_status launch(const fs_format *f, const call &c)
{
    const fs_launch_geometry geo = fs_launch_geometry_for(f, 1);
    const fs_walk a = fs_walk_of(f, geo);
    float *stats = c.work + fs_part_floats(f, c.heads, c.N);
    k_heads_forward<DT, V, KS, NT><<<dim3(geo.nbx, c.heads), 64, fs_bias_lds_bytes(c.bias.n_buckets, c.bias.reach), c.st>>>(
        a, c.X, c.Y, c.H, c.share, c.d, c.N, c.sl2, c.bias, c.drop, c.out, c.lse, c.work, stats);
    FS_LAUNCH_CHECK();
    if (f->n_split_windows > 0) {
        const int64_t blocks = f->n_split_windows * ((c.N + 31) / 32);
        if (blocks >= ((int64_t)1 << 31)) return FS_ERR_TOO_LARGE;
        k_merge_parts<DT, V><<<dim3((unsigned)blocks, c.heads), 64, 0, c.st>>>((const int4 *)f->split_windows, c.work, stats, (int)f->n_split_items, c.N,
                                                                                  c.out, c.drop.factor, f->M, c.lse);
        FS_LAUNCH_CHECK();
    }
    return FS_OK;
}

template <int DT, int V, int KS>
fs_status launch_n(const fs_format *f, const call &c)
{
    return c.N <= 32 ? launch<DT, V, KS, 2>(f, c) : c.N <= 64 ? launch<DT, V, KS, 4>(f, c) : launch<DT, V, KS, 8>(f, c);
}
template <int DT, int V>
fs_status launch_d(const fs_format *f, const call &c)
{
    return c.d <= 32 ? launch_n<DT, V, 1>(f, c) : c.d <= 64 ? launch_n<DT, V, 2>(f, c) : launch_n<DT, V, 4>(f, c);
}
template <int DT>
fs_status launch_v(const fs_format *f, const call &c)
{
    return f->V == 4 ? launch_d<DT, 4>(f, c) : f->V == 8 ? launch_d<DT, 8>(f, c) : launch_d<DT, 16>(f, c);
}

}  // namespace

fs_status fs_zero_heads_launch(const fs_head_matrix *m, int64_t rows, int64_t columns, int heads, float *d_lse, hipStream_t st)
{
    if (rows == 0) return FS_OK;
    const int64_t blocks = (rows * (columns / 8) + 255) / 256;
    k_zero_heads<<<dim3((unsigned)blocks, heads), 256, 0, st>>>(fs_operand_of(m), rows, (int)(columns / 8), d_lse);
    FS_LAUNCH_CHECK();
    return FS_OK;
}

size_t fs_attention_forward_floats(const fs_format *f, int64_t heads, int64_t N)
{
    return fs_part_floats(f, heads, N + 2);  // the tiles, and a maximum and a sum per row
}

fs_status fs_attention_forward_launch(const fs_format *f, int heads, int kv_heads, int d, int N, float scale, const fs_head_matrix *X,
                                      const fs_head_matrix *Y, const fs_head_matrix *H, const fs_bucket_bias *bias, const fs_dropout *drop,
                                      const fs_head_matrix *out, float *lse, void *work, hipStream_t st)
{
    if (f->nvec == 0) return fs_zero_heads_launch(out, f->M, N, heads, lse, st);
    const call c = {heads, heads / kv_heads, d, N, scale * 1.44269504088896340736f, fs_operand_of(X), fs_operand_of(Y), fs_operand_of(H), fs_operand_of(out),
                    fs_bias_of(bias), fs_drop_of(drop), lse, (float *)work, st};
    return f->dtype == FS_F16 ? launch_v<FS_F16>(f, c) : launch_v<FS_BF16>(f, c);
}
