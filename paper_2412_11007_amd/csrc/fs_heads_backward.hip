// The gradients of attention with several heads, a bucket bias and dropout, in two walks that compute the scores again.
//
//   P = exp(s - lse),  D_i = g_i . out_i,  dS = P * (Z * (g_i . h_j) - D_i)
//   by rows of A     dX_i = scale * sum_j dS y_j,  dtable[k] = sum of dS over bucket k
//   by columns of A  dY_j = scale * sum_i dS x_i,  dH_j = sum_i Z P g_i          (rows of A^T, on its own format)
//
// Both walks are the forward pass's: per block of 32 vectors two operands are gathered (Y and H by rows, X and the gradient g of
// out by columns), put to LDS, and used from there twice -- as they are against the window's rows in registers (scores and g . h,
// contracted over the columns) and transposed against dS and Z P (the gradients, contracted over the vectors).  So a walk reads what
// the forward pass reads, and nothing is kept of the scores; no atomics, since a walk's outputs belong to its windows.
//
// The walk by rows has lse and D per window row; it computes D when it meets the window and leaves {lse, D} per row and head
// for the walk by columns, which gathers them beside the rows.  D comes from the rounded out: its error of half a step of the
// element type in each product is of the size of the errors of Z P and dS, which are rounded for the matrix cores.  fp16 holds Z P scaled by
// 2^12: probabilities are at most 1, and those of rows with thousands of entries would lie among its subnormal numbers; and dS by a power of two
// of its row that follows the largest (fs_round8_up; both walks together 1 to 3 % slower than without: lognormal graph 938 us for 922).
//
// dtable: the block's dS pass through LDS, its stored elements are dealt out to the lanes, and each adds to one of 16 columns of a table of
// fp32 sums, kSumColumns for each bucket.  Four lanes share a column and take turns, kept apart by fences (a column for each lane, 8 KB
// with 32 buckets: gradients of a lognormal graph 1068 us for 1017; atomics on LDS: 51 us for 15 in the same sums over a value array).  A wavefront
// leaves one sum per bucket, and those are added in the order of the work list.
//
// By columns the query heads that share keys and values are walked inside a block, one after the other, into the same accumulators.
//
// Bounds, with 64 columns of both kinds, bias and dropout: on a lognormal graph of 262 k rows, two heads, the fabric (by rows 465 us, 2.9 GB
// fetched, 6.9 TB/s; by columns 546 us, 3.3 GB, 6.7 TB/s, lines for the 8 bytes {lse, D} of a row among them); on a sequence of 4096
// with a window of 256, eight heads on two, instructions and too few wavefronts to hide a block's chain (53 and 58 us, 51 % and 39 % of the
// issue slots; by columns 1.3 wavefronts a SIMD on average).  Wavefronts a SIMD: by rows four up to 64 columns, three up to KS * NT = 8; by
// columns, with two tiles of accumulators and of gathered rows, three up to 64 columns (four spill: 501 us by rows became 562 so, before
// addresses were worked out where they are used).
#include <type_traits>

#include "fs_common.h"
#include "fs_heads.h"

namespace {

constexpr int kSumColumns = 16;  // of the table of sums in LDS, for each bucket
__host__ __device__ constexpr float fs_weight_scale(int dtype) { return dtype == FS_F16 ? 4096.f : 1.f; }  // of Z P

// Rows far from zero.  Beside a maximum of a thousand an fp32 lse holds too little of the logarithm of a row's sum for exp(s - lse) to add up to
// one, beside a mask of -1e9 nothing of it.  Of such rows, of |lse| > kFar, the maximum and the logarithm of the sum of 2^(s - maximum) are worked
// out again and subtracted one after the other.  A wavefront of the walk by rows looks for them in its item's windows before it begins and
// leaves both beside {lse, D}, for rows from kFarLeft on, with the maximum for lse.  The walk by columns finds them by what stands for their lse
// there, in units of log2 (kFarFound): of a far row it is at most 24 from lse, log2 of the most entries of a row, so above 1418; of those not left there
// at most 1399.
constexpr float kFar = 1000.f, kFarLeft = 970.f, kFarFound = 1410.f;
__device__ __forceinline__ bool is_far(float lse, float limit) { return fabsf(lse) > limit && fabsf(lse) < INFINITY; }

// Of the window's rows in lanes (j, g): the maximum of the scores, in units of log2, and the logarithm of the sum of 2^(s - maximum).  `at`: any block
// slot of the window.  All blocks of the window are walked, whatever item they belong to, with the products of the walk itself (the same bits:
// far from zero one more would be worth more than all), Y's rows straight from memory, the next block's indices on their way.  1.4 us a block: a
// sequence of 4096 with 256 entries a row 75 us for 52; a row of 262 k entries, whose 1024 wavefronts each walk all of it, 12 ms for 0.15.
template <int DT, int V, int KS>
__device__ __forceinline__ float2 far_rows(const fs_walk &a, int at, const unsigned char *Xb, uint32_t x_pitch, const unsigned char *Yb, uint32_t y_pitch, int d,
                                           float sl2, const fs_bias_args &bias, const float *table, const uint8_t *lut, int lane)
{
    const int j = lane & 15, g = lane >> 4;
    fs_frag xf[KS];
    fs_load_window<V>(xf, Xb, x_pitch, d, a.blk_desc[at].z, a.M, lane);
    while (!(a.blk_desc[at].y & 512)) at--;
    auto columns = [&](const int4 &desc) -> int { return a.vec_col[max(min(desc.x + min(lane & 31, (desc.y & 255) - 1), a.nvec - 1), 0)]; };
    int4 desc = a.blk_desc[at];
    int cols = columns(desc);
    uint32_t bits = a.row_bits[(int64_t)at * V + (j & (V - 1))];
    float m = -INFINITY, l = 0.f;
#pragma unroll 1
    for (;;) {
        const int4 here = desc;
        const int of = cols;
        const uint32_t m8 = j < V ? bits >> (8 * g) : 0u;
        const bool last = here.y & 256;
        if (!last) {  // the next block's, while this one's rows are on their way
            desc = a.blk_desc[++at];
            cols = columns(desc);
            bits = a.row_bits[(int64_t)at * V + (j & (V - 1))];
        }
        fs_frag y[2][KS];
#pragma unroll
        for (int t = 0; t < 2; t++) {
            const unsigned char *row = Yb + fs_mul24((uint32_t)__shfl(of, 8 * (j >> 2) + (j & 3) + 4 * t, 64), y_pitch);
#pragma unroll
            for (int ks = 0; ks < KS; ks++) {
                y[t][ks].u = fs_u4{0u, 0u, 0u, 0u};
                if (32 * ks + 8 * g < d) y[t][ks].u = *reinterpret_cast<const fs_u4 *>(row + 64 * ks + 16 * g);
            }
        }
        float v[8], top = m;
#pragma unroll
        for (int t = 0; t < 2; t++) {
            fs_f4 sc = fs_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ks++) sc = fs_mfma_16x16x32<DT>(y[t][ks], xf[ks], sc);
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const int x = 4 * t + k, col = __shfl(of, 8 * g + x, 64);
                const float bias_of = bias.n_buckets > 0 ? table[fs_bucket_of(lut, bias.reach, bias.shift, here.z * V + j, col)] : 0.f;
                v[x] = m8 >> x & 1u ? fmaf(sc[k], sl2, bias_of) : -INFINITY;
                top = fmaxf(top, v[x]);
            }
        }
        const float use = top == -INFINITY ? 0.f : top;
        l *= __builtin_amdgcn_exp2f(m - use);
#pragma unroll
        for (int x = 0; x < 8; x++) l += __builtin_amdgcn_exp2f(v[x] - use);
        m = top;
        if (last) break;
    }
    const float top = fs_row_max(m);
    l = fs_row_sum(l * __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top)));
    return make_float2(top, __builtin_amdgcn_logf(l));
}

template <int DT, int V, int KS, int NT>
__global__ void __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(KS <= 2 && NT <= 4 ? 4 : KS * NT <= 8 ? 3 : 2)))
k_heads_rows(fs_walk a, fs_operand X, fs_operand Y, fs_operand H, fs_operand out, fs_operand G, const float *__restrict__ lse, int share, int d, int N,
             float sl2, float scale, fs_bias_args bias, fs_drop_args drop, fs_operand dX, float2 *__restrict__ row_stats, float2 *far,
             float *__restrict__ part, float *__restrict__ bucket_sums)
{
    using tile_y = fs_gathered<32 * KS>;
    using tile_h = fs_gathered<16 * NT>;
    constexpr int KN = NT / 2, COLS = kSumColumns;
    __shared__ __attribute__((aligned(16))) unsigned char lds[tile_y::kBytes > tile_h::kBytes ? tile_y::kBytes : tile_h::kBytes];  // H's rows, then Y's
    __shared__ __attribute__((aligned(16))) int lds_cols[32];
    __shared__ float2 lds_far[16];  // by window row
    __shared__ fs_entries<V> entries;
    extern __shared__ __attribute__((aligned(16))) unsigned char dyn[];
    float *table = reinterpret_cast<float *>(dyn);
    uint8_t *lut = dyn + 4 * bias.n_buckets;
    float *sums = reinterpret_cast<float *>(dyn + (fs_bias_lds_bytes(bias.n_buckets, bias.reach) + 15) / 16 * 16);

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
    if (bucket_sums) {
        bucket_sums += ((int64_t)head * a.n_items + turn) * bias.n_buckets;
        if (nblk == 0) {
            for (int i = lane; i < bias.n_buckets; i += 64) bucket_sums[i] = 0.f;
            return;
        }
        for (int i = lane; i < bias.n_buckets * COLS; i += 64) sums[i] = 0.f;
    }
    if (nblk == 0) return;
    int slot = it.z;
    const int j = lane & 15, g = lane >> 4;
    const int4 my_desc = a.blk_desc[it.x + min(lane, nblk - 1)];
    auto block = [&](int i) -> BlockDesc { return fs_item_block(my_desc, i, nblk); };
    const unsigned char *Xb = X.p + head * X.head, *Yb = Y.p + head / share * Y.head, *Hb = H.p + head / share * H.head;
    const unsigned char *Gb = G.p + head * G.head, *Ob = out.p + head * out.head;
    const uint32_t y_colb = tile_y::column_bytes(lane, d), h_colb = tile_h::column_bytes(lane, N);

    int cols0 = fs_first_cols(a, it, lane);
    BlockDesc d0 = block(0), d1 = block(1);
    cols0 = fs_cut_cols(cols0, d0.kb, lane);
    int cols1 = fs_block_cols(a, d1, lane);
    uint32_t bits0 = fs_row_bits<V>(a, it.x, 0, nblk, lane);
    // of the window: X's and g's rows, and lse (in units of log2) and D of row j
    fs_frag xf[KS], gf[KN], of[KN];
    float my_lse = 0.f;
    auto load_window = [&](int w) {
        fs_load_window<V>(xf, Xb, X.pitch, d, w, a.M, lane);
        fs_load_window<V>(gf, Gb, G.pitch, N, w, a.M, lane);
    };
    auto load_stats = [&](int w) {
        fs_load_window<V>(of, Ob, out.pitch, N, w, a.M, lane);
        const int j = fs_lane_here(lane) & 15;
        const int64_t row = (int64_t)w * V + j;
        if (j < V && row < a.M) my_lse = lse[(int64_t)head * a.M + row];
    };
    load_window(d0.w);
    load_stats(d0.w);
    // whether the item's windows have a far row
    bool item_far = false;
    {
        const float *of = lse + (int64_t)head * a.M;
        const int last = min((__builtin_amdgcn_readlane(my_desc.z, nblk - 1) + 1) * V, (int)a.M) - 1;
        for (int first = d0.w * V; first <= last; first += 64) item_far |= is_far(of[min(first + lane, last)], kFarLeft);
    }
    tile_y y;
    tile_h h;
    y.load(Yb, Y.pitch, y_colb, cols0, lane);
    h.load(Hb, H.pitch, h_colb, cols0, lane);
    item_far = __builtin_amdgcn_ballot_w64(item_far);
    if (__builtin_expect(item_far, 0)) {
        FS_WAVE_SYNC();
        for (int i = 0; i < nblk; i++) {  // (a window's wavefronts all leave the same)
            if (i > 0 && !block(i).first) continue;
            const int64_t row = (int64_t)block(i).w * V + j;
            const float2 got = far_rows<DT, V, KS>(a, it.x + i, Xb, X.pitch, Yb, Y.pitch, d, sl2, bias, table, lut, lane);
            const float of_row = j < V && row < a.M ? lse[(int64_t)head * a.M + row] : 0.f;
            if (g == 0 && is_far(of_row, kFarLeft))
                far[(int64_t)head * a.M + row] = is_far(of_row, kFar) ? got : make_float2(of_row * 1.44269504088896340736f, 0.f);
        }
        __threadfence();
    }
    const bool looks_up = bias.n_buckets > 0 || drop.state;

    fs_f4 acc[2 * KS];
    fs_clear(acc);
    float up = kUpUnset;  // of acc
    bool from_first = d0.first, new_window = true;
    float lse2 = 0.f, D = 0.f;
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
        int n_entries = 0;
        if (looks_up) {
            n_entries = entries.make_list(bits0, lane, drop.state);
            entries.template look_up<false>(n_entries, lane, d0.w * V, cols0, lds_cols, bias, table, lut, drop, key);
        }
        h.put(lds, lane, N);
        if constexpr (MORE) h.load(Hb, H.pitch, h_colb, cols1, lane);
        FS_WAVE_SYNC();
        fs_f4 sc[2], gp[2];
#pragma unroll
        for (int t = 0; t < 2; t++) gp[t] = tile_h::template contract<DT>(lds, t, lane, gf);
        FS_WAVE_SYNC();
        y.put(lds, lane, d);
        if constexpr (MORE) y.load(Yb, Y.pitch, y_colb, cols1, lane);
        FS_WAVE_SYNC();
#pragma unroll
        for (int t = 0; t < 2; t++) sc[t] = tile_y::template contract<DT>(lds, t, lane, xf);
        if (new_window) {
            const int j = fs_lane_here(lane) & 15, row = d0.w * V + j;
            D = 0.f;
#pragma unroll
            for (int ks = 0; ks < KN; ks++)
#pragma unroll
                for (int k = 0; k < 8; k++) D = fmaf(fs_widen<DT>(gf[ks].e[k]), fs_widen<DT>(of[ks].e[k]), D);
            D = fs_row_sum(D);
            // a row of which nothing is left: exp(s - lse) has to come out as zero
            lse2 = my_lse == -INFINITY ? INFINITY : my_lse * 1.44269504088896340736f;
            if (__builtin_expect(item_far, 0)) {
                const bool left = j < V && row < a.M && is_far(my_lse, kFarLeft);
                const float2 of_row = left ? far[(int64_t)head * a.M + row] : make_float2(lse2, 0.f);
                lse2 = of_row.x;
                if (const int l = fs_lane_here(lane); l < 16) lds_far[l] = of_row;
                FS_WAVE_SYNC();
            }
            if (d0.first && g == 0 && j < V && row < a.M) row_stats[(int64_t)head * a.M + row] = make_float2(lse2, D);
            if (__builtin_expect(item_far, 0)) lse2 = 0.f;  // (see below)
        }
        new_window = MORE && d1.w != d0.w;
        if (new_window) load_window(d1.w);
        const uint32_t m8 = bits0 >> (8 * g);
        float ds[8];
        uint2 kept8 = make_uint2(~0u, ~0u);
        if (looks_up) {
            if (drop.state) kept8 = entries.kept_bytes(lane);
            entries.values(ds, lane);
        } else {
#pragma unroll
            for (int x = 0; x < 8; x++) ds[x] = 0.f;
        }
        if (__builtin_expect(item_far, 0)) {  // the entries' exponents in place of their biases, beside a score and an lse of zero
            const float2 of_row = lds_far[fs_lane_here(lane) & 15];
#pragma unroll
            for (int x = 0; x < 8; x++) {
                ds[x] = (fmaf(sc[x >> 2][x & 3], sl2, ds[x]) - of_row.x) - of_row.y;
                sc[x >> 2][x & 3] = 0.f;
            }
        }
#pragma unroll
        for (int x = 0; x < 8; x++) {
            const uint32_t kept = fs_kept_mask(kept8, x);
            const float p = __builtin_amdgcn_exp2f(fmaf(sc[x >> 2][x & 3], sl2, ds[x]) - lse2);
            const float gz = __uint_as_float(kept & __float_as_uint(gp[x >> 2][x & 3]));
            ds[x] = __uint_as_float(fs_bit_mask(m8, x) & __float_as_uint(p * fmaf(gz, drop.factor, -D)));
        }
        if (bucket_sums) {
            FS_WAVE_SYNC();
            entries.put_values(ds, lane);
            FS_WAVE_SYNC();
            const int l = fs_lane_here(lane);
            for (int r0 = 0; r0 < n_entries; r0 += 64) {
                const bool mine = r0 + l < n_entries;
                const int code = mine ? entries.list[r0 + l] : 0;
                const float v = entries.value[(code >> 5 & 15) * entries.kPitch + (code & 31)];
                float *cell = sums + COLS * (code >> 9) + (l & (COLS - 1));
#pragma unroll
                for (int turn_ = 0; turn_ < 64 / COLS; turn_++) {  // no two lanes of a turn share a cell; the fence keeps the turns apart,
                    if (mine && l / COLS == turn_) *cell += v;     // which look like one to a compiler that sees a lane at a time
                    FS_WAVE_SYNC();
                }
            }
        }
        const fs_frag sp = fs_round8_up<DT>(ds, up, acc);
        if (d0.kb > 0) {
#pragma unroll
            for (int t = 0; t < 2 * KS; t++) acc[t] = fs_mfma_16x16x32<DT>(tile_y::transposed(lds, t, lane), sp, acc[t]);
        }
        FS_WAVE_SYNC();
        if (new_window) load_stats(d1.w);
        if (d0.last || !MORE) {
            if (d0.last && from_first) {
                fs_store_window<DT, V, 32 * KS>(lds, acc, scale * fs_down<DT>(up), dX.p + head * dX.head, dX.pitch, d, d0.w, a.M, lane);
            } else {
                fs_scale_down<DT>(acc, up);
                fs_store_part<V>(part + (int64_t)head * a.n_slots * V * d, slot, d, acc, lane);
                slot++;
            }
            fs_clear(acc);
            up = kUpUnset;
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
    if (bucket_sums) {
        FS_WAVE_SYNC();
        fs_store_bucket_sums<COLS>(sums, bias.n_buckets, lane, bucket_sums);
    }
}

// By columns: `a` walks A^T, its vectors are rows of A (`rows` of them) and its window rows columns.
template <int DT, int V, int KS, int NT>
__global__ void __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(KS <= 2 && NT <= 4 ? 3 : 2)))
k_heads_cols(fs_walk a, int64_t rows, fs_operand X, fs_operand Y, fs_operand H, fs_operand G, const float2 *__restrict__ row_stats, const float2 *__restrict__ far,
             int share, int d, int N, float sl2, float scale, fs_bias_args bias, fs_drop_args drop, fs_operand dY, fs_operand dH, float *__restrict__ part_y,
             float *__restrict__ part_h)
{
    using tile_x = fs_gathered<32 * KS>;
    using tile_g = fs_gathered<16 * NT>;
    constexpr int KN = NT / 2;
    constexpr float kWeight = fs_weight_scale(DT);
    __shared__ __attribute__((aligned(16))) unsigned char lds_x[tile_x::kBytes];
    __shared__ __attribute__((aligned(16))) unsigned char lds_g[tile_g::kBytes];
    __shared__ __attribute__((aligned(16))) int lds_rows[32];
    __shared__ __attribute__((aligned(16))) float2 lds_stats[32];
    __shared__ fs_entries<V> entries;
    extern __shared__ __attribute__((aligned(16))) unsigned char dyn[];
    float *table = reinterpret_cast<float *>(dyn);  // of `share` heads
    uint8_t *lut = dyn + 4 * bias.n_buckets * share;

    const int lane = threadIdx.x, kv = blockIdx.y;
    const int turn = __builtin_amdgcn_readfirstlane(fs_launch_turn<1>(blockIdx.x, a.slice, a.n_swz));
    if (turn >= a.n_items) return;
    const int4 it = a.items[turn];
    if (bias.n_buckets > 0) {
        fs_load_buckets(bias, lut, lane, 64);
        for (int i = lane; i < bias.n_buckets * share; i += 64)
            table[i] = fs_bias_log2(fs_widen<DT>(bias.table[(kv * share + i / bias.n_buckets) * bias.ld + i % bias.n_buckets]));
    }
    fs_key keys = fs_key{0u, 0u};  // lane i: that of the group's head i
    if (drop.state) {
        const uint64_t seed = (uint64_t)drop.state[0], at = (uint64_t)drop.state[1];
        keys = fs_threefry<20>(fs_key{(uint32_t)seed, (uint32_t)(seed >> 32)}, (uint32_t)at, (uint32_t)(at >> 32));
        keys = fs_threefry<20>(keys, (uint32_t)(kv * share + lane), 0u);
    }
    const int nblk = it.y;
    if (nblk == 0) return;
    int slot = it.z;
    const int j = lane & 15, g = lane >> 4;
    const int4 my_desc = a.blk_desc[it.x + min(lane, nblk - 1)];
    auto block = [&](int i) -> BlockDesc { return fs_item_block(my_desc, i, nblk); };
    const unsigned char *Yb = Y.p + kv * Y.head, *Hb = H.p + kv * H.head;
    const uint32_t x_colb = tile_x::column_bytes(lane, d), g_colb = tile_g::column_bytes(lane, N);

    tile_x x_;
    tile_g g_;
    float2 st;
    auto gather = [&](int member, int row_of_lane) {  // of query head kv * share + member
        const int head = kv * share + member;
        x_.load(X.p + head * X.head, X.pitch, x_colb, row_of_lane, lane);
        g_.load(G.p + head * G.head, G.pitch, g_colb, row_of_lane, lane);
        st = row_stats[head * rows + row_of_lane];
    };
    int rows0 = fs_first_cols(a, it, lane);
    BlockDesc d0 = block(0), d1 = block(1);
    rows0 = fs_cut_cols(rows0, d0.kb, lane);
    int rows1 = fs_block_cols(a, d1, lane);
    uint32_t bits0 = fs_row_bits<V>(a, it.x, 0, nblk, lane), bits1 = fs_row_bits<V>(a, it.x, 1, nblk, lane);
    fs_frag yf[KS], hf[KN];
    fs_load_window<V>(yf, Yb, Y.pitch, d, d0.w, a.M, lane);
    fs_load_window<V>(hf, Hb, H.pitch, N, d0.w, a.M, lane);
    gather(0, rows0);
    fs_f4 acc_y[2 * KS], acc_h[NT];
    fs_clear(acc_y);
    fs_clear(acc_h);
    float up = kUpUnset;  // of acc_y
    bool from_first = d0.first;
    const bool looks_up = bias.n_buckets > 0 || drop.state;
    int step = 0, member = 0, n_entries = 0;
    for (;;) {  // a head of a block at a time
        const bool block_done = member + 1 == share, done = block_done && step + 1 == nblk;
        x_.put(lds_x, lane, d);
        g_.put(lds_g, lane, N);
        if (const int l = fs_lane_here(lane); l < 32) {
            lds_rows[l] = rows0;
            lds_stats[l] = st;
        }
        const float lse_here = st.x;  // of vector l mod 32
        BlockDesc d2 = d1;
        int rows2 = rows1;
        uint32_t bits2 = bits1;
        gather(block_done ? 0 : member + 1, block_done ? rows1 : rows0);  // (behind the last block: its own rows once more)
        if (block_done) {
            d2 = block(step + 2);
            rows2 = fs_block_cols(a, d2, lane);
            bits2 = fs_row_bits<V>(a, it.x, step + 2, nblk, lane);
        }
        FS_WAVE_SYNC();
        if (looks_up) {
            const fs_key key = fs_key{(uint32_t)__builtin_amdgcn_readlane((int)keys.k0, member), (uint32_t)__builtin_amdgcn_readlane((int)keys.k1, member)};
            if (member == 0) n_entries = entries.make_list(bits0, lane, drop.state);
            entries.template look_up<true>(n_entries, lane, d0.w * V, rows0, lds_rows, bias, table + member * bias.n_buckets, lut, drop, key);
        }
        fs_f4 sc[2], gp[2];
#pragma unroll
        for (int t = 0; t < 2; t++) {
            sc[t] = tile_x::template contract<DT>(lds_x, t, lane, yf);
            gp[t] = tile_g::template contract<DT>(lds_g, t, lane, hf);
        }
        if (block_done && d1.w != d0.w) {
            fs_load_window<V>(yf, Yb, Y.pitch, d, d1.w, a.M, lane);
            fs_load_window<V>(hf, Hb, H.pitch, N, d1.w, a.M, lane);
        }
        const uint32_t m8 = bits0 >> (8 * g);
        float ds[8], w[8];
        uint2 kept8 = make_uint2(~0u, ~0u);
        if (looks_up) {
            if (drop.state) kept8 = entries.kept_bytes(lane);
            entries.values(ds, lane);
        } else {
#pragma unroll
            for (int x = 0; x < 8; x++) ds[x] = 0.f;
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(is_far(lse_here, kFarFound)) != 0, 0)) {
            // the exponents of far rows' entries in place of their biases, beside a score and an lse of zero; the logarithms by way of lds_rows, which
            // this head's entries are done with
            const int l = fs_lane_here(lane);
            if (l < 32) lds_rows[l] = is_far(lse_here, kFarFound) ? __float_as_int(far[(int64_t)(kv * share + member) * rows + rows0].y) : 0;
            FS_WAVE_SYNC();
#pragma unroll
            for (int x = 0; x < 8; x++) {
                const float of_row = lds_stats[8 * g + x].x;
                if (!is_far(of_row, kFarFound)) continue;
                ds[x] = (fmaf(sc[x >> 2][x & 3], sl2, ds[x]) - of_row) - __int_as_float(lds_rows[8 * g + x]);
                sc[x >> 2][x & 3] = 0.f;
            }
            FS_WAVE_SYNC();
            if (l < 32 && is_far(lse_here, kFarFound)) lds_stats[l].x = 0.f;
            FS_WAVE_SYNC();
        }
#pragma unroll
        for (int x = 0; x < 8; x++) {
            const uint32_t stored = fs_bit_mask(m8, x), kept = stored & fs_kept_mask(kept8, x);
            const float2 rs = lds_stats[8 * g + x];
            const float p = __builtin_amdgcn_exp2f(fmaf(sc[x >> 2][x & 3], sl2, ds[x]) - rs.x);
            w[x] = __uint_as_float(kept & __float_as_uint(p * kWeight));
            const float gz = __uint_as_float(kept & __float_as_uint(gp[x >> 2][x & 3]));
            ds[x] = __uint_as_float(stored & __float_as_uint(p * fmaf(gz, drop.factor, -rs.y)));
        }
        const fs_frag sy = fs_round8_up<DT>(ds, up, acc_y), sh = fs_round8<DT>(w);
        if (d0.kb > 0) {
#pragma unroll
            for (int t = 0; t < 2 * KS; t++) acc_y[t] = fs_mfma_16x16x32<DT>(tile_x::transposed(lds_x, t, lane), sy, acc_y[t]);
#pragma unroll
            for (int t = 0; t < NT; t++) acc_h[t] = fs_mfma_16x16x32<DT>(tile_g::transposed(lds_g, t, lane), sh, acc_h[t]);
        }
        FS_WAVE_SYNC();
        if (!block_done) {
            member++;
            continue;
        }
        member = 0;
        if (d0.last || done) {
            if (d0.last && from_first) {
                fs_store_window<DT, V, 32 * KS>(lds_x, acc_y, scale * fs_down<DT>(up), dY.p + kv * dY.head, dY.pitch, d, d0.w, a.M, lane);
                fs_store_window<DT, V, 16 * NT>(lds_g, acc_h, drop.factor / kWeight, dH.p + kv * dH.head, dH.pitch, N, d0.w, a.M, lane);
            } else {
                fs_scale_down<DT>(acc_y, up);
                fs_store_part<V>(part_y + (int64_t)kv * a.n_slots * V * d, slot, d, acc_y, lane);
                fs_store_part<V>(part_h + (int64_t)kv * a.n_slots * V * N, slot, N, acc_h, lane);
                slot++;
            }
            fs_clear(acc_y);
            fs_clear(acc_h);
            up = kUpUnset;
        }
        if (done) break;
        if (d0.last) from_first = true;
        step++;
        d0 = d1;
        d1 = d2;
        rows0 = rows1;
        rows1 = rows2;
        bits0 = bits1;
        bits1 = bits2;
    }
}

struct call {
    int heads, kv_heads, d, N, n_grad;  // n_grad: buckets whose gradient is asked for, or 0
    float scale;
    fs_operand X, Y, H, out, G, dX, dY, dH;
    const float *lse;
    void *table_grad;
    fs_bias_args bias;
    fs_drop_args drop;
    float *work;
    hipStream_t st;
};

// What is left after the walks, in one launch: the partial tiles of cut windows are added and the wavefronts' sums per bucket
// gathered into a few.
struct Parts {  // of one output
    const int4 *split_windows;
    const float *tiles;
    fs_operand out;
    int64_t rows;
    float factor;
    int V, n_slots, columns, chunks, groups, heads;  // groups: workgroups, one for a window and 32 columns
};
struct Sums {
    const float *from;
    float *to;
    int n, n_buckets, groups, heads;
};

template <int DT>
__device__ __forceinline__ void add_parts(const Parts &p, int group, int head)
{
    __shared__ __attribute__((aligned(16))) uint16_t out_t[16][32 + 8];
    const int V = p.V, lane = threadIdx.x;
    const int4 sw = p.split_windows[group / p.chunks];  // {window, first slot, slots}
    const int c0 = group % p.chunks * 32, nc = min(32, p.columns - c0);
    const int64_t tile4 = (int64_t)V * p.columns / 4;
    const fs_f4 *src0 = reinterpret_cast<const fs_f4 *>(p.tiles) + ((int64_t)head * p.n_slots + sw.y) * tile4 + (c0 / 4) * V;
    for (int idx = lane; idx < nc / 4 * V; idx += 64) {  // in storage order: 16-column tile, 4-column group, row
        const int ct = idx / (4 * V), rem = idx - ct * 4 * V, g = rem / V, j = rem - g * V;
        fs_f4 sum = fs_f4{0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < sw.z; k += 16) {  // sixteen loads in flight, added in slot order
            fs_f4 v[16];
#pragma unroll
            for (int u = 0; u < 16; u++) v[u] = src0[idx + (int64_t)min(k + u, sw.z - 1) * tile4];
#pragma unroll
            for (int u = 0; u < 16; u++)
                if (k + u < sw.z) sum += v[u];
        }
        uint2 o;
        o.x = fs_pack2<DT>(sum[0] * p.factor, sum[1] * p.factor);
        o.y = fs_pack2<DT>(sum[2] * p.factor, sum[3] * p.factor);
        *reinterpret_cast<uint2 *>(&out_t[j][16 * ct + 4 * g]) = o;
    }
    __syncthreads();
    for (int t = lane; t < V * (nc / 8); t += 64) {
        const int j = t / (nc / 8), c8 = t - j * (nc / 8);
        const int64_t row = (int64_t)sw.x * V + j;
        if (row < p.rows)
            __builtin_nontemporal_store(*reinterpret_cast<const fs_u4 *>(&out_t[j][8 * c8]),
                                        reinterpret_cast<fs_u4 *>(p.out.p + head * p.out.head + row * p.out.pitch + 2 * (c0 + 8 * c8)));
    }
}

__device__ __forceinline__ void add_sums(const Sums &s, int group, int head)  // a contiguous share of the wavefronts' sums
{
    const int share = (s.n + s.groups - 1) / s.groups, i0 = group * share, i1 = min(s.n, i0 + share);
    for (int b = threadIdx.x; b < s.n_buckets; b += 64) {
        const float *from = s.from + (int64_t)head * s.n * s.n_buckets + b;
        float t = 0.f;
        for (int i = i0; i < i1; i += 8) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; k++) v[k] = from[(int64_t)min(i + k, i1 - 1) * s.n_buckets];
#pragma unroll
            for (int k = 0; k < 8; k++) t += i + k < i1 ? v[k] : 0.f;
        }
        s.to[((int64_t)head * s.groups + group) * s.n_buckets + b] = t;
    }
}

template <int DT>
__global__ void __launch_bounds__(64) k_heads_finish(Parts x, Parts y, Parts h, Sums s)
{
    int group = blockIdx.x;
    const int head = blockIdx.y;
    if (group < x.groups) {
        if (head < x.heads) add_parts<DT>(x, group, head);
        return;
    }
    group -= x.groups;
    if (group < y.groups) {
        if (head < y.heads) add_parts<DT>(y, group, head);
        return;
    }
    group -= y.groups;
    if (group < h.groups) {
        if (head < h.heads) add_parts<DT>(h, group, head);
        return;
    }
    add_sums(s, group - h.groups, head);
}

// Where the workspace's pieces lie, in floats: {lse, D} per row and head, what far rows leave beside, the wavefronts' sums per bucket and the groups
// they are gathered into, the partial tiles of the three outputs.
struct Pieces {
    size_t far, sums, grouped, x, y, h, total;
    int groups;
};
Pieces pieces_of(const fs_format *f, const fs_format *t, int64_t heads, int64_t kv_heads, int64_t d, int64_t N, int64_t n_grad)
{
    Pieces p;
    p.groups = (int)std::min<int64_t>(1024, (f->n_items + 31) / 32);
    p.far = 2 * (size_t)heads * (size_t)f->M;
    p.sums = fs_align_up(2 * p.far, 4);
    p.grouped = p.sums + fs_align_up((size_t)heads * (size_t)f->n_items * (size_t)n_grad, 4);
    p.x = p.grouped + fs_align_up(fs_bucket_sums_floats(heads, p.groups, n_grad), 4);  // (with room for the sums' own launches)
    p.y = p.x + fs_part_floats(f, heads, d);
    p.h = p.y + fs_part_floats(t, kv_heads, d);
    p.total = p.h + fs_part_floats(t, kv_heads, N);
    return p;
}

Parts parts_of(const fs_format *f, const float *tiles, int columns, int heads, const fs_operand &out, float factor)
{
    const int chunks = (columns + 31) / 32;
    return Parts{(const int4 *)f->split_windows, tiles, out, f->M, factor, f->V, (int)f->n_split_items, columns, chunks, (int)(f->n_split_windows * chunks), heads};
}

template <int DT, int V, int KS, int NT>
fs_status rows_launch(const fs_format *f, const call &c, const Pieces &at)
{
    const fs_launch_geometry geo = fs_launch_geometry_for(f, 1);
    const size_t lds = (fs_bias_lds_bytes(c.bias.n_buckets, c.bias.reach) + 15) / 16 * 16 + (size_t)c.n_grad * 4 * kSumColumns;
    k_heads_rows<DT, V, KS, NT><<<dim3(geo.nbx, c.heads), 64, lds, c.st>>>(fs_walk_of(f, geo), c.X, c.Y, c.H, c.out, c.G, c.lse, c.heads / c.kv_heads, c.d, c.N,
                                                                          c.scale * 1.44269504088896340736f, c.scale, c.bias, c.drop, c.dX, (float2 *)c.work,
                                                                          (float2 *)(c.work + at.far), c.work + at.x,
                                                                          c.n_grad > 0 ? c.work + at.sums : nullptr);
    FS_LAUNCH_CHECK();
    return FS_OK;
}

template <int DT, int V, int KS, int NT>
fs_status cols_launch(const fs_format *f, const fs_format *t, const call &c, const Pieces &at)
{
    const fs_launch_geometry geo = fs_launch_geometry_for(t, 1);
    const int share = c.heads / c.kv_heads;
    const size_t lds = c.bias.n_buckets > 0 ? fs_bias_lds_bytes(c.bias.n_buckets, c.bias.reach) + 4 * (size_t)c.bias.n_buckets * (share - 1) : 0;
    k_heads_cols<DT, V, KS, NT><<<dim3(geo.nbx, c.kv_heads), 64, lds, c.st>>>(fs_walk_of(t, geo), f->M, c.X, c.Y, c.H, c.G, (const float2 *)c.work,
                                                                             (const float2 *)(c.work + at.far), share, c.d, c.N,
                                                                             c.scale * 1.44269504088896340736f, c.scale, c.bias, c.drop, c.dY, c.dH,
                                                                             c.work + at.y, c.work + at.h);
    FS_LAUNCH_CHECK();
    return FS_OK;
}

template <int DT>
fs_status finish(const fs_format *f, const fs_format *t, const call &c, const Pieces &at)
{
    const Parts x = parts_of(f, c.work + at.x, c.d, c.heads, c.dX, c.scale), y = parts_of(t, c.work + at.y, c.d, c.kv_heads, c.dY, c.scale),
                h = parts_of(t, c.work + at.h, c.N, c.kv_heads, c.dH, c.drop.factor / fs_weight_scale(DT));
    const Sums s = {c.work + at.sums, c.work + at.grouped, (int)f->n_items, c.n_grad, c.n_grad > 0 ? at.groups : 0, c.heads};
    const int64_t blocks = (int64_t)x.groups + y.groups + h.groups + s.groups;
    if (blocks > 0) {
        k_heads_finish<DT><<<dim3((unsigned)blocks, c.heads), 64, 0, c.st>>>(x, y, h, s);
        FS_LAUNCH_CHECK();
    }
    return c.n_grad > 0 ? fs_bucket_sums_launch(DT, c.heads, at.groups, c.n_grad, c.work + at.grouped, c.table_grad, c.st) : FS_OK;
}

// The two formats may have windows of different heights.
template <int DT, int KS, int NT>
fs_status launch(const fs_format *f, const fs_format *t, const call &c)
{
    const Pieces at = pieces_of(f, t, c.heads, c.kv_heads, c.d, c.N, c.n_grad);
    fs_status s = f->V == 4   ? rows_launch<DT, 4, KS, NT>(f, c, at)
                  : f->V == 8 ? rows_launch<DT, 8, KS, NT>(f, c, at)
                              : rows_launch<DT, 16, KS, NT>(f, c, at);
    if (s == FS_OK)
        s = t->V == 4   ? cols_launch<DT, 4, KS, NT>(f, t, c, at)
            : t->V == 8 ? cols_launch<DT, 8, KS, NT>(f, t, c, at)
                        : cols_launch<DT, 16, KS, NT>(f, t, c, at);
    return s == FS_OK ? finish<DT>(f, t, c, at) : s;
}
template <int DT, int KS>
fs_status launch_n(const fs_format *f, const fs_format *t, const call &c)
{
    return c.N <= 32 ? launch<DT, KS, 2>(f, t, c) : c.N <= 64 ? launch<DT, KS, 4>(f, t, c) : launch<DT, KS, 8>(f, t, c);
}
template <int DT>
fs_status launch_d(const fs_format *f, const fs_format *t, const call &c)
{
    return c.d <= 32 ? launch_n<DT, 1>(f, t, c) : c.d <= 64 ? launch_n<DT, 2>(f, t, c) : launch_n<DT, 4>(f, t, c);
}

}  // namespace

size_t fs_attention_backward_floats(const fs_format *f, const fs_format *t, int64_t heads, int64_t kv_heads, int64_t d, int64_t N, int64_t n_grad)
{
    return pieces_of(f, t, heads, kv_heads, d, N, n_grad).total;
}

fs_status fs_attention_backward_launch(const fs_format *f, const fs_format *t, int heads, int kv_heads, int d, int N, float scale, const fs_head_matrix *X,
                                       const fs_head_matrix *Y, const fs_head_matrix *H, const fs_bucket_bias *bias, const fs_dropout *drop,
                                       const fs_head_matrix *out, const float *lse, const fs_head_matrix *G, const fs_head_matrix *dX,
                                       const fs_head_matrix *dY, const fs_head_matrix *dH, void *table_grad, void *work, hipStream_t st)
{
    if (f->nvec == 0) {
        fs_status s = fs_zero_heads_launch(dX, f->M, d, heads, nullptr, st);
        if (s == FS_OK) s = fs_zero_heads_launch(dY, f->K, d, kv_heads, nullptr, st);
        if (s == FS_OK) s = fs_zero_heads_launch(dH, f->K, N, kv_heads, nullptr, st);
        return s != FS_OK || !table_grad ? s : fs_bucket_sums_launch(f->dtype, heads, 0, bias->n_buckets, (float *)work, table_grad, st);
    }
    const call c = {heads, kv_heads, d, N, table_grad ? bias->n_buckets : 0, scale,
                    fs_operand_of(X), fs_operand_of(Y), fs_operand_of(H), fs_operand_of(out), fs_operand_of(G), fs_operand_of(dX), fs_operand_of(dY), fs_operand_of(dH),
                    lse, table_grad, fs_bias_of(bias), fs_drop_of(drop), (float *)work, st};
    return f->dtype == FS_F16 ? launch_d<FS_F16>(f, t, c) : launch_d<FS_BF16>(f, t, c);
}
