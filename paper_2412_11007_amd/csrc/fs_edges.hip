// A bucket bias and dropout on value arrays in the vals_blk layout, and the gradient of the bias table.
//
// bias      out = scale * in + table[bucket(column - row - shift)]
// dropout   out = in * factor where the entry is kept, else zero (and the same on a gradient)
// gradient  dtable[k] = sum of g over the entries of bucket k
//
// A block is V x kb consecutive elements, row by row.  A lane takes eight of them, sixteen bytes, so that a wave-wide load or store
// moves 1 KB of consecutive blocks (16 / V of them at full width) whatever their width; the row and the place of an element
// follow from its number and kb.  Which elements A stores is read from blk_row_bits, the columns of the block's vectors from
// vec_col; both pass through LDS.  Bias and dropout run near a copy's rate (R-MAT of 2^18 rows, bias: 29 us, 132 MB, 4.5 TB/s; lognormal
// graph, two heads, dropout: 83 us, 362 MB, 4.4 TB/s).
//
// The gradient adds into a table in LDS of fp32 sums, n_buckets x 64 with a column for each lane, or n_buckets x 16 with four lanes a column
// that take turns: no two lanes add to a sum at once.  A sum's summands come in the order in which its wavefront walks the blocks, the
// columns of a bucket are added in a fixed order at the end, and the wavefronts' tables by a second launch, so the result does not depend
// on timing.  The walk is bound by the chain value -> column -> bucket -> sum, so wavefronts count: where A stores less than half of the
// places, those that it stores are dealt out to the lanes and the narrow table lets 32 wavefronts of a CU work instead of 16 (32 buckets,
// R-MAT of 2^18 rows 42 us -> 33, lognormal graph 44 -> 31, uniform 36 -> 28); where it stores more, turns and dealing cost more than they
// bring (sequence of 8192 with a window of 384, two heads: 17 us -> 19).
#include <algorithm>

#include "fs_common.h"
#include "fs_heads.h"
#include "fs_tile.h"

namespace {

enum { OP_BIAS = 0, OP_DROPOUT = 1, OP_GRADIENT = 2, OP_GRADIENT_LISTED = 3 };

constexpr int kWaves = 4;  // of a workgroup; gradients: one

// Columns of a gradient's table of sums.
constexpr int sum_columns(int op) { return op == OP_GRADIENT_LISTED ? 16 : 64; }

// Whether A stores less than half of its blocks' places.
bool mostly_empty(const fs_format *f) { return 2 * f->nnz < f->V * f->nvec; }

// Wavefronts for one head's gradient: as many as the chip's LDS holds, of which each takes up to 2688 B (640 B without a list), its table of
// sums and, where the kernel is launched, that of the buckets.  A few more would wait for the first ones' end (R-MAT of 2^18 rows, 60
// buckets: 51 us with 5224 wavefronts, 39 with the 5120 that are resident).
int gradient_waves(int heads, int n_buckets, int op, int lut)
{
    const int lds = ((op == OP_GRADIENT_LISTED ? 2688 : 640) + lut + 4 * sum_columns(op) * n_buckets + 1279) / 1280 * 1280;
    return std::max(256, 256 * std::min(32, 160 * 1024 / lds) / std::max(heads, 1));
}

template <int DT, int V, int OP>
__global__ void __launch_bounds__(OP >= OP_GRADIENT ? 64 : 64 * kWaves)
k_edges(const int4 *__restrict__ blk_desc, int n_blocks, const uint32_t *__restrict__ row_bits, const int32_t *__restrict__ vec_col, int nvec,
        const uint16_t *in, uint16_t *out, int64_t n_el, float scale, fs_bias_args bias, fs_drop_args drop, float *__restrict__ sums)
{
    constexpr bool GRADIENT = OP >= OP_GRADIENT, LISTED = OP == OP_DROPOUT || OP == OP_GRADIENT_LISTED;
    constexpr int COLUMNS = sum_columns(OP);
    constexpr int WAVES = GRADIENT ? 1 : kWaves;
    constexpr int PER = 16 / V;    // blocks of a round
    constexpr int LANES = 4 * V;   // lanes of a block
    __shared__ __attribute__((aligned(16))) int cols_all[WAVES][PER][32];
    __shared__ uint32_t bits_all[WAVES][16];
    // LISTED: the blocks' {first row, kb's reciprocal | kb}, the places of a round's stored elements, and by place whether they are kept, or
    // their values
    __shared__ int2 blocks_all[WAVES][PER];
    __shared__ __attribute__((aligned(16))) uint16_t list_all[LISTED ? WAVES : 1][512];
    __shared__ __attribute__((aligned(16))) uint8_t kept_all[OP == OP_DROPOUT ? WAVES : 1][512];
    __shared__ __attribute__((aligned(16))) uint16_t values[512];
    extern __shared__ __attribute__((aligned(16))) unsigned char dyn[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, head = blockIdx.y;
    float *table = reinterpret_cast<float *>(dyn);                   // OP_BIAS: of the head
    uint8_t *lut = dyn + (OP == OP_BIAS ? bias.n_buckets * 4 : 0);
    float *table_of_sums = reinterpret_cast<float *>(dyn + (2 * bias.reach + 1 + 15) / 16 * 16);  // GRADIENT
    float *mine = table_of_sums + lane % COLUMNS;                                                  // + COLUMNS * bucket
    in += head * n_el;
    if constexpr (!GRADIENT) out += head * n_el;
    int *cols = cols_all[wave][lane / LANES];
    int2 *block_of = blocks_all[wave];
    uint32_t *bits = bits_all[wave] + (lane / LANES) * V;
    const int e0 = 8 * (lane % LANES);  // of the block

    fs_key key = fs_key{0u, 0u};
    if constexpr (OP == OP_DROPOUT) {
        key = fs_drop_key(drop, head);
    } else {
        fs_load_buckets(bias, lut, threadIdx.x, WAVES * 64);
        if constexpr (OP == OP_BIAS) {
            for (int i = threadIdx.x; i < bias.n_buckets; i += WAVES * 64) table[i] = fs_widen<DT>(bias.table[head * bias.ld + i]);
        } else {
            for (int i = lane; i < bias.n_buckets * COLUMNS; i += 64) table_of_sums[i] = 0.f;
        }
        __syncthreads();
    }
    const int step = gridDim.x * WAVES * PER;
    int x0 = (blockIdx.x * WAVES + wave) * PER;
    int4 ahead = blk_desc[min(x0 + lane / LANES, n_blocks - 1)];  // descriptors are read a round ahead (values too: slower, a third fewer wavefronts fit)
    for (; x0 < n_blocks; x0 += step) {
        const int x = x0 + lane / LANES;
        const int4 desc = ahead;
        ahead = blk_desc[min(x + step, n_blocks - 1)];
        const int kb = x < n_blocks ? desc.y & 255 : 0, row0 = desc.z * V;
        const int64_t first = (int64_t)V * desc.x;
        const int own = min(8, V * kb - e0);  // elements of the lane: eight, four (V = 4, odd width) or none
        fs_frag v;
        v.u = fs_u4{0u, 0u, 0u, 0u};
        if (own == 8) v.u = *reinterpret_cast<const fs_u4_unaligned *>(in + first + e0);
        else if (own == 4) v.s[0] = __builtin_bit_cast(fs_s4, *reinterpret_cast<const fs_u2_unaligned *>(in + first + e0));
        // the block's columns, and its rows' occupancy
        for (int c = lane % LANES; c < 32; c += LANES) cols[c] = vec_col[max(min(desc.x + min(c, kb - 1), nvec - 1), 0)];
        if (lane % LANES < V) bits[lane % LANES] = row_bits[(int64_t)min(x, n_blocks - 1) * V + lane % LANES];
        FS_WAVE_SYNC();
        const uint32_t inv = kb == 32 ? 2048u : (uint32_t)(65536.f * __builtin_amdgcn_rcpf((float)max(kb, 1))) + 1u;  // e / kb = e * inv >> 16 for e < 512
        auto row_of = [&](int k) -> int { return min((int)((uint32_t)(e0 + k) * inv >> 16), V - 1); };
        uint32_t m8 = 0;
        if (kb == 32) {
            m8 = bits[e0 >> 5] >> (e0 & 31) & 255u;
        } else if (own > 0) {
#pragma unroll
            for (int k = 0; k < 8; k++) {
                const int r = row_of(k);
                if (k < own) m8 |= (bits[r] >> (e0 + k - r * kb) & 1u) << k;
            }
        }
        // the buckets of the lane's eight places: their reads do not wait for one another
        auto buckets = [&](int (&bucket)[8]) {
            if (kb == 32) {
                const int4 lo = *reinterpret_cast<const int4 *>(cols + (e0 & 31)), hi = *reinterpret_cast<const int4 *>(cols + (e0 & 31) + 4);
                const int col[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                for (int k = 0; k < 8; k++) bucket[k] = fs_bucket_of(lut, bias.reach, bias.shift, row0 + (e0 >> 5), col[k]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; k++) {
                    const int r = row_of(k);
                    bucket[k] = fs_bucket_of(lut, bias.reach, bias.shift, row0 + r, cols[(e0 + k - r * kb) & 31]);
                }
            }
        };
        if constexpr (!LISTED) {
            int bucket[8];
            buckets(bucket);
            if constexpr (OP == OP_BIAS) {
                float y[8];
#pragma unroll
                for (int k = 0; k < 8; k++) y[k] = table[bucket[k]];
#pragma unroll
                for (int k = 0; k < 8; k++) y[k] = m8 >> k & 1u ? fmaf(scale, fs_widen<DT>(v.e[k]), y[k]) : 0.f;
                v.u = fs_u4{fs_pack2<DT>(y[0], y[1]), fs_pack2<DT>(y[2], y[3]), fs_pack2<DT>(y[4], y[5]), fs_pack2<DT>(y[6], y[7])};
            } else {
#pragma unroll
                for (int k = 0; k < 8; k++)
                    if (m8 >> k & 1u) mine[COLUMNS * bucket[k]] += fs_widen<DT>(v.e[k]);
            }
        } else {
            // the stored elements are dealt out to the lanes: an eighth of the places in a power-law graph (lane by lane, for as long as the
            // one with most has any: dropout of a lognormal graph, two heads, 124 us for 83)
            uint16_t *list = list_all[wave];
            const int own_n = __popc(m8);
            int sum = own_n;
            sum += __builtin_amdgcn_update_dpp(0, sum, 0x111, 0xF, 0xF, true);  // row_shr:1, 2, 4, 8
            sum += __builtin_amdgcn_update_dpp(0, sum, 0x112, 0xF, 0xF, true);
            sum += __builtin_amdgcn_update_dpp(0, sum, 0x114, 0xF, 0xF, true);
            sum += __builtin_amdgcn_update_dpp(0, sum, 0x118, 0xF, 0xF, true);
            sum += __builtin_amdgcn_update_dpp(0, sum, 0x142, 0xA, 0xF, true);  // row_bcast:15, 31
            sum += __builtin_amdgcn_update_dpp(0, sum, 0x143, 0xC, 0xF, true);
            const int n = __builtin_amdgcn_readlane(sum, 63);
            int at = sum - own_n;
            for (uint32_t m = m8; m; m &= m - 1) list[at++] = (uint16_t)(8 * lane + __builtin_ctz(m));
            if (lane % LANES == 0) block_of[lane / LANES] = make_int2(row0, (int)inv << 8 | kb);
            if constexpr (GRADIENT) *reinterpret_cast<fs_u4 *>(values + 8 * lane) = v.u;
            FS_WAVE_SYNC();
            for (int i0 = 0; i0 < n; i0 += 64) {
                const bool some = i0 + lane < n;
                const int place = some ? list[i0 + lane] : 0, b = place / (8 * LANES), e = place % (8 * LANES);
                const int2 of = block_of[b];
                const int r = (uint32_t)e * ((uint32_t)of.y >> 8) >> 16, c = e - r * (of.y & 255);
                const int row = of.x + r, col = cols_all[wave][b][c & 31];
                if constexpr (OP == OP_DROPOUT) {
                    if (some) kept_all[wave][place] = fs_threefry<13>(key, (uint32_t)row, (uint32_t)col).k0 >= drop.below;
                } else {
                    float *cell = mine + COLUMNS * fs_bucket_of(lut, bias.reach, bias.shift, row, col);
                    const float g = fs_widen<DT>(values[place]);
#pragma unroll
                    for (int turn = 0; turn < 64 / COLUMNS; turn++) {
                        if (some && lane / COLUMNS == turn) *cell += g;
                        FS_WAVE_SYNC();
                    }
                }
            }
            if constexpr (OP == OP_DROPOUT) {
                FS_WAVE_SYNC();
                const uint2 mine8 = *reinterpret_cast<const uint2 *>(kept_all[wave] + 8 * lane);
                float y[8];
#pragma unroll
                for (int k = 0; k < 8; k++) {
                    const uint32_t kept = (k < 4 ? mine8.x : mine8.y) >> (8 * (k & 3)) & m8 >> k & 1u;
                    y[k] = kept ? fs_widen<DT>(v.e[k]) * drop.factor : 0.f;
                }
                v.u = fs_u4{fs_pack2<DT>(y[0], y[1]), fs_pack2<DT>(y[2], y[3]), fs_pack2<DT>(y[4], y[5]), fs_pack2<DT>(y[6], y[7])};
            }
        }
        if constexpr (!GRADIENT) {
            if (own == 8) *reinterpret_cast<fs_u4_unaligned *>(out + first + e0) = v.u;
            else if (own == 4) *reinterpret_cast<fs_u2_unaligned *>(out + first + e0) = __builtin_bit_cast(fs_u2, v.s[0]);
        }
        FS_WAVE_SYNC();
    }
    if constexpr (GRADIENT) {
        float *to = sums + ((int64_t)head * gridDim.x + blockIdx.x) * bias.n_buckets;
        FS_WAVE_SYNC();
        fs_store_bucket_sums<COLUMNS>(table_of_sums, bias.n_buckets, lane, to);
    }
}

// Adds n tables of n_buckets sums, a contiguous share of them per workgroup: thread (r, b) those r, r + R, ... of its share, R = 1024
// over the buckets' power of two; then the R sums of a bucket in order.  DT < 0: to fp32 tables, one a workgroup.
template <int DT>
__global__ void __launch_bounds__(1024) k_bucket_sums(const float *__restrict__ sums, int n, int n_buckets, int log2_buckets, void *__restrict__ to)
{
    __shared__ float part[1024];
    const int b = threadIdx.x & ((1 << log2_buckets) - 1), r = threadIdx.x >> log2_buckets, R = 1024 >> log2_buckets;
    const int head = blockIdx.y, share = (n + gridDim.x - 1) / gridDim.x, i0 = blockIdx.x * share, i1 = min(n, i0 + share);
    const float *from = sums + (int64_t)head * n * n_buckets + min(b, n_buckets - 1);
    float t = 0.f;
    for (int i = i0 + r; i < i1; i += 8 * R) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; k++) v[k] = from[(int64_t)min(i + k * R, i1 - 1) * n_buckets];
#pragma unroll
        for (int k = 0; k < 8; k++) t += i + k * R < i1 ? v[k] : 0.f;
    }
    part[threadIdx.x] = t;
    __syncthreads();
    if (r > 0 || b >= n_buckets) return;
    for (int k = 1; k < R; k++) t += part[(k << log2_buckets) + b];
    const int64_t at = ((int64_t)head * gridDim.x + blockIdx.x) * n_buckets + b;
    if constexpr (DT < 0) ((float *)to)[at] = t;
    else ((uint16_t *)to)[at] = fs_round_bits<DT>(t);
}

template <int DT, int V, int OP>
fs_status launch(const fs_format *f, int heads, const uint16_t *in, uint16_t *out, float scale, const fs_bias_args &bias,
                 const fs_drop_args &drop, float *work, hipStream_t st)
{
    const int64_t rounds = f->nvec > 0 ? (f->n_blocks + 16 / V - 1) / (16 / V) : 0;
    const int lut = (2 * bias.reach + 1 + 15) / 16 * 16;
    if constexpr (OP >= OP_GRADIENT) {
        const unsigned waves = (unsigned)std::min<int64_t>(rounds, gradient_waves(heads, bias.n_buckets, OP, lut));
        if (waves > 0)
            k_edges<DT, V, OP><<<dim3(waves, heads), 64, lut + 4 * sum_columns(OP) * bias.n_buckets, st>>>(
                (const int4 *)f->blk_desc, (int)f->n_blocks, f->blk_row_bits, f->vec_col, (int)f->nvec, in, nullptr, (int64_t)V * f->nvec, scale, bias, drop, work);
        FS_LAUNCH_CHECK();
        return fs_bucket_sums_launch(f->dtype, heads, (int)waves, bias.n_buckets, work, out, st);
    }
    if (rounds == 0) return FS_OK;
    const unsigned groups = (unsigned)std::min<int64_t>((rounds + kWaves - 1) / kWaves, 256 * 8);
    k_edges<DT, V, OP><<<dim3(groups, heads), 64 * kWaves, OP == OP_BIAS ? lut + 4 * bias.n_buckets : 0, st>>>(
        (const int4 *)f->blk_desc, (int)f->n_blocks, f->blk_row_bits, f->vec_col, (int)f->nvec, in, out, (int64_t)V * f->nvec, scale, bias, drop, nullptr);
    FS_LAUNCH_CHECK();
    return FS_OK;
}

template <int OP>
fs_status launch_any(const fs_format *f, int heads, const void *in, void *out, float scale, const fs_bias_args &bias, const fs_drop_args &drop,
                     void *work, hipStream_t st)
{
#define FS_EDGES(DT, ROWS) \
    if (f->dtype == DT && f->V == ROWS) return launch<DT, ROWS, OP>(f, heads, (const uint16_t *)in, (uint16_t *)out, scale, bias, drop, (float *)work, st)
    FS_EDGES(FS_F16, 4);
    FS_EDGES(FS_F16, 8);
    FS_EDGES(FS_F16, 16);
    FS_EDGES(FS_BF16, 4);
    FS_EDGES(FS_BF16, 8);
    FS_EDGES(FS_BF16, 16);
#undef FS_EDGES
    return FS_ERR_UNSUPPORTED;
}

}  // namespace

fs_status fs_bucket_sums_launch(int dtype, int heads, int n, int n_buckets, float *sums, void *grad, hipStream_t st)
{
    int log2_buckets = 0;
    while (1 << log2_buckets < n_buckets) log2_buckets++;
    if (((int64_t)n << log2_buckets) > 64 * 1024) {  // one workgroup a head adds 64 sums a thread in 4 us; two launches take 6 and 2.5 us more of the host
        float *part = sums + (size_t)heads * n * n_buckets;
        k_bucket_sums<-1><<<dim3(kBucketSumGroups, heads), 1024, 0, st>>>(sums, n, n_buckets, log2_buckets, part);
        FS_LAUNCH_CHECK();
        sums = part;
        n = kBucketSumGroups;
    }
    if (dtype == FS_BF16) k_bucket_sums<FS_BF16><<<dim3(1, heads), 1024, 0, st>>>(sums, n, n_buckets, log2_buckets, grad);
    else k_bucket_sums<FS_F16><<<dim3(1, heads), 1024, 0, st>>>(sums, n, n_buckets, log2_buckets, grad);
    FS_LAUNCH_CHECK();
    return FS_OK;
}

fs_status fs_edge_bias_launch(const fs_format *f, int heads, const void *in, float scale, const fs_bucket_bias *b, void *out, hipStream_t st)
{
    return launch_any<OP_BIAS>(f, heads, in, out, scale, fs_bias_of(b), fs_drop_of(nullptr), nullptr, st);
}

fs_status fs_edge_dropout_launch(const fs_format *f, int heads, const void *in, const fs_dropout *d, void *out, hipStream_t st)
{
    return launch_any<OP_DROPOUT>(f, heads, in, out, 1.f, fs_bias_of(nullptr), fs_drop_of(d), nullptr, st);
}

size_t fs_edge_bias_backward_floats(const fs_format *f, int heads, int n_buckets)
{
    const int op = mostly_empty(f) ? OP_GRADIENT_LISTED : OP_GRADIENT;
    const int64_t rounds = (f->n_blocks + 16 / f->V - 1) / (16 / f->V);
    return fs_bucket_sums_floats(heads, std::min<int64_t>(rounds, gradient_waves(heads, n_buckets, op, 0)), n_buckets);
}

fs_status fs_edge_bias_backward_launch(const fs_format *f, int heads, const void *g, const fs_bucket_bias *b, void *grad, void *work, hipStream_t st)
{
    const fs_bias_args bias = fs_bias_of(b);
    const fs_drop_args drop = fs_drop_of(nullptr);
    return mostly_empty(f) ? launch_any<OP_GRADIENT_LISTED>(f, heads, g, grad, 1.f, bias, drop, work, st)
                           : launch_any<OP_GRADIENT>(f, heads, g, grad, 1.f, bias, drop, work, st);
}
