// Device pieces shared by the kernels of attention with several heads, a bucket bias and dropout (fs_heads.hip,
// fs_heads_backward.hip) and by the same steps on value arrays (fs_edges.hip).
//
// Bias.  The bias of an entry is that of the bucket of its clamped relative position column - row - shift.  The buckets of
// all 2 * reach + 1 positions are a table of bytes that the caller made (any rule, exact at its borders); it and the head's
// biases, widened to fp32, are copied to LDS when a workgroup starts, so that an entry costs two LDS reads.
//
// Dropout.  An entry is dropped where a word drawn for (head, row, column) is below p * 2^32.  The generator is Threefry-2x32
// (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): additions, rotations and exclusive ors,
// all of them full-rate instructions here (a Philox of the same paper takes 20 quarter-rate multiplications a call), with the 13
// rounds that the paper reports to pass its batteries for entries and the default 20 for keys.  The counter is (row, column): no
// mask is stored, and the kernels that walk A by rows, those that walk A^T and the ones on value arrays draw the same one.
#pragma once

#include <algorithm>

#include "fs_common.h"
#include "fs_tile.h"

namespace {

template <int DT>
__device__ __forceinline__ float fs_widen(uint16_t bits)
{
    if (DT == FS_F16) return (float)__builtin_bit_cast(_Float16, bits);
    return __uint_as_float((uint32_t)bits << 16);
}

struct fs_key {
    uint32_t k0, k1;
};

// Threefry-2x32: both words of the counter (c0, c1) under a key.
template <int ROUNDS>
__host__ __device__ __forceinline__ fs_key fs_threefry(fs_key key, uint32_t c0, uint32_t c1)
{
    constexpr int turn[8] = {13, 15, 26, 6, 17, 29, 16, 24};
    const uint32_t ks[3] = {key.k0, key.k1, key.k0 ^ key.k1 ^ 0x1BD11BDAu};
    uint32_t a = c0 + key.k0, b = c1 + key.k1;
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) {
        a += b;
        b = (b << turn[i % 8] | b >> (32 - turn[i % 8])) ^ a;
        if (i % 4 == 3) {
            a += ks[(i / 4 + 1) % 3];
            b += ks[(i / 4 + 2) % 3] + (uint32_t)(i / 4 + 1);
        }
    }
    return fs_key{a, b};
}

// The lane's number as something that is not known ahead of a loop: addresses that only a window's end needs are worked out there, where they
// would be kept over all blocks otherwise, in registers that spill (and a spilled register's load waits for the gathers before it).
__device__ __forceinline__ int fs_lane_here(int lane)
{
    asm volatile("" : "+v"(lane));
    return lane;
}

// Reductions over the four lanes of a row, l, l ^ 16, l ^ 32 and l ^ 48: rows of sixteen lanes, then halves of the wavefront, change places in
// two copies of a register (no LDS traffic, no address).
__device__ __forceinline__ float fs_row_max(float v)
{
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float fs_row_sum(float v)
{
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// What the kernels are given of a bias and of a dropout (n_buckets = 0, state null: none).
struct fs_bias_args {
    const uint16_t *table;
    const uint8_t *bucket;
    int64_t ld;
    int n_buckets, reach, shift;
};
struct fs_drop_args {
    const int64_t *state;  // seed and step
    uint32_t below;        // an entry whose word is below is dropped
    float factor;          // 1 / (1 - p)
};

__device__ __forceinline__ fs_key fs_drop_key(const fs_drop_args &d, int head)
{
    fs_key k = fs_key{0u, 0u};
    if (d.state) {
        const uint64_t seed = (uint64_t)d.state[0], step = (uint64_t)d.state[1];
        k = fs_threefry<20>(fs_key{(uint32_t)seed, (uint32_t)(seed >> 32)}, (uint32_t)step, (uint32_t)(step >> 32));
        k = fs_threefry<20>(k, (uint32_t)head, 0u);
    }
    return fs_key{(uint32_t)__builtin_amdgcn_readfirstlane((int)k.k0), (uint32_t)__builtin_amdgcn_readfirstlane((int)k.k1)};
}

// Bytes of LDS for a head's biases and the buckets of the positions.
__host__ __device__ __forceinline__ int fs_bias_lds_bytes(int n_buckets, int reach)
{
    return n_buckets > 0 ? n_buckets * 4 + (2 * reach + 1 + 3) / 4 * 4 : 0;
}

// The buckets of the positions as bytes, four at a time (`bucket` is 4-byte aligned), no index past the table's end.
__device__ __forceinline__ void fs_load_buckets(const fs_bias_args &b, uint8_t *lut, int thread, int threads)
{
    const int n = 2 * b.reach + 1;
    const uint32_t most = (uint32_t)b.n_buckets - 1;
    for (int i = thread; i < (n + 3) / 4; i += threads) {
        uint32_t v = 0;
        if (4 * i + 4 <= n) v = reinterpret_cast<const uint32_t *>(b.bucket)[i];
        else
            for (int k = 0; 4 * i + k < n; k++) v |= (uint32_t)b.bucket[4 * i + k] << (8 * k);
        uint32_t o = 0;
#pragma unroll
        for (int k = 0; k < 4; k++) o |= min(v >> (8 * k) & 255u, most) << (8 * k);
        reinterpret_cast<uint32_t *>(lut)[i] = o;
    }
}

// Bucket of the entry (row, col).  Rows and columns are below 2^31; the subtraction of the shift saturates.
__device__ __forceinline__ int fs_bucket_of(const uint8_t *lut, int reach, int shift, int row, int col)
{
    const int r = __builtin_elementwise_sub_sat(col - row, shift);
    return lut[min(max(r, -reach), reach) + reach];
}

// A wavefront's table of COLS sums per bucket (a power of two) -> one sum per bucket.  The order of the columns differs from
// bucket to bucket, so that the lanes read different banks, and is always the same.
template <int COLS>
__device__ __forceinline__ void fs_store_bucket_sums(const float *table, int n_buckets, int lane, float *__restrict__ to)
{
    for (int b = lane; b < n_buckets; b += 64) {
        float t = 0.f;
#pragma unroll 8
        for (int c = 0; c < COLS; c++) t += table[COLS * b + ((c + b) & (COLS - 1))];
        to[b] = t;
    }
}

// ln 2 * (m + log2 l): the log-sum-exp of a row whose scores, in units of log2, have the maximum m and the sum l of 2^(. - m).
// A row without entries, or with nothing but minus infinities, has minus infinity.
__device__ __forceinline__ float fs_log_sum(float m, float l)
{
    return l == 0.f ? -INFINITY : 0.693147180559945309f * (m + __builtin_amdgcn_logf(l));
}

// A bias in units of log2.  A finite one stays finite: bf16's lowest value is a mask, but no minus infinity.
__device__ __forceinline__ float fs_bias_log2(float b)
{
    const float t = b * 1.44269504088896340736f;
    return __builtin_isfinite(b) ? fminf(fmaxf(t, -3.402823466e38f), 3.402823466e38f) : t;
}

// Host side: the checked arguments as the kernels take them.
inline fs_bias_args fs_bias_of(const fs_bucket_bias *b)
{
    if (!b) return fs_bias_args{nullptr, nullptr, 0, 0, 0, 0};
    return fs_bias_args{(const uint16_t *)b->d_table, b->d_bucket, b->ld, b->n_buckets, b->reach, (int)b->shift};
}
inline fs_drop_args fs_drop_of(const fs_dropout *d)
{
    if (!d || d->p == 0.0) return fs_drop_args{nullptr, 0u, 1.f};
    return fs_drop_args{d->d_state, (uint32_t)(d->p * 4294967296.0), (float)(1.0 / (1.0 - d->p))};
}

// Sums over `n` tables go through this many partial ones (0: straight).
constexpr int kBucketSumGroups = 64;
inline size_t fs_bucket_sums_floats(int64_t heads, int64_t n, int64_t n_buckets) { return (size_t)heads * (size_t)(n + kBucketSumGroups) * (size_t)n_buckets; }

}  // namespace

// grad[h][b] = sum over i < n of sums[h][i][b], rounded to the element type; `sums` is followed by room for the partial ones
// (fs_bucket_sums_floats in all).  In fs_edges.hip.
fs_status fs_bucket_sums_launch(int dtype, int heads, int n, int n_buckets, float *sums, void *grad, hipStream_t st);

// ---------------------------------------------------------------------------------------------------------------------------
// The block walk of the attention kernels

namespace {

// The work list and the pattern, as the kernels take them.
struct fs_walk {
    const int4 *items;
    const int4 *blk_desc;
    const int32_t *vec_col;
    const uint32_t *row_bits;
    int64_t M;
    int n_items, nvec, n_slots, slice, n_swz;
};
inline fs_walk fs_walk_of(const fs_format *f, const fs_launch_geometry &geo)
{
    return fs_walk{(const int4 *)f->items_by_cost, (const int4 *)f->blk_desc, f->vec_col, f->blk_row_bits, f->M,
                   (int)f->n_items, (int)f->nvec, (int)f->n_split_items, geo.slice, geo.n_swz};
}

// A matrix per head whose rows are gathered or held: byte strides.
struct fs_operand {
    unsigned char *p;
    int64_t head;
    uint32_t pitch;
};
inline fs_operand fs_operand_of(const fs_head_matrix *m) { return fs_operand{(unsigned char *)m->d, 2 * m->head, (uint32_t)(2 * m->ld)}; }

// 32 gathered rows of up to NC columns on their way to LDS: 16 bytes a lane, neighbouring lanes on one row; in LDS the layout of the
// staged tile (lds_row), where they are read as they are (contraction over the columns) and transposed (over the rows).
// Columns from `width` on are zeros.
template <int NC>
struct fs_gathered {
    static constexpr int LPR = NC / 8, RPI = 64 / LPR, NLD = 32 / RPI, RS = NC * 2;
    static constexpr int kBytes = (lds_row<RS>(31) + RS + 15) / 16 * 16;
    fs_u4 r[NLD];

    // cols: lane l holds the row number of vector l (mod 32); colb: the lane's column_bytes()
    __device__ __forceinline__ void load(const unsigned char *base, uint32_t pitch, uint32_t colb, int cols, int lane)
    {
#pragma unroll
        for (int l = 0; l < NLD; l++) {
            const int row = __shfl(cols, l * RPI + lane / LPR, 64);
            r[l] = *reinterpret_cast<const fs_u4 *>(base + (fs_mul24((uint32_t)row, pitch) + colb));
        }
    }
    static __device__ __forceinline__ uint32_t column_bytes(int lane, int width) { return 2 * (uint32_t)min((lane % LPR) * 8, width - 8); }
    __device__ __forceinline__ void put(unsigned char *lds, int lane, int width) const
    {
        unsigned char *to = lds + lds_row<RS>(lane / LPR) + (lane % LPR) * 16;
        if (width == NC) {
#pragma unroll
            for (int l = 0; l < NLD; l++) *reinterpret_cast<fs_u4 *>(to + lds_row<RS>(l * RPI)) = r[l];
        } else {
            const bool in = (lane % LPR) * 8 < width;
#pragma unroll
            for (int l = 0; l < NLD; l++) *reinterpret_cast<fs_u4 *>(to + lds_row<RS>(l * RPI)) = in ? r[l] : fs_u4{0u, 0u, 0u, 0u};
        }
    }
    // tile t of the products with an operand held in registers: lane (j, g) gets vectors 8g + 4t .. +3 of window row j
    template <int DT, int STEPS>
    static __device__ __forceinline__ fs_f4 contract(const unsigned char *lds, int t, int lane, const fs_frag (&held)[STEPS])
    {
        const int j = lane & 15, g = lane >> 4;
        const unsigned char *rd = lds + lds_row<RS>(8 * (j >> 2) + (j & 3)) + 4 * t * (RS + 32) + 16 * g;
        fs_f4 acc = fs_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < STEPS; ks++) {
            fs_frag a;
            a.u = *reinterpret_cast<const fs_u4 *>(rd + 64 * ks);
            acc = fs_mfma_16x16x32<DT>(a, held[ks], acc);
        }
        return acc;
    }
    // 16-column tile t, transposed: the operand that is multiplied with a weight per (vector, window row)
    static __device__ __forceinline__ fs_frag transposed(const unsigned char *lds, int t, int lane)
    {
        const int g = lane >> 4;
        const unsigned char *rd = lds + lds_row<RS>(8 * g + ((lane & 15) >> 2)) + 8 * (lane & 3);
        fs_frag a;
#pragma unroll
        for (int h = 0; h < 2; h++)
            a.s[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((fs_s4 __attribute__((address_space(3))) *)(rd + lds_row<RS>(4 * h) + 32 * t));
        return a;
    }
};

// A window's rows in operand layout: lane (j, g) holds columns 32ks + 8g .. +7 of row w * V + j; rows past V or the last, and columns
// past `width`, are zeros.  Lanes without a row load nothing: in this layout a load takes the vector-memory unit a cycle per lane.
template <int V, int STEPS>
__device__ __forceinline__ void fs_load_window(fs_frag (&held)[STEPS], const unsigned char *base, uint32_t pitch, int width, int w, int64_t rows, int lane_)
{
    const int lane = fs_lane_here(lane_);
    const int j = lane & 15, g = lane >> 4;
    const int64_t row = (int64_t)w * V + j;
#pragma unroll
    for (int ks = 0; ks < STEPS; ks++) held[ks].u = fs_u4{0u, 0u, 0u, 0u};
    if (j < V && row < rows) {
        const uint32_t at = fs_mul24((uint32_t)row, pitch) + 16 * g;
#pragma unroll
        for (int ks = 0; ks < STEPS; ks++)
            if (32 * ks + 8 * g < width) held[ks].u = *reinterpret_cast<const fs_u4 *>(base + (at + 64 * ks));
    }
}

// The columns of a block's vectors, lane l that of vector l mod 32; vectors past the block's width repeat its last one.
__device__ __forceinline__ int fs_block_cols(const fs_walk &a, const BlockDesc &b, int lane)
{
    return a.vec_col[max(min(b.s + min(lane & 31, b.kb - 1), a.nvec - 1), 0)];
}

// The same for the first block of an item, whose first vector stands in the item's record: the load is issued beside the descriptor's, not
// after it (fs_first_cols), and cut to the block's width when that is known.
__device__ __forceinline__ int fs_first_cols(const fs_walk &a, const int4 &item, int lane) { return a.vec_col[min(item.w + (lane & 31), a.nvec - 1)]; }
__device__ __forceinline__ int fs_cut_cols(int cols, int kb, int lane)
{
    const int last = __builtin_amdgcn_readlane(cols, max(kb - 1, 0));
    return (lane & 31) < kb ? cols : last;
}

// Occupancy of window row j in block i of an item: bit c, the row stores the block's vector c (none for lanes past V).
template <int V>
__device__ __forceinline__ uint32_t fs_row_bits(const fs_walk &a, int first_slot, int i, int nblk, int lane)
{
    const int j = lane & 15;
    const uint32_t m = a.row_bits[(int64_t)(first_slot + min(i, nblk - 1)) * V + (j & (V - 1))];
    return i < nblk && j < V ? m : 0u;
}

// What an entry needs beside its score -- a bias from its bucket, a word of the generator -- takes about 70 instructions.  In the
// scores' layout a lane has eight places, and taken place by place they were most of a block's: of a power-law graph an eighth of
// the places are stored, and with eight rows a window half the lanes have none.  So every lane takes one entry at a time from a list in LDS
// or one place at a time in row order, without a list: where more than half of the block is stored; with four rows, whose 128 places are
// two turns; with eight rows and no dropout, where a place costs less than the list's chain (one row of 1028 entries, eight heads, 12.1 us with
// the list, 10.5 without; R-MAT of 65 k rows 48 and 45; with dropout, R-MAT of 131 k rows, gradients 156 with and 171 without).  The results go to two
// V x 32 tiles, the biases and whether dropout keeps the entry.  (The latter as the lowest bit of the bias would set apart what is kept and what is
// dropped in the softmax itself: beside a bias far from zero that bit is worth more than the scores.)
template <int V>
struct fs_entries {
    static constexpr int kPitch = 36;  // floats from a row of `value` to the next: rows start in different banks
    uint16_t list[32 * V];             // vector | row << 5 | bucket << 9
    float value[V * kPitch] __attribute__((aligned(16)));
    uint8_t kept[32 * V] __attribute__((aligned(8)));  // 1 or 0; without dropout not written

    // m: occupancy of row j.  Returns how many of the list's elements to take, the same in all lanes.
    __device__ __forceinline__ int make_list(uint32_t m, int lane_, bool draws)
    {
        if (V == 4 || (V == 8 && !draws)) return 32 * V;
        const int lane = fs_lane_here(lane_);
        const int j = lane & 15, g = lane >> 4;
        const int own = __popc(m);
        int sum = own;  // over the rows up to j
        sum += __builtin_amdgcn_update_dpp(0, sum, 0x111, 0xF, 0xF, true);  // row_shr:1
        sum += __builtin_amdgcn_update_dpp(0, sum, 0x112, 0xF, 0xF, true);
        sum += __builtin_amdgcn_update_dpp(0, sum, 0x114, 0xF, 0xF, true);
        sum += __builtin_amdgcn_update_dpp(0, sum, 0x118, 0xF, 0xF, true);
        const int n = __builtin_amdgcn_readlane(sum, 15);
        if (n > 16 * V) return 32 * V;
        int at = sum - own + __popc(m & ((1u << (8 * g)) - 1u));
        for (uint32_t m8 = m >> (8 * g) & 255u; m8; m8 &= m8 - 1) list[at++] = (uint16_t)(8 * g + __builtin_ctz(m8) | j << 5);
        return n;
    }
    // T: window rows are columns of A.  cols: lane l holds the column (T: row) of vector l mod 32; lds_cols the same in LDS.
    template <bool T>
    __device__ __forceinline__ void look_up(int n, int lane_, int row0, int cols, const int *lds_cols, const fs_bias_args &b, const float *table,
                                            const uint8_t *lut, const fs_drop_args &drop, fs_key key)
    {
        const int lane = fs_lane_here(lane_);
        auto bucket = [&](int j, int col) -> int { return fs_bucket_of(lut, b.reach, b.shift, T ? col : row0 + j, T ? row0 + j : col); };
        auto keep = [&](int j, int col) -> uint8_t {
            return fs_threefry<13>(key, (uint32_t)(T ? col : row0 + j), (uint32_t)(T ? row0 + j : col)).k0 >= drop.below ? 1 : 0;
        };
        if (n == 32 * V) {
            const int c = lane & 31, j0 = lane >> 5;
            constexpr int P = V / 2 < 4 ? V / 2 : 4;  // side by side
#pragma unroll
            for (int i0 = 0; i0 < V / 2; i0 += P) {
                float v[P];
                if (b.n_buckets > 0) {
                    int k[P];
#pragma unroll
                    for (int i = 0; i < P; i++) k[i] = bucket(2 * (i0 + i) + j0, cols);
#pragma unroll
                    for (int i = 0; i < P; i++) {
                        v[i] = table[k[i]];
                        list[64 * (i0 + i) + lane] = (uint16_t)(64 * (i0 + i) + lane | k[i] << 9);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < P; i++) v[i] = 0.f;
                }
                if (drop.state) {
#pragma unroll
                    for (int i = 0; i < P; i++) kept[64 * (i0 + i) + lane] = keep(2 * (i0 + i) + j0, cols);
                }
#pragma unroll
                for (int i = 0; i < P; i++) value[(2 * (i0 + i) + j0) * kPitch + c] = v[i];
            }
        } else {
            FS_WAVE_SYNC();
            for (int r = lane; r < n; r += 64) {
                const int code = list[r] & 511, c = code & 31, j = code >> 5;
                const int col = lds_cols[c];
                float v = 0.f;
                if (b.n_buckets > 0) {
                    const int k = bucket(j, col);
                    v = table[k];
                    list[r] = (uint16_t)(code | k << 9);
                }
                if (drop.state) kept[code] = keep(j, col);
                value[j * kPitch + c] = v;
            }
        }
        FS_WAVE_SYNC();
    }
    // of the lane's places, row j, vectors 8g .. 8g+7: whether they are kept, in bit 0 of a byte each
    __device__ __forceinline__ uint2 kept_bytes(int lane_) const
    {
        const int lane = fs_lane_here(lane_);
        return *reinterpret_cast<const uint2 *>(kept + 32 * (lane & (V - 1)) + 8 * (lane >> 4));
    }
    // and their biases
    __device__ __forceinline__ void values(float (&v)[8], int lane_) const
    {
        const int lane = fs_lane_here(lane_);
        const fs_f4 *from = reinterpret_cast<const fs_f4 *>(value + (lane & (V - 1)) * kPitch + 8 * (lane >> 4));
        const fs_f4 lo = from[0], hi = from[1];
#pragma unroll
        for (int x = 0; x < 4; x++) {
            v[x] = lo[x];
            v[4 + x] = hi[x];
        }
    }
    __device__ __forceinline__ void put_values(const float (&v)[8], int lane_)
    {
        const int lane = fs_lane_here(lane_);
        if ((lane & 15) >= V) return;
        fs_f4 *to = reinterpret_cast<fs_f4 *>(value + (lane & 15) * kPitch + 8 * (lane >> 4));
        to[0] = fs_f4{v[0], v[1], v[2], v[3]};
        to[1] = fs_f4{v[4], v[5], v[6], v[7]};
    }
};

// Place x of kept_bytes as 0 or ~0.
__device__ __forceinline__ uint32_t fs_kept_mask(const uint2 &bytes, int x) { return (uint32_t)__builtin_amdgcn_sbfe((int)(x < 4 ? bytes.x : bytes.y), 8 * (x & 3), 1); }

// Bit x of m as 0 or ~0, and a choice by it.
__device__ __forceinline__ uint32_t fs_bit_mask(uint32_t m, int x) { return (uint32_t)__builtin_amdgcn_sbfe((int)m, x, 1); }
__device__ __forceinline__ float fs_choose(uint32_t mask, float a, float b) { return __uint_as_float((mask & __float_as_uint(a)) | (~mask & __float_as_uint(b))); }

// 1 / v for a power of two.
__device__ __forceinline__ float fs_inverse_power(float v) { return __uint_as_float((254u << 23) - __float_as_uint(v)); }

template <int NT>
__device__ __forceinline__ void fs_clear(fs_f4 (&acc)[NT])
{
#pragma unroll
    for (int t = 0; t < NT; t++) acc[t] = fs_f4{0.f, 0.f, 0.f, 0.f};
}

template <int DT>
__device__ __forceinline__ fs_frag fs_round8(const float (&p)[8])
{
    fs_frag o;
    o.u = fs_u4{fs_pack2<DT>(p[0], p[1]), fs_pack2<DT>(p[2], p[3]), fs_pack2<DT>(p[4], p[5]), fs_pack2<DT>(p[6], p[7])};
    return o;
}
// What that rounding leaves, rounded as well: the two together hold p to twice the bits.
template <int DT>
__device__ __forceinline__ fs_frag fs_round8_rest(const float (&p)[8], const fs_frag &rounded)
{
    float rest[8];
#pragma unroll
    for (int x = 0; x < 8; x++) rest[x] = p[x] - fs_widen<DT>(rounded.e[x]);
    return fs_round8<DT>(rest);
}

// dS for the matrix cores.  fp16 holds it times a power of two `up` of the window row (the four lanes of a row have the same), and the row's
// accumulators are sums of as much: an entry of a row of thousands, or of a small gradient, would be 0 or one of few subnormal numbers otherwise, a
// large one an infinity, where their sums are numbers.  `up` brings the largest |dS| seen in the row to 2^11 .. 2^12 when it is set and lasts up to
// 2^15; then the accumulators change with it, as a softmax's do with its maximum.  So what an entry loses below the normal numbers is at most
// 2^-36 of the row's largest.  A row that has seen nothing but zeros has kUpUnset.  bf16 has fp32's exponents and is rounded as it is.
constexpr float kUpUnset = 0x1p120f;
template <int DT, int NT>
__device__ __forceinline__ fs_frag fs_round8_up(const float (&ds)[8], float &up, fs_f4 (&acc)[NT])
{
    if constexpr (DT == FS_BF16) return fs_round8<DT>(ds);
    float top = 0.f;
#pragma unroll
    for (int x = 0; x < 8; x++) top = fmaxf(top, fabsf(ds[x]));
    if (__builtin_amdgcn_ballot_w64(top * up > 0x1p15f)) {  // rare: a row's first block, and a few in which it grows
        top = fs_row_max(top);
        const float to = top * up > 0x1p15f ? __uint_as_float((265u - (__float_as_uint(top) >> 23)) << 23) : up;  // 2^11 over top's power of two
        const float by = to * fs_inverse_power(up);
#pragma unroll
        for (int t = 0; t < NT; t++) acc[t] = acc[t] * by;
        up = to;
    }
    float v[8];
#pragma unroll
    for (int x = 0; x < 8; x++) v[x] = ds[x] * up;
    return fs_round8<DT>(v);
}
// What takes `up` out of the accumulators.
template <int DT>
__device__ __forceinline__ float fs_down(float up) { return DT == FS_BF16 ? 1.f : fs_inverse_power(up); }
template <int DT, int NT>
__device__ __forceinline__ void fs_scale_down(fs_f4 (&acc)[NT], float up)
{
    if constexpr (DT == FS_BF16) return;
#pragma unroll
    for (int t = 0; t < NT; t++) acc[t] = acc[t] * fs_down<DT>(up);
}

// Accumulators -> rounded rows of an output of up to NC columns, by way of the tile's LDS.
template <int DT, int V, int NC>
__device__ __forceinline__ void fs_store_window(unsigned char *lds, const fs_f4 (&acc)[NC / 16], float factor, unsigned char *base, uint32_t pitch,
                                                int width, int w, int64_t rows, int lane_)
{
    using tile = fs_gathered<NC>;
    const int lane = fs_lane_here(lane_);
    FS_WAVE_SYNC();
    fs_round_tile_to_lds<DT, V, NC / 16, tile::RS>(lds, acc, lane & 15, lane >> 4, factor);
    FS_WAVE_SYNC();
    fs_store_tile_rows<V, tile::RPI, tile::RS>(lds + lds_row<tile::RS>(lane / tile::LPR) + (lane % tile::LPR) * 16, (uint16_t *)base, pitch / 2, w, rows,
                                               width, lane / tile::LPR, (lane % tile::LPR) * 8);
    FS_WAVE_SYNC();
}

// Accumulators -> partial tile `slot` of a head's tiles of `width` columns.
template <int V, int NT>
__device__ __forceinline__ void fs_store_part(float *tiles, int slot, int width, const fs_f4 (&acc)[NT], int lane_)
{
    const int lane = fs_lane_here(lane_);
    const int j = lane & 15, g = lane >> 4;
    fs_store_partial_tile<V, NT>(tiles, slot, width, (uint32_t)((g * V + j) * 16), acc, j < V, NT * 16 <= width, 0, g);
}

// Floats of the partial tiles of one kernel.
inline size_t fs_part_floats(const fs_format *f, int64_t heads, int64_t columns) { return (size_t)heads * (size_t)f->n_split_items * (size_t)f->V * (size_t)columns; }

}  // namespace
