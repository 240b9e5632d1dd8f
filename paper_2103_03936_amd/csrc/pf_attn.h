// What the attention kernels share: arguments, matrix operands, tiles in LDS, the bias by distance.
//
// Orientation.  A product of 32 x 32 leaves lane l with column l % 32 and the rows 8 (i / 4) + 4 (l / 32) + i % 4,
// i = 0 .. 15, of the result.  Forward and for dQ the scores are formed transposed (rows: keys, columns: queries), so that
// a lane has one query: its maximum, sum, position and masks are scalars of the lane, and a row statistic needs one exchange
// between the two halves of the wave.  What a lane holds of P is then, without any exchange, the right operand of the next
// product, O^T = V^T P^T, if that product takes its contraction index in the same order, 16 keys at a time:
// {4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3} in the half h.  The left operand, V^T, is read from LDS in that order (for bf16
// with the transposing reads).  For dK and dV the scores are formed with rows: queries, columns: keys, and the same holds.
#pragma once

#include "pf_attn_bias.h"
#include "pf_overlap.h"
#include "pf_tile.h"

namespace pf {

struct AttnArgs {
    const void *Q, *K, *V, *dO, *Oin;
    void *O, *dQ, *dK, *dV;
    const float *table, *lse_in;
    float *lse, *stat, *tab; // stat[B, Hq][records]: what dK and dV need of each 32 queries (StatRecord); tab[Hq][B * tiles][buckets]: sums of dS per workgroup
    int records;
    const int *q_start, *q_len, *kv_len;
    int B, Lq, Lk, Hq, Hkv, G, D, causal, buckets, two_sided, tiles;
    float scale;
    i64 qs[3], ks[3], vs[3]; // strides: sequence, token, head
    // few queries: the split of the keys and where its parts go (partial O, maxima and sums), what the rows' biases are relative to
    int splits, rows, tile_heads;
    float *part_o, *part_ml, *part_shift;
    AttnBuckets bk;
};

// Of 32 queries: P = exp2((S - shift) - rest), S with its bias (base 2); shift is infinity where a query takes no part
struct StatRecord {
    float before[32], after[32]; // the bias of a key far before, far after the query, less shift and rest
    float neg_delta[32], shift[32], neg_rest[32];
    float with_rest[32]; // [0]: whether a rest is not zero
};

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// ------------------------------------------------------------------ matrix operands
template <typename T>
struct Frag;
template <>
struct Frag<bf16_t> {
    bf16x8_t v;
};
template <>
struct Frag<float> {
    float v[8];
};

__device__ __forceinline__ void mma(f32x16_t &c, const Frag<bf16_t> &a, const Frag<bf16_t> &b)
{
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x16_t &c, const Frag<float> &a, const Frag<float> &b)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], c, 0, 0, 0);
}

// Operand with the index along the rows and the contraction along 16 columns from `col` on, `row` the lane's row in global
// memory; h = lane / 32.  (The halves share the 16 columns in an order of their own, the same for both operands.)  Zeros where the row does not exist (ok) or has no such column (head_dim is a multiple of 8)
__device__ __forceinline__ Frag<bf16_t> row_frag_global(const bf16_t *row, int col, int D, int h, bool ok)
{
    Frag<bf16_t> f;
    f.v = bf16x8_t{};
    if (ok && col + 8 * h < D) f.v = *(const bf16x8_t *)(row + col + 8 * h);
    return f;
}
__device__ __forceinline__ Frag<float> row_frag_global(const float *row, int col, int D, int h, bool ok)
{
    Frag<float> f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
    if (ok && col + 4 * h < D) a = *(const float4 *)(row + col + 4 * h);
    if (ok && col + 8 + 4 * h < D) b = *(const float4 *)(row + col + 8 + 4 * h);
    f.v[0] = a.x, f.v[1] = a.y, f.v[2] = a.z, f.v[3] = a.w, f.v[4] = b.x, f.v[5] = b.y, f.v[6] = b.z, f.v[7] = b.w;
    return f;
}

// Eight values of a result (its registers 8 c .. 8 c + 7) as the operand for rows 16 c .. 16 c + 15; bf16: rounded to
// nearest even, the one rounding of P and dS, half a step of 2^-8 each
__device__ __forceinline__ void pack(const f32x16_t &x, int c, Frag<bf16_t> &f)
{
    union {
        uint32_t u[4];
        bf16x8_t v;
    } w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w.u[i] = pack_bf16x2(x[8 * c + 2 * i], x[8 * c + 2 * i + 1]);
    f.v = w.v;
}
__device__ __forceinline__ void pack(const f32x16_t &x, int c, Frag<float> &f)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) f.v[i] = x[8 * c + i];
}

// A value that is taken to change here (what follows from it is not kept in registers over a loop)
__device__ __forceinline__ int anew(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}
__device__ __forceinline__ float anew(float x)
{
    asm volatile("" : "+v"(x));
    return x;
}
// Values that are worked out here, whatever branch uses them later (the compiler would put them off to behind the branch)
__device__ __forceinline__ void here(Frag<bf16_t> &f)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    u32x4 w = __builtin_bit_cast(u32x4, f.v);
    asm volatile("" : "+v"(w));
    f.v = __builtin_bit_cast(bf16x8_t, w);
}
__device__ __forceinline__ void here(Frag<float> &f)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(f.v[e]));
}

// Four adjacent values
__device__ __forceinline__ void put4(float *p, float a, float b, float c, float d) { *(float4 *)p = make_float4(a, b, c, d); }
__device__ __forceinline__ void put4(bf16_t *p, float a, float b, float c, float d)
{
    *(uint2 *)p = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
}

// ------------------------------------------------------------------ tiles
// The transposing read.  __restrict__: nothing writes there meanwhile; without it every such read waits for all fetches into
// LDS that are on their way (so does a read of a struct such as float4, which is why the tiles and tables here are read as
// vectors of the language)
typedef __attribute__((address_space(3))) bf16x4_t LdsBf16x4;
__device__ inline bf16x4_t read_turned(const LdsBf16x4 *__restrict__ p) { return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsBf16x4 *)p); }

// ROWS rows of DP columns in LDS, fetched by THREADS threads straight into it (no registers; a wave's fetches end with
// fetched()).  A fetch puts the lanes' 16-byte pieces one after the other, so there is no padding: piece c of row r lies at
// c ^ turn(r).  The tile is read in two ways, as an operand by rows (bf16: 16 lanes that a cycle serves have one piece of 16
// rows) and by columns (the transposing reads: 32 lanes that a cycle serves have four adjacent pieces of four rows; float:
// 32 adjacent values of two rows, four apart), and turn() lets each way meet each of the 64 banks once (float of 32
// columns: twice).
constexpr int ATTN_MAX_STRIDE = 1 << 22; // elements from one token to the next
template <typename T, int DP, int ROWS, int THREADS>
struct Tile {
    static_assert((int64_t)ROWS * ATTN_MAX_STRIDE * sizeof(T) <= 1 << 30, "offsets of 31 bits, what is skipped included"); // 128 rows of bf16, 64 of float
    static constexpr int VEC = 16 / sizeof(T), PITCH = DP == 96 ? 128 : DP, CHUNKS = PITCH / VEC, PIECES = ROWS * CHUNKS, N = (PIECES + THREADS - 1) / THREADS;
    static constexpr int BYTES = PIECES * 16, SIZE = ROWS * PITCH;
    static_assert(PIECES % 64 == 0, "whole waves of pieces");
    uint32_t at[N]; // bytes from the tile's first row to the thread's pieces
    static __device__ __forceinline__ int turn(int row)
    {
        if constexpr (sizeof(T) == 2) {
            if constexpr (CHUNKS == 16) return (row & 3) << 2 | (row >> 2 & 3);
            if constexpr (CHUNKS == 8) return (row >> 1 & 1) << 2 | (row >> 2 & 3);
            return row >> 2 & 3;
        }
        if constexpr (CHUNKS == 8) return row >> 1 & 7;
        return (row >> 2 & 1) << 3 | (row >> 3 & 1) << 2 | (row & 3);
    }
    // elements `stride` from one row to the next, D columns (the others are zeros)
    __device__ __forceinline__ Tile(i64 stride, int D, int t)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = t + i * THREADS, row = p / CHUNKS, col = ((p % CHUNKS) ^ turn(row)) * VEC;
            at[i] = col < D ? (uint32_t)(row * (int)stride + col) * (uint32_t)sizeof(T) : BUF_OUT;
        }
    }
    // ROWS rows from `first` on (the same for all threads), zeros from row `rows` on: the descriptor ends with the last row.
    // wave: the thread's wave among those of THREADS.  The first `skip` rows are zeros: the descriptor begins behind them.
    __device__ __forceinline__ void fetch(T *lds, const T *first, i64 stride, int rows, int D, int wave, int skip = 0) const
    {
        typedef __attribute__((address_space(3))) void *lds_ptr;
        const int n = rows < ROWS ? rows : ROWS;
        const BufSrc src(first + skip * stride, n > skip ? ((n - 1 - skip) * (int)stride + D) * (int)sizeof(T) : 0);
        const uint32_t gone = skip * (uint32_t)stride * (uint32_t)sizeof(T); // (what is out of range stays so: both are below 2^30)
        const auto offset = [&](uint32_t x) { return x < gone ? BUF_OUT : x - gone; };
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (PIECES % THREADS == 0 || i * THREADS + wave * 64 < PIECES)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(src.r, (lds_ptr)((char *)lds + (i * THREADS + wave * 64) * 16), 16, (int)offset(at[i]), 0, 0, 0);
    }
    // Where a lane reads, in bytes from the tile's start.  turn() permutes bits, so that a step along a row is an exclusive or of
    // the place (tiles lie at multiples of their rows' lengths): one number for a lane and constants, not an address for every read.
    static constexpr int RB = PITCH * (int)sizeof(T); // bytes from one row to the next
    static __device__ __forceinline__ int row_place(int lane)
    {
        const int row = lane & 31;
        return row * RB + ((lane >> 5) ^ turn(row)) * 16;
    }
    static __device__ __forceinline__ int col_place(int lane)
    {
        if constexpr (sizeof(T) == 2) {
            const int g = lane >> 4, i = lane & 15, row = 4 * (g >> 1) + (i >> 2);
            return row * RB + ((2 * (g & 1) + (i >> 1 & 1)) ^ turn(row)) * 16 + 8 * (i & 1);
        }
        const int row = 4 * (lane >> 5);
        return row * RB + ((lane >> 2 & 7) ^ turn(row)) * 16 + 4 * (lane & 3);
    }
    // Operand with the index along the 32 rows from r0 on and the contraction along columns 16 c ..; at: row_place plus the
    // bytes from `lds` to the tile
    static __device__ __forceinline__ Frag<T> by_rows(const char *lds, int at, int r0, int c)
    {
        Frag<T> f;
        const char *const p = lds + r0 * RB;
        if constexpr (sizeof(T) == 2) {
            f.v = *(const bf16x8_t *)(p + (at ^ (32 * c)));
        } else {
            const f32x4_t x = *(const f32x4_t *)(p + (at ^ (64 * c))), y = *(const f32x4_t *)(p + (at ^ (64 * c + 32)));
#pragma unroll
            for (int e = 0; e < 4; ++e) f.v[e] = x[e], f.v[4 + e] = y[e];
        }
        return f;
    }
    // Operand with the index along the columns 32 d .. 32 d + 31 and the contraction along rows r0 .. r0 + 15 (r0 a multiple
    // of 16), in the order in which a product's result lies in the lanes; at: col_place plus the bytes to the tile
    static __device__ __forceinline__ Frag<T> by_cols(const char *lds, int at, int r0, int d)
    {
        Frag<T> f;
        const char *const p = lds + r0 * RB;
        if constexpr (sizeof(T) == 2) {
            const bf16x4_t x = read_turned((const LdsBf16x4 *)(p + (at ^ (64 * d)))),
                           y = read_turned((const LdsBf16x4 *)(p + 8 * RB + (at ^ (64 * d + 16 * turn(8)))));
#pragma unroll
            for (int e = 0; e < 4; ++e) f.v[e] = x[e], f.v[4 + e] = y[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int row = (e & 3) + 8 * (e >> 2);
                f.v[e] = *(const float *)(p + row * RB + (at ^ (128 * d + 16 * turn(row))));
            }
        }
        return f;
    }
};
// This wave's fetches have arrived (a barrier after it tells the others)
__device__ __forceinline__ void fetched() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// ------------------------------------------------------------------ lengths and positions
__device__ __forceinline__ int clamped(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
struct AttnLens {
    int nq, nk, start;
    __device__ __forceinline__ AttnLens(const AttnArgs &a, int b)
    {
        nq = a.q_len ? clamped(a.q_len[b], 0, a.Lq) : a.Lq;
        nk = a.kv_len ? clamped(a.kv_len[b], 0, a.Lk) : a.Lk;
        start = a.q_start ? clamped(a.q_start[b], -(1 << 30), 1 << 30) : 0;
    }
};

// Bucket of the distance key - query, within +-far.  Sixteen borders at a time: a loop over single ones waits for each.
__device__ __forceinline__ int bucket_of(const AttnArgs &a, int dist)
{
    const int n = dist < 0 ? -dist : dist;
    int u = 0;
    for (int k = 0; k < a.bk.borders; k += 16) {
#pragma unroll
        for (int i = 0; i < 16; ++i) u += n >= a.bk.border[k + i];
    }
    u = n < a.bk.exact ? n : a.bk.exact + u;
    return dist <= 0 ? u : a.two_sided ? u + a.bk.side : 0;
}
// of the distances -far and far
__device__ __forceinline__ int bucket_before(const AttnArgs &a) { return a.bk.side - 1; }
__device__ __forceinline__ int bucket_after(const AttnArgs &a) { return a.two_sided ? 2 * a.bk.side - 1 : 0; }

// The bias of query head `head` in a bucket, times log2(e); finite values stay finite (a table may hold the type's lowest)
__device__ __forceinline__ float bias_of(const AttnArgs &a, int bucket, int head)
{
    const float x = a.table[(i64)bucket * a.Hq + head], y = x * LOG2E;
    return __builtin_isinf(y) && !__builtin_isinf(x) ? __builtin_copysignf(3.4028234e38f, x) : y;
}
// A bias (base 2) from here on takes so many digits that what is added to it loses more than float's sums do.  Softmax does not
// change with what a whole row shares: where the largest bias that a row sees is such a one, all of the row's are taken relative to it.
constexpr float ATTN_LARGE = 1024.f;
__device__ __forceinline__ bool is_large(float x) { return fabsf(x) >= ATTN_LARGE && !__builtin_isinf(x); }
// bias[far + d], d = -far .. far: the head's bias at distance d (further ones have that of +-far), times log2(e).  Whether the
// thread met a large one.
__device__ __forceinline__ bool fill_bias(const AttnArgs &a, float *bias, int head, int t, int threads)
{
    bool large = false;
    for (int i = t; i <= 2 * a.bk.far; i += threads) {
        const float x = bias_of(a, bucket_of(a, i - a.bk.far), head);
        bias[i] = x;
        large |= is_large(x);
    }
    return large;
}
// Whether any thread of four waves has x: each wave leaves its answer before a barrier, all read them behind it
__device__ __forceinline__ void leave(int *flags, bool x, int wave, int lane)
{
    const int any = __any(x);
    if (lane == 0) flags[wave] = any;
}
__device__ __forceinline__ bool left(const int *flags, int waves)
{
    int any = 0;
    for (int k = 0; k < waves; ++k) any |= flags[k];
    return __builtin_amdgcn_readfirstlane(any) != 0;
}
// What the biases of a row that sees the distances lo .. hi are taken relative to; at(d) is the row's bias at distance d
template <class F>
__device__ __forceinline__ float row_shift(int lo, int hi, int far, F at)
{
    float top = -INFINITY;
    if (lo <= hi)
        for (int d = clamped(lo, -far, far); d <= clamped(hi, -far, far); ++d) top = fmaxf(top, at(d));
    return is_large(top) ? top : 0.f;
}

// Scores of a block at an edge or near the diagonal: s scale + (bias (base 2) - less); register e holds the distance
// rel + step (8 (e / 4) + e % 4), what is further than `most` is not seen.  less(e): of its row
template <bool BIAS, class F>
__device__ __forceinline__ void finish_scores_by(f32x16_t &s, float scale, F less, const float *bias, int far, int rel, int step, int most)
{
    float y[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = BIAS ? bias[clamped(rel + step * (8 * (e >> 2) + (e & 3)), -far, far) + far] : 0.f;
    __builtin_amdgcn_sched_barrier(0); // (all reads first)
#pragma unroll
    for (int e = 0; e < 16; ++e)
        s[e] = fminf(s[e] * scale + (y[e] - less(e)), rel + step * (8 * (e >> 2) + (e & 3)) > most ? -INFINITY : INFINITY);
}
// the lane has one query
template <bool BIAS>
__device__ __forceinline__ void finish_scores(f32x16_t &s, float scale, float less, const float *bias, int far, int rel, int step, int most)
{
    finish_scores_by<BIAS>(s, scale, [&](int) { return less; }, bias, far, rel, step, most);
}
// register e has the query 8 (e / 4) + e % 4 of those whose values lie at `less`, in LDS
template <bool BIAS>
__device__ __forceinline__ void finish_scores(f32x16_t &s, float scale, const float *less, const float *bias, int far, int rel, int step, int most)
{
    f32x4_t x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = *(const f32x4_t *)(less + 8 * e);
    finish_scores_by<BIAS>(s, scale, [&](int e) { return x[e / 4][e % 4]; }, bias, far, rel, step, most);
}

// XCDs take workgroups in turn: consecutive pieces of work (the tiles of a head, which share keys and values) go to one XCD
// and its L2.  A bijection for any number of workgroups.
__device__ __forceinline__ unsigned xcd_order(unsigned id, unsigned n)
{
    const unsigned x = id & 7, per = n >> 3, more = n & 7;
    return x * per + (x < more ? x : more) + (id >> 3);
}

// The wave's number, known to be one for all its lanes (what is decided by it is a branch, not a mask)
__device__ __forceinline__ int wave_of(int t) { return __builtin_amdgcn_readfirstlane(t >> 6); }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); } // (one instruction, 1 ulp)

// ------------------------------------------------------------------ host
int attn_split_fwd(const pf_attention_desc *d, AttnArgs &a, void *workspace, hipStream_t s); // few queries (pf_attn_split.hip)
int attn_split_count(const pf_attention_desc *d); // 0: the ordinary kernel
size_t attn_split_bytes(const pf_attention_desc *d);
int attn_check(const pf_attention_desc *d);
// A launch of 2^32 threads or more does not exist
inline bool too_many(i64 blocks, int threads) { return blocks * threads >= (i64)1 << 32; }
void attn_fill(const pf_attention_desc *d, AttnArgs &a);
// What the tensors of a call take in memory
struct AttnAreas {
    const pf_attention_desc *d;
    const AttnArgs &a;
    int64_t elem() const { return d->dtype == PF_BF16 ? 2 : 4; }
    Area queries(const void *p) const { return Area(p, d->B, a.Lq, a.Hq, a.qs, a.D, elem()); }
    Area keys(const void *p, const i64 (&s)[3]) const { return Area(p, d->B, a.Lk, a.Hkv, s, a.D, elem()); }
    Area dense_queries(const void *p) const { return Area(p, d->B * d->Lq * a.Hq * a.D * elem()); }
    Area dense_keys(const void *p) const { return Area(p, d->B * d->Lk * a.Hkv * a.D * elem()); }
    Area rows(const void *p) const { return Area(p, d->B * d->Lq * a.Hq * 4); }
    Area table(const void *p) const { return Area(a.buckets ? p : nullptr, (int64_t)a.buckets * a.Hq * 4); }
};

} // namespace pf
