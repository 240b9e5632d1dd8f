// Attention forward of few queries over many keys (decoding, a chunk of new tokens): the keys of a sequence are split between
// workgroups and the parts joined.
//
// Bound by reading keys and values.  The query heads of one key head, and their queries, are the rows r of one product (query
// head r / Lq, query r % Lq), 32 to a workgroup, so that keys and values are read once for all heads that share them.
// A wave takes 32 keys at a time, in tiles of LDS that are its own, and the next 32 are on their way while these are used; no wave
// waits for another before the end.  (K straight into the operand's registers meant loads of 32 bytes of 32 rows each, eight
// times over: a decoding step of 32 sequences of up to 4096 keys took 85 us, not 78; today 62 to 75, 4.7 TB/s; in float,
// where two waves to a compute unit are all that LDS holds, 289, and 131 with heads of 64.)  The waves' and then
// the workgroups' results are joined by their maxima and sums in a fixed order.
#include "pf_attn.h"

namespace pf {

constexpr int SPLIT_WAVES = 2;

template <typename T, int DP>
struct SplitLds {
    static constexpr int NW = SPLIT_WAVES, JOIN = DP * 33 * 4, TILES = 4 * NW * Tile<T, DP, 32, 64>::BYTES;
    static constexpr int AREA = JOIN > TILES ? JOIN : TILES;
};

// What a workgroup without keys writes: an empty part, or (the only part) rows of zeros
template <typename T>
__device__ __forceinline__ void leave_nothing(const AttnArgs &a, int bk, int tile, int split, int b, int kv, int t, int threads)
{
    if (a.splits > 1) {
        float *const ml = a.part_ml + (((i64)bk * a.tiles + tile) * a.splits + split) * 64;
        if (t < 64) ml[t] = t & 1 ? 0.f : -INFINITY;
        return;
    }
    for (int x = t; x < 32 * a.D; x += threads) {
        const int r = tile * 32 + x / a.D, c = x % a.D, g = r / a.Lq, i = r - g * a.Lq;
        if (r >= a.rows) break;
        ((T *)a.O)[(((i64)b * a.Lq + i) * a.Hq + kv * a.G + g) * a.D + c] = from_float<T>(0.f);
        if (c == 0 && a.lse) a.lse[((i64)b * a.Hq + kv * a.G + g) * a.Lq + i] = -INFINITY;
    }
}

template <typename T, int DP, bool BIAS>
__global__ __launch_bounds__(64 * SPLIT_WAVES, sizeof(T) * DP <= 256 ? 2 : 1) void attn_split_kernel(AttnArgs a)
{
    constexpr int NW = SPLIT_WAVES;
    using Tl = Tile<T, DP, 32, 64>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    float *const ml = (float *)(lds + SplitLds<T, DP>::AREA); // [2][NW][32]: the waves' maxima and sums
    float *const tab = ml + 2 * NW * 32;                      // [buckets][heads of the tile]: the bias (base 2)
    uint8_t *const lut = (uint8_t *)(tab + a.buckets * a.tile_heads); // bucket of each distance from -far to far
    const int t = threadIdx.x, wave = wave_of(t), lane = t & 63, col = lane & 31, h = lane >> 5;
    T *const own_tiles = (T *)(lds + 4 * wave * Tl::BYTES); // two of keys and two of values, this wave's own

    const unsigned w = xcd_order(blockIdx.x, gridDim.x);
    const int split = w % a.splits, tile = w / a.splits % a.tiles, bk = w / a.splits / a.tiles, b = bk / a.Hkv, kv = bk - b * a.Hkv;
    const AttnLens n(a, b);
    const int r = tile * 32 + col, g = r / a.Lq, i = r - g * a.Lq, head = kv * a.G + g;
    const bool row = r < a.rows, ok = row && i < n.nq;
    // the queries of the tile, from i0 to i1: all of them where it passes from one head to the next
    const int r1 = (tile * 32 + 32 < a.rows ? tile * 32 + 32 : a.rows) - 1, first_head = kv * a.G + tile * 32 / a.Lq;
    const bool one_head = tile * 32 / a.Lq == r1 / a.Lq;
    const int i0 = one_head ? tile * 32 % a.Lq : 0, i1 = one_head ? r1 % a.Lq : a.Lq - 1;
    const int pos = i + n.start, pmin = n.start + i0, pmax = n.start + i1;
    int keys = i0 < n.nq ? n.nk : 0;
    if (a.causal && pmax + 1 < keys) keys = pmax + 1 < 0 ? 0 : pmax + 1;
    const int all = (keys + 31) / 32, per = (all + a.splits - 1) / a.splits;
    const int first = split * per, end = first + per < all ? first + per : all; // groups of 32 keys

    const int far = a.bk.far;
    float flat_before = 0.f, flat_after = 0.f;
    if (first >= end) { // (no keys: nothing but an empty part to leave)
        leave_nothing<T>(a, bk, tile, split, b, kv, t, 64 * NW);
        return;
    }
    const T *const Kp = (const T *)a.K + b * a.ks[0] + kv * a.ks[2], *const Vp = (const T *)a.V + b * a.vs[0] + kv * a.vs[2];
    Frag<T> q[DP / 16];
    {
        const T *const Qp = (const T *)a.Q + b * a.qs[0] + (i64)head * a.qs[2] + i * a.qs[1];
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) q[c] = row_frag_global(Qp, 16 * c, a.D, h, ok);
    }
    const float sl2 = a.scale * LOG2E;
    f32x16_t o[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) o[d] = f32x16_t{};
    float m = -INFINITY, sum = 0.f;

    const Tl kl(a.ks[1], a.D, lane), vl(a.vs[1], a.D, lane);
    const int rows = Tl::row_place(lane) + 4 * wave * Tl::BYTES, cols = Tl::col_place(lane) + (4 * wave + 2) * Tl::BYTES;
    const auto fetch = [&](int k, int turn) {
        kl.fetch(own_tiles + turn * Tl::SIZE, Kp + (i64)(32 * k) * a.ks[1], a.ks[1], keys - 32 * k, a.D, 0);
        vl.fetch(own_tiles + (2 + turn) * Tl::SIZE, Vp + (i64)(32 * k) * a.vs[1], a.vs[1], keys - 32 * k, a.D, 0);
    };
    if (first + wave < end) fetch(first + wave, 0);
    __shared__ int large[NW];
    if constexpr (BIAS) {
        for (int k = t; k <= 2 * far; k += 64 * NW) lut[k] = (uint8_t)bucket_of(a, k - far);
        const int heads = a.tile_heads < (kv + 1) * a.G - first_head ? a.tile_heads : (kv + 1) * a.G - first_head;
        bool any = false;
        for (int k = t; k < a.buckets * a.tile_heads; k += 64 * NW) {
            const float x = k % a.tile_heads < heads ? bias_of(a, k / a.tile_heads, first_head + k % a.tile_heads) : 0.f;
            tab[k] = x;
            any |= is_large(x);
        }
        leave(large, any, wave, lane);
    }
    const float *const mine = tab + (row ? head - first_head : 0);
    float shift = 0.f; // what the row's biases, and its maximum, are relative to (in all parts the same: by all keys that it sees)
    if constexpr (BIAS) {
        __syncthreads();
        if (__builtin_expect(left(large, NW), 0))
            shift = row_shift(-pos, a.causal && n.nk > pos ? 0 : n.nk - 1 - pos, far, [&](int x) { return mine[lut[far + x] * a.tile_heads]; });
        flat_before = mine[bucket_before(a) * a.tile_heads] - shift;
        flat_after = mine[bucket_after(a) * a.tile_heads] - shift;
    }
    for (int k = first + wave, turn = 0; k < end; k += NW, turn ^= 1) {
        const int k0 = 32 * k;
        f32x16_t acc = {};
        fetched();
        if (k + NW < end) fetch(k + NW, turn ^ 1);
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) mma(acc, Tl::by_rows(lds, rows + turn * Tl::BYTES, 0, c), q[c]);
        const bool edge = k0 + 32 > n.nk || (a.causal && k0 + 31 > pmin);
        const bool near = BIAS && k0 + 31 - pmin > -far && k0 - pmax < far;
        const float flat = k0 >= pmin ? flat_after : flat_before;
        float top = -INFINITY;
        f32x16_t s = acc;
        if (near) {
            const int rel = k0 + 4 * h - pos;
            int u[16];
            float y[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) u[e] = lut[clamped(rel + 8 * (e >> 2) + (e & 3), -far, far) + far];
            __builtin_amdgcn_sched_barrier(0); // (all reads of a kind first)
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = mine[u[e] * a.tile_heads];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = s[e] * sl2 + (y[e] - shift);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = s[e] * sl2 + (BIAS ? flat : 0.f);
        }
        if (edge) {
            const int rel = k0 + 4 * h - pos, most = a.causal && n.nk > pos ? 0 : n.nk - 1 - pos; // distances; the furthest seen
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = fminf(s[e], rel + 8 * (e >> 2) + (e & 3) > most ? -INFINITY : INFINITY);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[e]);
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m, top), base = m_new == -INFINITY ? 0.f : m_new;
        if (__any(m_new > m)) {
            const float f = exp2_fast(m - base);
            sum *= f;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[d][e] *= f;
            m = m_new;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = exp2_fast(s[e] - base);
            sum += s[e];
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            Frag<T> p;
            pack(s, c, p);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) mma(o[d], Tl::by_cols(lds, cols + turn * Tl::BYTES, 16 * c, d), p);
        }
    }
    sum += __shfl_xor(sum, 32);
    if (h == 0) {
        ml[wave * 32 + col] = m;
        ml[(NW + wave) * 32 + col] = sum;
    }
    __syncthreads(); // (all waves are done with their tiles, too)
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int k = 0; k < NW; ++k) top = fmaxf(top, ml[k * 32 + col]);
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int k = 0; k < NW; ++k) total += ml[(NW + k) * 32 + col] * exp2_fast(ml[k * 32 + col] - base);
    const float f = exp2_fast(m - base);
    float *const join = (float *)lds; // [DP][33]
    for (int k = 0; k < NW; ++k) {
        if (wave == k && row) {
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float *const p = join + (32 * d + 8 * (e >> 2) + 4 * h + (e & 3)) * 33 + col;
                    *p = k ? *p + o[d][e] * f : o[d][e] * f;
                }
        }
        __syncthreads();
    }
    // the rows, one after the other: adjacent lanes have adjacent columns of one row
    const i64 piece = ((i64)bk * a.tiles + tile) * a.splits + split;
    if (wave == 0 && h == 0 && a.splits > 1) {
        a.part_ml[(piece * 32 + col) * 2] = top;
        a.part_ml[(piece * 32 + col) * 2 + 1] = total;
        if (split == 0) a.part_shift[((i64)bk * a.tiles + tile) * 32 + col] = shift; // (if any part has keys, this one has)
    }
    if (wave == 0 && h == 0 && a.splits == 1 && a.lse && row)
        a.lse[((i64)b * a.Hq + head) * a.Lq + i] = ok && total != 0.f ? (top + __builtin_amdgcn_logf(total)) * LN2 + shift * LN2 : -INFINITY;
    if (a.splits == 1 && wave == 0 && h == 0) ml[col] = ok && total != 0.f ? 1.f / total : 0.f;
    __syncthreads();
    for (int x = t; x < (r1 - tile * 32 + 1) * DP; x += 64 * NW) {
        const int rr = x / DP, c = x % DP;
        if (c >= a.D) continue;
        if (a.splits > 1) {
            a.part_o[(piece * 32 + rr) * DP + c] = join[c * 33 + rr];
        } else {
            const int gg = (tile * 32 + rr) / a.Lq, ii = tile * 32 + rr - gg * a.Lq;
            const float inv = ml[rr];
            ((T *)a.O)[(((i64)b * a.Lq + ii) * a.Hq + kv * a.G + gg) * a.D + c] = from_float<T>(inv != 0.f ? join[c * 33 + rr] * inv : 0.f);
        }
    }
}

// The parts of one row, joined: one wave to a row
template <typename T>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, int DP)
{
    const int lane = threadIdx.x & 63;
    const i64 all = (i64)blockIdx.x * 4 + (threadIdx.x >> 6); // (b, kv) a.rows + r
    if (all >= (i64)a.B * a.Hkv * a.rows) return;
    const int bk = (int)(all / a.rows), r = (int)(all - (i64)bk * a.rows), b = bk / a.Hkv, kv = bk - b * a.Hkv;
    const int g = r / a.Lq, i = r - g * a.Lq, head = kv * a.G + g;
    const i64 piece = ((i64)bk * a.tiles + r / 32) * a.splits;
    const float *const ml = a.part_ml + (piece * 32 + r % 32) * 2, *const po = a.part_o + (piece * 32 + r % 32) * DP;
    // lane s: part s (and s + 64 ..)
    float top = -INFINITY, total = 0.f;
    for (int s = lane; s < a.splits; s += 64) top = fmaxf(top, ml[s * 64]);
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float base = top == -INFINITY ? 0.f : top;
    float o[2] = {0.f, 0.f};
    const int c0 = lane < a.D ? lane : 0, c1 = lane + 64 < a.D ? lane + 64 : 0;
    for (int s0 = 0; s0 < a.splits; s0 += 8) { // eight parts on their way at a time, added in their order
        float f[8], y[8], z[8], w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int s = s0 + k < a.splits ? s0 + k : a.splits - 1;
            f[k] = ml[s * 64], w[k] = ml[s * 64 + 1];
            y[k] = po[(i64)s * 32 * DP + c0], z[k] = po[(i64)s * 32 * DP + c1];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            // A part without a key that the row sees has left no values, only the sum 0.  (Not told by its maximum: that of
            // scores that are all NaN is -infinity, too, and their sum is NaN.)
            if (s0 + k < a.splits && w[k] != 0.f) {
                const float g = exp2_fast(f[k] - base);
                total += w[k] * g;
                o[0] += y[k] * g;
                o[1] += z[k] * g;
            }
        }
    }
    const AttnLens n(a, b);
    const bool some = i < n.nq && total != 0.f;
    T *const O = (T *)a.O + (((i64)b * a.Lq + i) * a.Hq + head) * a.D;
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (lane + 64 * k < a.D) O[lane + 64 * k] = from_float<T>(some ? o[k] / total : 0.f);
    if (a.lse && lane == 0) a.lse[((i64)b * a.Hq + head) * a.Lq + i] = some ? (top + __builtin_amdgcn_logf(total)) * LN2 + a.part_shift[piece / a.splits * 32 + r % 32] * LN2 : -INFINITY;
}

// ------------------------------------------------------------------ host
static i64 row_tiles(const pf_attention_desc *d) { return (d->Lq * (d->heads_q / d->heads_kv) + 31) / 32; }
static int padded(int D) { return (D + 31) / 32 * 32; }
// The most heads that 32 rows touch, of G heads with Lq rows each
static int heads_of_tile(i64 Lq, int G) { return (int)(G < 31 / Lq + 2 ? G : 31 / Lq + 2); }
// LDS of a workgroup: tiles, the waves' maxima and sums, the bias of the tile's heads by bucket and the bucket of each distance
static size_t split_lds(size_t area, int buckets, int heads, int far)
{
    return area + 2 * SPLIT_WAVES * 32 * sizeof(float) + (buckets ? (size_t)buckets * heads * sizeof(float) + 2 * far + 1 : 0);
}
// Float rows of more than 64 values fill 128 KB with tiles: 256 buckets of 32 heads do not fit beside them.  The ordinary kernel has
// one head's bias in LDS and takes any.
static bool split_fits(const pf_attention_desc *d)
{
    const int DP = padded(d->head_dim), heads = heads_of_tile(d->Lq, d->heads_q / d->heads_kv);
    const bool bf16 = d->dtype == PF_BF16;
    const size_t area = DP == 32 ? (bf16 ? SplitLds<bf16_t, 32>::AREA : SplitLds<float, 32>::AREA)
                      : DP == 64 ? (bf16 ? SplitLds<bf16_t, 64>::AREA : SplitLds<float, 64>::AREA)
                      : DP == 96 ? (bf16 ? SplitLds<bf16_t, 96>::AREA : SplitLds<float, 96>::AREA)
                                 : (bf16 ? SplitLds<bf16_t, 128>::AREA : SplitLds<float, 128>::AREA);
    // (no border lies behind max_distance; 16 bytes of the kernel's own)
    return split_lds(area, d->buckets, heads, d->max_distance) + 16 <= 160 * 1024;
}
int attn_split_count(const pf_attention_desc *d)
{
    if (d->Lk == 0 || !split_fits(d)) return 0;
    if (d->Lq * (d->heads_q / d->heads_kv) > 32) {
        // More rows than one product takes: where the ordinary kernel has few tiles of 128 queries and many keys for each.  us, 128
        // queries, bf16, heads of 128: 4 tiles of 8192 keys 98 ordinary and 22 split, 32 of 8192 100 and 63, 64 of 8192 103 and 102, 16 of
        // 2048 31 and 23, 32 of 2048 32 and 36, 8 of 1024 20 and 17, 8 of 512 14 and 17; float, heads of 64: 8 of 600 33 and 23, 16 of
        // 600 33 and 24, 32 of 600 33 and 31, 32 of 2048 86 and 57, 64 of 2048 87 and 93, 32 of 8192 321 and 161; of 128: 16 of 600 59 and 37, 32 of 600
        // 59 and 65, 32 of 2048 163 and 124, 64 of 2048 164 and 204, 32 of 8192 618 and 356.
        const i64 tiles = d->B * d->heads_q * ((d->Lq + 127) / 128);
        if (tiles > 64 || tiles * (d->dtype == PF_BF16 ? 128 : 32) > d->Lk) return 0;
    }
    const i64 base = d->B * d->heads_kv * row_tiles(d);
    // pieces of 256 keys or more; sequences differ in length, so that there are more pieces (1024) than places for them
    // (512: 32 sequences of up to 4096 keys took 78 us with 512 pieces, 76 with 1024, 82 with 2048)
    i64 n = (1024 + base - 1) / base, most = (d->Lk + 255) / 256;
    n = n < most ? n : most;
    return (int)(n < 1 ? 1 : n > 256 ? 256 : n);
}
size_t attn_split_bytes(const pf_attention_desc *d)
{
    const int n = attn_split_count(d);
    if (n <= 1) return 0;
    const i64 pieces = d->B * d->heads_kv * row_tiles(d) * n;
    return align_up((size_t)pieces * 32 * 2 * sizeof(float)) + align_up((size_t)pieces * 32 * padded(d->head_dim) * sizeof(float)) +
           align_up((size_t)pieces / n * 32 * sizeof(float));
}

template <typename T, int DP>
static int attn_split_launch(const AttnArgs &a, hipStream_t s)
{
    const unsigned blocks = (unsigned)a.B * a.Hkv * a.tiles * a.splits;
    if (too_many(blocks, 64 * SPLIT_WAVES)) return PF_ERR_UNSUPPORTED;
    const size_t lds = split_lds(SplitLds<T, DP>::AREA, a.buckets, a.tile_heads, a.bk.far);
    int st = PF_OK;
    if (a.buckets)
        PF_LAUNCH_LDS(st, "attn_split", (attn_split_kernel<T, DP, true>), dim3(blocks), dim3(64 * SPLIT_WAVES), lds, s, a);
    else
        PF_LAUNCH_LDS(st, "attn_split", (attn_split_kernel<T, DP, false>), dim3(blocks), dim3(64 * SPLIT_WAVES), lds, s, a);
    if (a.splits > 1) {
        const i64 rows = (i64)a.B * a.Hkv * a.rows;
        PF_LAUNCH(st, "attn_join", attn_join_kernel<T>, dim3((unsigned)((rows + 3) / 4)), dim3(256), s, a, DP);
    }
    return st;
}

int attn_split_fwd(const pf_attention_desc *d, AttnArgs &a, void *workspace, hipStream_t s)
{
    a.splits = attn_split_count(d);
    a.rows = a.Lq * a.G;
    a.tiles = (a.rows + 31) / 32;
    a.tile_heads = heads_of_tile(a.Lq, a.G);
    const int DP = padded(a.D);
    if (a.splits > 1) {
        const size_t pieces = (size_t)a.B * a.Hkv * a.tiles * a.splits;
        a.part_ml = (float *)workspace;
        a.part_o = (float *)((char *)workspace + align_up(pieces * 32 * 2 * sizeof(float)));
        a.part_shift = (float *)((char *)a.part_o + align_up(pieces * 32 * DP * sizeof(float)));
    }
    if (d->dtype == PF_BF16)
        return DP == 32 ? attn_split_launch<bf16_t, 32>(a, s) : DP == 64 ? attn_split_launch<bf16_t, 64>(a, s)
             : DP == 96 ? attn_split_launch<bf16_t, 96>(a, s) : attn_split_launch<bf16_t, 128>(a, s);
    return DP == 32 ? attn_split_launch<float, 32>(a, s) : DP == 64 ? attn_split_launch<float, 64>(a, s)
         : DP == 96 ? attn_split_launch<float, 96>(a, s) : attn_split_launch<float, 128>(a, s);
}

} // namespace pf
