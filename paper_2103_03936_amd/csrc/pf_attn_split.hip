// Attention forward of few queries over many keys (decoding): the keys of a sequence are split between workgroups and
// the parts joined.
//
// Bound by reading keys and values.  The query heads of one key head, and their few queries, are the columns of one
// product (row r of the group: query head r / Lq, query r % Lq), so that keys and values are read once for all of them.
// A wave takes 32 keys at a time: K goes from memory straight into the operand's registers, V through 32 rows of LDS that are the
// wave's own (its columns are needed transposed), and the next 32 keys are on their way while these are used; no wave waits
// for another before the end.  The waves' and then the workgroups' results are joined by their maxima and sums in a fixed order.
#include "pf_attn.h"

namespace pf {

// float rows are twice as long: two waves, not four, share the LDS of a workgroup
template <typename T>
constexpr int SPLIT_WAVES = sizeof(T) == 2 ? 4 : 2;

template <typename T, int DP>
struct SplitLds {
    static constexpr int NW = SPLIT_WAVES<T>, JOIN = DP * 33 * 4, TILES = 2 * NW * Tile<T, DP, 32, 64>::BYTES;
    static constexpr int AREA = JOIN > TILES ? JOIN : TILES;
};

template <typename T, int DP, bool BIAS>
__global__ __launch_bounds__(64 * SPLIT_WAVES<T>) void attn_split_kernel(AttnArgs a)
{
    constexpr int NW = SPLIT_WAVES<T>;
    using Tl = Tile<T, DP, 32, 64>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    float *const ml = (float *)(lds + SplitLds<T, DP>::AREA); // [2][NW][32]: the waves' maxima and sums
    uint8_t *const lut = (uint8_t *)(ml + 2 * NW * 32);       // bucket of each distance from -far to far
    const int t = threadIdx.x, wave = wave_of(t), lane = t & 63, col = lane & 31, h = lane >> 5;
    T *const vb = (T *)(lds + 2 * wave * Tl::BYTES); // two tiles of this wave's own

    const unsigned w = xcd_order(blockIdx.x, gridDim.x);
    const int split = w % a.splits, tile = w / a.splits % a.tiles, bk = w / a.splits / a.tiles, b = bk / a.Hkv, kv = bk - b * a.Hkv;
    const AttnLens n(a, b);
    const int r = tile * 32 + col, g = r / a.Lq, i = r - g * a.Lq, head = kv * a.G + g;
    const bool row = r < a.rows, ok = row && i < n.nq;
    const int pos = i + n.start, pmin = n.start, pmax = n.start + a.Lq - 1;
    int keys = n.nk;
    if (a.causal && pmax + 1 < keys) keys = pmax + 1 < 0 ? 0 : pmax + 1;
    const int all = (keys + 31) / 32, per = (all + a.splits - 1) / a.splits;
    const int first = split * per, end = first + per < all ? first + per : all; // groups of 32 keys

    const int far = a.bk.far;
    float flat_before = 0.f, flat_after = 0.f;
    if constexpr (BIAS) {
        for (int k = t; k <= 2 * far; k += 64 * NW) lut[k] = (uint8_t)bucket_of(a, k - far);
        if (row) {
            flat_before = bias_of(a, bucket_of(a, -far), head);
            flat_after = bias_of(a, bucket_of(a, far), head);
        }
        __syncthreads();
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

    const Tl vl(a.vs[1], a.D, lane);
    const int cols = Tl::col_place(lane);
    Frag<T> kr[DP / 16];
    const uint32_t kat = (uint32_t)(col * (int)a.ks[1]) * (uint32_t)sizeof(T);
    const auto fetch = [&](int k, int turn) {
        const int rows = n.nk - 32 * k < 32 ? n.nk - 32 * k : 32;
        const BufSrc src(Kp + (i64)(32 * k) * a.ks[1], ((rows - 1) * (int)a.ks[1] + a.D) * (int)sizeof(T));
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) kr[c] = row_frag_buffer(src, kat, 16 * c, a.D, h, (T *)nullptr);
        vl.fetch(vb + turn * Tl::SIZE, Vp + (i64)(32 * k) * a.vs[1], a.vs[1], n.nk - 32 * k, a.D, 0);
    };
    if (first + wave < end) fetch(first + wave, 0);
    for (int k = first + wave, turn = 0; k < end; k += NW, turn ^= 1) {
        const int k0 = 32 * k;
        f32x16_t acc = {};
        fetched(); // (K's registers, too)
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) mma(acc, kr[c], q[c]);
        if (k + NW < end) fetch(k + NW, turn ^ 1);
        const bool edge = k0 + 32 > n.nk || (a.causal && k0 + 31 > pmin);
        const bool near = BIAS && k0 + 31 - pmin > -far && k0 - pmax < far;
        const float flat = k0 >= pmin ? flat_after : flat_before;
        f32x16_t s;
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int j = k0 + 8 * (e >> 2) + 4 * h + (e & 3);
            float x = acc[e] * sl2;
            if constexpr (BIAS) {
                if (near)
                    x += row ? bias_of(a, lut[clamped(j - pos, -far, far) + far], head) : 0.f;
                else
                    x += flat;
            }
            if (edge && (j >= n.nk || (a.causal && j > pos))) x = -INFINITY;
            s[e] = x;
            top = fmaxf(top, x);
        }
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
            for (int d = 0; d < DP / 32; ++d) mma(o[d], Tl::by_cols(lds, cols + (2 * wave + turn) * Tl::BYTES, 16 * c, d), p);
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
        if (wave == k) {
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
    }
    if (wave == 0 && h == 0 && a.splits == 1 && a.lse && row)
        a.lse[((i64)b * a.Hq + head) * a.Lq + i] = ok && total > 0.f ? (top + __builtin_amdgcn_logf(total)) * LN2 : -INFINITY;
    if (a.splits == 1 && wave == 0 && h == 0) ml[col] = ok && total > 0.f ? 1.f / total : 0.f;
    __syncthreads();
    for (int x = t; x < 32 * DP; x += 64 * NW) {
        const int rr = x / DP, c = x % DP;
        if (tile * 32 + rr >= a.rows || c >= a.D) continue;
        if (a.splits > 1) {
            a.part_o[(piece * 32 + rr) * DP + c] = join[c * 33 + rr];
        } else {
            const int gg = (tile * 32 + rr) / a.Lq, ii = tile * 32 + rr - gg * a.Lq;
            const float inv = ml[rr];
            ((T *)a.O)[(((i64)b * a.Lq + ii) * a.Hq + kv * a.G + gg) * a.D + c] = from_float<T>(inv > 0.f ? join[c * 33 + rr] * inv : 0.f);
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
    float top = -INFINITY, total = 0.f;
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, ml[s * 64]);
    const float base = top == -INFINITY ? 0.f : top;
    float o[2] = {0.f, 0.f};
    for (int s = 0; s < a.splits; ++s) {
        const float f = exp2_fast(ml[s * 64] - base);
        total += ml[s * 64 + 1] * f;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int c = lane + 64 * k;
            if (c < a.D) o[k] += po[(i64)s * 32 * DP + c] * f;
        }
    }
    const AttnLens n(a, b);
    const bool some = i < n.nq && total > 0.f;
    T *const O = (T *)a.O + (((i64)b * a.Lq + i) * a.Hq + head) * a.D;
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (lane + 64 * k < a.D) O[lane + 64 * k] = from_float<T>(some ? o[k] / total : 0.f);
    if (a.lse && lane == 0) a.lse[((i64)b * a.Hq + head) * a.Lq + i] = some ? (top + __builtin_amdgcn_logf(total)) * LN2 : -INFINITY;
}

// ------------------------------------------------------------------ host
int attn_split_count(const pf_attention_desc *d)
{
    const i64 rows = d->Lq * (d->heads_q / d->heads_kv);
    if (rows > 32 || d->Lk == 0) return 0;
    const i64 base = d->B * d->heads_kv * ((rows + 31) / 32);
    // three workgroups to a compute unit, each with 256 keys or more
    i64 n = (768 + base - 1) / base, most = (d->Lk + 255) / 256;
    n = n < most ? n : most;
    return (int)(n < 1 ? 1 : n > 256 ? 256 : n);
}
static int padded(int D) { return (D + 31) / 32 * 32; }
size_t attn_split_bytes(const pf_attention_desc *d)
{
    const int n = attn_split_count(d);
    if (n <= 1) return 0;
    const i64 rows = d->Lq * (d->heads_q / d->heads_kv), pieces = d->B * d->heads_kv * ((rows + 31) / 32) * n;
    return align_up((size_t)pieces * 32 * 2 * sizeof(float)) + align_up((size_t)pieces * 32 * padded(d->head_dim) * sizeof(float));
}

template <typename T, int DP>
static int attn_split_launch(const AttnArgs &a, hipStream_t s)
{
    const unsigned blocks = (unsigned)a.B * a.Hkv * a.tiles * a.splits;
    const size_t lds = SplitLds<T, DP>::AREA + 2 * SPLIT_WAVES<T> * 32 * sizeof(float) + (a.buckets ? 2 * a.bk.far + 1 : 0);
    int st = PF_OK;
    if (a.buckets)
        PF_LAUNCH_LDS(st, "attn_split", (attn_split_kernel<T, DP, true>), dim3(blocks), dim3(64 * SPLIT_WAVES<T>), lds, s, a);
    else
        PF_LAUNCH_LDS(st, "attn_split", (attn_split_kernel<T, DP, false>), dim3(blocks), dim3(64 * SPLIT_WAVES<T>), lds, s, a);
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
    const int DP = padded(a.D);
    if (a.splits > 1) {
        const size_t pieces = (size_t)a.B * a.Hkv * a.tiles * a.splits;
        a.part_ml = (float *)workspace;
        a.part_o = (float *)((char *)workspace + align_up(pieces * 32 * 2 * sizeof(float)));
    }
    if (d->dtype == PF_BF16)
        return DP == 32 ? attn_split_launch<bf16_t, 32>(a, s) : DP == 64 ? attn_split_launch<bf16_t, 64>(a, s)
             : DP == 96 ? attn_split_launch<bf16_t, 96>(a, s) : attn_split_launch<bf16_t, 128>(a, s);
    return DP == 32 ? attn_split_launch<float, 32>(a, s) : DP == 64 ? attn_split_launch<float, 64>(a, s)
         : DP == 96 ? attn_split_launch<float, 96>(a, s) : attn_split_launch<float, 128>(a, s);
}

} // namespace pf
