// Norms of queries and keys per head with the position rotation: pf_qk_norm_rotate_*.
//
// Bound by memory: forward reads and writes each value once, backward reads two and writes one.  A wave takes one token at a
// time, all its heads: a lane holds W pairs of a head (the two values that a rotation mixes are always in one lane), the
// head_dim / (2 W) lanes of a head add up its squares between them, and 64 / lanes heads are worked on while the next are on
// their way.  The angles belong to the token alone: the wave forms each one once, in double, and its heads read cosine and sine
// from LDS.  2 x 8191 tokens of 40 heads of 128 in bf16: forward 60 us, backward 113 (5.6 and 4.5 TB/s of what they read and
// write; some of it is still in the caches); without the loads ahead 68 and 117.
#include <math.h>
#include <string.h>

#include "pf_gemm.h"
#include "pf_overlap.h"

namespace pf {

struct QkArgs {
    const void *Q, *K, *dQo, *dKo;
    void *Qo, *Ko, *dQ, *dK;
    const float *gamma[2]; // queries', keys'
    const int *positions; // given, or any address that can be read
    int given;
    float *partial; // backward: sums of gamma gradients per workgroup [blocks][2][D]
    int tokens, L, heads[2], D, R, norm;
    float eps;
    i64 in[2][3], out[2][3], din[2][3]; // strides of Q, K, of Qo, Ko (dQo, dKo) and of dQ, dK
    double turns[128];       // revolutions per position of each pair
};

// W values as they lie in memory
template <typename T, int W>
struct Raw {
    uint32_t w[W * sizeof(T) / 4];
    __device__ __forceinline__ void load(const T *p) { __builtin_memcpy(w, __builtin_assume_aligned(p, sizeof(T) * W < 16 ? sizeof(T) * W : 16), sizeof(T) * W); }
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        return bf16_bits_to_float((uint16_t)(w[i / 2] >> (16 * (i & 1))));
    }
};
template <typename T, int W>
__device__ __forceinline__ void put_values(T *p, const float *x)
{
    if constexpr (sizeof(T) == 4) {
        __builtin_memcpy(__builtin_assume_aligned(p, sizeof(T) * W), x, sizeof(T) * W);
    } else {
        uint32_t w[W / 2];
#pragma unroll
        for (int i = 0; i < W / 2; ++i) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
        __builtin_memcpy(__builtin_assume_aligned(p, sizeof(T) * W), w, sizeof(T) * W);
    }
}
// The W pairs of a lane: from o1 and o2 (halves), or from o1 on, one after the other (pairs)
template <typename T, int W, bool PAIRS>
struct Pairs {
    Raw<T, PAIRS ? 2 * W : W> x, y; // (pairs: x alone)
    __device__ __forceinline__ void load(const T *head, int o1, int o2)
    {
        x.load(head + o1);
        if constexpr (!PAIRS) y.load(head + o2);
    }
    __device__ __forceinline__ float a(int i) const { return PAIRS ? x[2 * i] : x[i]; }
    __device__ __forceinline__ float b(int i) const
    {
        if constexpr (PAIRS) return x[2 * i + 1];
        return y[i];
    }
};
template <typename T, int W, bool PAIRS>
__device__ __forceinline__ void put_pairs(T *head, int o1, int o2, const float *a, const float *b)
{
    if constexpr (PAIRS) {
        float x[2 * W];
        constexpr int N = 16 / sizeof(T) < 2 * W ? 16 / sizeof(T) : 2 * W;
#pragma unroll
        for (int i = 0; i < W; ++i) x[2 * i] = a[i], x[2 * i + 1] = b[i];
#pragma unroll
        for (int i = 0; i < 2 * W; i += N) put_values<T, N>(head + o1 + i, x + i);
    } else {
        put_values<T, W>(head + o1, a);
        put_values<T, W>(head + o2, b);
    }
}

// Sum over the 2^log lanes of a head (log is one number for the wave).  Within 16 lanes the other addend comes with the addition.
template <int CTRL>
__device__ __forceinline__ float with_lane(float x)
{
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float head_sum(float x, int log)
{
    if (log > 0) x = with_lane<0xb1>(x);  // lanes 1 0 3 2
    if (log > 1) x = with_lane<0x4e>(x);  // 2 3 0 1
    if (log > 2) x = with_lane<0x141>(x); // 7 .. 0 of 8: the four that a quad lacks
    if (log > 3) x = with_lane<0x140>(x); // 15 .. 0 of 16
    if (log > 4) x += __shfl_xor(x, 16);
    if (log > 5) x += __shfl_xor(x, 32);
    return x;
}

// cos, sin of the token's angles into LDS (the wave's own part).  The angle in revolutions, its fraction within 1/2 of zero,
// in double: a position of 2^31 leaves 2^-22 of a revolution's digits, float alone would have none left at 2^24.
// turns: revolutions per position of the pairs lane and lane + 64.
__device__ __forceinline__ void token_angles(int pairs, int pos, const double (&turns)[2], float2 *cs, int lane)
{
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (64 * k >= pairs) break;
        double t = (double)pos * turns[k];
        t -= rint(t);
        float s, c;
        sincospif(2.f * (float)t, &s, &c);
        if (lane + 64 * k < pairs) cs[lane + 64 * k] = make_float2(c, s);
    }
}

// T, W pairs to a lane, PAIRS, BWD
template <typename T, int W, bool PAIRS, bool BWD>
__global__ __launch_bounds__(256, 4) void qk_norm_kernel(QkArgs a, int log)
{
    __shared__ __attribute__((aligned(16))) float2 cs_all[4][128];
    __shared__ __attribute__((aligned(16))) float gam[2][256];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    float2 *cs = cs_all[wave]; // cosine and sine for each pair
    const int D = a.D, half = a.R / 2;
    const int slot = lane >> log, slots = 64 >> log, all = a.heads[0] + a.heads[1];
    // The lane's first pair.  Lanes behind the end of a head, and heads behind the last, do the work of the last one once more:
    // loads and stores are the same for all lanes and without branches, so that it is known how many are on their way and none is
    // waited for that need not be.
    const int own = (lane & ((1 << log) - 1)) * W, part = own < D / 2 ? own : D / 2 - W;
    const bool in_head = own < D / 2;
    const bool turned = part < half; // (W divides R / 2: a lane's pairs are turned or not, all of them)
    const int o1 = PAIRS ? 2 * part : turned ? part : a.R + part - half;
    const int o2 = PAIRS ? 0 : o1 + (turned ? half : (D - a.R) / 2);
    const float inv_d = 1.f / (float)D;

    // Where a token's heads begin: the same for the whole wave, up to the lane's head
    const auto place = [&](const void *q, const void *k, const i64 (&sq)[3], const i64 (&sk)[3], int b, int l, int hh) {
        const T *const q0 = (const T *)q + b * sq[0] + l * sq[1], *const k0 = (const T *)k + b * sk[0] + l * sk[1];
        const bool key = hh >= a.heads[0];
        return (key ? k0 : q0) + (key ? hh - a.heads[0] : hh) * (key ? sk[2] : sq[2]);
    };
    // What is read of a token's heads h0 .. h0 + slots: on its way while the angles, or the heads before, are worked on
    struct Item {
        int b, l, pos;
        Pairs<T, W, PAIRS> x, y;
    };
    const int step = gridDim.x * 4;
    const auto load = [&](Item &m, int token, int h0) {
        token = token < a.tokens ? token : a.tokens - 1;
        m.b = token / a.L, m.l = token - m.b * a.L;
        m.pos = a.positions[a.given ? token : 0];
        const int hh = h0 + slot < all ? h0 + slot : all - 1;
        m.x.load(place(a.Q, a.K, a.in[0], a.in[1], m.b, m.l, hh), o1, o2);
        if constexpr (BWD) m.y.load(place(a.dQo, a.dKo, a.out[0], a.out[1], m.b, m.l, hh), o1, o2);
    };
    const double turns[2] = {lane < half ? a.turns[lane] : 0.0, lane + 64 < half ? a.turns[lane + 64] : 0.0};
    int token = blockIdx.x * 4 + wave;
    Item first, second;
    load(first, token, 0);
    for (int i = threadIdx.x; i < 2 * D; i += 256) {
        const int k = i >= D, j = k ? i - D : i;
        gam[k][j] = a.norm && a.gamma[k] ? a.gamma[k][j] : 1.f;
    }
    for (int i = half + lane; i < D / 2; i += 64) cs[i] = make_float2(1.f, 0.f);
    __syncthreads();
    float ga[2][W], gb[2][W]; // gradients of gamma: this lane's values of all heads that it sees, queries and keys
    if constexpr (BWD) {
#pragma unroll
        for (int i = 0; i < W; ++i) ga[0][i] = ga[1][i] = gb[0][i] = gb[1][i] = 0.f;
    }
    int h0 = 0;
    // works on m, on whose way the next item is
    const auto turn = [&](const Item &m, Item &next) {
        int token1 = token, h1 = h0 + slots;
        if (h1 >= all) h1 = 0, token1 += step;
        load(next, token1, h1);
        if (h0 == 0) {
            __builtin_amdgcn_wave_barrier();
            token_angles(half, a.given ? m.pos : m.l, turns, cs, lane);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
        const int hh = h0 + slot < all ? h0 + slot : all - 1, k = hh >= a.heads[0];
        const bool on = in_head && h0 + slot < all;
        float rstd = 1.f;
        if (a.norm) {
            float q = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) q += m.x.a(i) * m.x.a(i) + m.x.b(i) * m.x.b(i);
            rstd = 1.f / sqrtf(head_sum(in_head ? q : 0.f, log) * inv_d + a.eps);
        }
        const float *const g1 = gam[k] + o1, *const g2 = gam[k] + o2;
        const float2 *const angle = cs + part;
        float ya[W], yb[W], dot = 0.f;
        float p[W], r[W]; // backward: terms of gamma's gradients
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float c = angle[i].x, s = angle[i].y, gma = PAIRS ? g1[2 * i] : g1[i], gmb = PAIRS ? g1[2 * i + 1] : g2[i];
            const float xa = m.x.a(i) * rstd, xb = m.x.b(i) * rstd;
            if constexpr (!BWD) {
                const float u = xa * gma, v = xb * gmb;
                ya[i] = u * c - v * s;
                yb[i] = u * s + v * c;
            } else { // the turn taken back, then dx = rstd (w - xh mean(w xh)), w = gamma du
                const float u = m.y.a(i) * c + m.y.b(i) * s, v = m.y.b(i) * c - m.y.a(i) * s;
                p[i] = u * xa, r[i] = v * xb;
                ya[i] = u * gma;
                yb[i] = v * gmb;
                dot += ya[i] * xa + yb[i] * xb;
            }
        }
        if constexpr (BWD) {
            if (h0 < a.heads[0]) {
#pragma unroll
                for (int i = 0; i < W; ++i) ga[0][i] += on && !k ? p[i] : 0.f, gb[0][i] += on && !k ? r[i] : 0.f;
            }
            if (h0 + slots > a.heads[0]) {
#pragma unroll
                for (int i = 0; i < W; ++i) ga[1][i] += on && k ? p[i] : 0.f, gb[1][i] += on && k ? r[i] : 0.f;
            }
        }
        if (BWD && a.norm) {
            const float mean = head_sum(in_head ? dot : 0.f, log) * inv_d;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                ya[i] = rstd * (ya[i] - m.x.a(i) * rstd * mean);
                yb[i] = rstd * (yb[i] - m.x.b(i) * rstd * mean);
            }
        }
        T *const out = BWD ? (T *)place(a.dQ, a.dK, a.din[0], a.din[1], m.b, m.l, hh) : (T *)place(a.Qo, a.Ko, a.out[0], a.out[1], m.b, m.l, hh);
        put_pairs<T, W, PAIRS>(out, o1, o2, ya, yb);
        token = token1, h0 = h1;
    };
    while (token < a.tokens) {
        turn(first, second);
        if (token < a.tokens) turn(second, first);
    }
    if constexpr (BWD) {
        if (!a.partial) return;
        // this workgroup's sums: the lanes of a wave that hold the same values, then the four waves, always in one order
        __shared__ float sums[4][2][256];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                float p = ga[k][i], q = gb[k][i];
                for (int o = 1 << log; o < 64; o <<= 1) {
                    p += __shfl_xor(p, o);
                    q += __shfl_xor(q, o);
                }
                if (slot == 0 && in_head) {
                    sums[wave][k][PAIRS ? o1 + 2 * i : o1 + i] = p;
                    sums[wave][k][PAIRS ? o1 + 2 * i + 1 : o2 + i] = q;
                }
            }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * D; i += 256) {
            const int k = i >= D, j = k ? i - D : i;
            a.partial[(i64)blockIdx.x * 2 * D + i] = (sums[0][k][j] + sums[1][k][j]) + (sums[2][k][j] + sums[3][k][j]);
        }
    }
}

// The workgroups' sums to dgamma: one workgroup per value, in double and always in one order.  Bound by latency: a lane's loads
// are on their way together (one wave that loaded one by one took 6.7 us for 1024 workgroups, this 3.9).  Where queries and keys
// share their gamma (dq == dk) a value is the sum of both, in one workgroup.
__global__ __launch_bounds__(256) void qk_gamma_kernel(const float *partial, int blocks, int D, float *dq, float *dk, int accumulate)
{
    __shared__ double part[2][4];
    const int t = threadIdx.x, values = dq == dk ? 2 : 1, j = blockIdx.x < D ? blockIdx.x : blockIdx.x - D;
    for (int v = 0; v < values; ++v) {
        const int i = blockIdx.x + v * D;
        float x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = t + 256 * k < blocks ? partial[(i64)(t + 256 * k) * 2 * D + i] : 0.f;
        double s = ((double)x[0] + (double)x[1]) + ((double)x[2] + (double)x[3]);
        for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
        if ((t & 63) == 0) part[v][t >> 6] = s;
    }
    __syncthreads();
    float *const out = blockIdx.x < D ? dq : dk;
    if (t || !out) return;
    double s = (part[0][0] + part[0][1]) + (part[0][2] + part[0][3]);
    if (values == 2) s += (part[1][0] + part[1][1]) + (part[1][2] + part[1][3]);
    out[j] = accumulate ? out[j] + (float)s : (float)s;
}

// ------------------------------------------------------------------ host
static int qk_check(const pf_qk_norm_desc *d)
{
    if (!d) return PF_ERR_NULL;
    if (d->B < 0 || d->L < 0 || d->heads_q <= 0 || d->heads_k < 0 || d->head_dim <= 0 || d->rot_dim < 0) return PF_ERR_SHAPE;
    if (d->dtype != PF_F32 && d->dtype != PF_BF16) return PF_ERR_UNSUPPORTED;
    if (d->norm != PF_NORM_NONE && d->norm != PF_NORM_RMS) return PF_ERR_UNSUPPORTED;
    if (d->rotation != PF_ROT_HALVES && d->rotation != PF_ROT_PAIRS) return PF_ERR_UNSUPPORTED;
    if (d->head_dim % 8 || d->head_dim > 256 || d->rot_dim % 4 || d->rot_dim > d->head_dim) return PF_ERR_UNSUPPORTED;
    if (d->rot_dim && !(d->theta > 0 && isfinite(d->theta))) return PF_ERR_UNSUPPORTED;
    if (d->norm && !(d->eps >= 0 && isfinite(d->eps))) return PF_ERR_UNSUPPORTED;
    const i64 heads = (i64)d->heads_q + d->heads_k;
    if (d->B && d->L && (d->L > INT32_MAX / 2 / d->B || d->B * d->L > INT32_MAX / 2 / heads)) return PF_ERR_UNSUPPORTED;
    const int unit = 16 / (d->dtype == PF_BF16 ? 2 : 4);
    for (const int64_t *s : {d->q_stride, d->k_stride, d->qo_stride, d->ko_stride, d->dq_stride, d->dk_stride})
        for (int i = 0; i < 3; ++i)
            if (s[i] < 0 || s[i] % unit) return PF_ERR_UNSUPPORTED;
    return PF_OK;
}
static void strides_of(const int64_t *s, i64 L, int heads, int D, i64 (&out)[3])
{
    const bool dense = !s[0] && !s[1] && !s[2];
    out[2] = dense ? D : s[2];
    out[1] = dense ? (i64)heads * D : s[1];
    out[0] = dense ? L * heads * D : s[0];
}
constexpr int QK_SUMS = 1024; // (qk_gamma_kernel's lanes hold as many)
static int qk_blocks(const pf_qk_norm_desc *d, bool bwd)
{
    // Four tokens (one per wave) to a workgroup.  Backward, a workgroup leaves 2 D sums behind, so that there are at most
    // four to a compute unit, each going through many tokens.
    const i64 blocks = (d->B * d->L + 3) / 4, most = bwd ? QK_SUMS : 1 << 20;
    return (int)(blocks < most ? blocks : most);
}
static void qk_fill(const pf_qk_norm_desc *d, QkArgs &a)
{
    a.tokens = (int)(d->B * d->L);
    a.L = (int)d->L;
    a.heads[0] = d->heads_q;
    a.heads[1] = d->heads_k;
    a.D = d->head_dim;
    a.R = d->rot_dim;
    a.norm = d->norm == PF_NORM_RMS;
    a.eps = d->eps;
    strides_of(d->q_stride, d->L, d->heads_q, d->head_dim, a.in[0]);
    strides_of(d->k_stride, d->L, d->heads_k, d->head_dim, a.in[1]);
    strides_of(d->qo_stride, d->L, d->heads_q, d->head_dim, a.out[0]);
    strides_of(d->ko_stride, d->L, d->heads_k, d->head_dim, a.out[1]);
    strides_of(d->dq_stride, d->L, d->heads_q, d->head_dim, a.din[0]);
    strides_of(d->dk_stride, d->L, d->heads_k, d->head_dim, a.din[1]);
    // a model calls with one theta and size again and again: 64 powers would cost more than a small call's launch
    static thread_local struct {
        int R;
        double theta, turns[128];
    } known = {0, 0, {}};
    if (a.R && (known.R != a.R || known.theta != d->theta)) {
        for (int i = 0; i < a.R / 2; ++i) known.turns[i] = pow(d->theta, -2.0 * i / a.R) / (2.0 * M_PI);
        known.R = a.R;
        known.theta = d->theta;
    }
    for (int i = 0; i < a.R / 2; ++i) a.turns[i] = known.turns[i];
}

template <typename T, int W, bool BWD>
static int qk_launch_w(const QkArgs &a, bool pairs, int blocks, hipStream_t s)
{
    int log = 0, st = PF_OK;
    while ((1 << log) * W < a.D / 2) ++log; // lanes of a head
    if (pairs)
        PF_LAUNCH(st, BWD ? "qk_norm_bwd" : "qk_norm_fwd", (qk_norm_kernel<T, W, true, BWD>), dim3(blocks), dim3(256), s, a, log);
    else
        PF_LAUNCH(st, BWD ? "qk_norm_bwd" : "qk_norm_fwd", (qk_norm_kernel<T, W, false, BWD>), dim3(blocks), dim3(256), s, a, log);
    return st;
}
// Four pairs to a lane if they divide the turned part and the rest, two otherwise.  (Eight bf16 pairs make 16-byte accesses, but
// backward then holds 165 registers, not 110: 64 x 128 tokens of 16 heads of 64 took 31.1 us, not 30.4, and 2 x 8191 tokens of 40
// heads of 128 177 us, not 173.)
template <bool BWD>
static int qk_launch(const QkArgs &a, int dtype, bool pairs, int blocks, hipStream_t s)
{
    const auto whole = [&](int w) { return a.R / 2 % w == 0 && a.D / 2 % w == 0; };
    if (dtype == PF_BF16) {
        if (whole(4)) return qk_launch_w<bf16_t, 4, BWD>(a, pairs, blocks, s);
        return qk_launch_w<bf16_t, 2, BWD>(a, pairs, blocks, s);
    }
    if (whole(4)) return qk_launch_w<float, 4, BWD>(a, pairs, blocks, s);
    return qk_launch_w<float, 2, BWD>(a, pairs, blocks, s);
}

// The queries' or keys' outputs of one direction: an output may be one of its own inputs, element for element
static bool meets_other(const Area &out, std::initializer_list<Area> own, std::initializer_list<Area> others)
{
    for (const Area &x : own)
        if (!x.same(out) && meet(x, out)) return true;
    return outputs_meet({out}, others);
}

} // namespace pf

extern "C" {

using namespace pf;

int pf_qk_norm_rotate_fwd(const pf_qk_norm_desc *d, const void *Q, const void *K, const void *gamma_q, const void *gamma_k,
                          const void *positions, void *Qo, void *Ko, void *stream)
{
    const int status = qk_check(d);
    if (status != PF_OK) return status;
    if (d->B == 0 || d->L == 0) return PF_OK;
    if (!Q || !Qo || (d->heads_k && (!K || !Ko))) return PF_ERR_NULL;
    if (any_misaligned({Q, Qo}, 16) || (d->heads_k && any_misaligned({K, Ko}, 16)) || any_misaligned({gamma_q, gamma_k, positions}, 4))
        return PF_ERR_UNSUPPORTED;
    QkArgs a = {};
    qk_fill(d, a);
    a.Q = Q, a.K = K, a.Qo = Qo, a.Ko = Ko;
    a.gamma[0] = (const float *)gamma_q;
    a.gamma[1] = (const float *)gamma_k;
    a.positions = (const int *)(positions ? positions : Qo);
    a.given = positions != nullptr;
    const auto area = [&](const void *p, int k, const i64 (&s)[3]) {
        return Area(p, d->B, d->L, a.heads[k], s, a.D, d->dtype == PF_BF16 ? 2 : 4);
    };
    const Area q = area(Q, 0, a.in[0]), k = area(K, 1, a.in[1]), qo = area(Qo, 0, a.out[0]), ko = area(Ko, 1, a.out[1]);
    if (meets_other(qo, {q}, {k, ko}) || meets_other(ko, {k}, {q})) return PF_ERR_UNSUPPORTED;
    return qk_launch<false>(a, d->dtype, d->rotation == PF_ROT_PAIRS, qk_blocks(d, false), (hipStream_t)stream);
}

size_t pf_qk_norm_rotate_bwd_workspace_bytes(const pf_qk_norm_desc *d)
{
    if (qk_check(d) != PF_OK || d->B == 0 || d->L == 0 || d->norm == PF_NORM_NONE) return 0;
    return align_up((size_t)qk_blocks(d, true) * 2 * d->head_dim * sizeof(float));
}

int pf_qk_norm_rotate_bwd(const pf_qk_norm_desc *d, const void *Q, const void *K, const void *gamma_q, const void *gamma_k,
                          const void *positions, const void *dQo, const void *dKo, void *dQ, void *dK, void *dgamma_q,
                          void *dgamma_k, int accumulate, void *workspace, size_t workspace_bytes, void *stream)
{
    const int status = qk_check(d);
    if (status != PF_OK) return status;
    const bool norm = d->norm == PF_NORM_RMS, sums = norm && (dgamma_q || (d->heads_k && dgamma_k));
    if (any_misaligned({gamma_q, gamma_k, positions, dgamma_q, dgamma_k}, 4)) return PF_ERR_UNSUPPORTED;
    int st = PF_OK;
    if (d->B == 0 || d->L == 0) {
        if (!norm || accumulate) return PF_OK;
        st = launch_zero_f32((hipStream_t)stream, (float *)dgamma_q, d->head_dim);
        if (st == PF_OK && d->heads_k) st = launch_zero_f32((hipStream_t)stream, (float *)dgamma_k, d->head_dim);
        return st;
    }
    if (!dQo || !dQ || (norm && !Q) || (d->heads_k && (!dKo || !dK || (norm && !K)))) return PF_ERR_NULL;
    if (any_misaligned({Q, dQo, dQ}, 16) || (d->heads_k && any_misaligned({K, dKo, dK}, 16)) || any_misaligned({workspace}, 256))
        return PF_ERR_UNSUPPORTED;
    if (sums && (!workspace || workspace_bytes < pf_qk_norm_rotate_bwd_workspace_bytes(d))) return PF_ERR_WORKSPACE;
    QkArgs a = {};
    qk_fill(d, a);
    a.Q = Q, a.K = K, a.dQo = dQo, a.dKo = dKo, a.dQ = dQ, a.dK = dK;
    a.gamma[0] = (const float *)gamma_q;
    a.gamma[1] = (const float *)gamma_k;
    a.positions = (const int *)(positions ? positions : dQo);
    a.given = positions != nullptr;
    if (!norm) { // (the values are not needed: what is read once may be read twice)
        a.Q = dQo, a.K = dKo;
        memcpy(a.in, a.out, sizeof a.in);
    }
    const auto area = [&](const void *p, int k, const i64 (&s)[3]) {
        return Area(p, d->B, d->L, a.heads[k], s, a.D, d->dtype == PF_BF16 ? 2 : 4);
    };
    const Area q = area(a.Q, 0, a.in[0]), k = area(a.K, 1, a.in[1]), dqo = area(dQo, 0, a.out[0]), dko = area(dKo, 1, a.out[1]),
               dq = area(dQ, 0, a.din[0]), dk = area(dK, 1, a.din[1]), gq(sums ? dgamma_q : nullptr, d->head_dim * 4),
               gk(sums && d->heads_k ? dgamma_k : nullptr, d->head_dim * 4);
    if (meets_other(dq, {q, dqo}, {k, dko, dk}) || meets_other(dk, {k, dko}, {q, dqo})) return PF_ERR_UNSUPPORTED;
    if (meets_other(gq, {gk}, {q, k, dqo, dko, dq, dk}) || meets_other(gk, {gq}, {q, k, dqo, dko, dq, dk})) return PF_ERR_UNSUPPORTED;
    a.partial = sums ? (float *)workspace : nullptr;
    const int blocks = qk_blocks(d, true);
    st = qk_launch<true>(a, d->dtype, d->rotation == PF_ROT_PAIRS, blocks, (hipStream_t)stream);
    float *const dgq = (float *)dgamma_q, *const dgk = d->heads_k ? (float *)dgamma_k : nullptr;
    if (sums)
        PF_LAUNCH(st, "qk_gamma", qk_gamma_kernel, dim3((dgq == dgk ? 1 : 2) * d->head_dim), dim3(256), (hipStream_t)stream, a.partial, blocks,
                  d->head_dim, dgq, dgk, accumulate);
    return st;
}

} // extern "C"
