// Norms of queries and keys per head with the position rotation: pf_qk_norm_rotate_*.
//
// Bound by memory: forward reads and writes each value once, backward reads two and writes one.  A wave takes one token at a
// time, all its heads: a lane holds W pairs of a head (the two values that a rotation mixes are always in one lane), the
// head_dim / (2 W) lanes of a head add up its squares between them, and 64 / lanes heads are in flight.  The angles belong
// to the token alone: the wave forms each one once, in double, and its heads read cosine and sine from LDS.
#include <math.h>

#include "pf_gemm.h"

namespace pf {

struct QkArgs {
    const void *Q, *K, *dQo, *dKo;
    void *Qo, *Ko, *dQ, *dK;
    const float *gamma[2]; // queries', keys'
    const int *positions;
    float *partial; // backward: sums of gamma gradients per workgroup [blocks][2][D]
    int tokens, L, heads[2], D, R, norm;
    float eps;
    i64 in[2][3], out[2][3], din[2][3]; // strides of Q, K, of Qo, Ko (dQo, dKo) and of dQ, dK
    double turns[128];       // revolutions per position of each pair
};

template <typename T, int W>
__device__ __forceinline__ void get_values(const T *p, float *x)
{
    if constexpr (sizeof(T) == 4) {
        __builtin_memcpy(x, __builtin_assume_aligned(p, sizeof(T) * W), sizeof(T) * W);
    } else {
        uint32_t w[W / 2];
        __builtin_memcpy(w, __builtin_assume_aligned(p, sizeof(T) * W), sizeof(T) * W);
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = bf16_bits_to_float((uint16_t)(w[i / 2] >> (16 * (i & 1))));
    }
}
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
// The W pairs of a lane: a[] and b[], from o1 and o2 (halves), or from o1 on, one after the other (pairs)
template <typename T, int W, bool PAIRS>
__device__ __forceinline__ void get_pairs(const T *head, int o1, int o2, float *a, float *b)
{
    if constexpr (PAIRS) {
        float x[2 * W];
        constexpr int N = 16 / sizeof(T) < 2 * W ? 16 / sizeof(T) : 2 * W; // (16 bytes at a time)
#pragma unroll
        for (int i = 0; i < 2 * W; i += N) get_values<T, N>(head + o1 + i, x + i);
#pragma unroll
        for (int i = 0; i < W; ++i) a[i] = x[2 * i], b[i] = x[2 * i + 1];
    } else {
        get_values<T, W>(head + o1, a);
        get_values<T, W>(head + o2, b);
    }
}
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

// Sum over the 2^log lanes of a head
__device__ __forceinline__ float head_sum(float x, int log)
{
    for (int o = 0; o < log; ++o) x += __shfl_xor(x, 1 << o);
    return x;
}

// cos, sin of the token's angles into LDS (the wave's own part).  The angle in revolutions, its fraction within 1/2 of zero,
// in double: a position of 2^31 leaves 2^-22 of a revolution's digits, float alone would have none left at 2^24.
__device__ __forceinline__ void token_angles(const QkArgs &a, int pos, float2 *cs, int lane)
{
    for (int i = lane; i < a.R / 2; i += 64) {
        double t = (double)pos * a.turns[i];
        t -= rint(t);
        float s, c;
        sincospif(2.f * (float)t, &s, &c);
        cs[i] = make_float2(c, s);
    }
}

// T, W pairs to a lane, PAIRS, BWD
template <typename T, int W, bool PAIRS, bool BWD>
__global__ __launch_bounds__(256) void qk_norm_kernel(QkArgs a, int log)
{
    __shared__ float2 cs_all[4][128];
    __shared__ float gam[2][256];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    float2 *cs = cs_all[wave];
    const int D = a.D, half = a.R / 2, part = (lane & ((1 << log) - 1)) * W; // the lane's first pair
    const int slot = lane >> log, slots = 64 >> log, all = a.heads[0] + a.heads[1];
    const bool in_head = part < D / 2;
    const bool turned = part < half; // (W divides R / 2: a lane's pairs are turned or not, all of them)
    const int o1 = PAIRS ? 2 * part : turned ? part : a.R + part - half;
    const int o2 = PAIRS ? 0 : o1 + (turned ? half : (D - a.R) / 2);
    if (a.norm)
        for (int i = threadIdx.x; i < 2 * D; i += 256) {
            const int k = i >= D, j = k ? i - D : i;
            gam[k][j] = a.gamma[k] ? a.gamma[k][j] : 1.f;
        }
    __syncthreads();
    float ga[2][W], gb[2][W]; // gradients of gamma: this lane's values of all heads that it sees, queries and keys
    if constexpr (BWD) {
#pragma unroll
        for (int i = 0; i < W; ++i) ga[0][i] = ga[1][i] = gb[0][i] = gb[1][i] = 0.f;
    }
    for (int token = blockIdx.x * 4 + wave; token < a.tokens; token += gridDim.x * 4) {
        const int b = token / a.L, l = token - b * a.L;
        __builtin_amdgcn_wave_barrier();
        token_angles(a, a.positions ? a.positions[token] : l, cs, lane);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        for (int h0 = 0; h0 < all; h0 += slots) {
            const int hh = h0 + slot;
            const bool on = in_head && hh < all;
            const int k = hh >= a.heads[0], h = k ? hh - a.heads[0] : hh;
            float xa[W], xb[W], ya[W], yb[W];
            const T *x = (const T *)(k ? a.K : a.Q) + b * a.in[k][0] + l * a.in[k][1] + h * a.in[k][2];
            const i64 at_out = b * a.out[k][0] + l * a.out[k][1] + h * a.out[k][2];
#pragma unroll
            for (int i = 0; i < W; ++i) xa[i] = xb[i] = ya[i] = yb[i] = 0.f;
            if (on && (!BWD || a.norm)) get_pairs<T, W, PAIRS>(x, o1, o2, xa, xb);
            if constexpr (BWD) {
                if (on) get_pairs<T, W, PAIRS>((const T *)(k ? a.dKo : a.dQo) + at_out, o1, o2, ya, yb);
            }
            float rstd = 1.f;
            if (a.norm) {
                float q = 0.f;
#pragma unroll
                for (int i = 0; i < W; ++i) q += xa[i] * xa[i] + xb[i] * xb[i];
                rstd = 1.f / sqrtf(head_sum(q, log) / (float)D + a.eps);
            }
            float c[W], s[W], gma[W], gmb[W];
#pragma unroll
            for (int i = 0; i < W; ++i) c[i] = 1.f, s[i] = 0.f, gma[i] = gmb[i] = 1.f;
            if (on && turned) {
#pragma unroll
                for (int i = 0; i < W; ++i) c[i] = cs[part + i].x, s[i] = cs[part + i].y;
            }
            if (on && a.norm) {
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    gma[i] = gam[k][PAIRS ? o1 + 2 * i : o1 + i];
                    gmb[i] = gam[k][PAIRS ? o1 + 2 * i + 1 : o2 + i];
                }
            }
            if constexpr (!BWD) {
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const float u = xa[i] * rstd * gma[i], v = xb[i] * rstd * gmb[i];
                    ya[i] = u * c[i] - v * s[i];
                    yb[i] = u * s[i] + v * c[i];
                }
                if (on) put_pairs<T, W, PAIRS>((T *)(k ? a.Ko : a.Qo) + at_out, o1, o2, ya, yb);
            } else {
                float dot = 0.f;
#pragma unroll
                for (int i = 0; i < W; ++i) { // the turn taken back, then dx = rstd (w - xh mean(w xh)), w = gamma du
                    const float u = ya[i] * c[i] + yb[i] * s[i], v = yb[i] * c[i] - ya[i] * s[i];
                    if (a.norm) {
                        xa[i] *= rstd;
                        xb[i] *= rstd;
                        ga[0][i] += k ? 0.f : u * xa[i];
                        gb[0][i] += k ? 0.f : v * xb[i];
                        ga[1][i] += k ? u * xa[i] : 0.f;
                        gb[1][i] += k ? v * xb[i] : 0.f;
                    }
                    ya[i] = u * gma[i];
                    yb[i] = v * gmb[i];
                    dot += ya[i] * xa[i] + yb[i] * xb[i];
                }
                if (a.norm) {
                    const float mean = head_sum(dot, log) / (float)D;
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        ya[i] = rstd * (ya[i] - xa[i] * mean);
                        yb[i] = rstd * (yb[i] - xb[i] * mean);
                    }
                }
                T *dx = (T *)(k ? a.dK : a.dQ) + b * a.din[k][0] + l * a.din[k][1] + h * a.din[k][2];
                if (on) put_pairs<T, W, PAIRS>(dx, o1, o2, ya, yb);
            }
        }
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

// The workgroups' sums to dgamma: one workgroup of 64 lanes per value, in double and always in one order
__global__ __launch_bounds__(64) void qk_gamma_kernel(const float *partial, int blocks, int D, float *dq, float *dk, int accumulate)
{
    const int i = blockIdx.x, lane = threadIdx.x;
    double s = 0.0;
    for (int b = lane; b < blocks; b += 64) s += (double)partial[(i64)b * 2 * D + i];
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    float *out = i < D ? dq : dk;
    const int j = i < D ? i : i - D;
    if (lane == 0 && out) out[j] = accumulate ? out[j] + (float)s : (float)s;
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
    if (d->B && d->L && (d->L > INT32_MAX / d->B || d->B * d->L > INT32_MAX / heads)) return PF_ERR_UNSUPPORTED;
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
static int qk_blocks(const pf_qk_norm_desc *d, bool bwd)
{
    // Four tokens (one per wave) to a workgroup.  Backward, a workgroup leaves 2 D sums behind, so that there are at most
    // four to a compute unit, each going through many tokens.
    const i64 blocks = (d->B * d->L + 3) / 4, most = bwd ? 1024 : 1 << 20;
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
// As many pairs to a lane as make 16-byte accesses (halves: W values from each half), if they divide the turned part and
// the rest; two otherwise
template <bool BWD>
static int qk_launch(const QkArgs &a, int dtype, bool pairs, int blocks, hipStream_t s)
{
    const auto whole = [&](int w) { return a.R / 2 % w == 0 && a.D / 2 % w == 0; };
    if (dtype == PF_BF16) {
        if (whole(8)) return qk_launch_w<bf16_t, 8, BWD>(a, pairs, blocks, s);
        if (whole(4)) return qk_launch_w<bf16_t, 4, BWD>(a, pairs, blocks, s);
        return qk_launch_w<bf16_t, 2, BWD>(a, pairs, blocks, s);
    }
    if (whole(4)) return qk_launch_w<float, 4, BWD>(a, pairs, blocks, s);
    return qk_launch_w<float, 2, BWD>(a, pairs, blocks, s);
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
    a.positions = (const int *)positions;
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
    a.positions = (const int *)positions;
    a.partial = sums ? (float *)workspace : nullptr;
    const int blocks = qk_blocks(d, true);
    st = qk_launch<true>(a, d->dtype, d->rotation == PF_ROT_PAIRS, blocks, (hipStream_t)stream);
    if (sums)
        PF_LAUNCH(st, "qk_gamma", qk_gamma_kernel, dim3(2 * d->head_dim), dim3(64), (hipStream_t)stream, a.partial, blocks, d->head_dim,
                  (float *)dgamma_q, d->heads_k ? (float *)dgamma_k : nullptr, accumulate);
    return st;
}

} // extern "C"
