// Attention with a relative position bias by buckets, backward: pf_attention_bwd.
//
// P is formed again from the scores and lse.  Two kernels, neither of which adds into memory that another workgroup writes, so
// that results do not depend on an order: the first has queries in its columns and makes dQ, delta and the sums of dS by
// distance; the second has keys in its columns and makes dK and dV, going through the query heads of a key head.  They form S
// and dP each (seven products where one kernel with atomic sums of dQ would have five).
//
// delta = sum P dP of a row is sum O dO, too, but O is rounded to bf16 there and P was before O was formed: dS is off by
// 2^-9 of delta then, which is below what rounding dS itself costs dQ and dK, but not good enough for dtable, a float32 sum over
// all pairs in which the rows' errors would stay.  With a table gradient the first kernel therefore goes over its keys twice, for
// delta in float32 first.
#include "pf_attn.h"
#include "pf_gemm.h"

namespace pf {

template <typename T>
constexpr int BWD_KEYS = sizeof(T) == 2 ? 64 : 32; // keys (queries) of a tile

constexpr int DIAG = 33; // floats from one row of a 32 x 32 block of dS to the next in LDS

template <typename T, int DP>
struct BwdLds {
    using Tl = Tile<T, DP, BWD_KEYS<T>, 256>;
    static size_t dq(int far, bool bias, bool tab)
    {
        return 2 * Tl::BYTES + (bias ? (2 * far + 1) * 4 : 0) + (tab ? 4 * 32 * DIAG * 4 + 4 * (2 * far + 1) * 4 : 0);
    }
    static size_t dkv(int far, bool bias) { return 2 * Tl::BYTES + 2 * BWD_KEYS<T> * 4 + (bias ? (2 * far + 1) * 4 : 0); }
};

// dQ, delta and the sums of dS by distance; a workgroup has 128 queries of one head.  TAB: with the gradient of the table
template <typename T, int DP, bool BIAS, bool TAB>
__global__ __launch_bounds__(256, DP * sizeof(T) <= (TAB ? 128 : sizeof(T) == 2 ? 256 : 320) ? 2 : 1) void attn_dq_kernel(AttnArgs a)
{
    constexpr int KT = BWD_KEYS<T>, SUB = KT / 32;
    using Tl = Tile<T, DP, KT, 256>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int far = a.bk.far, span = 2 * far + 1;
    T *const kt = (T *)lds, *const vt = (T *)(lds + Tl::BYTES);
    float *const bias = (float *)(lds + 2 * Tl::BYTES);
    float *const diag_all = bias + span, *const sums_all = diag_all + 4 * 32 * DIAG; // [4][32][DIAG], [4][span]

    const unsigned w = xcd_order(blockIdx.x, gridDim.x);
    const int tile = a.tiles - 1 - (int)(w % a.tiles), bh = w / a.tiles, b = bh / a.Hq, head = bh - b * a.Hq;
    const int t = threadIdx.x, wave = wave_of(t), lane = t & 63, col = lane & 31, h = lane >> 5;
    float *const diag = diag_all + wave * 32 * DIAG, *const sums = sums_all + wave * span;
    const AttnLens n(a, b);
    const int i0 = tile * 128 + wave * 32, i = i0 + col;
    const bool ok = i < n.nq;
    const T *const Kp = (const T *)a.K + b * a.ks[0] + head / a.G * a.ks[2], *const Vp = (const T *)a.V + b * a.vs[0] + head / a.G * a.vs[2];
    int keys = n.nk;
    if (tile * 128 >= n.nq) keys = 0;
    const int block_last = (tile * 128 + 128 < n.nq ? tile * 128 + 128 : n.nq) - 1 + n.start;
    if (a.causal && block_last + 1 < keys) keys = block_last + 1 < 0 ? 0 : block_last + 1;
    const int last = (i0 + 32 < n.nq ? i0 + 32 : n.nq) - 1, pmin = i0 + n.start, pmax = last + n.start, pos = i + n.start;
    const bool idle = i0 >= n.nq;

    if (BIAS && keys > 0) fill_bias(a, bias, head, t, 256);
    if constexpr (TAB)
        for (int x = t; x < 4 * span; x += 256) sums_all[x] = 0.f;
    const i64 at = (((i64)b * a.Lq + i) * a.Hq + head) * a.D, stat = ((i64)b * a.Hq + head) * a.Lq + i;
    Frag<T> q[DP / 16], g[DP / 16];
    {
        const T *const Qp = (const T *)a.Q + b * a.qs[0] + head * a.qs[2] + i * a.qs[1], *const Gp = (const T *)a.dO + at;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
            q[c] = row_frag_global(Qp, 16 * c, a.D, h, ok);
            g[c] = row_frag_global(Gp, 16 * c, a.D, h, ok);
        }
    }
    // exp2(S - lse) is 0 for a query that takes no part
    float lse2 = INFINITY;
    if (ok) {
        const float x = a.lse_in[stat];
        if (x > -INFINITY) lse2 = x * LOG2E;
    }
    float delta = 0.f;
    if constexpr (!TAB) {
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
            const Frag<T> x = row_frag_global((const T *)a.Oin + at, 16 * c, a.D, h, ok);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta += (float)x.v[e] * (float)g[c].v[e];
        }
        delta += __shfl_xor(delta, 32);
    }
    const float sl2 = a.scale * LOG2E;
    f32x16_t dq[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) dq[d] = f32x16_t{};
    float before = 0.f, after = 0.f; // sums of dS in blocks that are further than `far` off

    const Tl kr(a.ks[1], a.D, t), vr(a.vs[1], a.D, t);
    for (int pass = TAB ? 0 : 1; pass < 2; ++pass) {
        float row = 0.f;
        for (int k0 = 0; k0 < keys; k0 += KT) {
            __syncthreads();
            kr.fetch(kt, Kp + (i64)k0 * a.ks[1], a.ks[1], n.nk - k0, a.D, wave);
            vr.fetch(vt, Vp + (i64)k0 * a.vs[1], a.vs[1], n.nk - k0, a.D, wave);
            fetched();
            __syncthreads();
            if (idle || (a.causal && k0 > pmax)) continue;
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                const int ks = k0 + 32 * u;
                const bool edge = ks + 32 > n.nk || (a.causal && ks + 31 > pmin);
                const bool near = BIAS && ks + 31 - pmin > -far && ks - pmax < far;
                const float flat = BIAS ? bias[ks >= pmin ? 2 * far : 0] : 0.f;
                f32x16_t s = {}, dp = {};
                #pragma unroll
                for (int c = 0; c < DP / 16; ++c) {
                    mma(s, Tl::by_rows(kt, 32 * u, c, lane), q[c]);
                    mma(dp, Tl::by_rows(vt, 32 * u, c, lane), g[c]);
                }
                float ds[16];
                const float base = flat - lse2;
#pragma unroll
                for (int e = 0; e < 16; ++e) ds[e] = s[e];
                if (edge || near) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int j = ks + 8 * (e >> 2) + 4 * h + (e & 3);
                        ds[e] = exp2_fast(ds[e] * sl2 + ((BIAS ? bias[clamped(j - pos, -far, far) + far] : 0.f) - lse2));
                        if (j >= n.nk || (a.causal && j > pos)) ds[e] = 0.f;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) ds[e] = exp2_fast(ds[e] * sl2 + base);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) { // (first pass: delta is 0, and the sum of these is delta)
                    ds[e] *= dp[e] - delta;
                    if (TAB && pass == 0) row += ds[e];
                }
                if (TAB && pass == 0) continue;
                if constexpr (TAB) {
                    if (near) {
                        // along the diagonals of the block: lane x has the distance x - 31 from that of its corner
#pragma unroll
                        for (int e = 0; e < 16; ++e) diag[(8 * (e >> 2) + 4 * h + (e & 3)) * DIAG + col] = ds[e];
                        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                        __builtin_amdgcn_wave_barrier();
                        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                        float y = 0.f;
#pragma unroll
                        for (int c = 0; c < 32; ++c) {
                            const int r = c + lane - 31;
                            const float v = diag[clamped(r, 0, 31) * DIAG + c];
                            y += r >= 0 && r < 32 ? v : 0.f;
                        }
                        const int dist = ks - pmin + lane - 31;
                        // distances beyond far share their sum's place: one lane after the other would be needed, so those go to
                        // the lanes' own sums
                        if (lane < 63) {
                            if (dist <= -far)
                                before += y;
                            else if (dist >= far)
                                after += y;
                            else
                                sums[dist + far] += y;
                        }
                        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                        __builtin_amdgcn_wave_barrier();
                        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                    } else {
                        float y = 0.f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) y += ds[e];
                        if (ks >= pmin)
                            after += y;
                        else
                            before += y;
                    }
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    Frag<T> p;
                    pack(ds, c, p);
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) mma(dq[d], Tl::by_cols(kt, 32 * u + 16 * c, d, lane), p);
                }
            }
        }
        if (TAB && pass == 0) delta = row + __shfl_xor(row, 32);
        __syncthreads(); // (the tiles are free for the next pass)
    }
    if (i < a.Lq) {
        T *const out = (T *)a.dQ + at;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int c = 32 * d + 8 * (e >> 2) + 4 * h;
                float v[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = ok ? dq[d][e + x] * a.scale : 0.f;
                if (c < a.D) put4(out + c, v[0], v[1], v[2], v[3]);
            }
        if (h == 0) a.delta[stat] = ok ? delta : 0.f;
    }
    if constexpr (TAB) {
        for (int o = 32; o; o >>= 1) {
            before += __shfl_xor(before, o);
            after += __shfl_xor(after, o);
        }
        if (lane == 0) {
            sums[0] += before;
            sums[2 * far] += after;
        }
        __syncthreads();
        for (int x = t; x < span; x += 256) sums_all[x] = (sums_all[x] + sums_all[span + x]) + (sums_all[2 * span + x] + sums_all[3 * span + x]);
        __syncthreads();
        float *const out = a.tab + (((i64)head * a.B + b) * a.tiles + tile) * a.buckets;
        for (int u = t; u < a.buckets; u += 256) {
            // the distances of bucket u: lo .. hi of its side, the last one's up to far
            const int v = a.two_sided && u >= a.bk.side ? u - a.bk.side : u, e = a.bk.exact;
            int lo = v, hi = v;
            if (v >= e) {
                lo = v == e ? e : a.bk.border[v - e - 1];
                hi = v == a.bk.side - 1 ? far : a.bk.border[v - e] - 1;
            }
            float y = 0.f;
            if (a.two_sided && u >= a.bk.side) {
                for (int x = lo < 1 ? 1 : lo; x <= hi; ++x) y += sums_all[far + x];
            } else {
                for (int x = lo; x <= hi; ++x) y += sums_all[far - x];
                if (u == 0 && !a.two_sided)
                    for (int x = 1; x <= far; ++x) y += sums_all[far + x];
            }
            out[u] = y;
        }
    }
}

// dK and dV: a workgroup has 128 keys of one key head, a wave 32 of them
template <typename T, int DP, bool BIAS>
__global__ __launch_bounds__(256, DP * sizeof(T) <= 128 ? 2 : 1) void attn_dkv_kernel(AttnArgs a)
{
    constexpr int QT = BWD_KEYS<T>, SUB = QT / 32;
    using Tl = Tile<T, DP, QT, 256>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    T *const qt = (T *)lds, *const gt = (T *)(lds + Tl::BYTES);
    float *const lse_t = (float *)(lds + 2 * Tl::BYTES), *const delta_t = lse_t + QT, *const bias = delta_t + QT;

    const unsigned w = xcd_order(blockIdx.x, gridDim.x);
    const int tile = (int)(w % a.tiles), bk = w / a.tiles, b = bk / a.Hkv, kv = bk - b * a.Hkv;
    const int t = threadIdx.x, wave = wave_of(t), lane = t & 63, col = lane & 31, h = lane >> 5;
    const AttnLens n(a, b);
    const int far = a.bk.far, j0 = tile * 128 + wave * 32, j = j0 + col;
    const bool ok = j < n.nk;
    Frag<T> k[DP / 16], v[DP / 16];
    {
        const T *const Kp = (const T *)a.K + b * a.ks[0] + kv * a.ks[2] + j * a.ks[1], *const Vp = (const T *)a.V + b * a.vs[0] + kv * a.vs[2] + j * a.vs[1];
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
            k[c] = row_frag_global(Kp, 16 * c, a.D, h, ok);
            v[c] = row_frag_global(Vp, 16 * c, a.D, h, ok);
        }
    }
    const float sl2 = a.scale * LOG2E;
    f32x16_t dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) dk[d] = dv[d] = f32x16_t{};

    // the first query that sees a key of the workgroup
    int begin = 0;
    if (a.causal) begin = clamped(tile * 128 - n.start, 0, a.Lq) / QT * QT;
    if (tile * 128 >= n.nk) begin = n.nq;
    const i64 qrow = (i64)a.Hq * a.D;
    const Tl qr(a.qs[1], a.D, t), gr(qrow, a.D, t);
    for (int g0 = 0; g0 < a.G; ++g0) {
        const int head = kv * a.G + g0;
        const T *const Qp = (const T *)a.Q + b * a.qs[0] + head * a.qs[2], *const Gp = (const T *)a.dO + ((i64)b * a.Lq * a.Hq + head) * a.D;
        const i64 stat = ((i64)b * a.Hq + head) * a.Lq;
        if (BIAS && begin < n.nq) {
            __syncthreads(); // (the last head's bias is not used any more)
            fill_bias(a, bias, head, t, 256);
        }
        for (int i0 = begin; i0 < n.nq; i0 += QT) {
            __syncthreads();
            qr.fetch(qt, Qp + (i64)i0 * a.qs[1], a.qs[1], n.nq - i0, a.D, wave);
            gr.fetch(gt, Gp + (i64)i0 * qrow, qrow, n.nq - i0, a.D, wave);
            if (t < QT) {
                const int i = i0 + t;
                const float x = i < n.nq ? a.lse_in[stat + i] : -INFINITY;
                lse_t[t] = x > -INFINITY ? x * LOG2E : INFINITY;
                delta_t[t] = i < n.nq ? a.delta[stat + i] : 0.f;
            }
            fetched();
            __syncthreads();
            if (j0 >= n.nk) continue;
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                const int p0 = i0 + 32 * u + n.start; // the position of the first row
                if (a.causal && p0 + 31 < j0) continue;
                const bool edge = j0 + 32 > n.nk || (a.causal && j0 + 31 > p0);
                const bool near = BIAS && j0 + 31 - p0 > -far && j0 - (p0 + 31) < far;
                const float flat = BIAS ? bias[j0 >= p0 ? 2 * far : 0] : 0.f;
                f32x16_t s = {}, dp = {};
                #pragma unroll
                for (int c = 0; c < DP / 16; ++c) {
                    mma(s, Tl::by_rows(qt, 32 * u, c, lane), k[c]);
                    mma(dp, Tl::by_rows(gt, 32 * u, c, lane), v[c]);
                }
                float p[16], ds[16];
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4) {
                    const float4 l4 = *(const float4 *)(lse_t + 32 * u + 8 * e4 + 4 * h);
                    const float ll[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
                    for (int x = 0; x < 4; ++x) p[4 * e4 + x] = ll[x];
                }
                if (edge || near) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int pos = p0 + 8 * (e >> 2) + 4 * h + (e & 3);
                        p[e] = exp2_fast(s[e] * sl2 + ((BIAS ? bias[clamped(j - pos, -far, far) + far] : 0.f) - p[e]));
                        if (j >= n.nk || (a.causal && j > pos)) p[e] = 0.f;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) p[e] = exp2_fast(s[e] * sl2 + (flat - p[e]));
                }
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4) {
                    const float4 d4 = *(const float4 *)(delta_t + 32 * u + 8 * e4 + 4 * h);
                    const float dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                    for (int x = 0; x < 4; ++x) ds[4 * e4 + x] = p[4 * e4 + x] * (dp[4 * e4 + x] - dd[x]);
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    Frag<T> f;
                    pack(p, c, f);
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) mma(dv[d], Tl::by_cols(gt, 32 * u + 16 * c, d, lane), f);
                    pack(ds, c, f);
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) mma(dk[d], Tl::by_cols(qt, 32 * u + 16 * c, d, lane), f);
                }
            }
        }
    }
    if (j >= a.Lk) return;
    const i64 at = (((i64)b * a.Lk + j) * a.Hkv + kv) * a.D;
    T *const ok_ = (T *)a.dK + at, *const ov = (T *)a.dV + at;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int c = 32 * d + 8 * (e >> 2) + 4 * h;
            if (c >= a.D) continue;
            put4(ok_ + c, dk[d][e] * a.scale, dk[d][e + 1] * a.scale, dk[d][e + 2] * a.scale, dk[d][e + 3] * a.scale);
            put4(ov + c, dv[d][e], dv[d][e + 1], dv[d][e + 2], dv[d][e + 3]);
        }
}

// dtable[u][head] from the workgroups' sums: one wave to a value, in double and always in one order
__global__ __launch_bounds__(64) void attn_table_kernel(const float *tab, int parts, int buckets, int heads, float *dtable, int accumulate)
{
    const int u = blockIdx.x % buckets, head = blockIdx.x / buckets, lane = threadIdx.x;
    double y = 0.0;
    for (int p = lane; p < parts; p += 64) y += (double)tab[((i64)head * parts + p) * buckets + u];
    for (int o = 32; o; o >>= 1) y += __shfl_xor(y, o);
    float *const out = dtable + (i64)u * heads + head;
    if (lane == 0) *out = accumulate ? *out + (float)y : (float)y;
}

// ------------------------------------------------------------------ host
template <typename T, int DP>
static int attn_bwd_launch(AttnArgs &a, float *dtable, int accumulate, hipStream_t s)
{
    const bool bias = a.buckets > 0, tab = bias && dtable;
    int st = PF_OK;
    a.tiles = (a.Lq + 127) / 128;
    const int parts = a.B * a.tiles;
    const dim3 grid((unsigned)a.B * a.Hq * a.tiles);
    const size_t lds = BwdLds<T, DP>::dq(a.bk.far, bias, tab);
    if (a.Lq > 0) {
        if (tab)
            PF_LAUNCH_LDS(st, "attn_dq_tab", (attn_dq_kernel<T, DP, true, true>), grid, dim3(256), lds, s, a);
        else if (bias)
            PF_LAUNCH_LDS(st, "attn_dq", (attn_dq_kernel<T, DP, true, false>), grid, dim3(256), lds, s, a);
        else
            PF_LAUNCH_LDS(st, "attn_dq", (attn_dq_kernel<T, DP, false, false>), grid, dim3(256), lds, s, a);
    }
    if (a.Lk > 0) {
        a.tiles = (a.Lk + 127) / 128;
        const dim3 kgrid((unsigned)a.B * a.Hkv * a.tiles);
        const size_t klds = BwdLds<T, DP>::dkv(a.bk.far, bias);
        if (bias)
            PF_LAUNCH_LDS(st, "attn_dkv", (attn_dkv_kernel<T, DP, true>), kgrid, dim3(256), klds, s, a);
        else
            PF_LAUNCH_LDS(st, "attn_dkv", (attn_dkv_kernel<T, DP, false>), kgrid, dim3(256), klds, s, a);
    }
    if (tab)
        PF_LAUNCH(st, "attn_table", attn_table_kernel, dim3((unsigned)a.buckets * a.Hq), dim3(64), s, a.tab, parts, a.buckets, a.Hq, dtable, accumulate);
    return st;
}
static size_t delta_bytes(const pf_attention_desc *d) { return align_up((size_t)d->B * d->heads_q * d->Lq * sizeof(float)); }

} // namespace pf

extern "C" {

using namespace pf;

size_t pf_attention_bwd_workspace_bytes(const pf_attention_desc *d)
{
    if (attn_check(d) != PF_OK || d->B == 0 || d->Lq == 0) return 0;
    return delta_bytes(d) + align_up((size_t)d->heads_q * d->B * ((d->Lq + 127) / 128) * d->buckets * sizeof(float));
}

int pf_attention_bwd(const pf_attention_desc *d, const void *Q, const void *K, const void *V, const void *table, const void *q_start,
                     const void *q_len, const void *kv_len, const void *O, const void *lse, const void *dO, void *dQ, void *dK, void *dV,
                     void *dtable, int accumulate, void *workspace, size_t workspace_bytes, void *stream)
{
    const int status = attn_check(d);
    if (status != PF_OK) return status;
    if (any_misaligned({table, q_start, q_len, kv_len, lse, dtable}, 4)) return PF_ERR_UNSUPPORTED;
    const hipStream_t s = (hipStream_t)stream;
    if (d->B == 0) {
        if (!dtable || !d->buckets || accumulate) return PF_OK;
        return launch_zero_f32(s, (float *)dtable, (i64)d->buckets * d->heads_q);
    }
    if ((d->Lq && (!Q || !O || !lse || !dO || !dQ)) || (d->Lk && (!K || !V || !dK || !dV)) || (d->buckets && !table)) return PF_ERR_NULL;
    for (const void *p : {Q, O, dO, (const void *)dQ})
        if (d->Lq && any_misaligned({p}, 16)) return PF_ERR_UNSUPPORTED;
    for (const void *p : {K, V, (const void *)dK, (const void *)dV})
        if (d->Lk && any_misaligned({p}, 16)) return PF_ERR_UNSUPPORTED;
    if (any_misaligned({workspace}, 256)) return PF_ERR_UNSUPPORTED;
    const size_t need = pf_attention_bwd_workspace_bytes(d);
    if (need && (!workspace || workspace_bytes < need)) return PF_ERR_WORKSPACE;
    AttnArgs a = {};
    attn_fill(d, a);
    a.Q = Q, a.K = K, a.V = V, a.Oin = O, a.dO = dO, a.dQ = dQ, a.dK = dK, a.dV = dV;
    a.table = (const float *)table;
    a.lse_in = (const float *)lse;
    a.q_start = (const int *)q_start;
    a.q_len = (const int *)q_len;
    a.kv_len = (const int *)kv_len;
    a.delta = (float *)workspace;
    a.tab = (float *)((char *)workspace + delta_bytes(d));
    const int DP = (a.D + 31) / 32 * 32;
    float *const dt = d->buckets ? (float *)dtable : nullptr;
    if (d->dtype == PF_BF16)
        return DP == 32 ? attn_bwd_launch<bf16_t, 32>(a, dt, accumulate, s) : DP == 64 ? attn_bwd_launch<bf16_t, 64>(a, dt, accumulate, s)
             : DP == 96 ? attn_bwd_launch<bf16_t, 96>(a, dt, accumulate, s) : attn_bwd_launch<bf16_t, 128>(a, dt, accumulate, s);
    return DP == 32 ? attn_bwd_launch<float, 32>(a, dt, accumulate, s) : DP == 64 ? attn_bwd_launch<float, 64>(a, dt, accumulate, s)
         : DP == 96 ? attn_bwd_launch<float, 96>(a, dt, accumulate, s) : attn_bwd_launch<float, 128>(a, dt, accumulate, s);
}

} // extern "C"
