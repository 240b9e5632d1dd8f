// Attention with a relative position bias by buckets, forward: pf_attention_fwd.
//
// A workgroup has 128 queries of one head, a wave 32 of them in its columns (pf_attn.h); keys and values pass through LDS
// in tiles, the next ones on their way while this one is used.  Where that makes too few workgroups, it has 64, and two waves
// share their queries, each with half of the keys of a tile.  One pass over the keys with the running maximum and
// sum of each query; the score matrix, the bias and P exist in registers only.
//
// Bound by the vector work of a tile beside its products: 2 x 4096 tokens of 16 heads of 128, causal, take 155 us, with the matrix unit
// busy 45 % of the time.  64 x 128 padded tokens of 8 heads of 64 take 12: launch, first loads and one or two tiles.
#include "pf_attn.h"

namespace pf {

template <typename T>
constexpr int KEYS = sizeof(T) == 2 ? 64 : 32; // keys of a tile

// One tile of queries.  A turn of the loop has the scores of its keys in registers; their exponentials are worked out while
// the matrix unit makes the next turn's scores, and the largest of those is found while it multiplies P and V.
// KW: waves that share queries.
template <typename T, int DP, bool BIAS, int KW>
__device__ __forceinline__ void attn_fwd_tile(const AttnArgs &a, char *lds, int b, int head, int tile)
{
    constexpr int KT = KEYS<T>, SUB = KT / 32, STEP = KT * KW, QUERIES = 128 / KW; // a wave's keys of a tile; all; the workgroup's queries
    using Tl = Tile<T, DP, STEP, 256>;
    T *const kb = (T *)lds, *const vb = kb + 2 * Tl::SIZE; // two tiles of keys, two of values
    float *const bias = (float *)(lds + 4 * Tl::BYTES);

    const int t = threadIdx.x, wave = wave_of(t), lane = t & 63, col = lane & 31, h = lane >> 5;
    const AttnLens n(a, b);
    const int kw = wave % KW, own = KT * kw;                           // the wave's keys begin there in a tile
    const int i0 = tile * QUERIES + wave / KW * 32, i = i0 + col; // the lane's query
    const bool ok = i < n.nq;

    const T *const Kp = (const T *)a.K + b * a.ks[0] + head / a.G * a.ks[2], *const Vp = (const T *)a.V + b * a.vs[0] + head / a.G * a.vs[2];
    // keys that some query of the workgroup sees, and that some query of the wave sees
    int keys = n.nk;
    if (tile * QUERIES >= n.nq) keys = 0;
    const int block_last = (tile * QUERIES + QUERIES < n.nq ? tile * QUERIES + QUERIES : n.nq) - 1 + n.start; // positions
    if (a.causal && block_last + 1 < keys) keys = block_last + 1 < 0 ? 0 : block_last + 1;
    const int last = (i0 + 32 < n.nq ? i0 + 32 : n.nq) - 1, pmin = i0 + n.start, pmax = last + n.start, pos = i + n.start;
    const int most = a.causal && n.nk > pos ? 0 : n.nk - 1 - pos; // the furthest distance seen
    int mine = i0 >= n.nq ? 0 : keys;
    if (a.causal && mine > 0 && pmax + 1 < mine) mine = pmax + 1 < 0 ? 0 : pmax + 1;

    const Tl kl(a.ks[1], a.D, t), vl(a.vs[1], a.D, t);
    const auto fetch_keys = [&](int k0, int odd) { kl.fetch(kb + odd * Tl::SIZE, Kp + (i64)k0 * a.ks[1], a.ks[1], keys - k0, a.D, wave); };
    const auto fetch_values = [&](int k0, int odd) { vl.fetch(vb + odd * Tl::SIZE, Vp + (i64)k0 * a.vs[1], a.vs[1], keys - k0, a.D, wave); };
    if (keys > 0) {
        fetch_keys(0, 0);
        fetch_values(0, 0);
        if (keys > STEP) fetch_keys(STEP, 1);
    }
    Frag<T> q[DP / 16];
    {
        const T *const Qp = (const T *)a.Q + b * a.qs[0] + head * a.qs[2] + i * a.qs[1];
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) q[c] = row_frag_global(Qp, 16 * c, a.D, h, ok);
    }
    __shared__ int large[4];
    if (BIAS && keys > 0) leave(large, fill_bias(a, bias, head, t, 256), wave, lane); // (behind the loads that it need not wait for)
    const float sl2 = a.scale * LOG2E;
    const int far = a.bk.far;
    f32x16_t o[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) o[d] = f32x16_t{};
    float m = -INFINITY, sum = 0.f; // the maximum that values are taken relative to (base 2); the sum of the lane's keys
    float top = -INFINITY;
    f32x16_t s0[SUB], s1[SUB];
    const int rows = Tl::row_place(lane) + own * Tl::RB, cols = Tl::col_place(lane) + own * Tl::RB; // (turn() repeats after 16 rows)
    constexpr int CH = DP / 16, SC = SUB * CH, DB = DP / 32, PV = 2 * SUB * DB, AHEAD = 3;
    fetched();
    __syncthreads();
    float shift = 0.f; // what the row's biases, and its maximum, are relative to
    if (BIAS && keys > 0 && __builtin_expect(left(large, 4), 0)) shift = row_shift(-pos, most, far, [&](int x) { return bias[far + x]; });
    if (own < mine) {
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            s0[u] = f32x16_t{};
#pragma unroll
            for (int c = 0; c < CH; ++c) mma(s0[u], Tl::by_rows(lds, rows, 32 * u, c), q[c]);
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s0[u][e]);
        }
    }
    __syncthreads();
    // the tile from key t0 on with the scores of the wave's keys in s; `odd`: which of the two places it is in
    const auto turn = [&](int t0, int odd, f32x16_t (&s)[SUB], f32x16_t (&next)[SUB]) {
        if (t0 + 2 * STEP < keys) fetch_keys(t0 + 2 * STEP, odd);
        if (t0 + STEP < keys) fetch_values(t0 + STEP, !odd);
        const int k0 = t0 + own;
        if (k0 < mine) {
            const bool edge = k0 + KT > n.nk || (a.causal && k0 + KT - 1 > pmin);
            const bool near = BIAS && k0 + KT - 1 - pmin > -far && k0 - pmax < far;
            const float flat = BIAS ? bias[k0 >= pmin ? 2 * far : 0] - shift : 0.f; // where no key is near
            // Away from the edges and the near keys, nothing is done to a product but one fused multiply-add on its way into
            // the exponential; the maximum is that of the products themselves.
            const bool plain = !edge && !near && sl2 > 0.f;
            if (plain) {
                top = top * sl2 + flat;
            } else {
                top = -INFINITY;
                const int rel = anew(k0 + 4 * h - pos); // distance of the first key that the lane holds
#pragma unroll
                for (int u = 0; u < SUB; ++u) {
                    finish_scores<BIAS>(s[u], sl2, shift, bias, far, rel + 32 * u, 1, most);
#pragma unroll
                    for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
                }
            }
            top = fmaxf(top, __shfl_xor(top, 32));
            // The maximum that values are taken relative to follows only when it is left by 2^8: sums and rounded P lose
            // nothing to a common factor, and most tiles spare the products their rescaling.
            if (__any(top > m + 8.f)) {
                const float m_new = fmaxf(m, top), f = exp2_fast(m - (m_new == -INFINITY ? 0.f : m_new));
                sum *= f;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[d][e] *= f;
                m = m_new;
            }
            const float base = m == -INFINITY ? 0.f : m, mul = plain ? sl2 : 1.f, add = plain ? flat - base : -base;
            // The order of what follows is fixed step by step: a step is one product, the read of the operand of the product
            // AHEAD steps on, and a share of the vector instructions.
            Frag<T> p[2 * SUB], ring[AHEAD + 1];
            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < SUB; ++u) next[u] = f32x16_t{};
            __builtin_amdgcn_sched_barrier(0);
            // the next keys' scores (of whatever lies there, after the last) beside this tile's exponentials
            const int ka = rows + (odd ? 0 : Tl::BYTES), va = cols + 2 * Tl::BYTES + (odd ? Tl::BYTES : 0);
            const auto operand = [&](int x) {
                return x < SC ? Tl::by_rows(lds, ka, 32 * (x / CH), x % CH) : Tl::by_cols(lds, va, 16 * ((x - SC) / DB), (x - SC) % DB);
            };
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) ring[x] = operand(x);
#pragma unroll
            for (int x = 0; x < SC; ++x) {
                ring[(x + AHEAD) % (AHEAD + 1)] = operand(x + AHEAD);
                mma(next[x / CH], ring[x % (AHEAD + 1)], q[x % CH]);
#pragma unroll
                for (int y = x * (16 * SUB) / SC; y < (x + 1) * (16 * SUB) / SC; ++y) {
                    const float z = exp2_fast(s[y / 16][y % 16] * mul + add);
                    s[y / 16][y % 16] = z;
                    part[y & 3] += z;
                    if (y % 8 == 7) pack(s[y / 16], y % 16 / 8, p[y / 8]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // P and V beside the largest of the next scores
            top = -INFINITY;
#pragma unroll
            for (int x = 0; x < PV; ++x) {
                if (x + AHEAD < PV) ring[(SC + x + AHEAD) % (AHEAD + 1)] = operand(SC + x + AHEAD);
                mma(o[x % DB], ring[(SC + x) % (AHEAD + 1)], p[x / DB]);
#pragma unroll
                for (int y = x * (16 * SUB) / PV; y < (x + 1) * (16 * SUB) / PV; ++y) top = fmaxf(top, next[y / 16][y % 16]);
                __builtin_amdgcn_sched_barrier(0);
            }
            sum += (part[0] + part[1]) + (part[2] + part[3]);
        }
        fetched();
        __syncthreads();
    };
    for (int t0 = 0; t0 < keys; t0 += 2 * STEP) {
        turn(t0, 0, s0, s1);
        if (t0 + STEP < keys) turn(t0 + STEP, 1, s1, s0);
    }
    sum += __shfl_xor(sum, 32);
    if constexpr (KW == 2) { // the second wave's part to the first (the loop ended with a barrier: the tiles' room is free)
        float *const part = (float *)lds + wave / KW * (DP / 2 + 2) * 64 + lane;
        if (kw == 1) {
            part[0] = m, part[64] = sum;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) part[(2 + 16 * d + e) * 64] = o[d][e];
        }
        __syncthreads();
        if (kw == 1) return;
        const float m1 = part[0], both = fmaxf(m, m1), base = both == -INFINITY ? 0.f : both;
        const float f = exp2_fast(m - base), f1 = exp2_fast(m1 - base);
        sum = sum * f + part[64] * f1;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[d][e] = o[d][e] * f + part[(2 + 16 * d + e) * 64] * f1;
        m = both;
    }
    if (i >= a.Lq) return;
    const bool some = ok && sum != 0.f;
    const float inv = some ? 1.f / sum : 0.f;
    T *const Op = (T *)a.O + (((i64)b * a.Lq + i) * a.Hq + head) * a.D;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int c = 32 * d + 8 * (e >> 2) + 4 * h;
            float v[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = some ? o[d][e + x] * inv : 0.f;
            if (c < a.D) put4(Op + c, v[0], v[1], v[2], v[3]);
        }
    if (a.lse && h == 0) a.lse[((i64)b * a.Hq + head) * a.Lq + i] = some ? (m + __builtin_amdgcn_logf(sum)) * LN2 + shift * LN2 : -INFINITY;
}

// paired: a workgroup has a long tile of queries and a short one (causal; a.tiles of them to a head), so that all take the
// same time
template <typename T, int DP, bool BIAS, int KW>
__global__ __launch_bounds__(256, sizeof(T) == 4 && DP > 64 ? 1 : 2) void attn_fwd_kernel(AttnArgs a, int paired)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const unsigned w = xcd_order(blockIdx.x, gridDim.x);
    const int each = paired ? (a.tiles + 1) / 2 : a.tiles, k = (int)(w % each), bh = w / each, b = bh / a.Hq, head = bh - b * a.Hq;
    const int other = paired && a.tiles - 1 - k != k ? 2 : 1;
#pragma unroll 1
    for (int pass = 0; pass < other; ++pass) {
        attn_fwd_tile<T, DP, BIAS, KW>(a, lds, b, head, pass ? k : a.tiles - 1 - k);
        __syncthreads();
    }
}

// ------------------------------------------------------------------ host
static bool strides_ok(const int64_t *s, int unit)
{
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || s[i] % unit) return false;
    return true;
}
static void strides_of(const int64_t *s, i64 L, int heads, int D, i64 (&out)[3])
{
    const bool dense = !s[0] && !s[1] && !s[2];
    out[2] = dense ? D : s[2];
    out[1] = dense ? (i64)heads * D : s[1];
    out[0] = dense ? L * heads * D : s[0];
}

int attn_check(const pf_attention_desc *d)
{
    if (!d) return PF_ERR_NULL;
    if (d->B < 0 || d->Lq < 0 || d->Lk < 0 || d->heads_q <= 0 || d->heads_kv <= 0 || d->head_dim <= 0) return PF_ERR_SHAPE;
    if (d->heads_q % d->heads_kv) return PF_ERR_SHAPE;
    if (d->dtype != PF_F32 && d->dtype != PF_BF16) return PF_ERR_UNSUPPORTED;
    if (d->head_dim % 8 || d->head_dim > 128) return PF_ERR_UNSUPPORTED;
    if (!isfinite(d->scale)) return PF_ERR_UNSUPPORTED;
    if (d->Lq >= 1 << 29 || d->Lk >= 1 << 29 || d->B > INT32_MAX / d->heads_q) return PF_ERR_UNSUPPORTED;
    // workgroups of 32 rows or keys at the least are counted in 32 bits
    if (d->B * d->heads_q > INT32_MAX / ((d->Lq + 31) / 32 + 1) || d->B * d->heads_kv > INT32_MAX / ((d->Lk + 31) / 32 + 1)) return PF_ERR_UNSUPPORTED;
    if (d->buckets) {
        const int side = d->bidirectional ? d->buckets / 2 : d->buckets;
        if (d->buckets < 0 || d->buckets > ATTN_MAX_BUCKETS || side < 2 || (d->bidirectional && d->buckets % 2)) return PF_ERR_UNSUPPORTED;
        if (d->max_distance <= side / 2 || d->max_distance > ATTN_MAX_DISTANCE) return PF_ERR_UNSUPPORTED;
    }
    const int unit = 16 / (d->dtype == PF_BF16 ? 2 : 4);
    if (!strides_ok(d->q_stride, unit) || !strides_ok(d->k_stride, unit) || !strides_ok(d->v_stride, unit)) return PF_ERR_UNSUPPORTED;
    // a tile of tokens is read through one descriptor, with offsets of 31 bits
    const i64 q = (i64)d->heads_q * d->head_dim, k = (i64)d->heads_kv * d->head_dim, most = ATTN_MAX_STRIDE - d->head_dim;
    if (q > most || k > most || d->q_stride[1] > most || d->k_stride[1] > most || d->v_stride[1] > most) return PF_ERR_UNSUPPORTED;
    return PF_OK;
}

void attn_fill(const pf_attention_desc *d, AttnArgs &a)
{
    a.B = (int)d->B, a.Lq = (int)d->Lq, a.Lk = (int)d->Lk;
    a.Hq = d->heads_q, a.Hkv = d->heads_kv, a.G = d->heads_q / d->heads_kv, a.D = d->head_dim;
    a.causal = d->causal != 0;
    a.buckets = d->buckets;
    a.two_sided = d->bidirectional != 0;
    a.scale = d->scale;
    strides_of(d->q_stride, d->Lq, d->heads_q, d->head_dim, a.qs);
    strides_of(d->k_stride, d->Lk, d->heads_kv, d->head_dim, a.ks);
    strides_of(d->v_stride, d->Lk, d->heads_kv, d->head_dim, a.vs);
    if (d->buckets) { // (a model has one bias: its borders are worked out once)
        static thread_local struct {
            int side, distance;
            AttnBuckets b;
        } known = {};
        const int side = d->bidirectional ? d->buckets / 2 : d->buckets;
        if (known.side != side || known.distance != d->max_distance) known = {side, d->max_distance, attn_buckets(side, d->max_distance)};
        a.bk = known.b;
    }
}

template <typename T, int DP, int KW>
static int attn_fwd_launch(AttnArgs &a, hipStream_t s)
{
    using Tl = Tile<T, DP, KEYS<T> * KW, 256>;
    a.tiles = (a.Lq + 128 / KW - 1) / (128 / KW);
    // two workgroups to a compute unit are resident: causal tiles are paired where there are more
    const bool paired = a.causal && (i64)a.B * a.Hq * a.tiles > 512;
    const unsigned blocks = (unsigned)a.B * a.Hq * (paired ? (a.tiles + 1) / 2 : a.tiles);
    if (too_many(blocks, 256)) return PF_ERR_UNSUPPORTED;
    const size_t lds = 4 * Tl::BYTES + (a.buckets ? (2 * a.bk.far + 1) * sizeof(float) : 0);
    int st = PF_OK;
    if (a.buckets)
        PF_LAUNCH_LDS(st, "attn_fwd", (attn_fwd_kernel<T, DP, true, KW>), dim3(blocks), dim3(256), lds, s, a, (int)paired);
    else
        PF_LAUNCH_LDS(st, "attn_fwd", (attn_fwd_kernel<T, DP, false, KW>), dim3(blocks), dim3(256), lds, s, a, (int)paired);
    return st;
}
// Two waves share queries where that makes no more workgroups than fit the card at once, two to a compute unit if the tiles of
// both fit its LDS (us, bf16, 8 heads: 2 x 1024 tokens of 64 columns, 128 tiles, 25 alone and 18 shared; 4 x 1024, 256 tiles,
// 26 and 23; 6 x 1024 34 and 33; 512 queries of 32 heads of 128 over 4096 keys, 128 tiles, 80 and 54; twice those 84 and 104; float,
// B x 512 tokens of 8 heads of 64: 128 tiles 49 and 29, 256 50 and 47, 512 83 and 90; of 128: 128 tiles 87 and 52, 256 89 and 101.  Of
// 320 tiles, which fill the card once and a quarter, shared ones are the faster in float, 82 and 70: not taken)
template <typename T, int DP>
static int attn_fwd_launch(AttnArgs &a, hipStream_t s)
{
    const bool few = (i64)a.B * a.Hq * ((a.Lq + 127) / 128) <= (DP <= 64 ? 256 : 128);
    return few ? attn_fwd_launch<T, DP, 2>(a, s) : attn_fwd_launch<T, DP, 1>(a, s);
}

} // namespace pf

extern "C" {

using namespace pf;

size_t pf_attention_fwd_workspace_bytes(const pf_attention_desc *d)
{
    if (attn_check(d) != PF_OK || d->B == 0 || d->Lq == 0) return 0;
    return attn_split_bytes(d);
}

int pf_attention_fwd(const pf_attention_desc *d, const void *Q, const void *K, const void *V, const void *table, const void *q_start,
                     const void *q_len, const void *kv_len, void *O, void *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    const int status = attn_check(d);
    if (status != PF_OK) return status;
    if (d->B == 0 || d->Lq == 0) return PF_OK;
    if (!Q || !O || (d->Lk && (!K || !V)) || (d->buckets && !table)) return PF_ERR_NULL;
    if (any_misaligned({Q, O, d->Lk ? K : nullptr, d->Lk ? V : nullptr}, 16) || any_misaligned({table, q_start, q_len, kv_len, lse}, 4) ||
        any_misaligned({workspace}, 256))
        return PF_ERR_UNSUPPORTED;
    const size_t need = attn_split_bytes(d);
    if (need && (!workspace || workspace_bytes < need)) return PF_ERR_WORKSPACE;
    AttnArgs a = {};
    attn_fill(d, a);
    const AttnAreas of{d, a};
    if (outputs_meet({of.dense_queries(O), of.rows(lse)}, {of.queries(Q), of.keys(K, a.ks), of.keys(V, a.vs), of.table(table)})) return PF_ERR_UNSUPPORTED;
    a.Q = Q, a.K = K, a.V = V, a.O = O;
    a.table = (const float *)table;
    a.lse = (float *)lse;
    a.q_start = (const int *)q_start;
    a.q_len = (const int *)q_len;
    a.kv_len = (const int *)kv_len;
    if (attn_split_count(d)) return attn_split_fwd(d, a, workspace, (hipStream_t)stream);
    const hipStream_t s = (hipStream_t)stream;
    const int DP = (a.D + 31) / 32 * 32;
    if (d->dtype == PF_BF16)
        return DP == 32 ? attn_fwd_launch<bf16_t, 32>(a, s) : DP == 64 ? attn_fwd_launch<bf16_t, 64>(a, s)
             : DP == 96 ? attn_fwd_launch<bf16_t, 96>(a, s) : attn_fwd_launch<bf16_t, 128>(a, s);
    return DP == 32 ? attn_fwd_launch<float, 32>(a, s) : DP == 64 ? attn_fwd_launch<float, 64>(a, s)
         : DP == 96 ? attn_fwd_launch<float, 96>(a, s) : attn_fwd_launch<float, 128>(a, s);
}

} // extern "C"
