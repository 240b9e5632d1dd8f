// One AdamW step over many tensors: pf_adamw_*.
//
// Every value is read and written once (28 bytes with 32-bit states, 16 with 8-bit ones, 2 more for a bf16 copy), so the
// step is bound by memory.  One launch takes all tensors: a table in device memory says which piece of which
// tensor a workgroup has.  A wave takes 256 consecutive values at a time, four per lane: they are the values that share a scale
// when states have 8 bits, so that a scale is a maximum over one wave's registers and nothing is read twice.
// 7.1 M values of six Transformer layers' factors with bf16 copies take 45.7 us at 32 bits, 61 M of a language model 212 us at 8: 4.6 to 4.7
// TB/s, what a copy reaches.
#include <string.h>

#include "pf_common.h"

namespace pf {

constexpr int ADAMW_CHUNK = 4096; // values of a workgroup: four rounds of its four waves
constexpr int ADAMW_BLOCK = 256;  // values that share a scale

struct AdamwHead {
    unsigned done; // workgroups of the running launch that have read `steps`
    unsigned pad[63];
};
struct AdamwTensor {
    float *p;
    const float *g;
    void *m, *v;
    float *ms, *vs;
    uint16_t *copy;
    i64 n;
    float wd;
    float pad;
};
struct AdamwChunk {
    unsigned tensor, index; // values index * ADAMW_CHUNK .. of that tensor
};
struct AdamwArgs {
    AdamwHead *head;
    const AdamwTensor *tensors;
    const AdamwChunk *chunks;
    const float *lr, *scale;
    i64 *steps;
    double beta1, beta2;
    float b1, b1c, b2, b2c, eps; // b1c = 1 - beta1, rounded once from double
};

typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));       // (4-byte aligned 16-byte accesses)
typedef uint16_t h4_any __attribute__((ext_vector_type(4), aligned(2)));

// The largest of the lanes' values in every lane
__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
    return x;
}

// The smallest power of two from 2^-126 on with top / scale <= 448 = 7/8 2^9, top finite and not negative
__device__ __forceinline__ float scale_of(float top)
{
    const uint32_t u = __float_as_uint(top);
    int e = (int)(u >> 23) - ((u & 0x7fffff) > 0x600000 ? 7 : 8); // biased; a subnormal top has e < 1
    if (e < 1) e = 1;
    return __uint_as_float((uint32_t)e << 23);
}
// 1 / scale, a power of two as well (scale <= 2^120, so that it is no subnormal)
__device__ __forceinline__ float inverse_of(float scale) { return __uint_as_float(0x7f000000u - __float_as_uint(scale)); }

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// Four values as e4m3 codes (nearest even); what is not finite becomes NaN
__device__ __forceinline__ uint32_t encode4(const float (&x)[4])
{
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
    uint32_t c = (uint32_t)w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (!finite(x[i])) c |= 0x7fu << (8 * i);
    return c;
}
__device__ __forceinline__ void decode4(uint32_t c, float (&x)[4])
{
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8((int)c, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)c, 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8((int)c, 3);
}

// x^n by squaring, in double: 1 - beta^t needs the digits, and a power function costs more than a workgroup's values
__device__ __forceinline__ double power(double x, i64 n)
{
    double r = 1.0;
    for (; n > 0; n >>= 1, x *= x)
        if (n & 1) r *= x;
    return r;
}

// ALL: the four values exist (else `n` of them)
template <bool ALL>
__device__ __forceinline__ void get4(const float *p, int n, float (&x)[4])
{
    if constexpr (ALL) {
        const f4_any v = *(const f4_any *)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i < n ? p[i] : 0.f;
    }
}
template <bool ALL>
__device__ __forceinline__ void put4(float *p, int n, const float (&x)[4])
{
    if constexpr (ALL) {
        const f4_any v = {x[0], x[1], x[2], x[3]};
        *(f4_any *)p = v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = x[i];
    }
}
template <bool ALL>
__device__ __forceinline__ uint32_t get_codes(const uint8_t *p, int n)
{
    if constexpr (ALL) return *(const uint32_t *)p;
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) c |= (uint32_t)p[i] << (8 * i);
    return c;
}
template <bool ALL>
__device__ __forceinline__ void put_codes(uint8_t *p, int n, uint32_t c)
{
    if constexpr (ALL) {
        *(uint32_t *)p = c;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = (uint8_t)(c >> (8 * i));
    }
}

// The values at .. at + 3 of tensor t in one lane, `n` of which exist; all 64 lanes of a wave come here together.
// Products and sums are rounded one by one (no fused multiply-add), as the formulas in the header have them: a state that
// is stored in 8 bits then does not depend on how the compiler pairs them.
template <int BITS, bool ALL>
__device__ __forceinline__ void adamw_four(const AdamwArgs &a, const AdamwTensor &t, i64 at, int n, float grad_scale, float keep, float step,
                                           float root)
{
#pragma clang fp contract(off)
    float p[4], g[4], m[4], v[4], r[4];
    const int lane = threadIdx.x & 63;
    if constexpr (ALL) n = 4;
    get4<ALL>(t.p + at, n, p);
    get4<ALL>(t.g + at, n, g);
    if constexpr (BITS == 32) {
        get4<ALL>((const float *)t.m + at, n, m);
        get4<ALL>((const float *)t.v + at, n, v);
    } else {
        const float ms = t.ms[at / ADAMW_BLOCK], vs = t.vs[at / ADAMW_BLOCK]; // (the wave's: its lanes have one block)
        decode4(get_codes<ALL>((const uint8_t *)t.m + at, n), m);
        decode4(get_codes<ALL>((const uint8_t *)t.v + at, n), v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = m[i] * ms;
            v[i] = v[i] * vs;
            v[i] = v[i] * v[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (a.scale) g[i] = g[i] * grad_scale;
        m[i] = a.b1 * m[i] + a.b1c * g[i];
        v[i] = a.b2 * v[i] + a.b2c * (g[i] * g[i]);
        r[i] = __builtin_sqrtf(v[i]);
        p[i] = p[i] * keep - step * (m[i] / (r[i] / root + a.eps));
    }
    put4<ALL>(t.p + at, n, p);
    if (t.copy) {
        if constexpr (ALL) {
            const uint32_t lo = pack_bf16x2(p[0], p[1]), hi = pack_bf16x2(p[2], p[3]);
            const h4_any c = {(uint16_t)lo, (uint16_t)(lo >> 16), (uint16_t)hi, (uint16_t)(hi >> 16)};
            *(h4_any *)(t.copy + at) = c;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) t.copy[at + i] = float_to_bf16_bits(p[i]);
        }
    }
    if constexpr (BITS == 32) {
        put4<ALL>((float *)t.m + at, n, m);
        put4<ALL>((float *)t.v + at, n, v);
    } else {
        float mt = 0.f, rt = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i < n && finite(m[i])) mt = fmaxf(mt, fabsf(m[i]));
            if (i < n && finite(r[i])) rt = fmaxf(rt, r[i]);
        }
        const float ms = scale_of(wave_max(mt)), vs = scale_of(wave_max(rt));
        const float mi = inverse_of(ms), vi = inverse_of(vs);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = m[i] * mi; // (exact: powers of two)
            r[i] = r[i] * vi;
            if (r[i] > 0.f) r[i] = fmaxf(r[i], 0x1p-9f); // the smallest code: m divided by a zero root would leap
        }
        put_codes<ALL>((uint8_t *)t.m + at, n, encode4(m));
        put_codes<ALL>((uint8_t *)t.v + at, n, encode4(r));
        if (lane == 0) {
            t.ms[at / ADAMW_BLOCK] = ms;
            t.vs[at / ADAMW_BLOCK] = vs;
        }
    }
}

template <int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwArgs a, unsigned chunks)
{
    const i64 t = *a.steps + 1;
    const double c1 = 1.0 - power(a.beta1, t), c2 = 1.0 - power(a.beta2, t);
    const float lr = *a.lr, step = (float)((double)lr / c1), root = (float)sqrt(c2);
    const float grad_scale = a.scale ? *a.scale : 1.f;
    if (blockIdx.x < chunks) {
        const AdamwChunk c = a.chunks[blockIdx.x];
        const AdamwTensor q = a.tensors[c.tensor];
        const float keep = (float)(1.0 - (double)lr * (double)q.wd);
        const i64 first = (i64)c.index * ADAMW_CHUNK;
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        for (int k = 0; k < ADAMW_CHUNK / 1024; ++k) {
            const i64 base = first + k * 1024 + wave * ADAMW_BLOCK, at = base + lane * 4;
            if (base >= q.n) break;
            if (base + ADAMW_BLOCK <= q.n)
                adamw_four<BITS, true>(a, q, at, 4, grad_scale, keep, step, root);
            else
                adamw_four<BITS, false>(a, q, at, (int)(q.n - at < 0 ? 0 : q.n - at > 4 ? 4 : q.n - at), grad_scale, keep, step, root);
        }
    }
    // The last workgroup to come here stores the step's number: all others have used theirs.
    __syncthreads();
    if (threadIdx.x == 0) {
        if (atomicAdd(&a.head->done, 1u) == gridDim.x - 1) {
            a.head->done = 0;
            *a.steps = t;
        }
    }
}

static int adamw_check(const pf_adamw_desc *d, const pf_adamw_tensor *q)
{
    if (!d || (!q && d->tensors > 0)) return PF_ERR_NULL;
    if (d->tensors < 0 || d->tensors > (1 << 24)) return PF_ERR_SHAPE;
    if (d->state_bits != 32 && d->state_bits != 8) return PF_ERR_UNSUPPORTED;
    if (!(d->beta1 >= 0 && d->beta1 < 1 && d->beta2 >= 0 && d->beta2 < 1 && d->eps >= 0)) return PF_ERR_UNSUPPORTED;
    i64 chunks = 0;
    for (i64 i = 0; q && i < d->tensors; ++i) {
        if (q[i].count < 0) return PF_ERR_SHAPE;
        chunks += (q[i].count + ADAMW_CHUNK - 1) / ADAMW_CHUNK;
        if (q[i].count == 0) continue;
        if (chunks >= (i64)1 << 31) return PF_ERR_SHAPE;
        if (!q[i].param || !q[i].grad || !q[i].m || !q[i].v) return PF_ERR_NULL;
        if (d->state_bits == 8 && (!q[i].m_scale || !q[i].v_scale)) return PF_ERR_NULL;
        if (any_misaligned({q[i].param, q[i].grad, q[i].m, q[i].v}, 4) || any_misaligned({q[i].copy}, 2)) return PF_ERR_UNSUPPORTED;
        if (d->state_bits == 8 && any_misaligned({q[i].m_scale, q[i].v_scale}, 4)) return PF_ERR_UNSUPPORTED;
    }
    return PF_OK;
}
static i64 adamw_chunks(const pf_adamw_desc *d, const pf_adamw_tensor *q)
{
    i64 n = 0;
    for (i64 i = 0; i < d->tensors; ++i) n += (q[i].count + ADAMW_CHUNK - 1) / ADAMW_CHUNK;
    return n;
}
// (records and pieces are multiples of 8 bytes: 4 bytes more tell a plan for 8-bit states, which a step must not take for the other)
static size_t adamw_bytes(i64 tensors, i64 chunks, int bits)
{
    return sizeof(AdamwHead) + sizeof(AdamwTensor) * (size_t)tensors + sizeof(AdamwChunk) * (size_t)chunks + (bits == 8 ? 4 : 0);
}

} // namespace pf

extern "C" {

using namespace pf;

size_t pf_adamw_plan_bytes(const pf_adamw_desc *d, const pf_adamw_tensor *tensors)
{
    if (adamw_check(d, tensors) != PF_OK) return 0;
    return adamw_bytes(d->tensors, adamw_chunks(d, tensors), d->state_bits);
}

int pf_adamw_plan_fill(const pf_adamw_desc *d, const pf_adamw_tensor *tensors, void *plan_host, size_t plan_bytes)
{
    const int status = adamw_check(d, tensors);
    if (status != PF_OK) return status;
    if (!plan_host || plan_bytes < adamw_bytes(d->tensors, adamw_chunks(d, tensors), d->state_bits)) return PF_ERR_WORKSPACE;
    char *p = (char *)plan_host;
    memset(p, 0, sizeof(AdamwHead));
    p += sizeof(AdamwHead);
    for (i64 i = 0; i < d->tensors; ++i, p += sizeof(AdamwTensor)) {
        const pf_adamw_tensor &q = tensors[i];
        const bool small = d->state_bits == 8;
        const AdamwTensor t = {(float *)q.param, (const float *)q.grad, q.m, q.v, small ? (float *)q.m_scale : nullptr,
                               small ? (float *)q.v_scale : nullptr, (uint16_t *)q.copy, q.count, q.weight_decay, 0.f};
        memcpy(p, &t, sizeof t);
    }
    for (i64 i = 0; i < d->tensors; ++i)
        for (i64 k = 0; k * ADAMW_CHUNK < tensors[i].count; ++k, p += sizeof(AdamwChunk)) {
            const AdamwChunk c = {(unsigned)i, (unsigned)k};
            memcpy(p, &c, sizeof c);
        }
    return PF_OK;
}

int pf_adamw_step(const pf_adamw_desc *d, void *plan, size_t plan_bytes, const void *lr, const void *grad_scale, void *steps, void *stream)
{
    if (!d || !lr || !steps) return PF_ERR_NULL;
    if (d->tensors < 0 || d->tensors > (1 << 24)) return PF_ERR_SHAPE;
    if (d->state_bits != 32 && d->state_bits != 8) return PF_ERR_UNSUPPORTED;
    if (!(d->beta1 >= 0 && d->beta1 < 1 && d->beta2 >= 0 && d->beta2 < 1 && d->eps >= 0)) return PF_ERR_UNSUPPORTED;
    if (any_misaligned({lr, grad_scale}, 4) || any_misaligned({steps}, 8) || any_misaligned({plan}, 256)) return PF_ERR_UNSUPPORTED;
    const size_t fixed = adamw_bytes(d->tensors, 0, d->state_bits);
    // the table's size says how many pieces it lists, and for which states: it is the size that pf_adamw_plan_bytes gave
    if (!plan || plan_bytes < fixed || (plan_bytes - fixed) % sizeof(AdamwChunk) != 0) return PF_ERR_WORKSPACE;
    const size_t chunks = (plan_bytes - fixed) / sizeof(AdamwChunk);
    if (chunks >= (size_t)1 << 31) return PF_ERR_WORKSPACE;
    AdamwArgs a;
    a.head = (AdamwHead *)plan;
    a.tensors = (const AdamwTensor *)((char *)plan + sizeof(AdamwHead));
    a.chunks = (const AdamwChunk *)((char *)plan + adamw_bytes(d->tensors, 0, 32));
    a.lr = (const float *)lr;
    a.scale = (const float *)grad_scale;
    a.steps = (i64 *)steps;
    a.beta1 = d->beta1;
    a.beta2 = d->beta2;
    a.b1 = (float)d->beta1;
    a.b1c = (float)(1.0 - d->beta1);
    a.b2 = (float)d->beta2;
    a.b2c = (float)(1.0 - d->beta2);
    a.eps = (float)d->eps;
    int st = PF_OK;
    const dim3 grid((unsigned)(chunks ? chunks : 1));
    if (d->state_bits == 32)
        PF_LAUNCH(st, "adamw", adamw_kernel<32>, grid, dim3(256), (hipStream_t)stream, a, (unsigned)chunks);
    else
        PF_LAUNCH(st, "adamw8", adamw_kernel<8>, grid, dim3(256), (hipStream_t)stream, a, (unsigned)chunks);
    return st;
}

} // extern "C"
