// Attention with a relative position bias by buckets, backward: pf_attention_bwd.
//
// P is formed again from the scores and lse.  Two kernels, neither of which adds into memory that another workgroup writes, so
// that results do not depend on an order: the first has queries in its columns and makes dQ, delta and the sums of dS by
// distance; the second has keys in its columns and makes dK and dV, going through the query heads of a key head.  They form S
// and dP each (seven products where one kernel with atomic sums of dQ would have five).
//
// 2 x 4096 tokens of 16 heads of 128, causal: dQ with the table 268 us (matrix unit busy 38 %; vector work beside the products),
// dK and dV 398 (29 %; accumulators and operands fill the registers, so that a unit has one wave and little overlaps).  64 x 128 padded
// tokens of 8 heads of 64: 23 and 17, launch and latency of one to four tiles.
//
// delta = sum P dP of a row is sum O dO, too, but O is rounded to bf16 there and P was before O was formed: dS is off by about
// 2^-9 of delta then.  For queries that see many keys that is below what rounding dS itself costs dQ and dK; where some see few,
// delta is formed from P and dP first.  For dtable, a float32 sum over all pairs in which the rows' errors would stay, it is never
// good enough.  What delta is off by is the sum of the row's dS, so that it is known once the row is through.
//
// P = exp2((S - shift) - rest), shift = lse (base 2) and rest = 0.  An lse of 1024 or more has lost digits that P needs (at 1e9, a bias on
// all keys that a query sees, it is known to +-64).  A tile with such a row goes through its keys before: shift is then the largest bias
// that the row sees, or else its largest score, and rest comes from the row's own sum.  S is not formed at its full size then:
// shift is taken off the bias before the product is added.
#include "pf_attn.h"
#include "pf_gemm.h"

namespace pf {

// A 32 x 32 block of dS in LDS, value (r, c) in row r at c - r + 31, so that a column holds a diagonal.  What no value is written
// to is zero from the start and stays so.
constexpr int DIAG = 32 * 64;

template <typename T, int DP, int KW>
struct DqLds {
    using Tl = Tile<T, DP, 32 * KW, 256>;
    // three groups of keys, two of values; with the table's gradient then, over them, two of each and the waves' blocks
    static constexpr size_t TILES = 4 * Tl::BYTES + 4 * DIAG * 4 > 5 * Tl::BYTES ? 4 * Tl::BYTES + 4 * DIAG * 4 : 5 * Tl::BYTES;
    static size_t bytes(int far, bool bias, bool tab)
    {
        return (tab ? TILES + 4 * (2 * far + 1) * 4 : 5 * Tl::BYTES) + (bias ? (2 * far + 1) * 4 : 0);
    }
};
// dK and dV: KW waves have keys of their own, QW share the queries
template <typename T, int DP, int KW, int QW>
struct DkvLds {
    using Tl = Tile<T, DP, 32 * QW, 64 * KW * QW>;
    static size_t bytes(int far, bool bias) { return 6 * Tl::BYTES + 3 * QW * sizeof(StatRecord) + (bias ? (2 * far + 1) * 4 : 0); }
};

// dQ, delta and the sums of dS by distance, for one tile of 128 queries of one head.  TAB: with the gradient of the table.
// KW: waves that share queries, each with 32 keys of a group of 32 KW (the tile has 128 / KW queries).
//
// A turn of the loop has S and dP of 32 keys in registers.  It works out dS while the matrix unit makes S and dP of the next 32,
// then adds dS K to dQ.  Three groups of keys and two of values are in LDS: those whose columns dQ needs, those whose rows S and dP
// need, and the keys on their way; a turn needs one barrier.
//
// With the table's gradient there are two passes.  The first takes delta from O; in the far blocks, where one bucket holds all
// distances, it keeps the sums of dS and of P of each row, and it sums all dS of a row: that sum is what delta is off by. The
// second pass goes over the near blocks alone, for their dS with the delta that is now exact (S and dP, two products of the
// first pass's three); the far sums are put right by their sums of P.
template <typename T, int DP, bool BIAS, bool TAB, int KW>
__device__ __forceinline__ void attn_dq_tile(const AttnArgs &a, char *lds, int b, int head, int tile)
{
    using Tl = Tile<T, DP, 32 * KW, 256>;
    constexpr int CH = DP / 16, DB = DP / 32, AHEAD = 2, STEP = 32 * KW, QUERIES = 128 / KW;
    const int far = a.bk.far, span = 2 * far + 1;
    T *const kb = (T *)lds, *const vb = kb + 3 * Tl::SIZE;
    // the waves' blocks of dS (second pass), their sums by distance [span]
    float *const diag_all = (float *)(lds + 4 * Tl::BYTES);
    float *const bias = (float *)(lds + (TAB ? DqLds<T, DP, KW>::TILES : 5 * Tl::BYTES)), *const sums_all = bias + span;

    const int t = threadIdx.x, wave = wave_of(t), lane = t & 63, col = lane & 31, h = lane >> 5;
    float *const diag = diag_all + wave * DIAG, *const sums = sums_all + wave * span;
    const AttnLens n(a, b);
    const int kw = wave % KW, own = 32 * kw; // the wave's keys begin there in a group
    const int i0 = tile * QUERIES + wave / KW * 32, i = i0 + col;
    const bool ok = i < n.nq;
    const T *const Kp = (const T *)a.K + b * a.ks[0] + head / a.G * a.ks[2], *const Vp = (const T *)a.V + b * a.vs[0] + head / a.G * a.vs[2];
    int keys = n.nk;
    if (tile * QUERIES >= n.nq) keys = 0;
    const int block_last = (tile * QUERIES + QUERIES < n.nq ? tile * QUERIES + QUERIES : n.nq) - 1 + n.start;
    if (a.causal && block_last + 1 < keys) keys = block_last + 1 < 0 ? 0 : block_last + 1;
    const int last = (i0 + 32 < n.nq ? i0 + 32 : n.nq) - 1, pmin = i0 + n.start, pmax = last + n.start, pos = i + n.start;
    int mine = i0 >= n.nq ? 0 : keys; // of the keys, those that the wave's queries see
    if (a.causal && mine > 0 && pmax + 1 < mine) mine = pmax + 1 < 0 ? 0 : pmax + 1;

    const int most = a.causal && n.nk > pos ? 0 : n.nk - 1 - pos; // the furthest distance seen

    const Tl kl(a.ks[1], a.D, t), vl(a.vs[1], a.D, t);
    const int rows = Tl::row_place(lane) + own * Tl::RB, cols = Tl::col_place(lane) + own * Tl::RB; // (turn() repeats after 16 rows)
    const auto fetch = [&](int j, int kslot, int vslot) {
        kl.fetch(kb + kslot * Tl::SIZE, Kp + (i64)(STEP * j) * a.ks[1], a.ks[1], keys - STEP * j, a.D, wave);
        vl.fetch(vb + vslot * Tl::SIZE, Vp + (i64)(STEP * j) * a.vs[1], a.vs[1], keys - STEP * j, a.D, wave);
    };
    const int groups = (keys + STEP - 1) / STEP; // of STEP keys
    // A query that sees few keys: there delta is not small beside dP, nor is what it is off by beside dP - delta (2 x 3 causal
    // tokens: dQ off by 6e-3, by 3e-3 with the exact one; the rounding of dS alone makes 2.4e-3 of any length)
    const int position0 = tile * QUERIES + n.start, fewest = a.causal && position0 + 1 < keys ? position0 + 1 : keys;
    const bool few = sizeof(T) == 2 && groups > 0 && fewest <= 128;
    bool plainly = few || (sizeof(T) == 4 && TAB);
    const auto fetch2 = [&](int j) { fetch(j, j & 1, (j & 1) - 1); }; // (two groups of keys, two of values)
    if (groups > 0) {
        if (plainly)
            fetch2(0);
        else
            fetch(0, 0, 0);
    }
    const i64 at = (((i64)b * a.Lq + i) * a.Hq + head) * a.D, stat = ((i64)b * a.Hq + head) * a.Lq + i;
    Frag<T> q[CH], g[CH];
    float delta = 0.f;
    {
        const T *const Qp = (const T *)a.Q + b * a.qs[0] + head * a.qs[2] + i * a.qs[1];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            q[c] = row_frag_global(Qp, 16 * c, a.D, h, ok);
            g[c] = row_frag_global((const T *)a.dO + at, 16 * c, a.D, h, ok);
            const Frag<T> x = row_frag_global((const T *)a.Oin + at, 16 * c, a.D, h, ok);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta += (float)x.v[e] * (float)g[c].v[e];
        }
        delta += __shfl_xor(delta, 32);
    }
    // A query that sees one key has dS = 0: here by dO = 0, not by what rounding leaves of dP - delta
    float kept = 0.f;
    if (pos + most == 0) {
        kept = delta, delta = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) g[c] = {};
    }
    // exp2(S - lse) is 0 for a query that takes no part
    float lse2 = INFINITY;
    if (ok) {
        const float x = a.lse_in[stat];
        if (x != -INFINITY) lse2 = x * LOG2E;
    }
    // A query that sees nothing takes no part, whatever its dO holds
    if (lse2 == INFINITY) {
        delta = kept = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) g[c] = {};
    }
    __shared__ int flags[4];
    const bool large = fabsf(lse2) >= ATTN_LARGE && lse2 != INFINITY;
    leave(flags, large, wave, lane);
    float shift = lse2, rest = 0.f;
    const float sl2 = a.scale * LOG2E;
    f32x16_t dq[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dq[d] = f32x16_t{};
    float before = 0.f, after = 0.f, before_p = 0.f, after_p = 0.f, off = 0.f; // far sums of dS and P; the sum of all dS

    const auto near_at = [&](int k0) { return BIAS && k0 + 31 - pmin > -far && k0 - pmax < far; };
    const auto finish = [&](f32x16_t &s, int k0) { finish_scores<BIAS>(s, sl2, shift, bias, far, anew(k0 + 4 * h - pos), 1, most); };
    if (BIAS && keys > 0) fill_bias(a, bias, head, t, 256); // (behind the loads that it need not wait for)
    if constexpr (TAB)
        for (int x = t; x < 4 * span; x += 256) sums_all[x] = 0.f;
    if (groups > 0) {
        fetched();
        __syncthreads();
    }
    // S of group j, finished, and dP on `start`, from what fetch2 fetched
    const auto form = [&](int j, float start, f32x16_t &s, f32x16_t &dp) {
        const int at_j = (j & 1) * Tl::BYTES + rows;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f, dp[e] = start;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            mma(s, Tl::by_rows(lds, at_j, 0, c), q[c]);
            mma(dp, Tl::by_rows(lds, 2 * Tl::BYTES + at_j, 0, c), g[c]);
        }
        finish(s, STEP * j + own);
    };
    // The sum (or the largest) over the waves that share queries (between two barriers the tiles' room is free)
    const auto over_waves = [&](float x, bool sum = true) {
        if constexpr (KW == 1) return x;
        float *const y = (float *)lds + DP * 64 + lane;
        y[wave * 64] = x;
        __syncthreads();
        const float u = y[(wave & ~1) * 64], v = y[(wave | 1) * 64];
        __syncthreads();
        return sum ? u + v : fmaxf(u, v);
    };
    // Over all keys, what f makes of a group's S and dP
    const auto over_keys = [&](auto f) {
#pragma unroll 1
        for (int j = 0; j < groups; ++j) {
            if (j + 1 < groups) fetch2(j + 1);
            if (STEP * j + own < mine) {
                f32x16_t s, dp;
                form(j, 0.f, s, dp);
                f(s, dp);
            }
            fetched();
            __syncthreads();
        }
    };
    const auto from_start = [&] {
        fetch2(0);
        fetched();
        __syncthreads();
    };
    const bool large_tile = groups > 0 && left(flags, 4);
    if (__builtin_expect(large_tile, 0)) {
        const bool by_bias = BIAS && large && (shift = row_shift(-pos, most, far, [&](int x) { return bias[far + x]; })) != 0.f;
        if (large && !by_bias) shift = 0.f;
        float top = 0.f, sum = 0.f, sum_dp = 0.f;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) { // the largest score, the largest relative to shift, the sums
            from_start();
            float x = pass < 2 ? -INFINITY : 0.f;
            over_keys([&](const f32x16_t &s, const f32x16_t &dp) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float p = exp2_fast(s[e] - top);
                    x = pass < 2 ? fmaxf(x, s[e]) : x + p;
                    sum_dp += pass < 2 ? 0.f : p * dp[e];
                }
            });
            const float y = __shfl_xor(x, 32);
            x = over_waves(pass < 2 ? fmaxf(x, y) : x + y, pass == 2);
            if (pass == 0 && large && !by_bias && x != -INFINITY) shift = x;
            if (pass == 1 && large && x != -INFINITY) top = x;
            sum = x;
        }
        sum_dp = over_waves(sum_dp + __shfl_xor(sum_dp, 32));
        if (large && sum != 0.f) {
            rest = top + __builtin_amdgcn_logf(sum);
            sum_dp /= sum;
        }
        delta = sum_dp; // (other rows: shift is lse, P is normalised)
        plainly = true;
        from_start();
    }
    // The sums of a near block's dS along its diagonals
    const auto diagonals = [&](int k0, const f32x16_t &ds) {
#pragma unroll
        for (int e = 0; e < 16; ++e) diag[(8 * (e >> 2) + 4 * h + (e & 3)) * 63 + col + 31] = ds[e];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        float v[32], y = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) v[r] = diag[r * 64 + lane];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int r = 0; r < 32; ++r) y += v[r];
        // (distances from far on have one place, several lanes' sums go there: by way of the lanes' own)
        const int dist = k0 - pmin + 31 - lane;
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
    };
    const auto clear_blocks = [&] { // (what no value of a block is written to stays zero)
        for (int x = t; x < DIAG; x += 256) ((f32x4_t *)diag_all)[x] = f32x4_t{};
    };
    if (few && !large_tile) { // delta = sum P dP
        delta = 0.f;
        over_keys([&](const f32x16_t &s, const f32x16_t &dp) {
#pragma unroll
            for (int e = 0; e < 16; ++e) delta += exp2_fast(s[e]) * dp[e];
        });
        delta = over_waves(delta + __shfl_xor(delta, 32));
        from_start();
    }
    // With the exact delta one pass makes dQ and the diagonals' sums.  (In float O is exact enough, and products of 64 cycles hide
    // no vector work worth the order above: 4 x 333 tokens of 8 heads of 64 took 43 us in two passes, 28 so.)
    if (plainly) {
        if constexpr (TAB) {
            clear_blocks();
            __syncthreads();
        }
#pragma unroll 1
        for (int j = 0; j < groups; ++j) {
            const int k0 = STEP * j + own;
            if (j + 1 < groups) fetch2(j + 1);
            if (k0 < mine) {
                f32x16_t s, dp;
                form(j, -delta, s, dp);
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = exp2_fast(s[e] - rest) * dp[e];
                if constexpr (TAB) {
                    if (near_at(k0)) {
                        diagonals(k0, s);
                    } else {
                        float y = 0.f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) y += s[e];
                        (k0 >= pmin ? after : before) += y;
                    }
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    Frag<T> f;
                    pack(s, c, f);
#pragma unroll
                    for (int d = 0; d < DB; ++d) mma(dq[d], Tl::by_cols(lds, (j & 1) * Tl::BYTES + cols, 16 * c, d), f);
                }
            }
            fetched();
            __syncthreads();
        }
    }
    f32x16_t sA = {}, sB = {}, dpA = {}, dpB = {};
    int slot = 2; // of group j
    const auto turn = [&](int j, f32x16_t &s, f32x16_t &dp, f32x16_t &next, f32x16_t &dnext) {
        const int s1 = slot == 2 ? 0 : slot + 1, s2 = slot == 0 ? 2 : slot - 1; // of groups j + 1, j + 2
        const int k0 = STEP * j + own; // the wave's first key
        if (j + 2 < groups) fetch(j + 2, s2, j & 1);
        const bool now = j >= 0 && k0 < mine, then = k0 + STEP < mine;
        if (now || then) {
            const int krow = s1 * Tl::BYTES + rows, vrow = (3 + ((j + 1) & 1)) * Tl::BYTES + rows, kcol = slot * Tl::BYTES + cols;
            // S and dP in turn, then dQ: 16 keys after 16 keys
            const auto operand = [&](int x) {
                return x < 2 * CH ? Tl::by_rows(lds, x & 1 ? vrow : krow, 0, x / 2) : Tl::by_cols(lds, kcol, 16 * ((x - 2 * CH) / DB), (x - 2 * CH) % DB);
            };
            const bool near = near_at(k0), plain = !near && k0 + 32 <= n.nk && !(a.causal && k0 + 31 > pmin);
            const float flat = BIAS ? bias[k0 >= pmin ? 2 * far : 0] : 0.f;
            if (now && !plain) finish(s, k0);
            const float mul = plain ? sl2 : 1.f, add = plain ? flat - shift : 0.f;
            const float start = anew(-delta); // (dP is formed on -delta: dS = P (dP - delta))
#pragma unroll
            for (int e = 0; e < 16; ++e) next[e] = 0.f, dnext[e] = start;
            Frag<T> ring[AHEAD + 1], f[2];
            float sum = 0.f, sum_p = 0.f;
            __builtin_amdgcn_sched_barrier(0);
            // S and dP of the next keys (step 2 c: S, columns 16 c ..; 2 c + 1: dP) beside dS of these
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) ring[x] = operand(x);
#pragma unroll
            for (int x = 0; x < 2 * CH; ++x) {
                ring[(x + AHEAD) % (AHEAD + 1)] = operand(x + AHEAD);
                if (x & 1)
                    mma(dnext, ring[x % (AHEAD + 1)], g[x / 2]);
                else
                    mma(next, ring[x % (AHEAD + 1)], q[x / 2]);
#pragma unroll
                for (int e = x * 16 / (2 * CH); e < (x + 1) * 16 / (2 * CH); ++e) {
                    const float p = exp2_fast(s[e] * mul + add);
                    s[e] = p * dp[e];
                    if constexpr (TAB) {
                        sum = anew(sum + s[e]);
                        sum_p = anew(sum_p + p);
                    }
                    if (e % 8 == 7) {
                        pack(s, e / 8, f[e / 8]);
                        here(f[e / 8]);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (now) {
                if constexpr (TAB) {
                    off += sum;
                    if (!near) {
                        if (k0 >= pmin) {
                            after += sum;
                            after_p += sum_p;
                        } else {
                            before += sum;
                            before_p += sum_p;
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = 0; x < 2 * DB; ++x) {
                    if (x + AHEAD < 2 * DB) ring[(2 * CH + x + AHEAD) % (AHEAD + 1)] = operand(2 * CH + x + AHEAD);
                    mma(dq[x % DB], ring[(2 * CH + x) % (AHEAD + 1)], f[x / DB]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        slot = s1;
        fetched();
        __syncthreads();
    };
    int start = -1; // (a number to the compiler: it would unroll the first turn for its own)
    asm volatile("" : "+s"(start));
    for (int j = plainly ? groups : start; j < groups; j += 2) {
        turn(j, sA, dpA, sB, dpB);
        if (j + 1 < groups) turn(j + 1, sB, dpB, sA, dpA);
    }
    if constexpr (KW == 2) { // the second wave's dQ to the first (the loop ended with a barrier)
        float *const part = (float *)lds + wave / KW * (DP / 2) * 64 + lane;
        if (kw == 1) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) part[(16 * d + e) * 64] = dq[d][e];
        }
        __syncthreads();
        if (kw == 0) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) dq[d][e] += part[(16 * d + e) * 64];
        }
        off = over_waves(off);
    }
    if (i < a.Lq && kw == 0) {
        T *const out = (T *)a.dQ + at;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int c = 32 * d + 8 * (e >> 2) + 4 * h;
                float v[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = ok ? dq[d][e + x] * a.scale : 0.f;
                if (c < a.D) put4(out + c, v[0], v[1], v[2], v[3]);
            }
    }
    if constexpr (TAB) {
        off += __shfl_xor(off, 32);
        delta += off;
        before -= off * before_p;
        after -= off * after_p;
    }
    if (kw == 0) { // the wave's record, of queries behind the last, too
        StatRecord *const out = (StatRecord *)a.stat + ((i64)b * a.Hq + head) * a.records + i0 / 32;
        const bool table = BIAS && groups > 0, with_rest = __any(rest != 0.f);
        if (h == 0) {
            out->before[col] = ((table ? bias[0] : 0.f) - shift) - rest;
            out->after[col] = ((table ? bias[2 * far] : 0.f) - shift) - rest;
            out->neg_delta[col] = ok ? -(delta + kept) : 0.f;
            out->shift[col] = shift;
            out->neg_rest[col] = -rest;
            if (col == 0) out->with_rest[0] = with_rest ? 1.f : 0.f;
        }
    }
    if constexpr (TAB) {
        // the near blocks once more: STEP begin + STEP - 1 > first position - far, STEP (end - 1) < last position + far
        int begin = 0, end = groups;
        const int lo = tile * QUERIES + n.start - far - (STEP - 1), hi = block_last + far;
        if (lo >= 0) begin = lo / STEP + 1;
        if (plainly || hi <= 0)
            end = 0;
        else if ((hi + STEP - 1) / STEP < end)
            end = (hi + STEP - 1) / STEP;
        if (begin < end) {
            clear_blocks();
            fetch2(begin);
            fetched();
            __syncthreads();
        }
        for (int j = begin; j < end; ++j) {
            const int k0 = STEP * j + own;
            if (j + 1 < end) fetch2(j + 1);
            if (k0 < mine && near_at(k0)) {
                f32x16_t s, dp;
                form(j, -delta, s, dp);
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = exp2_fast(s[e]) * dp[e];
                diagonals(k0, s);
            }
            fetched();
            __syncthreads();
        }
        for (int o = 32; o; o >>= 1) {
            before += __shfl_xor(before, o);
            after += __shfl_xor(after, o);
        }
        __syncthreads();
        if (lane == 0) {
            sums[0] += before;
            sums[2 * far] += after;
        }
        __syncthreads();
        for (int x = t; x < span; x += 256) sums_all[x] = (sums_all[x] + sums_all[span + x]) + (sums_all[2 * span + x] + sums_all[3 * span + x]);
        __syncthreads();
        float *const out = a.tab + (((i64)head * a.B + b) * a.tiles + tile) * a.buckets;
        // eight lanes to a bucket
        for (int x = t; x < 8 * a.buckets; x += 256) {
            // the distances of bucket u: lo .. hi of its side, the last one's up to far
            const int u = x / 8, sub = x & 7, v = a.two_sided && u >= a.bk.side ? u - a.bk.side : u, e = a.bk.exact;
            int lo = v, hi = v;
            if (v >= e) {
                lo = v == e ? e : a.bk.border[v - e - 1];
                hi = v == a.bk.side - 1 ? far : a.bk.border[v - e] - 1;
            }
            float y = 0.f;
            if (a.two_sided && u >= a.bk.side) {
                for (int z = (lo < 1 ? 1 : lo) + sub; z <= hi; z += 8) y += sums_all[far + z];
            } else {
                for (int z = lo + sub; z <= hi; z += 8) y += sums_all[far - z];
                if (u == 0 && !a.two_sided)
                    for (int z = 1 + sub; z <= far; z += 8) y += sums_all[far + z];
            }
            for (int o = 4; o; o >>= 1) y += __shfl_xor(y, o);
            if (sub == 0) out[u] = y;
        }
    }
}

// paired: a long tile of queries and a short one to a workgroup, as forward
template <typename T, int DP, bool BIAS, bool TAB, int KW>
__global__ __launch_bounds__(256, DP * sizeof(T) <= 256 ? 2 : 1) void attn_dq_kernel(AttnArgs a, int paired)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const unsigned w = xcd_order(blockIdx.x, gridDim.x);
    const int each = paired ? (a.tiles + 1) / 2 : a.tiles, k = (int)(w % each), bh = w / each, b = bh / a.Hq, head = bh - b * a.Hq;
    const int count = paired && a.tiles - 1 - k != k ? 2 : 1;
#pragma unroll 1
    for (int x = 0; x < count; ++x) {
        attn_dq_tile<T, DP, BIAS, TAB, KW>(a, lds, b, head, x ? k : a.tiles - 1 - k);
        __syncthreads();
    }
}

// dtable[u][head] from the tiles' sums: one wave to a value, in double and always in one order
struct TableSum {
    float *dtable; // or none
    int parts, accumulate;
    unsigned after; // the workgroups of the launch that come before these
};
__device__ __forceinline__ void attn_table(const AttnArgs &a, const TableSum &z, int value, int lane)
{
    if (value >= a.buckets * a.Hq) return;
    const int u = value % a.buckets, head = value / a.buckets;
    double y = 0.0;
    for (int p = lane; p < z.parts; p += 64) y += (double)a.tab[((i64)head * z.parts + p) * a.buckets + u];
    for (int o = 32; o; o >>= 1) y += __shfl_xor(y, o);
    float *const out = z.dtable + (i64)u * a.Hq + head;
    if (lane == 0) *out = z.accumulate ? *out + (float)y : (float)y;
}

// dK and dV: a workgroup has 32 KW keys of one key head, a wave 32 of them in its columns; the query heads of the key head one
// after the other, each in groups of 32 QW queries, of which a wave has 32.  As above, dS and P of 32 queries are worked out
// while S and dP of the next are made.  The waves that share keys add up what they have at the end.
template <typename T, int DP, bool BIAS, int KW, int QW>
__global__ __launch_bounds__((64 * KW * QW), (DP * sizeof(T) <= 128 ? 2 : 1)) void attn_dkv_kernel(AttnArgs a, TableSum z)
{
    constexpr int ROWS = 32 * QW, THREADS = 64 * KW * QW, KEYS = 32 * KW;
    using Tl = Tile<T, DP, ROWS, THREADS>;
    constexpr int CH = DP / 16, DB = DP / 32, AHEAD = DP * sizeof(T) <= 128 ? 3 : sizeof(T) == 2 ? 6 : 3; // (one wave to a unit needs more on the way)
    extern __shared__ __attribute__((aligned(16))) char lds[];
    T *const qb = (T *)lds, *const gb = qb + 3 * Tl::SIZE;
    StatRecord *const stats = (StatRecord *)(lds + 6 * Tl::BYTES); // [3][QW]
    float *const bias = (float *)(stats + 3 * QW);

    if (blockIdx.x >= z.after) return attn_table(a, z, (int)(blockIdx.x - z.after) * KW * QW + (threadIdx.x >> 6), threadIdx.x & 63);
    const unsigned w = xcd_order(blockIdx.x, z.after);
    const int tile = (int)(w % a.tiles), bk = w / a.tiles, b = bk / a.Hkv, kv = bk - b * a.Hkv;
    const int t = threadIdx.x, wave = wave_of(t), lane = t & 63, col = lane & 31, h = lane >> 5;
    const AttnLens n(a, b);
    const int kw = wave % KW, r0 = 32 * (wave / KW); // the wave's keys; its rows of a group
    const int far = a.bk.far, j0 = tile * KEYS + kw * 32, j = j0 + col;
    const bool ok = j < n.nk;
    const int most = !ok ? INT32_MIN : a.causal ? 0 : INT32_MAX; // the furthest distance from which the key is seen
    Frag<T> k[CH], v[CH];
    {
        const T *const Kp = (const T *)a.K + b * a.ks[0] + kv * a.ks[2] + j * a.ks[1], *const Vp = (const T *)a.V + b * a.vs[0] + kv * a.vs[2] + j * a.vs[1];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            k[c] = row_frag_global(Kp, 16 * c, a.D, h, ok);
            v[c] = row_frag_global(Vp, 16 * c, a.D, h, ok);
        }
    }
    const float sl2 = a.scale * LOG2E;
    f32x16_t dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = dv[d] = f32x16_t{};

    const i64 grow = (i64)a.Hq * a.D;
    const Tl ql(a.qs[1], a.D, t), gl(grow, a.D, t);
    const int rows = Tl::row_place(lane) + r0 * Tl::RB, cols = Tl::col_place(lane) + r0 * Tl::RB; // (turn() repeats after 16 rows)
    // the groups of queries that see a key of the workgroup; the first query that sees one of the wave
    int begin = 0, mine = 0, hidden = 0; // the first `hidden` queries see nothing: they are not read (0 times NaN is not 0)
    const int end = (n.nq + ROWS - 1) / ROWS;
    if (a.causal) {
        hidden = clamped(-n.start, 0, n.nq);
        begin = clamped(tile * KEYS - n.start, 0, a.Lq) / ROWS;
        mine = clamped(j0 - n.start, 0, a.Lq);
    }
    if (tile * KEYS >= n.nk) begin = end;
    if (j0 >= n.nk) mine = a.Lq;
    for (int g0 = 0; g0 < a.G && begin < end; ++g0) {
        const int head = kv * a.G + g0;
        const T *const Qp = (const T *)a.Q + b * a.qs[0] + head * a.qs[2], *const Gp = (const T *)a.dO + ((i64)b * a.Lq * a.Hq + head) * a.D;
        const StatRecord *const records = (const StatRecord *)a.stat + ((i64)b * a.Hq + head) * a.records;
        const auto fetch = [&](int x, int slot, int skip) {
            ql.fetch(qb + slot * Tl::SIZE, Qp + (i64)(ROWS * x) * a.qs[1], a.qs[1], n.nq - ROWS * x, a.D, wave, skip);
            gl.fetch(gb + slot * Tl::SIZE, Gp + (i64)(ROWS * x) * grow, grow, n.nq - ROWS * x, a.D, wave, skip);
            // the group's records, 16 bytes a lane
            typedef __attribute__((address_space(3))) void *lds_ptr;
            const BufSrc src(records + QW * x, QW * sizeof(StatRecord));
            if (16 * t < QW * (int)sizeof(StatRecord))
                __builtin_amdgcn_raw_ptr_buffer_load_lds(src.r, (lds_ptr)((char *)(stats + QW * slot) + 1024 * wave), 16, 16 * t, 0, 0, 0);
        };
        int slot = (begin + 2) % 3;
        fetch(begin, begin % 3, hidden > ROWS * begin ? hidden - ROWS * begin : 0);
        if constexpr (BIAS) fill_bias(a, bias, head, t, THREADS);
        fetched();
        __syncthreads();
        f32x16_t sA = {}, sB = {}, dpA = {}, dpB = {};
        const auto turn = [&](int x0, f32x16_t &s, f32x16_t &dp, f32x16_t &next, f32x16_t &dnext) {
            const int s1 = slot == 2 ? 0 : slot + 1, s2 = slot == 0 ? 2 : slot - 1;
            if (x0 + 2 < end) fetch(x0 + 2, s2, 0);
            const int i0 = ROWS * x0 + r0; // the wave's first query
            const bool now = x0 >= begin && i0 < n.nq && i0 + 31 >= mine, then = x0 + 1 < end && i0 + ROWS < n.nq && i0 + ROWS + 31 >= mine;
            if (now || then) {
                // S and dP in turn, then dV and dK in turn, 16 rows after 16 rows
                const int qrow = s1 * Tl::BYTES + rows, grow_at = qrow + 3 * Tl::BYTES, qcol = slot * Tl::BYTES + cols, gcol = qcol + 3 * Tl::BYTES;
                const auto operand = [&](int x) {
                    const int y = x - 2 * CH;
                    return x < 2 * CH ? Tl::by_rows(lds, x & 1 ? grow_at : qrow, 0, x / 2) : Tl::by_cols(lds, y & 1 ? qcol : gcol, 16 * (y / (2 * DB)), y / 2 % DB);
                };
                const StatRecord &own = stats[QW * slot + wave / KW];
                const float *const st1 = stats[QW * s1 + wave / KW].neg_delta + 4 * h;
                const int p0 = i0 + n.start; // the position of the first row
                const bool edge = j0 + 32 > n.nk || (a.causal && j0 + 31 > p0);
                const bool near = BIAS && j0 + 31 - p0 > -far && j0 - (p0 + 31) < far;
                const bool plain = !edge && !near && __builtin_amdgcn_readfirstlane(own.with_rest[0]) == 0;
                if (now && !plain) finish_scores<BIAS>(s, sl2, own.shift + 4 * h, bias, far, anew(j - p0 - 4 * h), -1, most);
                // what is added to the products: with a far key its bias, too
                const float mul = plain ? sl2 : 1.f, *const st = (plain ? j0 >= p0 ? own.after : own.before : own.neg_rest) + 4 * h;
#pragma unroll
                for (int e = 0; e < 16; e += 4) { // (dP is formed on -delta: dS = P (dP - delta))
                    const f32x4_t y = *(const f32x4_t *)(st1 + 2 * e);
                    next[e] = next[e + 1] = next[e + 2] = next[e + 3] = 0.f;
                    dnext[e] = y[0], dnext[e + 1] = y[1], dnext[e + 2] = y[2], dnext[e + 3] = y[3];
                }
                Frag<T> ring[AHEAD + 1], fp[2], fs[2];
                f32x16_t p;
                f32x4_t l4 = *(const f32x4_t *)st;
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = 0; x < AHEAD; ++x) ring[x] = operand(x);
#pragma unroll
                for (int x = 0; x < 2 * CH; ++x) {
                    ring[(x + AHEAD) % (AHEAD + 1)] = operand(x + AHEAD);
                    if (x & 1)
                        mma(dnext, ring[x % (AHEAD + 1)], v[x / 2]);
                    else
                        mma(next, ring[x % (AHEAD + 1)], k[x / 2]);
#pragma unroll
                    for (int e = x * 16 / (2 * CH); e < (x + 1) * 16 / (2 * CH); ++e) {
                        p[e] = exp2_fast(s[e] * mul + l4[e % 4]);
                        s[e] = p[e] * dp[e];
                        if (e % 8 == 7) {
                            pack(p, e / 8, fp[e / 8]);
                            pack(s, e / 8, fs[e / 8]);
                            here(fp[e / 8]);
                            here(fs[e / 8]);
                        }
                        if (e % 4 == 3 && e < 15) l4 = *(const f32x4_t *)(st + 2 * (e + 1));
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (now) {
#pragma unroll
                    for (int x = 0; x < 4 * DB; ++x) {
                        if (x + AHEAD < 4 * DB) ring[(2 * CH + x + AHEAD) % (AHEAD + 1)] = operand(2 * CH + x + AHEAD);
                        if (x & 1)
                            mma(dk[x / 2 % DB], ring[(2 * CH + x) % (AHEAD + 1)], fs[x / (2 * DB)]);
                        else
                            mma(dv[x / 2 % DB], ring[(2 * CH + x) % (AHEAD + 1)], fp[x / (2 * DB)]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
            slot = s1;
            fetched();
            __syncthreads();
        };
        for (int x0 = begin - 1; x0 < end; x0 += 2) {
            turn(x0, sA, dpA, sB, dpB);
            if (x0 + 1 < end) turn(x0 + 1, sB, dpB, sA, dpA);
        }
    }
    if constexpr (QW == 2) { // (the loop ended with a barrier: the tiles' room is free)
        float *const sum = (float *)lds + kw * DB * 2048 + lane;
        if (wave >= KW) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    sum[(16 * d + e) * 64] = dk[d][e];
                    sum[(16 * (DB + d) + e) * 64] = dv[d][e];
                }
        }
        __syncthreads();
        if (wave >= KW) return;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                dk[d][e] += sum[(16 * d + e) * 64];
                dv[d][e] += sum[(16 * (DB + d) + e) * 64];
            }
    }
    if (j >= a.Lk) return;
    const float scale = n.nk == 1 ? 0.f : a.scale; // (one key: P = 1 and dS = 0, not what rounding leaves of dP - delta)
    const i64 at = (((i64)b * a.Lk + j) * a.Hkv + kv) * a.D;
    T *const ok_ = (T *)a.dK + at, *const ov = (T *)a.dV + at;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int c = 32 * d + 8 * (e >> 2) + 4 * h;
            if (c >= a.D) continue;
            put4(ok_ + c, dk[d][e] * scale, dk[d][e + 1] * scale, dk[d][e + 2] * scale, dk[d][e + 3] * scale);
            put4(ov + c, dv[d][e], dv[d][e + 1], dv[d][e + 2], dv[d][e + 3]);
        }
}

// ------------------------------------------------------------------ host
template <typename T, int DP, int KW>
static int attn_dq_launch(AttnArgs &a, bool tab, hipStream_t s)
{
    int st = PF_OK;
    a.tiles = (a.Lq + 128 / KW - 1) / (128 / KW);
    const int paired = a.causal && (i64)a.B * a.Hq * a.tiles > 512; // (two workgroups to a compute unit are resident)
    const dim3 grid((unsigned)a.B * a.Hq * (paired ? (a.tiles + 1) / 2 : a.tiles));
    if (too_many(grid.x, 256)) return PF_ERR_UNSUPPORTED;
    const size_t lds = DqLds<T, DP, KW>::bytes(a.bk.far, a.buckets, tab);
    if (a.Lq == 0) return st;
    if (tab)
        PF_LAUNCH_LDS(st, "attn_dq_tab", (attn_dq_kernel<T, DP, true, true, KW>), grid, dim3(256), lds, s, a, paired);
    else if (a.buckets)
        PF_LAUNCH_LDS(st, "attn_dq", (attn_dq_kernel<T, DP, true, false, KW>), grid, dim3(256), lds, s, a, paired);
    else
        PF_LAUNCH_LDS(st, "attn_dq", (attn_dq_kernel<T, DP, false, false, KW>), grid, dim3(256), lds, s, a, paired);
    return st;
}
// Waves that share queries: as forward, two where that makes no more workgroups than fit the card at once (rows of more than 128
// bytes: one to a compute unit; of more than 256: no room for it).  us, bf16, 8 heads of 64 with the table: 2 x 1024 tokens, 128
// tiles, 50 alone and 33 shared; 4 x 1024, 256 tiles, 51 and 40; 6 x 1024 64 and 62; float, 8 x 512, 256 tiles, 105 and 117.
static int dq_sharing(i64 B, i64 Hq, i64 Lq, size_t row)
{
    return row <= 256 && B * Hq * ((Lq + 127) / 128) <= (row <= 128 ? 256 : 128) ? 2 : 1;
}
static int padded(int D) { return (D + 31) / 32 * 32; }
static i64 dq_tiles(i64 B, i64 Hq, i64 Lq, size_t row)
{
    const int queries = 128 / dq_sharing(B, Hq, Lq, row);
    return (Lq + queries - 1) / queries;
}

template <typename T, int DP, int KW, int QW>
static int attn_dkv_launch(AttnArgs &a, TableSum z, hipStream_t s)
{
    int st = PF_OK;
    a.tiles = (a.Lk + 32 * KW - 1) / (32 * KW);
    z.after = (unsigned)a.B * a.Hkv * a.tiles;
    // behind the workgroups for the keys, those that sum up the table's gradient (a launch of their own took 5 us)
    const dim3 grid(z.after + (z.dtable ? (a.buckets * a.Hq + KW * QW - 1) / (KW * QW) : 0));
    const size_t lds = DkvLds<T, DP, KW, QW>::bytes(a.bk.far, a.buckets);
    if (grid.x == 0) return st;
    if (a.buckets)
        PF_LAUNCH_LDS(st, "attn_dkv", (attn_dkv_kernel<T, DP, true, KW, QW>), grid, dim3(64 * KW * QW), lds, s, a, z);
    else
        PF_LAUNCH_LDS(st, "attn_dkv", (attn_dkv_kernel<T, DP, false, KW, QW>), grid, dim3(64 * KW * QW), lds, s, a, z);
    return st;
}

// Keys of a workgroup: 128, a wave's own 32 queries at a time, where that makes as many workgroups as fit the card at once (queries and
// dO are read half as often); 64 shared by two waves each where it does not, and with a causal mask, whose first keys have
// the most queries.  us, bf16: 64 x 128 tokens of 8 heads of 64, 512 tiles of 128, 19 and 24 with tiles of 64; 6 x 1024, 384 tiles,
// 54 and 51; 4 x 1024 with heads of 128, 256 tiles (one to a compute unit), 61 and 68; 2 x 4096 causal, 256 tiles, 675 and 408.
// (Six tiles of rows of more than 256 bytes leave no room for two waves' queries, nor for a second workgroup: four waves where
// there are more tiles of 64 keys than compute units.  16 x 512 tokens of 8 heads of 128: 320 us, with two waves 591)
static int dkv_keys(const pf_attention_desc *d, size_t row)
{
    const i64 heads = d->B * d->heads_kv;
    if (row > 256) return heads * ((d->Lk + 63) / 64) > 256 ? 128 : 64;
    return (!d->causal || d->Lk <= 128) && heads * ((d->Lk + 127) / 128) >= (row <= 128 ? 512 : 256) ? 128 : 64;
}

template <typename T, int DP>
static int attn_bwd_launch(AttnArgs &a, int keys, float *dtable, int accumulate, hipStream_t s)
{
    const bool bias = a.buckets > 0, tab = bias && dtable;
    int st;
    if constexpr (DP * sizeof(T) <= 256)
        st = dq_sharing(a.B, a.Hq, a.Lq, DP * sizeof(T)) == 2 ? attn_dq_launch<T, DP, 2>(a, tab, s) : attn_dq_launch<T, DP, 1>(a, tab, s);
    else
        st = attn_dq_launch<T, DP, 1>(a, tab, s);
    const int parts = a.B * a.tiles;
    if (st != PF_OK) return st;
    const TableSum z = {tab ? dtable : nullptr, parts, accumulate, 0};
    return keys == 128 ? attn_dkv_launch<T, DP, 4, 1>(a, z, s) : attn_dkv_launch<T, DP, 2, (DP * sizeof(T) > 256 ? 1 : 2)>(a, z, s);
}
// The workspace: records of each head's queries, whole tiles of them; the table's sums
struct BwdSpace {
    int records;
    size_t stat, tab;
    BwdSpace(const pf_attention_desc *d)
    {
        const size_t row = padded(d->head_dim) * (d->dtype == PF_BF16 ? 2 : 4), heads = (size_t)d->B * d->heads_q;
        const i64 tiles = dq_tiles(d->B, d->heads_q, d->Lq, row);
        records = (int)(tiles * (128 / dq_sharing(d->B, d->heads_q, d->Lq, row)) / 32);
        stat = align_up(heads * records * sizeof(StatRecord));
        tab = align_up(heads * tiles * d->buckets * sizeof(float));
    }
};

} // namespace pf

extern "C" {

using namespace pf;

size_t pf_attention_bwd_workspace_bytes(const pf_attention_desc *d)
{
    if (attn_check(d) != PF_OK || d->B == 0 || d->Lq == 0) return 0;
    const BwdSpace w(d);
    return w.stat + w.tab;
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
    // (the second launch, and the workgroups in it that sum up the table; the first one refuses by itself)
    const int keys = dkv_keys(d, padded(d->head_dim) * (d->dtype == PF_BF16 ? 2 : 4));
    if (too_many(d->B * d->heads_kv * ((d->Lk + keys - 1) / keys) + (i64)d->buckets * d->heads_q, 256)) return PF_ERR_UNSUPPORTED;
    AttnArgs a = {};
    attn_fill(d, a);
    const AttnAreas of{d, a};
    if (outputs_meet({of.dense_queries(dQ), of.dense_keys(dK), of.dense_keys(dV), of.table(dtable)},
                     {of.queries(Q), of.keys(K, a.ks), of.keys(V, a.vs), of.dense_queries(O), of.dense_queries(dO), of.rows(lse), of.table(table)}))
        return PF_ERR_UNSUPPORTED;
    a.Q = Q, a.K = K, a.V = V, a.Oin = O, a.dO = dO, a.dQ = dQ, a.dK = dK, a.dV = dV;
    a.table = (const float *)table;
    a.lse_in = (const float *)lse;
    a.q_start = (const int *)q_start;
    a.q_len = (const int *)q_len;
    a.kv_len = (const int *)kv_len;
    const BwdSpace w(d);
    a.records = w.records;
    a.stat = (float *)workspace;
    a.tab = (float *)((char *)workspace + w.stat);
    const int DP = (a.D + 31) / 32 * 32;
    float *const dt = d->buckets ? (float *)dtable : nullptr;
    if (d->dtype == PF_BF16)
        return DP == 32 ? attn_bwd_launch<bf16_t, 32>(a, keys, dt, accumulate, s) : DP == 64 ? attn_bwd_launch<bf16_t, 64>(a, keys, dt, accumulate, s)
             : DP == 96 ? attn_bwd_launch<bf16_t, 96>(a, keys, dt, accumulate, s) : attn_bwd_launch<bf16_t, 128>(a, keys, dt, accumulate, s);
    return DP == 32 ? attn_bwd_launch<float, 32>(a, keys, dt, accumulate, s) : DP == 64 ? attn_bwd_launch<float, 64>(a, keys, dt, accumulate, s)
         : DP == 96 ? attn_bwd_launch<float, 96>(a, keys, dt, accumulate, s) : attn_bwd_launch<float, 128>(a, keys, dt, accumulate, s);
}

} // extern "C"
