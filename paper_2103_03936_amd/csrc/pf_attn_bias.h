// Which distances share a bucket of the relative position bias (host arithmetic; the header pufferfish.h has the formula).
#pragma once

#include <math.h>
#include <stdint.h>

namespace pf {

constexpr int ATTN_MAX_BORDERS = 128, ATTN_MAX_DISTANCE = 1024, ATTN_MAX_BUCKETS = 256;

// One side's buckets: distance n < exact has bucket n, the others exact + (number of borders <= n); from `far` on the
// bucket is side - 1.  Behind the last border stand values that no distance reaches.
struct AttnBuckets {
    int side, exact, borders, far;
    uint16_t border[ATTN_MAX_BORDERS];
};

// x^nx y^ny in 32-bit digits, the lowest first: at most 256 factors of at most 1024 = 2^10, 2560 bits.  (No memory is asked for: the
// callers are entry points that C code calls, where nothing may be thrown.)
struct PowerProduct {
    uint32_t w[80];
    int n = 1;
    PowerProduct(uint32_t x, int nx, uint32_t y, int ny)
    {
        w[0] = 1;
        for (int i = 0; i < nx + ny; ++i) {
            const uint64_t f = i < nx ? x : y;
            uint64_t carry = 0;
            for (int j = 0; j < n; ++j) {
                carry += f * w[j];
                w[j] = (uint32_t)carry;
                carry >>= 32;
            }
            if (carry) w[n++] = (uint32_t)carry;
        }
    }
};
static_assert(ATTN_MAX_DISTANCE <= 1 << 10 && ATTN_MAX_BUCKETS / 2 <= 128, "digits of a PowerProduct");
// Whether a^m b^k >= c^k d^m, in whole numbers; k < m
inline bool power_product_ge(uint32_t a, int m, uint32_t b, int k, uint32_t c, uint32_t d)
{
    const PowerProduct l(a, m, b, k), r(c, k, d, m);
    if (l.n != r.n) return l.n > r.n;
    for (int i = l.n; i-- > 0;)
        if (l.w[i] != r.w[i]) return l.w[i] > r.w[i];
    return true;
}

// buckets >= 2 of one side, max_distance > buckets / 2
inline AttnBuckets attn_buckets(int side, int max_distance)
{
    AttnBuckets t = {};
    t.side = side;
    t.exact = side / 2;
    const int e = t.exact, m = side - e;
    for (int k = 1; k < m; ++k) {
        // the smallest n with (n / e)^m >= (max_distance / e)^k; where the root comes out next to a whole number, that
        // number is tried exactly
        const double x = e * pow((double)max_distance / e, (double)k / m), near = floor(x + 0.5);
        int n = (int)ceil(x);
        if (fabs(x - near) < 1e-6 * x)
            n = power_product_ge((uint32_t)near, m, (uint32_t)e, k, (uint32_t)max_distance, (uint32_t)e) ? (int)near : (int)near + 1;
        t.border[t.borders++] = (uint16_t)n;
    }
    for (int k = t.borders; k < ATTN_MAX_BORDERS; ++k) t.border[k] = 0xffff;
    t.far = t.borders ? t.border[t.borders - 1] : e;
    return t;
}

} // namespace pf
