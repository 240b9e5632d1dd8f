// Whether two tensors with strides have an element in common (host arithmetic).
#pragma once

#include <stdint.h>

#include <algorithm>
#include <initializer_list>

namespace pf {

// Rows of `row` bytes, `size` of them in each of the dimensions `stride` bytes apart (not negative)
struct Area {
    uint64_t at = 0;
    int64_t row = 0;
    int dims = 0;
    int64_t stride[3], size[3];
    Area() {}
    // no pointer, or no element: meets nothing
    Area(const void *p, int64_t bytes) : at((uint64_t)(uintptr_t)p), row(p ? bytes : 0) {}
    // [B, L, heads] rows of D elements of `elem` bytes; strides in elements
    template <class S>
    Area(const void *p, int64_t B, int64_t L, int64_t heads, const S (&s)[3], int64_t D, int64_t elem) : Area(p, D * elem)
    {
        const int64_t n[3] = {B, L, heads};
        for (int i = 0; i < 3; ++i) {
            if (n[i] == 0) row = 0;
            if (n[i] > 1 && s[i] > 0) stride[dims] = s[i] * elem, size[dims++] = n[i]; // (stride 0: the same row again and again)
        }
        for (int i = 0; i < dims; ++i) // the largest stride first
            for (int j = i + 1; j < dims; ++j)
                if (stride[j] > stride[i]) std::swap(stride[i], stride[j]), std::swap(size[i], size[j]);
        // rows that lie side by side are one, dimensions that continue each other are one
        while (dims && stride[dims - 1] == row) row *= size[--dims];
        for (int i = dims - 2; i >= 0; --i)
            if (stride[i] == stride[i + 1] * size[i + 1]) {
                size[i + 1] *= size[i];
                for (int j = i; j < dims - 1; ++j) stride[j] = stride[j + 1], size[j] = size[j + 1];
                --dims;
            }
    }
    uint64_t end() const
    {
        uint64_t x = at + row;
        for (int i = 0; i < dims; ++i) x += (size[i] - 1) * stride[i];
        return x;
    }
    bool same(const Area &o) const
    {
        return at == o.at && row == o.row && dims == o.dims && std::equal(stride, stride + dims, o.stride) && std::equal(size, size + dims, o.size);
    }
};

struct Difference { // whole numbers lo .. hi, times `step`
    int64_t step, lo, hi;
};
// Whether from + sum k_i step_i, lo_i <= k_i <= hi_i, comes within least .. most.  With strides that nest, each dimension leaves two or three
// k to try; `tries` bounds the work of others.
inline bool comes_within(int64_t from, const Difference *d, int n, int64_t least, int64_t most, int &tries)
{
    if (n == 0) return from >= least && from <= most;
    int64_t low = 0, high = 0; // what the smaller steps can add
    for (int i = 1; i < n; ++i) low += d[i].lo * d[i].step, high += d[i].hi * d[i].step;
    const auto floor_div = [](int64_t a, int64_t b) { return a >= 0 ? a / b : -((-a + b - 1) / b); };
    const int64_t first = std::max(d[0].lo, -floor_div(from + high - least, d[0].step)), last = std::min(d[0].hi, floor_div(most - from - low, d[0].step));
    for (int64_t k = first; k <= last; ++k) {
        if (--tries < 0) return false;
        if (comes_within(from + k * d[0].step, d + 1, n - 1, least, most, tries)) return true;
    }
    return false;
}
inline bool meet(const Area &a, const Area &b)
{
    if (a.row == 0 || b.row == 0 || a.end() <= b.at || b.end() <= a.at) return false;
    Difference d[6];
    int n = 0;
    for (int i = 0, j = 0; i < a.dims || j < b.dims;) { // both lists of strides, merged
        const int64_t s = std::max(i < a.dims ? a.stride[i] : 0, j < b.dims ? b.stride[j] : 0);
        d[n] = {s, 0, 0};
        for (; i < a.dims && a.stride[i] == s; ++i) d[n].lo -= a.size[i] - 1;
        for (; j < b.dims && b.stride[j] == s; ++j) d[n].hi += b.size[j] - 1;
        ++n;
    }
    int tries = 100000;
    return comes_within((int64_t)(b.at - a.at), d, n, 1 - b.row, a.row - 1, tries);
}

// Whether an output meets another one or an input
inline bool outputs_meet(std::initializer_list<Area> outputs, std::initializer_list<Area> inputs)
{
    for (auto o = outputs.begin(); o != outputs.end(); ++o) {
        for (auto x = outputs.begin(); x != o; ++x)
            if (meet(*x, *o)) return true;
        for (const Area &x : inputs)
            if (meet(x, *o)) return true;
    }
    return false;
}

} // namespace pf
