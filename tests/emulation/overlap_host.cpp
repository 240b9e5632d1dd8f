// The host arithmetic of overlapping tensors, for the test that calls it without a GPU.
#include "../../paper_2103_03936_amd/csrc/pf_overlap.h"

extern "C" int overlap_meet(const int64_t *a, const int64_t *b)
{ // at, B, L, heads, strides, D
    const auto area = [](const int64_t *x) {
        const int64_t s[3] = {x[4], x[5], x[6]};
        return pf::Area((const void *)(uintptr_t)(1000 + x[0]), x[1], x[2], x[3], s, x[7], 1);
    };
    return pf::meet(area(a), area(b));
}
