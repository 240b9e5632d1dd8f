// The host arithmetic of the relative position bias in a process whose memory has run out.
#include "../../paper_2103_03936_amd/csrc/pf_attn_bias.h"

#include <stdlib.h>

#include <new>

static bool out_of_memory;
void *operator new(size_t n)
{
    void *p = out_of_memory ? nullptr : malloc(n);
    if (!p) throw std::bad_alloc();
    return p;
}
void operator delete(void *p) noexcept { free(p); }
void operator delete(void *p, size_t) noexcept { free(p); }

// the sum of all borders, or -1 if anything was thrown
extern "C" int attention_borders(int side, int max_distance)
{
    int sum = 0;
    out_of_memory = true;
    try {
        const pf::AttnBuckets t = pf::attn_buckets(side, max_distance);
        for (int k = 0; k < t.borders; ++k) sum += t.border[k];
    } catch (...) {
        sum = -1;
    }
    out_of_memory = false;
    return sum;
}
