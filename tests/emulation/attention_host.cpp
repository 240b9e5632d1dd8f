// The host arithmetic of the relative position bias, for the test that calls it without a GPU.
#include "../../paper_2103_03936_amd/csrc/pf_attn_bias.h"

extern "C" int attention_bucket(int side, int max_distance, int n)
{
    const pf::AttnBuckets t = pf::attn_buckets(side, max_distance);
    if (n < t.exact) return n;
    int u = t.exact;
    for (int k = 0; k < t.borders; ++k) u += n >= t.border[k];
    return u;
}
extern "C" int attention_far(int side, int max_distance) { return pf::attn_buckets(side, max_distance).far; }
