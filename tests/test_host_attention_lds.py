"""Attention of few queries over many keys is given to the kernel that splits the keys only where its LDS fits a workgroup
(no GPU: that kernel is the one that needs a workspace)."""
import ctypes

import pytest

import paper_2103_03936_amd as pf

LDS = 160 * 1024


def _need(dtype, D, G, Lq, buckets, far):
    """Two waves' tiles of 32 keys and values, two of each, rows padded to 32, 64 or 128 values; 32 maxima and sums a wave; the bias of
    the heads that 32 rows touch; a byte for each distance."""
    row = 32 if D <= 32 else 64 if D <= 64 else 128
    heads = max(len({r // Lq for r in range(t, min(t + 32, Lq * G))}) for t in range(0, Lq * G, 32))
    return 2 * 4 * 32 * row * (4 if dtype == pf.PF_F32 else 2) + 2 * 2 * 32 * 4 + buckets * heads * 4 + 2 * far + 1


@pytest.mark.parametrize("dtype", [pf.PF_F32, pf.PF_BF16])
@pytest.mark.parametrize("D", [32, 64, 80, 128])
@pytest.mark.parametrize("G,Lq", [(1, 1), (8, 1), (32, 1), (33, 1), (64, 1), (8, 4), (40, 3), (1, 32)])
def test_split_fits(G, Lq, D, dtype):
    seen = set()
    for buckets, distance in ((0, 0), (32, 128), (64, 1024), (128, 1024), (256, 129), (256, 1024)):
        d = pf.pf_attention_desc(1, Lq, 16384, G, 1, D, 1, buckets, distance, 0, dtype, 1.0)
        need = _need(dtype, D, G, Lq, buckets, distance) if buckets else 0
        split = pf.lib.pf_attention_fwd_workspace_bytes(ctypes.byref(d)) > 0
        if need > LDS:
            assert not split, (buckets, distance, need)
        if need < LDS - 2048:  # (the last head of a tile may be counted although it is not touched)
            assert split, (buckets, distance, need)
        seen.add(split)
    assert True in seen
