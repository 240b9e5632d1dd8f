"""Overlapping outputs through the package: refused, with nothing written; slices that lie between each other are not."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_refused_and_taken():
    import paper_2103_03936_amd as pf
    B, L, H, D = 2, 9, 2, 32
    gen = torch.Generator("cuda").manual_seed(3)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    Q, K, V, dO = (new(B, L, H, D) for _ in range(4))
    O_, lse = pf.pf_attention_fwd(Q, K, V)
    want = pf.pf_attention_bwd(Q, K, V, O_, lse, dO)
    n = Q.numel()
    room = torch.full((4 * n,), 7.0, device="cuda")
    cut = lambda i: room[i:i + n].view(B, L, H, D)  # noqa: E731
    for out in ((cut(0), cut(n - 4), cut(2 * n)), (cut(0), cut(n), cut(0)), (cut(0), cut(n), cut(2 * n - 64))):
        with pytest.raises(pf.PfError):
            pf.pf_attention_bwd(Q, K, V, O_, lse, dO, out=out)
    with pytest.raises(pf.PfError):
        pf.pf_qk_norm_rotate_fwd(Q, K, out=(cut(0), cut(n - 4)))
    with pytest.raises(pf.PfError):
        pf.pf_qk_norm_rotate_fwd(Q, K, out=(K, Q))
    assert (room == 7).all()
    # the room between the heads of one buffer
    wide = torch.zeros(B, L, 3 * H, D, device="cuda")
    wide[:, :, :H], wide[:, :, H:2 * H] = Q, K
    y = pf.pf_qk_norm_rotate_fwd(Q, K)
    pf.pf_qk_norm_rotate_fwd(wide[:, :, :H], wide[:, :, H:2 * H], out=(wide[:, :, 2 * H:], wide[:, :, H:2 * H]))
    assert torch.equal(wide[:, :, 2 * H:], y[0]) and torch.equal(wide[:, :, H:2 * H], y[1]) and torch.equal(wide[:, :, :H], Q)
    got = pf.pf_attention_bwd(Q, K, V, O_, lse, dO, out=(cut(0), cut(n), cut(2 * n)))
    for a, b in zip(got[:3], want):
        assert torch.equal(a, b)
    assert (room[3 * n:] == 7).all()
    # the room behind the first sequence's keys of a cache
    cache = torch.zeros(B, 64, H, D, device="cuda")
    cache[:, :L] = K
    dq = cache.view(-1)[20 * H * D:20 * H * D + n].view(B, L, H, D)
    got = pf.pf_attention_bwd(Q, cache[:, :L], V, O_, lse, dO, out=(dq, None, None))
    assert got[0] is dq and all(torch.equal(a, b) for a, b in zip(got[:3], want)) and torch.equal(cache[:, :L], K)
