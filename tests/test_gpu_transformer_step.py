"""The operators together, as a factorized Transformer layer uses them: a training step (shared Q, K, V projection, norms and
rotation, attention over a padded batch, output projection and feed-forward block, all backward into one gradient buffer,
AdamW) against autograd in double, eager and captured; and a cache filled by a chunk and then token by token."""
import numpy as np
import pytest
import torch

from operator_bounds import E, assert_within, attention_bounds
from oracle import operators as O

pytestmark = pytest.mark.gpu

B, L, H, D, R, FF, NB, DIST = 3, 70, 2, 64, 32, 256, 32, 40
d, M = H * D, B * L
LENS = [70, 33, 1]
SHAPES = [("Vq", (3, d, R)), ("Uq", (3, d, R)), ("bq", (3, d)), ("gq", (D,)), ("gk", (D,)), ("table", (NB, H)), ("Vo", (d, R)),
          ("Uo", (d, R)), ("bo", (d,)), ("V1", (d, R)), ("U1", (FF, R)), ("b1", (FF,)), ("V2", (FF, R)), ("U2", (d, R)), ("b2", (d,))]
FLOAT = ("gq", "gk", "table")  # what the operators read as float32
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


class Layer:
    """Parameters in float32 with copies in the compute type, gradients in one buffer."""

    def __init__(self, dtype, bits, seed=5):
        import paper_2103_03936_amd as pf
        self.pf, self.dtype = pf, dtype
        g = torch.Generator().manual_seed(seed)
        self.p = {}
        for n, s in SHAPES:
            std = 1.0 / s[-2] ** 0.5 if n[0] == "V" else 1.0 / R ** 0.5 if n[0] == "U" else 0.5
            x = torch.randn(s, generator=g) * std + (1.0 if n[0] == "g" else 0.0)
            self.p[n] = x.to(torch.bfloat16).float().cuda()
        low = dtype == "bf16"
        self.c = {n: t.to(torch.bfloat16) if low and n not in FLOAT else t for n, t in self.p.items()}
        self.grads = pf.GradBuffer(SHAPES)
        names = [n for n, _ in SHAPES]
        self.opt = pf.AdamW([self.p[n] for n in names], [self.grads.views[n] for n in names], lr=1e-2, state_bits=bits,
                            copies=[self.c[n] if low and n not in FLOAT else None for n in names], weight_decay=0.1)
        self.lens = torch.tensor(LENS, dtype=torch.int32).cuda()

    def inputs(self, seed):
        g = torch.Generator().manual_seed(seed)
        return [torch.randn((M, d), generator=g).to(TYPES[self.dtype]).cuda() for _ in range(2)]

    def run(self, x, dy):
        """Forward and backward: (y, dx); parameter gradients in self.grads."""
        pf, c, heads = self.pf, self.c, lambda t: t.view(B, L, H, D)  # noqa: E731
        G = self.grads.zero().views
        at = dict(max_distance=DIST, q_len=self.lens, kv_len=self.lens)
        Y, Tq = pf.pf_lowrank_linear_shared_fwd(x, c["Vq"], c["Uq"], c["bq"])
        q, k, v = (heads(t) for t in Y)
        qr, kr = pf.pf_qk_norm_rotate_fwd(q, k, c["gq"], c["gk"])
        o, lse = pf.pf_attention_fwd(qr, kr, v, c["table"], **at)
        h, To = pf.pf_lowrank_linear_fwd_ep(o.view(M, d), c["Vo"], c["Uo"], c["bo"], residual=x)
        a, T1 = pf.pf_lowrank_linear_fwd_ep(h, c["V1"], c["U1"], c["b1"], act="relu")
        y, T2 = pf.pf_lowrank_linear_fwd_ep(a, c["V2"], c["U2"], c["b2"], residual=h)

        dz = pf.pf_lowrank_linear_bwd_ep(a, c["V2"], c["U2"], dy, T_saved=T2, x_is_relu=True, has_bias=True,
                                         grads=(G["U2"], G["V2"], G["b2"]))[0]
        dh = pf.pf_lowrank_linear_bwd_ep(h, c["V1"], c["U1"], dz, T_saved=T1, dX_add=dy, has_bias=True,
                                         grads=(G["U1"], G["V1"], G["b1"]))[0]
        do = pf.pf_lowrank_linear_bwd_ep(o.view(M, d), c["Vo"], c["Uo"], dh, T_saved=To, has_bias=True,
                                         grads=(G["Uo"], G["Vo"], G["bo"]))[0]
        dY = torch.empty_like(Y)
        dq, dk, dv = (heads(t) for t in dY)
        pf.pf_attention_bwd(qr, kr, v, o, lse, heads(do), c["table"], grads=G["table"], out=(dq, dk, dv), **at)
        pf.pf_qk_norm_rotate_bwd(q, k, dq, dk, c["gq"], c["gk"], grads=(G["gq"], G["gk"]), out=(dq, dk))
        dx = pf.pf_lowrank_linear_shared_bwd(x, c["Vq"], c["Uq"], dY, T_saved=Tq, has_bias=True, grads=(G["Uq"], G["Vq"], G["bq"]))[0]
        return y, dx + dh


class _Stored(torch.autograd.Function):
    """What storing a value and its gradient in a type does to them."""

    @staticmethod
    def forward(ctx, x, t):
        ctx.t = t
        return x.to(t).to(x.dtype)

    @staticmethod
    def backward(ctx, g):
        return g.to(ctx.t).to(g.dtype), None


def _double(layer, x, dy, stored):
    """The layer in double, {name: gradient}, y, dx; stored: the type that every operator's result is rounded to, or None."""
    keep = (lambda t: _Stored.apply(t, stored)) if stored is not None else (lambda t: t)
    p = {n: t.detach().cpu().double().requires_grad_() for n, t in layer.c.items()}
    x = x.detach().cpu().double().requires_grad_()
    heads = lambda t: t.view(B, L, H, D).transpose(1, 2)  # noqa: E731
    low = lambda x, V, U, b: keep(x @ V) @ U.T + b  # noqa: E731
    q, k, v = (heads(keep(low(x, p["Vq"][i], p["Uq"][i], p["bq"][i]))) for i in range(3))
    pos = torch.arange(L, dtype=torch.float64)
    turn = pos[:, None] * 10000.0 ** (-2.0 * torch.arange(D // 2, dtype=torch.float64) / D)

    def rotate(t, g):
        t = t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt() * g
        a, b = t[..., :D // 2], t[..., D // 2:]
        return keep(torch.cat([a * turn.cos() - b * turn.sin(), a * turn.sin() + b * turn.cos()], -1))

    dist = np.arange(L)[None, :] - np.arange(L)[:, None]
    bucket = torch.tensor([[O.bucket(int(e), NB, DIST, True) for e in row] for row in dist])
    s = rotate(q, p["gq"]) @ rotate(k, p["gk"]).transpose(-1, -2) / D ** 0.5 + p["table"][bucket].permute(2, 0, 1)
    seen = torch.arange(L)[None, :] < torch.tensor(LENS)[:, None]
    pr = keep(s.masked_fill(~seen[:, None, None, :], -torch.inf).softmax(-1)) * seen[:, None, :, None]
    o = keep(pr @ v).transpose(1, 2).reshape(M, d)
    h = keep(low(o, p["Vo"], p["Uo"], p["bo"]) + x)
    a = keep(low(h, p["V1"], p["U1"], p["b1"]).relu())
    y = keep(low(a, p["V2"], p["U2"], p["b2"]) + h)
    y.backward(dy.detach().cpu().double())
    return {n: t.grad for n, t in p.items()}, y.detach(), x.grad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_step_against_autograd(dtype):
    """As far from the double-precision layer as rounding every stored value takes that layer itself, times 4 (one draw of the
    roundings against another); float32 times 64: there a sum of up to 256 terms is rounded as often as it has terms, which
    makes 16 roundings of one in the mean, and they are not in the model."""
    layer = Layer(dtype, 32)
    x, dy = layer.inputs(1)
    grads, y64, dx64 = _double(layer, x, dy, None)
    rough, yr, dxr = _double(layer, x, dy, TYPES[dtype])
    y, dx = layer.run(x, dy)
    factor = 4 if dtype == "bf16" else 64
    for name, got, want, near in [("y", y, y64, yr), ("dx", dx, dx64, dxr)] + [
            (n, layer.grads.views[n], grads[n], rough[n]) for n, _ in SHAPES]:
        off, allowed = (got.cpu().double() - want).norm().item(), factor * (near - want).norm().item()
        if name == "b2":  # no stored value is on the way to it: a sum of M float32 terms is within (M + 1) E of their magnitudes' sum
            allowed = (M + 1) * E * dy.cpu().double().abs().sum(0).norm().item()
        assert off <= allowed, f"{name}: {off} off, allowed {allowed}, norm {want.norm().item()}"

    # the optimizer's step with the gradients as they are: p (1 - lr wd) and the update, about ten roundings each
    before = {n: t.cpu().double().numpy() for n, t in layer.p.items()}
    layer.opt.step()
    for n, _ in SHAPES:
        g, p = layer.grads.views[n].cpu().double().numpy(), before[n]
        want = O.adamw(p, g, 0 * p, 0 * p, 1, np.float64(np.float32(1e-2)), 0.9, 0.999, 1e-8, np.float64(np.float32(0.1)))[0]
        assert_within(layer.p[n], want, E * (4 * np.abs(p) + 32 * 1e-2), n)
        assert torch.equal(layer.c[n], layer.p[n].to(layer.c[n].dtype))


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_step(bits):
    """Whole steps from a graph, with eager work in between, make the same parameters bit for bit as eager steps."""
    one, two = Layer("bf16", bits), Layer("bf16", bits)
    x, dy = one.inputs(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one.run(x, dy)
        one.opt.step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    two.run(x, dy)
    two.opt.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = one.run(x, dy)
        one.opt.step()
    for seed in (2, 3, 4):
        fresh = one.inputs(seed)
        x.copy_(fresh[0])
        dy.copy_(fresh[1])
        one.opt.lr.fill_(1e-2 / seed)
        two.opt.lr.fill_(1e-2 / seed)
        graph.replay()
        y2, dx2 = two.run(*fresh)
        two.opt.step()
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(dx, dx2)
        for n, _ in SHAPES:
            assert torch.equal(one.grads.views[n], two.grads.views[n]), n
            assert torch.equal(one.p[n], two.p[n]) and torch.equal(one.c[n], two.c[n]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cache_by_chunk_and_by_token(dtype):
    """Keys go into a cache [B, heads, capacity, D] where the rotation writes them, a chunk first, then single tokens; each step's
    attention is that of the whole sequence.  Behind the tokens the cache holds NaN."""
    import paper_2103_03936_amd as pf
    n, hq, hk, cap, first = 57, 6, 2, 80, 50
    g = torch.Generator().manual_seed(9)
    new = lambda h: torch.randn((B, n, h, D), generator=g).to(TYPES[dtype]).cuda()  # noqa: E731
    Q, K, V = new(hq), new(hk), new(hk)
    table = torch.randn((NB, hq), generator=g).cuda()
    gam = [torch.rand((D,), generator=g).cuda() + 0.5 for _ in range(2)]
    skip = torch.tensor([0, 3, 11], dtype=torch.int32)  # tokens of each cache that were there before
    kc, vc = (torch.full((B, hk, cap, D), float("nan"), dtype=TYPES[dtype], device="cuda").transpose(1, 2) for _ in range(2))
    old = [torch.randn((B, 11, hk, D), generator=g).to(TYPES[dtype]).cuda() for _ in range(2)]
    for b in range(B):
        kc[b, :skip[b]], vc[b, :skip[b]] = old[0][b, :skip[b]], old[1][b, :skip[b]]
    where = skip[:, None] + torch.arange(n, dtype=torch.int32)
    qs, outs = [], []
    for lo, hi in [(0, first)] + [(i, i + 1) for i in range(first, n)]:
        q = torch.empty((B, hi - lo, hq, D), dtype=TYPES[dtype], device="cuda")
        for b in range(B):  # (every sequence's tokens go to a place of their own)
            at = slice(int(skip[b]) + lo, int(skip[b]) + hi)
            pf.pf_qk_norm_rotate_fwd(Q[b:b + 1, lo:hi], K[b:b + 1, lo:hi], *gam, positions=where[b:b + 1, lo:hi].contiguous().cuda(),
                                     out=(q[b:b + 1], kc[b:b + 1, at]))
            vc[b, at] = V[b, lo:hi]
        kv_len = (skip + hi).cuda()
        o, _ = pf.pf_attention_fwd(q, kc, vc, table, causal=True, max_distance=DIST, bidirectional=False,
                                   q_start=kv_len - (hi - lo), kv_len=kv_len)
        qs.append(q)
        outs.append(o)
    q, got = torch.cat(qs, 1), torch.cat(outs, 1)
    qw, kw = pf.pf_qk_norm_rotate_fwd(Q, K, *gam, positions=where.contiguous().cuda())
    assert torch.equal(q, qw)
    for b in range(B):
        assert torch.equal(kc[b, skip[b]:skip[b] + n], kw[b])
        m = int(skip[b]) + n
        f = lambda t: t.cpu().double().numpy()  # noqa: E731
        a = O.Attention(f(q[b:b + 1]), f(kc[b:b + 1, :m]), f(vc[b:b + 1, :m]), f(table), causal=True, max_distance=DIST,
                        bidirectional=False, q_start=skip[b:b + 1].numpy())
        assert_within(got[b:b + 1], a.O, attention_bounds(a, np.ones_like(a.O), dtype)[0], f"sequence {b}")
