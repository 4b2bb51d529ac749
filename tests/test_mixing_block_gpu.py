"""Layer normalisation, gated feed-forward block and dropout together, as a residual block uses them: forward, backward,
captured and replayed, on streams of their own, and its gradients against the formulas and against differences."""
import pytest
import torch

from paper_1812_07816_amd import ffn, glue

pytestmark = pytest.mark.gpu


class Block:
    """y = x + dropout(ffn(norm(x))) with buffers of its own."""

    def __init__(self, rows, C, F, dtype, p, seed=0, act="silu"):
        gen = torch.Generator().manual_seed(seed)
        r = lambda s, *shape: (torch.randn(*shape, generator=gen) * s)  # noqa: E731
        self.w1, self.w2 = r(C ** -0.5, 2 * F, C).to(dtype).cuda(), r(F ** -0.5, C, F).to(dtype).cuda()
        self.gamma, self.beta = (1 + r(0.1, C)).cuda(), r(0.1, C).cuda()
        self.desc, self.p, self.act = ffn.make_desc(rows, C, F, C, act, dtype), p, act
        new = lambda *s, d=dtype: torch.empty(s, dtype=d, device="cuda")  # noqa: E731
        self.n, self.f, self.y, self.dx, self.df, self.dn = (new(rows, C) for _ in range(6))
        self.gu, self.dgu, self.h = new(rows, 2 * F), new(rows, 2 * F), new(rows, F)
        self.stats = new(rows, 2, d=torch.float32)
        self.dw1, self.dw2, self.dgamma, self.dbeta = (new(*s, d=torch.float32) for s in ((2 * F, C), (C, F), (C,), (C,)))
        self.ws = torch.empty(max(max(ffn.workspace_bytes(self.desc, q) for q in range(3)), glue.layernorm_workspace(rows, C).numel(), 16), dtype=torch.uint8, device="cuda")
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def forward(self, x):
        glue.layernorm_fwd(x, self.gamma, self.beta, self.n, self.stats)
        ffn.ffn_fwd(self.desc, self.n, self.w1, self.w2, self.f, gu=self.gu, ws=self.ws)
        glue.dropout_fwd(self.f, self.p, 99, 4, residual=x, out=self.y, dev_offset=self.step)
        return self.y

    def backward(self, x, dy):
        glue.dropout_bwd(dy, self.p, 99, 4, da=self.df, dev_offset=self.step)
        ffn.ffn_dgrad(self.desc, self.df, self.w1, self.w2, self.gu, self.dn, self.dgu, self.h, ws=self.ws)
        ffn.ffn_wgrad(self.desc, self.n, self.dgu, self.h, self.df, self.dw1, self.dw2, ws=self.ws)
        glue.layernorm_bwd(self.dn, x, self.stats, self.gamma, self.dx, self.dgamma, self.dbeta, self.ws, add=dy)
        return [self.dx, self.dw1, self.dw2, self.dgamma, self.dbeta]


def formula(b, x, dy):
    """Output and gradients in 64 bits, with the mask taken from the kernel (a tensor of ones dropped)."""
    mask = glue.dropout_bwd(torch.ones(x.shape, device="cuda"), b.p, 99, 4, dev_offset=b.step).double().cpu()
    leaves = [t.double().cpu().requires_grad_() for t in (x, b.w1, b.w2, b.gamma, b.beta)]
    X, w1, w2, gamma, beta = leaves
    mean = X.mean(1, keepdim=True)
    n = (X - mean) / torch.sqrt((X - mean).square().mean(1, keepdim=True) + glue.IN_EPS) * gamma + beta
    g, u = (n @ w1.t()).chunk(2, 1)
    a = g * torch.sigmoid(g) if b.act == "silu" else g * torch.special.ndtr(g)
    y = X + ((a * u) @ w2.t()) * mask
    y.backward(dy.double().cpu())
    return y.detach(), [t.grad for t in leaves]


def rel(got, ref):
    return float((got.double().cpu() - ref).norm() / ref.norm())


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,C,F", [(1, 64, 128), (50, 40, 72), (333, 136, 264)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_gradients_against_the_formulas(device, rows, C, F, dtype, act):
    gen = torch.Generator().manual_seed(rows)
    x, dy = (torch.randn(rows, C, generator=gen).to(dtype).cuda() for _ in range(2))
    b = Block(rows, C, F, dtype, 0.25, act=act)
    y = b.forward(x)
    grads = b.backward(x, dy)
    ry, rg = formula(b, x, dy)
    # bf16: every tensor between two calls is rounded (half a step, 2^-8); in the 2-norm at most the sum of the roundings on the way:
    # n, gu and h, f, y forward; df, gu, dgu, dn, dx and n, h backward, each of which is passed on with a gain of at most 1.2 here.
    # fp32: 2^-24 each, and sums of up to 2 F + C terms.
    tol = 10 * 1.2 * 2.0 ** -8 if dtype == torch.bfloat16 else 1e-5
    assert rel(y, ry) <= tol
    for got, ref in zip(grads, rg):
        assert rel(got, ref) <= tol


def test_gradients_against_differences(device):
    """fp32: sum(y * dy) along the gradient of every input, central differences at h = 2^-9.  y's values are good to about 1e-6:
    300 * 64 of them with random signs move the sum by 1.4e-4, the quotient by 0.036, of a derivative of 1000 and more; the third
    derivative moves it by at most 2e-5 of itself (the formulas in 64 bits)."""
    rows, C, F = 300, 64, 96
    gen = torch.Generator().manual_seed(3)
    x, dy = (torch.randn(rows, C, generator=gen).cuda() for _ in range(2))
    b = Block(rows, C, F, torch.float32, 0.3)
    b.forward(x)
    grads = [g.clone() for g in b.backward(x, dy)]
    for i, (t, g) in enumerate(zip((x, b.w1, b.w2, b.gamma, b.beta), grads)):
        v = (g / g.norm() * t.numel() ** 0.5).contiguous()      # the direction of the gradient itself, of one per value
        h = 2.0 ** -9
        keep, got = t.clone(), []
        for s in (h, -h):
            t.copy_(keep + s * v)
            got.append(float((b.forward(x).double() * dy.double()).sum()))
        t.copy_(keep)
        want = float((g.double() * v.double()).sum())
        assert abs((got[0] - got[1]) / (2 * h) - want) <= 1e-3 * abs(want), i


@pytest.mark.parametrize("rows", [5, 200])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_captured_and_replayed(device, rows, dtype):
    """Two blocks captured into one graph, replayed between eager work on the same tensors: every replay gives the eager bits."""
    x, dy = torch.empty(rows, 72, dtype=dtype, device=device), torch.empty(rows, 72, dtype=dtype, device=device)
    b, e = Block(rows, 72, 136, dtype, 0.3), Block(rows, 72, 136, dtype, 0.3)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.forward(x)
        b.backward(x, dy)
    for i in range(4):
        x.normal_()
        dy.normal_()
        b.step.fill_(i)
        e.step.fill_(i)
        g.replay()
        ref = [e.forward(x)] + e.backward(x, dy)
        torch.cuda.synchronize()
        for p, q in zip([b.y, b.dx, b.dw1, b.dw2, b.dgamma, b.dbeta], ref):
            assert torch.equal(p, q), i


def test_streams_at_once(device):
    """Two blocks of different sizes on two streams give what they give one after the other."""
    x = [torch.randn(r, 64, device=device).bfloat16() for r in (700, 40)]
    blocks = [Block(r, 64, 256, torch.bfloat16, 0.1, seed=r) for r in (700, 40)]
    ref = [[t.clone() for t in [b.forward(v)] + b.backward(v, v)] for b, v in zip(blocks, x)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for b, v, s in zip(blocks, x, streams):
            with torch.cuda.stream(s):
                b.forward(v)
                b.backward(v, v)
    torch.cuda.synchronize()
    for b, r in zip(blocks, ref):
        for p, q in zip([b.y, b.dx, b.dw1, b.dw2, b.dgamma, b.dbeta], r):
            assert torch.equal(p, q)
