"""The feed-forward block and the normalisation on operands beyond 2 GiB, each along and across the contraction, and beyond 2^31
values: rows and columns at both ends against their formulas in 64 bits."""
import pytest
import torch

from paper_1812_07816_amd import ffn, glue
from tests.test_ffn_gpu import HALF, U, act64, close, sums

pytestmark = pytest.mark.gpu
GIB2 = 2 ** 31


def normal(shape, scale, dtype, device, seed):
    gen = torch.Generator(device=device).manual_seed(seed)
    return torch.randn(shape, generator=gen, device=device, dtype=torch.float32).mul_(scale).to(dtype)


def held(got, a, b, half, what):
    """got = a b within the sums' bound and one rounding."""
    ref, e = sums(a, b)
    close(got, ref, 1.01 * (half * ref.abs() + e), what)


def test_weights_and_gate_beyond_2_gib(device):
    """F = 65536: w1, w2, [g | u] and its gradient are of more than 2 GiB each; 8321 rows and one."""
    dt, half = torch.bfloat16, HALF[torch.bfloat16]
    rows, C, F, O = 8321, 8200, 65536, 16400
    x, dy = normal((rows, C), 1, dt, device, 1), normal((rows, O), 1, dt, device, 2)
    w1, w2 = normal((2 * F, C), C ** -0.5, dt, device, 3), normal((O, F), F ** -0.5, dt, device, 4)
    assert min(t.numel() for t in (w1, w2)) * 2 > GIB2 and rows * 2 * F * 2 > GIB2
    some, cols = [0, 255, 4097, 8191, rows - 1], [0, 31, 32, 40000, F - 1]
    d = ffn.make_desc(rows, C, F, O, "silu", dt)
    gu = torch.full((rows, 2 * F), float("nan"), dtype=dt, device=device)
    y = ffn.ffn_fwd(d, x, w1, w2, gu=gu)
    h = ffn.ffn_gate(d, x, w1)
    both = cols + [F + c for c in cols]
    held(gu[:, both], x.double(), w1[both].double().t(), half, "columns of [g | u]")
    held(gu[some], x[some].double(), w1.double().t(), half, "rows of [g | u]")
    held(y[some], h[some].double(), w2.double().t(), half, "rows of y")
    one = ffn.make_desc(1, C, F, O, "silu", dt)
    gu1 = torch.empty((1, 2 * F), dtype=dt, device=device)
    y1, h1 = ffn.ffn_fwd(one, x[-1:], w1, w2, gu=gu1), ffn.ffn_gate(one, x[-1:], w1)
    held(gu1, x[-1:].double(), w1.double().t(), half, "[g | u] of one row")
    held(y1, h1.double(), w2.double().t(), half, "y of one row")
    del y, h
    dx, dgu, h = ffn.ffn_dgrad(d, dy, w1, w2, gu)
    g, u = gu[some, :F].double(), gu[some, F:].double()
    a, da = act64(g, "silu")
    dh, e = sums(dy[some].double(), w2.double())
    close(h[some], a * u, 1.01 * (half * (a * u).abs() + 36 * U * (g * u).abs()) + 1e-30, "h")
    close(dgu[some, F:], dh * a, 1.01 * (half * (dh * a).abs() + e * a.abs() + 36 * U * (dh * g).abs()) + 1e-30, "du")
    close(dgu[some, :F], dh * u * da, 1.01 * ((half + 4 * U) * (dh * u * da).abs() + e * (u * da).abs() + 64 * U * (1 + g.abs()) * (dh * u).abs()) + 1e-30, "dg")
    held(dx[some], dgu[some].double(), w1.double(), half, "dx")
    dw1, dw2 = ffn.ffn_wgrad(d, x, dgu, h, dy)
    held(dw1[both], dgu[:, both].double().t().contiguous(), x.double(), 0, "rows of dw1")
    held(dw2[:, cols], dy.double().t().contiguous(), h[:, cols].double(), 0, "columns of dw2")


@pytest.mark.parametrize("dtype,rows", [(torch.bfloat16, 2 ** 20 + 37), (torch.float32, 2 ** 19 + 37)], ids=["bf16", "f32"])
def test_rows_beyond_2_gib(device, dtype, rows):
    """x and dy of more than 2 GiB, along the contraction forward and across it in the weight gradients."""
    C, F, half = 1040, 24, HALF[dtype]
    x, dy = normal((rows, C), 1, dtype, device, 1), normal((rows, C), 1, dtype, device, 2)
    assert x.numel() * x.element_size() > GIB2
    w1, w2 = normal((2 * F, C), C ** -0.5, dtype, device, 3), normal((C, F), F ** -0.5, dtype, device, 4)
    some = [0, 129, rows // 2, rows - 38, rows - 1]
    d = ffn.make_desc(rows, C, F, C, "silu", dtype)
    gu = torch.empty((rows, 2 * F), dtype=dtype, device=device)
    y, h = ffn.ffn_fwd(d, x, w1, w2, gu=gu), ffn.ffn_gate(d, x, w1)
    held(gu[some], x[some].double(), w1.double().t(), half, "[g | u]")
    held(y[some], h[some].double(), w2.double().t(), half, "y")
    del y
    dx, dgu, h = ffn.ffn_dgrad(d, dy, w1, w2, gu)
    dh, e = sums(dy[some].double(), w2.double())
    g = gu[some, :F].double()
    a = act64(g, "silu")[0]
    close(dgu[some, F:], dh * a, 1.01 * (half * (dh * a).abs() + e * a.abs() + 36 * U * (dh * g).abs()) + 1e-30, "du")
    held(dx[some], dgu[some].double(), w1.double(), half, "dx")
    del dx
    dw1, dw2 = ffn.ffn_wgrad(d, x, dgu, h, dy)
    cols = [0, 7, C - 1]
    held(dw1[:, cols], dgu.double().t().contiguous(), x[:, cols].double(), 0, "columns of dw1")
    held(dw2[cols], dy[:, cols].double().t().contiguous(), h.double(), 0, "rows of dw2")


@pytest.mark.parametrize("dtype,C", [(torch.bfloat16, 1032), (torch.float32, 1029)], ids=["bf16", "f32 odd"])
def test_normalisation_beyond_2_31_values(device, dtype, C):
    rows = 2 ** 31 // C + 4133
    x, dy = normal((rows, C), 1, dtype, device, 1), normal((rows, C), 1, dtype, device, 2)
    gamma, beta = normal((C,), 0.2, torch.float32, device, 3) + 1, normal((C,), 0.2, torch.float32, device, 4)
    y, stats = glue.layernorm_fwd(x, gamma, beta)
    some = [0, 1, rows // 3, rows - 4133, rows - 1]
    xd = x[some].double()
    mean = xd.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((xd - mean).square().mean(1, keepdim=True) + glue.IN_EPS)
    xhat = (xd - mean) * rstd
    # 64 roundings of a mean (32 sums in a lane, across the lanes, a product), twice that for the squares around it
    d_mean = 64 * U * xd.abs().mean(1, keepdim=True)
    d_rstd = 64 * U + 2 * rstd * (d_mean + U * xd.abs()).square().mean(1, keepdim=True).sqrt()
    ref = xhat * gamma.double() + beta.double()
    tol = HALF[dtype] * ref.abs() + gamma.double().abs() * (rstd * (d_mean + 2 * U * xd.abs()) + xhat.abs() * (d_rstd + 4 * U)) + 4 * U * beta.double().abs()
    close(y[some], ref, 1.01 * tol + 1e-30, "y")
    del y
    dx, dgamma, dbeta = glue.layernorm_bwd(dy, x, stats, gamma)
    m, r = stats[some, :1].double(), stats[some, 1:].double()
    xhat = (xd - m) * r
    g = dy[some].double() * gamma.double()
    ref = r * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    dxh = 2 * U * (xd.abs() + m.abs()) * r + 2 * U * xhat.abs()
    mg, mgx = g.abs().mean(1, keepdim=True), (g * xhat).abs().mean(1, keepdim=True)
    tol = r * (8 * U * g.abs() + 64 * U * mg + xhat.abs() * (64 * U * mgx + (g.abs() * dxh).mean(1, keepdim=True)) + (dxh + 8 * U * xhat.abs()) * mgx)
    close(dx[some], ref, 1.01 * ((HALF[dtype] + 4 * U) * ref.abs() + tol) + 1e-30, "dx")
    # sums over all rows, a piece at a time.  A lane adds every 2048th row (512 workgroups of 4 rows), the workgroup 4 lanes, the rest is in 64 bits
    s = {k: torch.zeros(C, dtype=torch.float64, device=device) for k in ("g", "ag", "b", "ab", "e")}
    for i in range(0, rows, 1 << 18):
        d = dy[i:i + (1 << 18)].double()
        q = stats[i:i + (1 << 18)].double()
        xp = x[i:i + (1 << 18)].double()
        z = (xp - q[:, :1]) * q[:, 1:]
        s["b"] += d.sum(0)
        s["ab"] += d.abs().sum(0)
        s["g"] += (d * z).sum(0)
        s["ag"] += (d * z).abs().sum(0)
        s["e"] += (d.abs() * (2 * U * (xp.abs() + q[:, :1].abs()) * q[:, 1:] + 2 * U * z.abs())).sum(0)
    n = rows / 2048 + 16
    close(dgamma, s["g"], 1.01 * (n * U * s["ag"] + s["e"]), "dgamma")
    close(dbeta, s["b"], 1.01 * n * U * s["ab"], "dbeta")
