"""The residual block y = x + dropout(ffn(norm(x))) run as a whole, forward and backward, each tensor on the way held against the
formula of its own step in 64 bits for the tensors that the step read: element by element, one rounding and the sums' bound."""
import pytest
import torch

from paper_1812_07816_amd import ffn, glue
from tests.test_ffn_gpu import HALF, U, act64, close, sums
from tests.test_mixing_block_gpu import Block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,C,F", [(1, 64, 128), (50, 40, 72), (333, 136, 264), (2000, 320, 1280)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_each_step_of_a_block(device, rows, C, F, dtype, act):
    half, p = HALF[dtype], 0.25
    gen = torch.Generator().manual_seed(rows + C)
    x, dy = (torch.randn(rows, C, generator=gen).to(dtype).to(device) for _ in range(2))
    b = Block(rows, C, F, dtype, p, act=act)
    y = b.forward(x)
    h_fwd = ffn.ffn_gate(b.desc, b.n, b.w1)
    dx, dw1, dw2, dgamma, dbeta = b.backward(x, dy)
    kept = glue.dropout_bwd(torch.ones_like(x), p, 99, 4, dev_offset=b.step) != 0
    scale = 65536 / round((1 - p) * 65536)
    D = lambda t: t.double()  # noqa: E731

    def held(got, q, w, what, h=half):
        ref, e = sums(q, w)
        close(got, ref, 1.01 * (h * ref.abs() + e), what)

    # n
    X = D(x)
    mean = X.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((X - mean).square().mean(1, keepdim=True) + glue.IN_EPS)
    xhat = (X - mean) * rstd
    d_mean = 64 * U * X.abs().mean(1, keepdim=True)
    d_rstd = 64 * U + 2 * rstd * (d_mean + U * X.abs()).square().mean(1, keepdim=True).sqrt()
    ref = xhat * D(b.gamma) + D(b.beta)
    tol = half * ref.abs() + D(b.gamma).abs() * (rstd * (d_mean + 2 * U * X.abs()) + xhat.abs() * (d_rstd + 4 * U)) + 4 * U * D(b.beta).abs()
    close(b.n, ref, 1.01 * tol + 1e-30, "n")
    # [g | u], h, f, y
    held(b.gu, D(b.n), D(b.w1).t(), "gu")
    r, e = sums(D(b.n), D(b.w1).t())
    g, u, eg, eu = r[:, :F], r[:, F:], e[:, :F], e[:, F:]
    a, ea = act64(g, act)[0], 1.13 * eg + 32 * U * g.abs()
    close(h_fwd, a * u, 1.01 * (half * (a * u).abs() + a.abs() * eu + u.abs() * ea + ea * eu + 4 * U * (a * u).abs()) + 1e-30, "h")
    held(b.f, D(h_fwd), D(b.w2).t(), "f")
    f = torch.where(kept, D(b.f) * scale, 0.0)
    close(y, X + f, 1.01 * ((half + 2 * U) * (X + f).abs() + 2 * U * f.abs()), "y")
    # df, h, [dg | du], dn
    ref = torch.where(kept, D(dy) * scale, 0.0)
    close(b.df, ref, 1.01 * (half + 2 * U) * ref.abs(), "df")
    g, u = D(b.gu[:, :F]), D(b.gu[:, F:])
    a, da = act64(g, act)
    close(b.h, a * u, 1.01 * (half * (a * u).abs() + 36 * U * (g * u).abs()) + 1e-30, "h again")
    dh, e = sums(D(b.df), D(b.w2))
    close(b.dgu[:, F:], dh * a, 1.01 * (half * (dh * a).abs() + e * a.abs() + 36 * U * (dh * g).abs()) + 1e-30, "du")
    close(b.dgu[:, :F], dh * u * da, 1.01 * ((half + 4 * U) * (dh * u * da).abs() + e * (u * da).abs() + 64 * U * (1 + g.abs()) * (dh * u).abs()) + 1e-30, "dg")
    held(b.dn, D(b.dgu), D(b.w1), "dn")
    # weights
    held(dw1, D(b.dgu).t().contiguous(), D(b.n), "dw1", 0)
    held(dw2, D(b.df).t().contiguous(), D(b.h), "dw2", 0)
    # dx, dgamma, dbeta
    m, q = D(b.stats[:, :1]), D(b.stats[:, 1:])
    xhat, dn = (X - m) * q, D(b.dn)
    gg = dn * D(b.gamma)
    ref = q * (gg - gg.mean(1, keepdim=True) - xhat * (gg * xhat).mean(1, keepdim=True)) + D(dy)
    dxh = 2 * U * (X.abs() + m.abs()) * q + 2 * U * xhat.abs()
    mg, mgx = gg.abs().mean(1, keepdim=True), (gg * xhat).abs().mean(1, keepdim=True)
    tol = q * (8 * U * gg.abs() + 64 * U * mg + xhat.abs() * (64 * U * mgx + (gg.abs() * dxh).mean(1, keepdim=True)) + (dxh + 8 * U * xhat.abs()) * mgx)
    close(dx, ref, 1.01 * (half * ref.abs() + tol + 4 * U * (D(dy).abs() + ref.abs())) + 1e-30, "dx")
    n = rows / 64 + 320      # (terms of a sum in 32 bits, at most)
    close(dgamma, (dn * xhat).sum(0), n * U * (dn * xhat).abs().sum(0) + (dn.abs() * dxh).sum(0) + 1e-30, "dgamma")
    close(dbeta, dn.sum(0), n * U * dn.abs().sum(0) + 1e-30, "dbeta")
