"""GELU and its derivative over the whole range of the gate, with bounds relative to their values: far below zero
g Phi(g) is small but not zero, and the sums of a product give any g."""
import pytest
import torch

from paper_1812_07816_amd import ffn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = 2.0 ** -122      # (smaller values may be cut to zero on the way)
DTYPES = [torch.float32, torch.bfloat16]


def phi_error(g, dtype):
    """Relative error of Phi(g).  fp32: erfc of a z = -g / sqrt 2 with two roundings, each of which moves it by up to 1 + 2 z^2 = 1 + g^2 of
    itself, and the function's own 8 units in the last place.  bf16: that of the approximation (2e-4) and of its exponential, whose
    argument carries three roundings of up to g^2 / 2, and some twelve units of the products around it."""
    return (2 * (1 + g * g) + 16) * U if dtype == torch.float32 else 2e-4 + (2 * g * g + 24) * U


def gates(dtype):
    g = torch.cat([torch.linspace(-12.5, 12.5, 4001), torch.tensor([-1e4, -40.0, -5.5, -1e-3, 0.0, 1e-3, 40.0, 1e4])])
    return g.to(dtype).unique()


def close(got, ref, tol, what):
    off = (got.cpu().double() - ref).abs()
    assert torch.isfinite(got).all(), what
    assert (off <= tol).all(), (what, float((off / tol).max()))


def functions(g):
    c = 0.5 * torch.special.erfc(-g / 2 ** 0.5)
    p = torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5
    return c, p


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [None, 40], ids=["all", "few"])
def test_forward(device, dtype, rows):
    """u = 1 and g from one product each: [g | u] is exact."""
    C, F = 8, 16
    g = gates(dtype)[:rows]
    x = torch.zeros((g.numel(), C), dtype=dtype)
    x[:, 0], x[:, 1] = g, 1
    w1 = torch.zeros((2 * F, C), dtype=dtype)
    w1[:F, 0], w1[F:, 1] = 1, 1
    d = ffn.make_desc(g.numel(), C, F, 8, "gelu", dtype)
    gu = torch.empty((g.numel(), 2 * F), dtype=dtype, device=device)
    h = ffn.ffn_gate(d, x.to(device), w1.to(device), gu=gu)
    assert torch.equal(gu.cpu(), torch.cat([g[:, None].expand(-1, F), torch.ones(g.numel(), F, dtype=dtype)], 1))
    g = g.double()[:, None].expand(-1, F)
    ref = g * functions(g)[0]
    close(h, ref, 1.01 * ref.abs() * (HALF[dtype] + phi_error(g, dtype) + 4 * U) + TINY, "h")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_data_gradient(device, dtype):
    """dh = 1 and u = 1: [dg | du] is [act' | act]."""
    C, F = 8, 16
    g = gates(dtype)
    dy = torch.zeros((g.numel(), 8), dtype=dtype)
    dy[:, 0] = 1
    w2 = torch.zeros((8, F), dtype=dtype)
    w2[0] = 1
    gu = torch.cat([g[:, None].expand(-1, F), torch.ones(g.numel(), F, dtype=dtype)], 1)
    d = ffn.make_desc(g.numel(), C, F, 8, "gelu", dtype)
    _, dgu, h = ffn.ffn_dgrad(d, dy.to(device), torch.zeros((2 * F, C), dtype=dtype, device=device), w2.to(device), gu.to(device))
    g = g.double()[:, None].expand(-1, F)
    c, p = functions(g)
    act, da = g * c, c + g * p
    tol = 1.01 * act.abs() * (HALF[dtype] + phi_error(g, dtype) + 4 * U) + TINY
    close(h, act, tol, "h")
    close(dgu[:, F:], act, tol, "du")
    # e^(-g^2 / 2): its argument carries three roundings at most, that is 1.5 g^2 U, and the function 4 units
    close(dgu[:, :F], da, 1.01 * (HALF[dtype] * da.abs() + (g * p).abs() * (2 * g * g + 12) * U + c * phi_error(g, dtype) + 4 * U * da.abs()) + TINY, "dg")
