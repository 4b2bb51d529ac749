"""The gated feed-forward block against its formulas in 64 bits: rows from one to several tiles, widths that no tile divides,
both types and activations, with and without what the backward pass needs."""
import pytest
import torch

from paper_1812_07816_amd import _lib, ffn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DTYPES = [torch.bfloat16, torch.float32]
# (rows, Cin, F, Cout)
SHAPES = [(1, 8, 8, 8), (1, 1024, 264, 64), (2, 64, 64, 64), (7, 40, 24, 48), (16, 320, 96, 40), (17, 72, 136, 320), (33, 136, 40, 8), (64, 256, 520, 256),
          (65, 128, 128, 128), (129, 8, 72, 264), (300, 200, 520, 200), (257, 328, 200, 72), (1000, 64, 256, 64), (513, 520, 1032, 136), (1331, 24, 88, 24),
          (2, 2048, 2056, 8), (5, 16, 4104, 1032)]


def act64(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    c = torch.special.ndtr(g)
    return g * c, c + g * torch.exp(-g * g / 2) * 0.3989422804014327


def inputs(rows, C, F, O, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed + rows + 7 * C + 13 * F)
    r = lambda s, *shape: (torch.randn(*shape, generator=gen) * s).to(dtype)  # noqa: E731
    return dict(x=r(1, rows, C), w1=r(C ** -0.5, 2 * F, C), w2=r(F ** -0.5, O, F), dy=r(1, rows, O), gu=r(1, rows, 2 * F), dgu=r(0.7, rows, 2 * F), h=r(0.7, rows, F))


def close(got, ref, tol, what=""):
    assert torch.isfinite(got).all(), what
    off = (got.to(ref.device).double() - ref).abs()
    assert (off <= tol).all(), (what, float((off - tol).max()), float((off / tol).max()))


def sums(a, b):
    """Product in 64 bits and the bound of fp32 sums in any order, each rounded or cut (2 U a sum)."""
    k = a.shape[1]
    return a @ b, 2 * U * (k + 1) * (a.abs() @ b.abs()) + 1e-30


def check_forward(device, rows, C, F, O, dtype, where="cpu"):
    """where: the device that forms the reference."""
    act = "gelu" if F % 16 else "silu"
    t = {k: v.to(where) for k, v in inputs(rows, C, F, O, dtype).items()}
    d = ffn.make_desc(rows, C, F, O, act, dtype)
    x, w1, w2 = (t[k].to(device) for k in ("x", "w1", "w2"))
    gu = torch.full((rows, 2 * F), float("nan"), dtype=dtype, device=device)
    y = ffn.ffn_fwd(d, x, w1, w2, gu=gu)
    h = ffn.ffn_gate(d, x, w1)
    ref, e = sums(t["x"].double(), t["w1"].double().t())
    close(gu, ref, 1.01 * (HALF[dtype] * ref.abs() + e), "gu")
    g, u, eg, eu = ref[:, :F], ref[:, F:], e[:, :F], e[:, F:]
    a, da = act64(g, act)
    # |act'| stays below 1.13; the functions and their products are good to 32 U of |g|
    ea = 1.13 * eg + 32 * U * g.abs()
    rh = a * u
    eh = HALF[dtype] * rh.abs() + a.abs() * eu + u.abs() * ea + ea * eu + 4 * U * rh.abs()
    close(h, rh, 1.01 * eh + 1e-30, "h")
    ry, ey = sums(rh, t["w2"].double().t())
    ey = ey + eh @ t["w2"].double().abs().t()
    close(y, ry, 1.01 * (HALF[dtype] * ry.abs() + ey), "y")
    assert torch.equal(ffn.ffn_fwd(d, x, w1, w2), y)      # without [g | u]
    h2, gu2 = torch.empty_like(h), torch.empty_like(gu)
    ffn.ffn_gate(d, x, w1, h2, gu2)
    assert torch.equal(h2, h) and torch.equal(gu2, gu)


def check_data_gradient(device, rows, C, F, O, dtype, where="cpu"):
    act = "silu" if F % 16 else "gelu"
    t = {k: v.to(where) for k, v in inputs(rows, C, F, O, dtype).items()}
    d = ffn.make_desc(rows, C, F, O, act, dtype)
    dx, dgu, h = ffn.ffn_dgrad(d, *(t[k].to(device) for k in ("dy", "w1", "w2", "gu")))
    g, u = t["gu"][:, :F].double(), t["gu"][:, F:].double()
    a, da = act64(g, act)
    rh = a * u
    close(h, rh, 1.01 * (HALF[dtype] * rh.abs() + 36 * U * (g * u).abs()) + 1e-30, "h")
    dh, e = sums(t["dy"].double(), t["w2"].double())
    rg, ru = dh * u * da, dh * a
    # act' is good to 64 U (1 + |g|)
    eg = HALF[dtype] * rg.abs() + e * (u * da).abs() + 64 * U * (1 + g.abs()) * (dh * u).abs() + 4 * U * rg.abs()
    eu = HALF[dtype] * ru.abs() + e * a.abs() + 36 * U * (dh * g).abs()
    rgu, egu = torch.cat([rg, ru], 1), 1.01 * torch.cat([eg, eu], 1) + 1e-30
    close(dgu, rgu, egu, "dgu")
    rx, ex = sums(rgu, t["w1"].double())
    ex = ex + egu @ t["w1"].double().abs()
    close(dx, rx, 1.01 * (HALF[dtype] * rx.abs() + ex), "dx")


def check_weight_gradient(device, rows, C, F, O, dtype, where="cpu"):
    t = {k: v.to(where) for k, v in inputs(rows, C, F, O, dtype).items()}
    d = ffn.make_desc(rows, C, F, O, "silu", dtype)
    args = [t[k].to(device) for k in ("x", "dgu", "h", "dy")]
    dw1, dw2 = ffn.ffn_wgrad(d, *args, dw1=torch.full((2 * F, C), float("nan"), device=device), dw2=torch.full((O, F), float("nan"), device=device))
    close(dw1, *sums(t["dgu"].double().t(), t["x"].double()), "dw1")
    close(dw2, *sums(t["dy"].double().t(), t["h"].double()), "dw2")
    again = ffn.ffn_wgrad(d, *args)
    assert torch.equal(again[0], dw1) and torch.equal(again[1], dw2)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,C,F,O", SHAPES)
def test_forward(device, rows, C, F, O, dtype):
    check_forward(device, rows, C, F, O, dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,C,F,O", SHAPES)
def test_data_gradient(device, rows, C, F, O, dtype):
    check_data_gradient(device, rows, C, F, O, dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,C,F,O", SHAPES + [(0, 16, 24, 8), (9000, 64, 72, 40)])
def test_weight_gradient(device, rows, C, F, O, dtype):
    check_weight_gradient(device, rows, C, F, O, dtype)


L, M, S, FEW = "tiles_256x256", "tiles_128x128", "tiles_64x128", "few_rows"
# a shape for each kernel of a product, with its contraction whole and in parts (0: any number of parts above one)
EACH = [("fwd", "bf16", (17612, 272, 352, 8), L, None), ("fwd", "bf16", (583, 8, 3656, 8), M, None), ("fwd", "bf16", (1132, 8, 160, 8), S, None),
        ("fwd", "bf16", (7536, 24, 280, 1776), None, (L, 1)), ("fwd", "bf16", (18684, 16, 2680, 144), None, (L, 0)), ("fwd", "bf16", (17204, 16, 8, 184), None, (M, 1)),
        ("fwd", "bf16", (9036, 16, 3088, 24), None, (M, 0)), ("fwd", "bf16", (40, 40, 8, 3160), None, (S, 1)), ("fwd", "bf16", (41, 104, 1544, 2728), None, (S, 0)),
        ("fwd", "bf16", (300, 200, 520, 200), FEW, (FEW, 1)),
        ("fwd", "f32", (799, 8, 2592, 8), M, None), ("fwd", "f32", (3159, 8, 24, 8), S, None), ("fwd", "f32", (300, 200, 520, 200), FEW, (FEW, 1)),
        ("fwd", "f32", (11640, 8, 8, 264), None, (M, 1)), ("fwd", "f32", (8470, 8, 936, 40), None, (M, 0)), ("fwd", "f32", (19, 120, 8, 3200), None, (S, 1)),
        ("fwd", "f32", (1, 8, 3552, 8), None, (S, 0)),
        ("dgrad", "bf16", (3725, 8, 3448, 736), L, None), ("dgrad", "bf16", (19587, 8, 136, 8), M, None), ("dgrad", "bf16", (3224, 3944, 136, 16), None, (L, 1)),
        ("dgrad", "bf16", (16702, 152, 1200, 32), None, (L, 0)), ("dgrad", "bf16", (16506, 160, 8, 16), None, (M, 1)), ("dgrad", "bf16", (10804, 8, 1200, 8), None, (M, 0)),
        ("dgrad", "bf16", (2, 8, 552, 8), S, (S, 0)), ("dgrad", "f32", (12818, 8, 296, 8), M, None), ("dgrad", "f32", (19045, 152, 8, 56), None, (M, 1)),
        ("dgrad", "f32", (4790, 8, 800, 8), None, (M, 0)),
        ("wgrad", "bf16", (272, 1512, 2528, 1808), None, ("pair " + L, 1)), ("wgrad", "bf16", (4645, 136, 3752, 144), None, ("pair " + L, 0)),
        ("wgrad", "bf16", (1, 440, 3968, 8), None, ("pair " + M, 1)), ("wgrad", "bf16", (14361, 8, 8, 1136), None, ("pair " + M, 0)),
        ("wgrad", "bf16", (1120, 8, 8, 8), None, ("pair " + S, 0)), ("wgrad", "bf16", (15379, 176, 3816, 8), L, (S, 0)), ("wgrad", "bf16", (331, 152, 2344, 3008), S, (M, 1)),
        ("wgrad", "f32", (2552, 24, 8, 3232), None, ("pair " + M, 0)), ("wgrad", "f32", (435, 8, 8, 16), None, ("pair " + S, 0)),
        ("wgrad", "f32", (4455, 8, 4096, 8), M, (S, 0)), ("wgrad", "f32", (386, 16, 1992, 1856), S, (S, 1))]


@pytest.mark.parametrize("way,dt,shape,first,second", EACH)
def test_each_kernel_with_whole_and_split_contractions(device, way, dt, shape, first, second):
    dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[dt]
    how = ffn.kernel_detail(ffn.make_desc(*shape, "silu", dtype), ("fwd", "dgrad", "wgrad").index(way)).split(", ")
    assert first is None or how[0].split(" parts")[0] == first, how
    if second is not None:
        name, parts = how[-1].split(" parts ")
        assert name == second[0] and (int(parts) > 1 if second[1] == 0 else int(parts) == second[1]), how
    {"fwd": check_forward, "dgrad": check_data_gradient, "wgrad": check_weight_gradient}[way](device, *shape, dtype, where=device)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
def test_what_is_not_finite_stays_in_its_row(device, dtype):
    """An infinity and a NaN in rows of x, beside the ends of tiles and of the contraction."""
    rows, C, F, O = 140, 72, 136, 40
    t = {k: v.to(device) for k, v in inputs(rows, C, F, O, dtype).items()}
    d = ffn.make_desc(rows, C, F, O, "silu", dtype)
    y = ffn.ffn_fwd(d, t["x"], t["w1"], t["w2"])
    bad = t["x"].clone()
    bad[127, C - 1], bad[128, 0] = float("inf"), float("nan")
    yb = ffn.ffn_fwd(d, bad, t["w1"], t["w2"])
    ok = [i for i in range(rows) if i not in (127, 128)]
    assert torch.equal(yb[ok], y[ok]) and torch.isnan(yb[128]).all()
    dx, dgu, h = ffn.ffn_dgrad(d, t["dy"], t["w1"], t["w2"], t["gu"])
    bad = t["dy"].clone()
    bad[3, 1], bad[139, O - 1] = float("nan"), float("inf")
    dxb, dgub, hb = ffn.ffn_dgrad(d, bad, t["w1"], t["w2"], t["gu"])
    ok = [i for i in range(rows) if i not in (3, 139)]
    assert torch.equal(dxb[ok], dx[ok]) and torch.equal(dgub[ok], dgu[ok]) and torch.equal(hb, h) and torch.isnan(dxb[3]).all()


@pytest.mark.parametrize("rows", [3, 70])
def test_rows_behind_the_last_stay_as_they_are(device, rows):
    C, F, O = 40, 72, 24
    t = {k: v.to(device) for k, v in inputs(rows, C, F, O, torch.bfloat16).items()}
    d = ffn.make_desc(rows, C, F, O, "silu", torch.bfloat16)
    bufs = [torch.full((rows + 130, n), 9.0, dtype=torch.bfloat16, device=device) for n in (O, 2 * F, C, 2 * F, F, F)]
    y, gu, dx, dgu, h, h2 = (b[:rows] for b in bufs)
    ffn.ffn_fwd(d, t["x"], t["w1"], t["w2"], y, gu=gu)
    ffn.ffn_gate(d, t["x"], t["w1"], h2)
    ffn.ffn_dgrad(d, t["dy"], t["w1"], t["w2"], t["gu"], dx, dgu, h)
    for b in bufs:
        assert (b[rows:] == 9).all() and not (b[:rows] == 9).all()


def test_leading_dimensions_and_workspace(device):
    """NDHWC tensors; a workspace one byte short is refused and nothing is written."""
    d = ffn.make_desc(2 * 3 * 4 * 5, 16, 24, 8, "gelu", torch.bfloat16)
    x = torch.randn(2, 3, 4, 5, 16, device=device).bfloat16()
    w1, w2 = torch.randn(48, 16, device=device).bfloat16(), torch.randn(8, 24, device=device).bfloat16()
    y = ffn.ffn_fwd(d, x, w1, w2)
    assert y.shape == (2, 3, 4, 5, 8) and torch.equal(y.view(-1, 8), ffn.ffn_fwd(d, x.view(-1, 16), w1, w2))
    need = ffn.workspace_bytes(d, ffn.PASS_FWD)
    out = torch.full((120, 8), 5.0, device=device).bfloat16()
    with pytest.raises(_lib.Mi3dError) as e:
        ffn.ffn_fwd(d, x, w1, w2, out, ws=torch.empty(need - 1, dtype=torch.uint8, device=device))
    assert e.value.status == -3 and (out == 5).all()
    ffn.ffn_fwd(d, x, w1, w2, out, ws=torch.empty(need, dtype=torch.uint8, device=device))
    assert torch.equal(out, y.view(-1, 8))
