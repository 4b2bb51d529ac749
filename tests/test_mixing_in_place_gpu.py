"""What the header allows in place: normalisation of odd widths, whose pieces overlap inside a row, in up to 512 lanes of several
wavefronts, and dropout onto its input and its residual.  The bits are those of the call with a result of its own."""
import pytest
import torch

from paper_1812_07816_amd import glue

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,C", [(700, 5), (3001, 9), (900, 67), (515, 333), (300, 1000), (130, 2047), (97, 2051), (40, 4095), (9, 8193), (5, 16383)])
def test_normalisation(device, rows, C, dtype):
    gen = torch.Generator().manual_seed(C)
    x, dy, add = (torch.randn(rows, C, generator=gen).to(dtype).to(device) for _ in range(3))
    gamma, beta = (torch.rand(C, generator=gen).to(device) for _ in range(2))
    y, stats = glue.layernorm_fwd(x, gamma, beta)
    z = x.clone()
    _, again = glue.layernorm_fwd(z, gamma, beta, y=z)
    assert torch.equal(z, y) and torch.equal(again, stats)
    ref = glue.layernorm_bwd(dy, x, stats, gamma, add=add)
    for where in ("dy", "x", "add"):
        t = dict(dy=dy.clone(), x=x.clone(), add=add.clone())
        got = glue.layernorm_bwd(t["dy"], t["x"], stats, gamma, dx=t[where], add=t["add"])
        assert all(torch.equal(a, b) for a, b in zip(got, ref)), where


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 7, 4099, 600001])
def test_dropout(device, n, dtype):
    gen = torch.Generator().manual_seed(n)
    a, res = (torch.randn(n, generator=gen).to(dtype).to(device) for _ in range(2))
    ref = glue.dropout_fwd(a, 0.3, 5, 6, residual=res)
    for where in ("a", "res"):
        t = dict(a=a.clone(), res=res.clone())
        assert torch.equal(glue.dropout_fwd(t["a"], 0.3, 5, 6, residual=t["res"], out=t[where]), ref), where
    own = a.clone()      # one tensor in all three places
    assert torch.equal(glue.dropout_fwd(own, 0.3, 5, 6, residual=own, out=own), glue.dropout_fwd(a, 0.3, 5, 6, residual=a))
    d = a.clone()
    assert torch.equal(glue.dropout_bwd(d, 0.3, 5, 6, da=d), glue.dropout_bwd(a, 0.3, 5, 6))
