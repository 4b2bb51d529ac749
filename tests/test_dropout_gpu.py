"""Dropout against the published generator in numpy: which values stay, what they are multiplied with, all lengths around the
pieces of eight, whole channels across sample borders, replays of a captured graph."""
import numpy as np
import pytest
import torch

from paper_1812_07816_amd import glue

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


def philox(i, offset, seed, rounds=10):
    """Words of Philox 4x32 for counters (i, offset), in Python's integers."""
    M = 0xFFFFFFFF
    c, k = [i & M, i >> 32, offset & M, offset >> 32], [seed & M, seed >> 32]
    for _ in range(rounds):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & M, (a >> 32) ^ c[3] ^ k[1], a & M]
        k = [(k[0] + 0x9E3779B9) & M, (k[1] + 0xBB67AE85) & M]
    return c


def numbers(n, seed, offset, first=0):
    out = []
    for i in range(first // 8, (first + n + 7) // 8):
        out += [h for w in philox(i, offset, seed) for h in (w & 0xFFFF, w >> 16)]
    return np.array(out[first % 8:first % 8 + n])


def reference(a, kept, limit, res=None):
    """One fp32 product and one sum, rounded to the type: what the header states, so the bits are known."""
    scale = np.float32(65536.0 / limit) if limit else np.float32(0)
    v = torch.where(kept, a.float() * float(scale), torch.zeros((), dtype=torch.float32))
    return v if res is None else v + res.float()


def test_the_generator_is_the_published_one():
    """Known answers of Philox 4x32-10 (counter and key of zeros, and of ones)."""
    assert philox(0, 0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    one = 0xFFFFFFFFFFFFFFFF
    assert philox(one, one, one) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("n,p,seed,offset", [(1, 0.5, 1, 0), (7, 0.5, 2, 1), (8, 0.1, 3, 2), (9, 0.9, 4, 3), (2047, 0.25, 5, 2 ** 40), (2049, 0.3, 2 ** 63 + 5, 2 ** 64 - 1),
                                             (20000, 0.0, 7, 0), (4096, 1.0, 8, 0), (10001, 1e-6, 9, 0), (1000, 0.99999, 10, 4)])
def test_values(device, n, p, seed, offset, dtype):
    gen = torch.Generator().manual_seed(n)
    a, res = torch.randn(n, generator=gen).to(dtype), torch.randn(n, generator=gen).to(dtype)
    limit = round((1 - float(np.float32(p))) * 65536)
    kept = torch.from_numpy(numbers(n, seed, offset) < limit)
    for r in (None, res):
        got = glue.dropout_fwd(a.to(device), p, seed, offset, residual=None if r is None else r.to(device)).cpu()
        ref = reference(a, kept, limit, r)
        # (the sum may be formed without rounding the product: half a step of either)
        tol = (2.0 ** -24 * ref.abs() + 2.0 ** -24 * reference(a, kept, limit).abs()).double() * 1.01 + (2.0 ** -8 * ref.abs().double() if dtype == torch.bfloat16 else 0)
        assert ((got.double() - ref.double()).abs() <= tol).all()
        if r is None:
            assert torch.equal(got != 0, kept & (a != 0))
            assert torch.equal(glue.dropout_bwd(a.to(device), p, seed, offset).cpu(), got)


def test_dropped_values_are_zero_whatever_they_were(device):
    n = 4099
    a = torch.full((n,), float("nan"))
    a[::2] = float("inf")
    kept = torch.from_numpy(numbers(n, 11, 5) < 32768)
    got = glue.dropout_fwd(a.to(device), 0.5, 11, 5).cpu()
    assert (got[~kept] == 0).all() and not torch.isfinite(got[kept]).any()
    assert (glue.dropout_fwd(a.to(device), 1.0, 11, 5, residual=torch.ones(n, device=device)) == 1).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("N,voxels,C", [(1, 1, 1), (2, 5, 1), (3, 7, 3), (2, 11, 8), (3, 13, 21), (2, 300, 24), (1, 5000, 64), (4, 9, 7), (2, 3, 1000), (2, 1, 5000), (5, 1, 9)])
def test_whole_channels(device, N, voxels, C, dtype):
    gen = torch.Generator().manual_seed(C)
    a = torch.randn((N, voxels, C), generator=gen).to(dtype)
    limit = round((1 - float(np.float32(0.3))) * 65536)
    kept = torch.from_numpy(numbers(N * C, 77, 3) < limit).view(N, 1, C)
    for out in (None, "in place"):
        x = a.to(device)
        got = glue.dropout_channels(x, 0.3, 77, 3, out=x if out else None).cpu()
        assert torch.equal(got, reference(a, kept.expand(a.shape), limit).to(dtype))


def test_far_numbers_of_a_long_tensor(device):
    """Values behind 2^31, drawn by their own number; and what lies behind the tensor stays."""
    n = 2 ** 31 + 4100
    a = torch.ones(n + 8, dtype=torch.bfloat16, device=device)
    glue.dropout_fwd(a[:n], 0.5, 123, 9, out=a[:n])
    for first in (0, 2 ** 31 - 1000, n - 2000):
        kept = torch.from_numpy(numbers(2000, 123, 9, first) < 32768)
        assert torch.equal(a[first:first + 2000].cpu() != 0, kept)
    assert (a[n:] == 1).all()


def test_share_of_kept_values_and_streams(device):
    a = torch.ones(1 << 22, device=device)
    masks = [glue.dropout_fwd(a, 0.3, s, o) != 0 for s, o in ((1, 0), (1, 1), (2, 0))]
    for m in masks:      # 5 standard deviations
        assert abs(m.double().mean().item() - 45875 / 65536) < 5 * (0.21 / (1 << 22)) ** 0.5
    for i in range(3):   # independent: both kept with the product of the probabilities
        both = (masks[i] & masks[i - 1]).double().mean().item()
        assert abs(both - (45875 / 65536) ** 2) < 5 * (0.25 / (1 << 22)) ** 0.5


def test_replays_of_a_graph_differ_by_the_number_in_memory(device):
    a = torch.randn(5000, device=device)
    out, ch, extra = torch.empty_like(a), torch.empty(2, 50, 50, device=device), torch.zeros(1, dtype=torch.int64, device=device)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        glue.dropout_fwd(a, 0.4, 5, 100, out=out, dev_offset=extra)
        glue.dropout_channels(a.view(2, 50, 50), 0.4, 5, 200, out=ch, dev_offset=extra)
        extra.add_(1)
    for i in range(4):
        a.normal_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, glue.dropout_fwd(a, 0.4, 5, 100 + i)), i
        assert torch.equal(ch, glue.dropout_channels(a.view(2, 50, 50), 0.4, 5, 200 + i)), i
