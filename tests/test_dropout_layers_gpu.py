"""Dropout of several layers in one captured graph whose replays share a step number in device memory."""
import pytest
import torch

from paper_1812_07816_amd import glue

pytestmark = pytest.mark.gpu
LAYERS, STEPS, SEED, P = 3, 5, 17, 0.5


def masks(device, offset_of):
    """[step][layer]: what a graph of all layers kept of ones, forward and backward pass alike."""
    one, step = torch.ones(4096, device=device), torch.zeros(1, dtype=torch.int64, device=device)
    outs = [torch.empty_like(one) for _ in range(LAYERS)]
    backs = [torch.empty_like(one) for _ in range(LAYERS)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for k in range(LAYERS):
            glue.dropout_fwd(one, P, SEED, offset_of(k), out=outs[k], dev_offset=step)
            glue.dropout_bwd(one, P, SEED, offset_of(k), da=backs[k], dev_offset=step)
    kept = []
    for t in range(STEPS):
        step.fill_(t)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, backs))
        kept.append([o != 0 for o in outs])
    return kept


def test_spaced_layers_never_draw_the_same_numbers(device):
    """offset = layer << 40: no two of the masks of all layers and steps are alike, and any two agree in half of their values
    (4096 values: 2048, standard deviation 32; six of them)."""
    kept = [m for step in masks(device, lambda k: k << 40) for m in step]
    for i, a in enumerate(kept):
        for b in kept[:i]:
            assert abs(int((a == b).sum()) - 2048) < 192
    eager = torch.ones(4096, device=device)
    assert torch.equal(kept[-1], glue.dropout_fwd(eager, P, SEED, (LAYERS - 1 << 40) + STEPS - 1) != 0)


def test_neighbouring_offsets_repeat_a_step_later(device):
    """The sum of offset and number is the stream: what the header warns of."""
    kept = masks(device, lambda k: k)
    for t in range(STEPS - 1):
        for k in range(LAYERS - 1):
            assert torch.equal(kept[t + 1][k], kept[t][k + 1])
