"""What the calls of the channel-mixing block refuse (no GPU: nothing is launched)."""
import ctypes

import pytest
import torch

from paper_1812_07816_amd import _lib, ffn, glue

A, INVALID, UNSUPPORTED, WORKSPACE = 1 << 20, -1, -2, -3      # an aligned address that is never looked at


def test_layernorm_refusals():
    l = _lib.lib()
    for f, b in ((l.mi3d_layernorm_fwd, l.mi3d_layernorm_bwd), (l.mi3d_layernorm_fwd_f32, l.mi3d_layernorm_bwd_f32)):
        assert f(A, A, A, 4, 0, 1e-5, A, A, None) == INVALID and f(A, A, A, 4, -8, 1e-5, A, A, None) == INVALID
        assert f(None, A, A, 4, 8, 1e-5, A, A, None) == INVALID and f(A, A, A, 4, 8, 1e-5, None, A, None) == INVALID
        assert f(A + 2, A, A, 4, 8, 1e-5, A, A, None) == INVALID and f(A, A, A, 4, 8, 1e-5, A, A + 4, None) == INVALID
        assert f(A, A, A, 4, 8, -1.0, A, A, None) == INVALID and f(A, A, A, 4, 8, float("nan"), A, A, None) == INVALID
        for C in (16385, 16392, 1 << 30):
            assert f(A, A, A, 4, C, 1e-5, A, A, None) == UNSUPPORTED, C
            assert l.mi3d_layernorm_workspace_bytes(4, C) == 0
        assert f(A, A, A, 1 << 40, 8, 1e-5, A, A, None) == UNSUPPORTED
        assert f(None, A, A, 0, 8, 1e-5, None, None, None) == 0
        need = l.mi3d_layernorm_workspace_bytes(4, 8)
        assert need > 0 and b(A, A, A, A, None, 4, 8, A, A, A, A, need - 1, None) == WORKSPACE
        assert b(A, A, None, A, None, 4, 8, A, A, A, A, need, None) == INVALID and b(A, A, A, A, A + 8, 4, 8, A, A, A, A, need, None) == INVALID
        assert b(A, A, A, A, None, 4, 8, A, None, A, A, need, None) == INVALID


def test_dropout_refusals():
    l = _lib.lib()
    for f, b, c in ((l.mi3d_dropout_fwd, l.mi3d_dropout_bwd, l.mi3d_dropout_channels), (l.mi3d_dropout_fwd_f32, l.mi3d_dropout_bwd_f32, l.mi3d_dropout_channels_f32)):
        for p in (-0.1, 1.5, float("nan")):
            assert f(A, None, A, 8, p, 0, 0, None, None) == INVALID and b(A, A, 8, p, 0, 0, None, None) == INVALID and c(A, A, 1, 1, 8, p, 0, 0, None, None) == INVALID
        assert f(None, None, A, 8, 0.5, 0, 0, None, None) == INVALID and f(A, A + 8, A, 8, 0.5, 0, 0, None, None) == INVALID
        assert f(A, None, A, 8, 0.5, 0, 0, A + 4, None) == INVALID and f(None, None, None, 0, 0.5, 0, 0, None, None) == 0
        assert b(A, None, 8, 0.5, 0, 0, None, None) == INVALID and b(A, A, 1 << 50, 0.5, 0, 0, None, None) == UNSUPPORTED
        assert c(A, A, 1, 1, 0, 0.5, 0, 0, None, None) == INVALID and c(A, A, -1, 1, 8, 0.5, 0, 0, None, None) == INVALID
        assert c(A, A, 1, 1, 65537, 0.5, 0, 0, None, None) == UNSUPPORTED and c(A, A, 65536, 1, 8, 0.5, 0, 0, None, None) == UNSUPPORTED
        assert c(A, A, 1, 1 << 30, 8, 0.5, 0, 0, None, None) == UNSUPPORTED and c(None, None, 0, 5, 8, 0.5, 0, 0, None, None) == 0


def test_ffn_refusals():
    l = _lib.lib()
    d = ffn.make_desc(10, 16, 24, 8, "silu", torch.bfloat16)
    r, need = ctypes.byref(d), [ffn.workspace_bytes(d, q) for q in range(3)]
    assert need[0] >= 10 * 24 * 2
    assert l.mi3d_ffn_fwd(r, A, A, A, A, None, A, need[0] - 1, None) == WORKSPACE and l.mi3d_ffn_fwd(r, A, A, A, A, None, None, 0, None) == WORKSPACE
    for i in range(4):
        args = [A] * 4
        args[i] = None
        assert l.mi3d_ffn_fwd(r, *args, None, A, need[0], None) == INVALID
        args[i] = A + 8
        assert l.mi3d_ffn_fwd(r, *args, None, A, need[0], None) == INVALID
        assert l.mi3d_ffn_wgrad(r, *args, A, A, A, need[2], None) == INVALID
    assert l.mi3d_ffn_gate(r, A, None, A, None, None) == INVALID and l.mi3d_ffn_gate(r, A, A, A, A + 2, None) == INVALID
    assert l.mi3d_ffn_dgrad(r, A, A, A, A, None, A, A, A, 1 << 30, None) == INVALID and l.mi3d_ffn_wgrad(r, A, A, A, A, A, None, A, 1 << 30, None) == INVALID
    for bad, st in ((dict(Cin=12), UNSUPPORTED), (dict(F=4), UNSUPPORTED), (dict(Cout=65544), UNSUPPORTED), (dict(rows=2 ** 31), UNSUPPORTED), (dict(act=7), UNSUPPORTED),
                    (dict(dtype=5), UNSUPPORTED), (dict(rows=-1), INVALID), (dict(F=0), INVALID), (dict(Cin=-8), INVALID)):
        e = type(d).from_buffer_copy(d)
        for k, v in bad.items():
            setattr(e, k, v)
        e = ctypes.byref(e)
        assert l.mi3d_ffn_fwd(e, A, A, A, A, None, A, 1 << 30, None) == st and l.mi3d_ffn_gate(e, A, A, A, None, None) == st, bad
        assert l.mi3d_ffn_dgrad(e, A, A, A, A, A, A, A, A, 1 << 30, None) == st and l.mi3d_ffn_wgrad(e, A, A, A, A, A, A, A, 1 << 30, None) == st, bad
        assert l.mi3d_ffn_workspace_bytes(e, 0) == 0
    assert l.mi3d_ffn_fwd(None, A, A, A, A, None, A, 1 << 30, None) == INVALID
    none = ctypes.byref(ffn.make_desc(0, 16, 24, 8, "gelu", torch.float32))
    assert l.mi3d_ffn_fwd(none, None, A, A, None, None, None, 0, None) == 0 and l.mi3d_ffn_dgrad(none, None, A, A, None, None, None, None, None, 0, None) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ffn_refuses_more_workgroups_than_a_launch_holds(dtype):
    """2^31 - 1 rows of eight channels are 2^24 tiles of 256 threads: 2^32, one more than a launch counts."""
    l, r = _lib.lib(), ctypes.byref(ffn.make_desc(2 ** 31 - 1, 8, 8, 8, "silu", dtype))
    assert l.mi3d_ffn_gate(r, A, A, A, None, None) == UNSUPPORTED and l.mi3d_ffn_fwd(r, A, A, A, A, None, A, 1 << 40, None) == UNSUPPORTED
    assert l.mi3d_ffn_dgrad(r, A, A, A, A, A, A, A, A, 1 << 40, None) == UNSUPPORTED


def test_kernel_detail_says_what_runs_and_refuses_what_a_call_refuses():
    l, buf = _lib.lib(), ctypes.create_string_buffer(64)
    d = ffn.make_desc(1, 1024, 4096, 1024, "silu", torch.bfloat16)
    assert ffn.kernel_detail(d, ffn.PASS_FWD) == "few_rows, few_rows parts 1"
    d = ffn.make_desc(16384, 1024, 4096, 1024, "gelu", torch.bfloat16)
    assert ffn.kernel_detail(d, ffn.PASS_DGRAD) == "tiles_256x256, tiles_256x256 parts 1" and ffn.workspace_bytes(d, ffn.PASS_DGRAD) == 0
    assert l.mi3d_ffn_kernel_detail(ctypes.byref(d), 3, buf, 64) == INVALID and l.mi3d_ffn_kernel_detail(ctypes.byref(d), 0, None, 64) == INVALID
    d.Cin = 12
    assert l.mi3d_ffn_kernel_detail(ctypes.byref(d), 0, buf, 64) == UNSUPPORTED


def test_plans_do_not_depend_on_what_was_asked_before():
    """A thread keeps its last plans: the same answers in any order and in other threads."""
    import random
    import threading
    r = random.Random(5)
    asks = [(ffn.make_desc(r.randint(1, 9000), 8 * r.randint(1, 200), 8 * r.randint(1, 400), 8 * r.randint(1, 200), "silu", r.choice([torch.bfloat16, torch.float32])), q)
            for _ in range(120) for q in range(3)]
    said = [(ffn.kernel_detail(*a), ffn.workspace_bytes(*a)) for a in asks]
    wrong = []

    def again(order):
        wrong.extend(i for i in order if (ffn.kernel_detail(*asks[i]), ffn.workspace_bytes(*asks[i])) != said[i])

    order = list(range(len(asks)))
    r.shuffle(order)
    threads = [threading.Thread(target=again, args=(o,)) for o in (order, order[::-1])]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_the_binding_refuses_before_the_library_is_called():
    """Tensors on the host, of another type or shape, or not dense."""
    x, g = torch.zeros(4, 8), torch.zeros(8)
    with pytest.raises(ValueError):
        glue.layernorm_fwd(x, g, g)
    with pytest.raises(ValueError):
        glue.layernorm_fwd(x.double(), g, g)
    with pytest.raises(ValueError):
        glue.layernorm_bwd(x, x, torch.zeros(4, 2), g, ws=torch.zeros(64, dtype=torch.uint8))
    with pytest.raises(ValueError):
        glue.dropout_fwd(x.t(), 0.5, 1)
    with pytest.raises(ValueError):
        glue.dropout_bwd(x.half(), 0.5, 1)
    with pytest.raises(ValueError):
        glue.dropout_channels(g, 0.5, 1)
    with pytest.raises(ValueError):
        ffn.ffn_fwd(ffn.make_desc(4, 8, 8, 8, "silu", torch.float32), x, torch.zeros(16, 8), torch.zeros(8, 8), ws=torch.zeros(1024, dtype=torch.uint8))
    with pytest.raises(KeyError):
        ffn.make_desc(4, 8, 8, 8, "tanh", torch.float32)


@pytest.mark.gpu
def test_the_binding_refuses_tensors_that_do_not_fit(device):
    x, g = torch.zeros(4, 8, device=device), torch.zeros(8, device=device)
    for bad in (dict(gamma=g[:4]), dict(gamma=g.bfloat16()), dict(y=torch.zeros(8, 4, device=device).t()), dict(y=x.cpu()), dict(stats=torch.zeros(4, device=device))):
        with pytest.raises(ValueError):
            glue.layernorm_fwd(**(dict(x=x, gamma=g, beta=g) | bad))
    with pytest.raises(ValueError):
        glue.dropout_fwd(x, 0.5, 1, residual=x[:2])
    with pytest.raises(ValueError):
        glue.dropout_fwd(x, 0.5, 1, dev_offset=torch.zeros(1, device=device))
    with pytest.raises(_lib.Mi3dError):
        glue.dropout_fwd(torch.zeros(40, device=device)[1:33], 0.5, 1)      # not 16-byte aligned
    with pytest.raises(_lib.Mi3dError):
        glue.dropout_fwd(x, 1.5, 1)
    d = ffn.make_desc(4, 8, 16, 8, "silu", torch.float32)
    w1, w2 = torch.zeros(32, 8, device=device), torch.zeros(8, 16, device=device)
    for a, b, c in ((x[:3], w1, w2), (x, w2, w1), (x, w1.t().contiguous().t(), w2), (x.bfloat16(), w1, w2)):
        with pytest.raises(ValueError):
            ffn.ffn_fwd(d, a, b, c)
