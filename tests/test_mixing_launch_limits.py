"""Products of the feed-forward block beside the 2^31 threads of a launch (no GPU: nothing is launched)."""
import ctypes

import pytest
import torch

from paper_1812_07816_amd import _lib, ffn

A, OK, UNSUPPORTED = 1 << 20, 0, -2      # an aligned address that is never looked at
FWD, DGRAD, WGRAD = range(3)


def detail(shape, pass_, dtype=torch.bfloat16):
    buf = ctypes.create_string_buffer(128)
    d = ffn.make_desc(*shape, "silu", dtype)
    return _lib.lib().mi3d_ffn_kernel_detail(ctypes.byref(d), pass_, buf, 128), buf.value.decode()


def test_tiles_of_more_rows_where_a_launch_cannot_hold_the_smaller_ones():
    """2^29 rows and 136 columns: 2^23 tiles of 128 x 128 in 256 threads are 2^31, one more than a launch counts; 2^21 of 256 x 256 in 512 are 2^30."""
    st, how = detail((2 ** 29, 8, 8, 136), FWD)
    assert st == OK and how.endswith("tiles_256x256 parts 1")
    st, how = detail((2 ** 29, 136, 8, 8), DGRAD)
    assert st == OK and how.endswith("tiles_256x256 parts 1")


# (rows, Cin, F, Cout): a first product that a launch holds, a second one that none does
@pytest.mark.parametrize("dtype,wide", [(torch.bfloat16, 264), (torch.float32, 136)], ids=["bf16", "f32"])
def test_a_call_whose_second_product_is_too_large_is_refused_before_its_first_one(dtype, wide):
    l, rows = _lib.lib(), 2 ** 29
    for shape, q in (((rows, 8, 8, wide), FWD), ((rows, wide, 8, 8), DGRAD)):
        d = ffn.make_desc(*shape, "silu", dtype)
        r = ctypes.byref(d)
        assert detail(shape, q, dtype)[0] == UNSUPPORTED and l.mi3d_ffn_workspace_bytes(r, q) == 0
        if q == FWD:
            assert l.mi3d_ffn_fwd(r, A, A, A, A, None, A, 1 << 50, None) == UNSUPPORTED
        else:
            assert l.mi3d_ffn_dgrad(r, A, A, A, A, A, A, A, A, 1 << 50, None) == UNSUPPORTED


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_kernel_detail_refuses_a_first_product_that_is_too_large(dtype):
    for q in (FWD, DGRAD):
        assert detail((2 ** 31 - 1, 8, 8, 8), q, dtype)[0] == UNSUPPORTED
    assert detail((2 ** 31 - 1, 8, 8, 8), WGRAD, dtype)[0] == OK      # (one tile, whatever the rows)
