"""Sides of maps near 2^31: refused before anything is launched where positions of the windows laid over them would pass an int.  No GPU needed."""
import ctypes

import pytest

from paper_2603_06738_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.library()


def refusals(lib, B, H, W, heads, d, M, s):
    size, masked = (B, H, W, heads, d), 0
    saved = (ctypes.c_void_p * 8)(*range(256, 256 * 9, 256))
    big = 1 << 62
    yield lib.rib_window_attn_fwd(256, 512, 768, 1024, 2048, *size, 16, M, s, 4096, 8192, None)
    yield lib.rib_window_attn_fwd_padded(256, 512, 768, 1024, 2048, 0, *size, 16, M, s, 4096, 8192, None)
    yield lib.rib_window_attn_bwd_padded(256, 512, 768, 1024, 2048, 0, 4096, 8192, 12288, *size, 16, M, s, 16384, 20480, 24576, 28672, 30720, 32768, big, None)
    yield lib.rib_window_attn_fwd_bucketed(256, 512, 768, 1024, 0, 9, 2048, 9, *size, M, s, masked, 4096, 8192, None)
    yield lib.rib_window_attn_bwd_bucketed(256, 512, 768, 1024, 0, 9, 2048, 9, 4096, 8192, 12288, *size, M, s, masked, 16384, 20480, 24576, 28672, 32768, big, None)
    yield lib.rib_window_attn_bwd_bucketed_checkpointed(saved, 1024, 0, 9, 2048, 9, 8192, 12288, *size, M, s, masked, 16384, 20480, 24576, 28672, 32768, big, None)


@pytest.mark.parametrize("H,W,M,s", [(2**31 - 1, 1, 16, 0), (2**31 - 1, 1, 16, 8), (1, 2**31 - 1, 7, 3), (2**31 - 16, 1, 16, 0), (1, 2**31 - 16, 16, 15), (2**31 - 5, 1, 1000, 0),
                                     (2**31 - 1, 2**31 - 1, 1024, 0)])
def test_sides_that_do_not_fit(lib, H, W, M, s):
    for rc in refusals(lib, 1, H, W, 1, 8, M, s):
        assert rc in (-2, -3)
    assert lib.rib_window_attn_bwd_bucketed_workspace(9, 9, 1, H, W, 1, 8, M) == 0
    assert lib.rib_window_attn_bwd_padded_workspace(0, 1, H, W, 1, 8, 16, M) == 0


def test_the_largest_sides(lib):
    """Just below, the shape is one that a call takes: its workspace has a size."""
    for H, M in ((2**31 - 32, 16), (2**31 - 15, 7)):
        assert lib.rib_window_attn_bwd_bucketed_workspace(9, 9, 1, H, 1, 1, 8, M) > 0
