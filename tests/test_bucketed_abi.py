"""Refusals of the calls for a bias by buckets and for 8-bit checkpoints: every one before anything is launched, so no GPU is needed."""
import ctypes

import pytest
import torch

from paper_2603_06738_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.library()


def fwd_args(**over):
    a = dict(q=256, k=512, v=768, bias=1024, dtype=0, stride=9, buckets=2048, count=9, B=1, H=32, W=32, heads=2, d=32, window=16, shift=0, masked=0, out=4096, lse=8192, stream=None)
    a.update(over)
    return list(a.values())


def bwd_args(**over):
    a = dict(q=256, k=512, v=768, bias=1024, dtype=0, stride=9, buckets=2048, count=9, out=4096, lse=8192, dout=12288, B=1, H=32, W=32, heads=2, d=32, window=16, shift=0,
             masked=0, dq=16384, dk=20480, dv=24576, dbias=28672, workspace=32768, bytes=1 << 30, stream=None)
    a.update(over)
    return list(a.values())


COMMON = [
    (dict(q=None), -1), (dict(bias=None), -1), (dict(buckets=None), -1), (dict(out=None), -1),
    (dict(count=0), -2), (dict(count=-1), -2), (dict(stride=8), -2), (dict(stride=-9), -2), (dict(shift=16), -2), (dict(shift=-1), -2), (dict(window=0), -2),
    (dict(B=0), -2), (dict(masked=1, H=40), -2), (dict(dtype=2), -3), (dict(dtype=-1), -3), (dict(d=65), -3),
    (dict(bias=1026), -4), (dict(buckets=2050), -4), (dict(k=520), -4), (dict(dtype=1, bias=1025), -4),
]


@pytest.mark.parametrize("over,code", COMMON)
def test_forward_refuses(lib, over, code):
    assert lib.rib_window_attn_fwd_bucketed(*fwd_args(**over)) == code


@pytest.mark.parametrize("over,code", COMMON + [(dict(lse=None), -1), (dict(dbias=None), -1), (dict(dv=None), -1), (dict(dbias=28674), -4), (dict(workspace=None), -5),
                                                (dict(bytes=16), -5), (dict(workspace=32768 + 16), -4)])
def test_backward_refuses(lib, over, code):
    assert lib.rib_window_attn_bwd_bucketed(*bwd_args(**over)) == code


def test_workspaces(lib):
    need = lib.rib_window_attn_bwd_bucketed_workspace
    assert need(9, 9, 1, 32, 32, 2, 32, 16) > 0 and need(0, 9, 1, 33, 31, 2, 5, 7) > 0
    assert need(8, 9, 1, 32, 32, 2, 32, 16) == 0 and need(0, 0, 1, 32, 32, 2, 32, 16) == 0 and need(0, 9, 1, 32, 32, 2, 65, 16) == 0
    images = 4 * 2 * 1 * 32 * 32 * 2 * 32
    assert lib.rib_window_attn_bwd_bucketed_checkpointed_workspace(9, 9, 1, 32, 32, 2, 32, 16) >= need(9, 9, 1, 32, 32, 2, 32, 16) + images
    assert lib.rib_window_attn_bwd_checkpointed_workspace(0, 1, 32, 32, 2, 32, 16, 16) >= lib.rib_window_attn_bwd_workspace(1, 32, 32, 2, 32, 16, 16) + images
    assert lib.rib_window_attn_bwd_checkpointed_workspace(0, 1, 32, 32, 2, 65, 16, 16) == 0


@pytest.mark.parametrize("over,code", [(dict(x=None), -1), (dict(codes=None), -1), (dict(scales=None), -1), (dict(rows=-1), -2), (dict(d=0), -2), (dict(d=65), -3),
                                       (dict(rows=(1 << 31) + 1), -3), (dict(x=264), -4), (dict(codes=520), -4), (dict(scales=772), -4), (dict(rows=0), 0)])
def test_checkpoints_refuse(lib, over, code):
    a = dict(x=256, codes=512, scales=768, rows=4, d=32)
    a.update(over)
    assert lib.rib_checkpoint_store(a["x"], a["rows"], a["d"], a["codes"], a["scales"], None) == code
    assert lib.rib_checkpoint_restore(a["codes"], a["scales"], a["rows"], a["d"], a["x"], None) == code


@pytest.mark.parametrize("over,code", [(dict(saved=None), -1), (dict(codes=None), -1), (dict(scales=None), -1), (dict(lse=None), -1), (dict(dout=None), -1), (dict(workspace=None), -5),
                                       (dict(bytes=64), -5), (dict(bytes=4 * 131072 + 64), -5), (dict(codes=260), -4), (dict(dq=264), -4), (dict(B=0), -2), (dict(shift=16), -2),
                                       (dict(masked=1, H=40), -2), (dict(d=65), -3)])
def test_backward_from_checkpoints_refuses(lib, over, code):
    a = dict(saved=1, codes=256, scales=512, lse=8192, dout=12288, B=1, H=32, W=32, heads=2, d=32, window=16, shift=0, masked=0, dq=16384, workspace=32768, bytes=1 << 30)
    a.update(over)
    saved = (ctypes.c_void_p * 8)(*([a["codes"], a["scales"]] * 4)) if a["saved"] else None
    shape = [a[k] for k in ("B", "H", "W", "heads", "d")]
    assert lib.rib_window_attn_bwd_checkpointed(saved, 1024, 2048, 0, a["lse"], a["dout"], *shape, 16, a["window"], a["shift"], a["masked"], a["dq"], 20480, 24576, 28672, 30720,
                                                a["workspace"], a["bytes"], None) == code
    assert lib.rib_window_attn_bwd_bucketed_checkpointed(saved, 1024, 0, 9, 2048, 9, a["lse"], a["dout"], *shape, a["window"], a["shift"], a["masked"], a["dq"], 20480, 24576, 28672,
                                                         a["workspace"], a["bytes"], None) == code


def test_the_binding_checks_its_tensors():
    q = torch.zeros(1, 4, 4, 2, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q must be"):
        binding.rib_window_attn_fwd_bucketed(q, q, q, torch.zeros(2, 3), torch.zeros(7, 7, dtype=torch.int32), 4)
    check = lambda bias, named, device="cpu": binding._check_bias(bias, named, 2, 4, torch.device(device))  # noqa: E731
    named = torch.zeros(7, 7, dtype=torch.int32)
    assert check(torch.zeros(2, 3), named) == (0, 3, 3) and check(torch.zeros(5, dtype=torch.bfloat16), named) == (1, 0, 5)
    for bias, m in ((torch.zeros(3, 3), named), (torch.zeros(2, 0), named), (torch.zeros(2, 3).half(), named), (torch.zeros(2, 6)[:, ::2], named), (torch.zeros(2, 3), named.long()),
                    (torch.zeros(2, 3), named[:6]), (torch.zeros(1, 2, 3), named)):
        with pytest.raises(ValueError):
            check(bias, m)
    with pytest.raises(ValueError):
        check(torch.zeros(2, 3), named, "meta")


def test_checkpoints_of_too_many_rows_are_refused(lib):
    """Sides whose product is beyond 64 bits as well."""
    saved = (ctypes.c_void_p * 8)(*range(256, 256 * 9, 256))
    for B, H, W, heads in ((1 << 16, 1 << 16, 16, 1), (1 << 30, 1 << 30, 1 << 30, 1 << 30), (1 << 30, 1 << 30, 16, 1 << 30)):
        assert lib.rib_window_attn_bwd_bucketed_checkpointed(saved, 1024, 0, 9, 2048, 9, 8192, 12288, B, H, W, heads, 32, 16, 0, 0, 16384, 20480, 24576, 28672, 32768, 1 << 62, None) in (-2, -3)
        assert lib.rib_window_attn_bwd_checkpointed(saved, 1024, 2048, 0, 8192, 12288, B, H, W, heads, 32, 16, 16, 0, 0, 16384, 20480, 24576, 28672, 30720, 32768, 1 << 62, None) in (-2, -3)
