"""What the calls of attention to states and of norms with rotation refuse: codes of the C calls (nothing is launched, pointers are never read), errors of the binding."""
import pytest
import torch

from paper_2603_06738_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.library()


CROSS = ("B", "H", "W", "heads", "kv_heads", "d", "L", "contexts")


def cross_args(backward, **over):
    a = dict(q=256, k=512, v=768, lengths=None, out=1024, lse=1280, dout=1536, dq=1792, dk=2048, dv=2304, B=2, H=8, W=8, heads=4, kv_heads=2, d=32, L=77, contexts=2,
             workspace=4096, bytes=1 << 40, stream=None)
    a.update(over)
    names = ("q", "k", "v", "lengths") + (("out", "lse", "dout") + CROSS + ("dq", "dk", "dv") if backward else CROSS + ("out", "lse")) + ("workspace", "bytes", "stream")
    return [a[n] for n in names]


REFUSED = [
    (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(out=None), -1),
    (dict(B=0), -2), (dict(H=-1), -2), (dict(W=0), -2), (dict(heads=0), -2), (dict(kv_heads=0), -2), (dict(d=0), -2), (dict(L=0), -2), (dict(L=-5), -2),
    (dict(kv_heads=3), -2), (dict(contexts=3), -2), (dict(contexts=0), -2),
    (dict(d=65), -3), (dict(heads=65, kv_heads=1), -3), (dict(H=1 << 16, W=1 << 16), -3), (dict(H=1 << 15, W=1 << 14, heads=2, kv_heads=2), -3),
    (dict(L=2 ** 31 - 1), -3), (dict(L=1 << 30, contexts=2), -3),
    (dict(q=264), -4), (dict(k=520), -4), (dict(v=770), -4), (dict(out=1032), -4), (dict(lse=1284), -4), (dict(lengths=514), -4), (dict(workspace=4112), -4),
]


@pytest.mark.parametrize("over,code", REFUSED)
@pytest.mark.parametrize("backward", [False, True])
def test_cross_attention_refuses(lib, over, code, backward):
    call = lib.rib_cross_attn_bwd if backward else lib.rib_cross_attn_fwd
    assert call(*cross_args(backward, **over)) == code


@pytest.mark.parametrize("over,code", [(dict(lse=None), -1), (dict(dout=None), -1), (dict(dq=None), -1), (dict(dk=None), -1), (dict(dv=None), -1), (dict(dout=1544), -4), (dict(dv=2306), -4),
                                       (dict(workspace=None, L=777), -5), (dict(bytes=100, L=777), -5)])
def test_cross_attention_backward_refuses(lib, over, code):
    assert lib.rib_cross_attn_bwd(*cross_args(True, **over)) == code


def test_cross_attention_forward_refuses_too_little_scratch(lib):
    # few rows and many keys: runs of keys are joined; rows that are no multiple of 16 bytes: copies
    for shape in (dict(B=1, H=1, W=1, contexts=1, L=5000), dict(d=30)):
        sizes = [int(x) for x in cross_args(False, **shape)[4:12]]
        need = binding.rib_cross_attn_fwd_workspace(*sizes)
        assert need > 0
        assert lib.rib_cross_attn_fwd(*cross_args(False, **shape, bytes=need - 1)) == -5
        assert lib.rib_cross_attn_fwd(*cross_args(False, **shape, workspace=None)) == -5


def test_cross_attention_workspace_of_a_refused_shape_is_0(lib):
    for over in (dict(d=65), dict(L=0), dict(kv_heads=3), dict(H=1 << 16, W=1 << 16)):
        sizes = [int(x) for x in cross_args(False, **over)[4:12]]
        assert binding.rib_cross_attn_fwd_workspace(*sizes) == 0 and binding.rib_cross_attn_bwd_workspace(*sizes) == 0


ROPE = ("B", "H", "W", "heads", "kv_heads", "d", "rot", "interleaved", "eps")


def rope_args(backward, **over):
    a = dict(q=256, q_stride=256, k=512, k_stride=256, q_weight=768, k_weight=1024, per_head=0, table=1280, dq_out=1536, dk_out=1792, B=2, H=8, W=8, heads=4, kv_heads=2, d=32,
             rot=32, interleaved=0, eps=1e-6, q_out=2048, k_out=2304, dq=2560, dq_stride=256, dk=2816, dk_stride=256, dq_weight=3088, dk_weight=3328, workspace=4096, bytes=1 << 40,
             stream=None)
    a.update(over)
    names = ("q", "q_stride", "k", "k_stride", "q_weight", "k_weight", "per_head", "table") + (
        ("dq_out", "dk_out") + ROPE + ("dq", "dq_stride", "dk", "dk_stride", "dq_weight", "dk_weight", "workspace", "bytes") if backward else ROPE + ("q_out", "k_out")) + ("stream",)
    return [a[n] for n in names]


@pytest.mark.parametrize("over,code", [
    (dict(q=None), -1), (dict(k=None), -1), (dict(kv_heads=0), -1), (dict(table=None), -1), (dict(rot=0), -1),
    (dict(B=0), -2), (dict(heads=-1), -2), (dict(kv_heads=-1), -2), (dict(d=0), -2), (dict(rot=34), -2), (dict(rot=31), -2), (dict(rot=-2), -2), (dict(eps=-1.0), -2), (dict(eps=float("nan")), -2),
    (dict(q_stride=127), -2), (dict(k_stride=63), -2), (dict(q_stride=-256), -2),
    (dict(d=65, q_stride=512), -3), (dict(H=1 << 16, W=1 << 16), -3), (dict(heads=65536, q_stride=1 << 22), -3),
    (dict(q=257), -4), (dict(k=513), -4), (dict(q_weight=772), -4), (dict(k_weight=1028), -4), (dict(table=1284), -4),
])
@pytest.mark.parametrize("backward", [False, True])
def test_norm_and_rotation_refuse(lib, over, code, backward):
    call = lib.rib_qk_norm_rope_bwd if backward else lib.rib_qk_norm_rope_fwd
    assert call(*rope_args(backward, **over)) == code


@pytest.mark.parametrize("over,code", [(dict(q_out=None), -1), (dict(k_out=None), -1), (dict(q_out=2056), -4), (dict(k_out=2312), -4)])
def test_norm_and_rotation_forward_refuse(lib, over, code):
    assert lib.rib_qk_norm_rope_fwd(*rope_args(False, **over)) == code


@pytest.mark.parametrize("over,code", [(dict(dq_out=None), -1), (dict(dk_out=None), -1), (dict(dq=None), -1), (dict(dk=None), -1), (dict(dq_weight=None), -1), (dict(dk_weight=None), -1),
                                       (dict(dq_stride=100), -2), (dict(dk_stride=1), -2), (dict(dq_out=1544), -4), (dict(dq=2561), -4), (dict(dq_weight=3076), -4), (dict(workspace=4104), -4),
                                       (dict(workspace=None), -5), (dict(bytes=16), -5)])
def test_norm_and_rotation_backward_refuse(lib, over, code):
    assert lib.rib_qk_norm_rope_bwd(*rope_args(True, **over)) == code


@pytest.mark.parametrize("over,code", [(dict(f=None), -1), (dict(table=None), -1), (dict(H=0), -2), (dict(W=-1), -2), (dict(pairs=0), -2), (dict(pairs=33), -3), (dict(y0=1 << 41), -3),
                                       (dict(x0=-(1 << 41)), -3), (dict(f=260), -4), (dict(table=516), -4)])
def test_table_refuses(lib, over, code):
    a = dict(f=256, H=8, W=8, pairs=16, y0=0, x0=0, magnitude=1.0, table=512, stream=None)
    a.update(over)
    assert lib.rib_rope_table(*a.values()) == code


def test_frequencies_refuse():
    for args in (dict(rot=0), dict(rot=7), dict(rot=8, base=0.0), dict(rot=8, scale=-1.0), dict(rot=8, scaling="other"), dict(rot=8, scaling="by_parts"), dict(rot=8, trained=100)):
        with pytest.raises(ValueError):
            binding.rib_rope_frequencies(device="cpu", **args)


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu():
    q = torch.zeros(1, 4, 4, 2, 32, dtype=torch.bfloat16)
    k = torch.zeros(1, 7, 2, 32, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.rib_cross_attn_fwd(q, k, k)
    with pytest.raises(ValueError):
        binding.rib_qk_norm_rope_fwd(q, q, torch.ones(32), torch.ones(32))
    with pytest.raises(ValueError):
        binding.rib_rope_table(torch.zeros(2, 8), 4, 4)
