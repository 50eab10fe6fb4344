"""Attention of a map's tokens to few states, whose scores are taken at once: what can go wrong in tiles that follow one another through few slots, against 64 bits."""
import pytest
import torch

import cross_util as ref
from paper_2603_06738_b200 import binding as rib
from test_gpu_cross_and_rope_calls import Guarded
from test_gpu_cross_attn import check_all, inputs, run_both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L", [1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 80, 95, 96, 97, 111, 112, 113, 127, 128, 129])
@pytest.mark.parametrize("heads,kv,d", [(2, 2, 32), (4, 2, 64), (3, 1, 20)])
def test_lengths(L, heads, kv, d):
    check_all(*inputs(2, 9, 17, heads, kv, d, L, seed=L))


@pytest.mark.parametrize("B,H,W,heads,kv,d", [(300, 1, 3, 2, 2, 32), (200, 1, 1, 16, 4, 64), (700, 1, 5, 1, 1, 24), (90, 3, 43, 3, 3, 32), (40, 13, 13, 12, 2, 40), (1, 1, 7, 1, 1, 8)])
def test_many_groups_of_few_tiles(B, H, W, heads, kv, d):
    """A slot's next tile lies several groups on; some of them have no keys, at both ends of a run among them."""
    q, k, v, dout = inputs(B, H, W, heads, kv, d, 50, seed=B)
    check_all(q, k, v, dout)
    lengths = torch.randint(0, 51, (B,), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(B))
    lengths[::3] = 0
    out, lse, _ = check_all(q, k, v, dout, lengths)
    assert (out[lengths == 0] == 0).all() and (lse[lengths == 0] == -torch.inf).all()


def test_no_keys_at_all():
    q, k, v, dout = inputs(5, 20, 30, 4, 2, 32, 100, seed=1)
    q.fill_(float("nan"))
    out, lse, (dq, dk, dv) = run_both(q, k, v, dout, torch.zeros(5, dtype=torch.int32, device="cuda"))
    assert (out == 0).all() and (lse == -torch.inf).all() and (dq == 0).all() and (dk == 0).all() and (dv == 0).all()


@pytest.mark.parametrize("d", [32, 64, 20])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_padding_has_no_influence(d, what):
    lengths = torch.tensor([0, 5, 64, 70, 99, 16], dtype=torch.int32, device="cuda")
    q, k, v, dout = inputs(6, 15, 19, 4, 2, d, 100, seed=3)
    clean = run_both(q, k, v, dout, lengths)
    for i, n in enumerate(lengths.tolist()):
        k[i, n:] = what
        v[i, n:] = what
    dirty = run_both(q, k, v, dout, lengths)
    for a, b in zip((*clean[:2], *clean[2]), (*dirty[:2], *dirty[2])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("scale", [8.0, 60.0])
@pytest.mark.parametrize("d", [32, 64])
def test_large_logits(scale, d):
    check_all(*inputs(2, 9, 17, 2, 2, d, 110, seed=11, scale=scale))


@pytest.mark.parametrize("heads,kv,d", [(2, 2, 32), (2, 2, 64), (6, 2, 24), (2, 1, 20)])
def test_rows_that_are_no_numbers_stay_alone(heads, kv, d):
    """A row's maximum is its own: nothing beside a NaN or an infinity changes."""
    q, k, v, _ = inputs(3, 16, 17, heads, kv, d, 100, seed=13)
    want, want_lse = rib.rib_cross_attn_fwd(q, k, v)
    q[0, 2, 3, 1, 0] = float("nan")
    q[1, 0, 0, 0, 1] = float("inf")
    k[2, 70, kv - 1, 0] = float("nan")
    got, lse = rib.rib_cross_attn_fwd(q, k, v)
    bad = torch.zeros(3, 16, 17, heads, dtype=torch.bool, device="cuda")
    bad[0, 2, 3, 1] = bad[1, 0, 0, 0] = True
    bad[2, :, :, heads - heads // kv:] = True
    assert got[bad].isnan().all()
    assert torch.equal(got[~bad], want[~bad])
    bad = bad.permute(0, 3, 1, 2)
    assert torch.equal(lse[~bad], want_lse[~bad])


def test_keys_of_minus_infinity_weigh_nothing():
    q, k, v, _ = inputs(1, 4, 4, 1, 1, 32, 120, seed=14)
    q[..., 0] = 1.0
    k[..., 0] = 0.0
    k[0, 0:70, 0, 0] = -float("inf")
    (exact, exact_lse), (bound, bound_lse) = ref.forward(q, k[:, 70:], v[:, 70:])
    out, lse = rib.rib_cross_attn_fwd(q, k, v)
    ref.check("out", out, exact, bound)
    ref.check("lse", lse, exact_lse, bound_lse)
    k[..., 0] = -float("inf")
    assert rib.rib_cross_attn_fwd(q, k, v)[0].isnan().all()


@pytest.mark.parametrize("heads,kv,d", [(2, 2, 32), (4, 1, 64), (3, 1, 24), (2, 2, 20)])
def test_rows_behind_the_last_token_are_left_alone(heads, kv, d):
    """Rows of a tile that are no tokens are not written."""
    q, k, v, _ = inputs(2, 5, 9, heads, kv, d, 40, seed=d)
    sizes = (2, 5, 9, heads, kv, d, 40, 2)
    need = rib.rib_cross_attn_fwd_workspace(*sizes)
    out, lse, ws = Guarded(q.shape, torch.bfloat16), Guarded((2, heads, 5, 9), torch.float32), Guarded((max(need, 1),), torch.uint8)
    pointers = [t.data_ptr() for t in (q, k, v)]
    assert rib.library().rib_cross_attn_fwd(*pointers, None, *sizes, out.t.data_ptr(), lse.t.data_ptr(), ws.t.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert out.intact() and lse.intact() and ws.intact()
    (want, want_lse), (bound, bound_lse) = ref.forward(q, k, v)
    ref.check("out", out.t, want, bound)
    ref.check("lse", lse.t, want_lse, bound_lse)


@pytest.mark.parametrize("d", [32, 64])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), 3e38])
def test_every_key_of_longer_sequences_counts(d, what):
    """A NaN or an infinity in any one key makes the rows that meet it NaN, whichever way that key's exponential is taken; a key whose logit is minus infinity weighs nothing."""
    L = 160
    q, k, v, _ = inputs(L, 2, 3, 1, 1, d, L, seed=d)
    q[..., 0] = q[..., 0].abs() + 0.1
    clean = rib.rib_cross_attn_fwd(q, k, v)[0]
    for j in range(L):
        k[j, j, 0, 0] = what
    out = rib.rib_cross_attn_fwd(q, k, v)[0]
    if what == 3e38:      # a finite logit, far above all others (or, with two channels' product beyond the type, infinite): all weight, or NaN
        for j in range(L):
            rows = out[j].flatten(0, 2)
            assert (rows.isnan().any(-1) | (rows == v[j, j, 0]).all(-1)).all()
    else:
        assert out.isnan().all()
    for j in range(L):
        k[j, j, 0, 0] = -float("inf")
    out, lse = rib.rib_cross_attn_fwd(q, k, v)
    keep = ~torch.eye(L, dtype=torch.bool, device="cuda")
    others = lambda x: torch.stack([x[j][keep[j]] for j in range(L)])  # noqa: E731
    (want, want_lse), (bound, bound_lse) = ref.forward(q, others(k), others(v))
    ref.check("out", out, want, bound)
    ref.check("lse", lse, want_lse, bound_lse)
    assert clean.isfinite().all()


@pytest.mark.parametrize("contexts", [1, 2, 5, 31, 32, 33, 63, 64, 65, 70])
def test_contexts_of_one_and_two_blocks_of_keys(contexts):
    """Whatever the order of the lengths: each context's gradients are its own, those without keys among them."""
    g = torch.Generator(device="cuda").manual_seed(contexts)
    q, k, v, dout = inputs(contexts, 5, 9, 3, 3, 32, 250, seed=contexts)
    lengths = torch.randint(0, 251, (contexts,), dtype=torch.int32, device="cuda", generator=g)
    lengths[torch.rand(contexts, device="cuda", generator=g) < 0.2] = 0
    for cut in (lengths, lengths.sort().values, lengths.sort(descending=True).values, torch.full_like(lengths, 128), torch.full_like(lengths, 129), torch.zeros_like(lengths)):
        check_all(q, k, v, dout, cut.contiguous())
