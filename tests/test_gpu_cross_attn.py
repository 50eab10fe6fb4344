"""Attention of a map's tokens to states of another length, forward and backward, against 64 bits."""
import pytest
import torch

import cross_util as ref
from paper_2603_06738_b200 import binding as rib

pytestmark = pytest.mark.gpu


def inputs(B, H, W, heads, kv, d, L, contexts=None, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    contexts = B if contexts is None else contexts
    q, dout = (normal(B, H, W, heads, d) for _ in range(2))
    k, v = (normal(contexts, L, kv, d) for _ in range(2))
    return [(t * s).bfloat16() for t, s in ((q, scale), (k, 1.0), (v, 1.0), (dout, 1.0))]


def run_both(q, k, v, dout, lengths=None, backward=True):
    out, lse = rib.rib_cross_attn_fwd(q, k, v, lengths=lengths)
    grads = rib.rib_cross_attn_bwd(q, k, v, out, lse, dout, lengths=lengths) if backward else ()
    torch.cuda.synchronize()
    assert rib.rib_query_status() == 0
    return out, lse, grads


def check_all(q, k, v, dout, lengths=None):
    out, lse, grads = run_both(q, k, v, dout, lengths)
    (want, want_lse), (bound, bound_lse) = ref.forward(q, k, v, lengths)
    ref.check("out", out, want, bound)
    ref.check("lse", lse, want_lse, bound_lse)
    wants, bounds = ref.backward(q, k, v, out, lse, dout, lengths)
    for name, got, want, bound in zip(("dq", "dk", "dv"), grads, wants, bounds):
        ref.check(name, got, want, bound)
    return out, lse, grads


@pytest.mark.parametrize("d", [8, 16, 24, 32, 40, 48, 56, 64])
def test_head_widths(d):
    check_all(*inputs(2, 9, 15, 2, 2, d, 100, seed=d))


@pytest.mark.parametrize("d", [1, 2, 5, 20, 30, 33, 63])
def test_widths_on_padded_copies(d):
    check_all(*inputs(2, 7, 11, 3, 3, d, 70, seed=d))


@pytest.mark.parametrize("L", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 1000])
def test_lengths_of_the_states(L):
    check_all(*inputs(1, 10, 13, 2, 2, 32, L, seed=L))


@pytest.mark.parametrize("H,W", [(1, 1), (1, 2), (3, 21), (8, 8), (5, 13), (8, 16), (3, 43), (16, 16), (37, 53)])
def test_sizes_of_the_map(H, W):
    check_all(*inputs(2, H, W, 2, 2, 32, 90, seed=H))


@pytest.mark.parametrize("heads,kv", [(1, 1), (2, 1), (3, 1), (6, 2), (5, 1), (8, 2), (12, 4), (64, 1), (33, 1)])
@pytest.mark.parametrize("d", [32, 64])
def test_grouped_heads(heads, kv, d):
    check_all(*inputs(2, 6, 9, heads, kv, d, 75, seed=heads))


@pytest.mark.parametrize("heads,kv,d", [(2, 2, 32), (4, 2, 64), (3, 3, 20)])
def test_one_context_for_the_batch(heads, kv, d):
    check_all(*inputs(5, 7, 9, heads, kv, d, 130, contexts=1, seed=d))


@pytest.mark.parametrize("d", [32, 64, 30])
@pytest.mark.parametrize("L", [64, 150, 700])
def test_ragged_lengths(d, L):
    lengths = torch.tensor([0, 1, 16, 17, L // 2, L - 1, L], dtype=torch.int32, device="cuda")
    q, k, v, dout = inputs(7, 6, 11, 2, 2, d, L, seed=L)
    out, lse, (dq, dk, dv) = check_all(q, k, v, dout, lengths)
    assert (out[0] == 0).all() and (lse[0] == -torch.inf).all() and (dq[0] == 0).all()
    for i, n in enumerate(lengths.tolist()):
        assert (dk[i, n:] == 0).all() and (dv[i, n:] == 0).all()


@pytest.mark.parametrize("d", [32, 64, 20])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_padding_has_no_influence(d, what):
    lengths = torch.tensor([0, 5, 64, 70, 129], dtype=torch.int32, device="cuda")
    q, k, v, dout = inputs(5, 5, 9, 4, 2, d, 200, seed=3)
    clean = run_both(q, k, v, dout, lengths)
    for i, n in enumerate(lengths.tolist()):
        k[i, n:] = what
        v[i, n:] = what
    dirty = run_both(q, k, v, dout, lengths)
    for a, b in zip((*clean[:2], *clean[2]), (*dirty[:2], *dirty[2])):
        assert torch.equal(a, b)


def test_lengths_outside_the_states_count_as_the_nearer_end():
    q, k, v, dout = inputs(3, 4, 5, 2, 2, 32, 80, seed=5)
    odd = run_both(q, k, v, dout, torch.tensor([-7, 81, 2 ** 31 - 1], dtype=torch.int32, device="cuda"))
    even = run_both(q, k, v, dout, torch.tensor([0, 80, 80], dtype=torch.int32, device="cuda"))
    for a, b in zip((*odd[:2], *odd[2]), (*even[:2], *even[2])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("B,heads,kv,d,L", [(1, 1, 1, 32, 5000), (2, 6, 6, 32, 3000), (3, 8, 2, 64, 2100), (64, 2, 2, 32, 300), (1, 4, 1, 16, 8192), (2, 64, 1, 64, 900), (2, 3, 3, 30, 1000)])
def test_single_tokens_over_long_contexts(B, heads, kv, d, L):
    lengths = torch.randint(1, L + 1, (B,), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(L))
    check_all(*inputs(B, 1, 1, heads, kv, d, L, seed=B))
    check_all(*inputs(B, 1, 1, heads, kv, d, L, seed=B), lengths)


@pytest.mark.parametrize("scale", [8.0, 60.0])
@pytest.mark.parametrize("d", [32, 64])
def test_large_logits(scale, d):
    check_all(*inputs(2, 9, 17, 2, 2, d, 260, seed=11, scale=scale))


def test_scores_that_grow_along_the_states():
    """The running maximum moves in every block."""
    q, k, v, dout = inputs(1, 8, 16, 2, 2, 32, 640, seed=12)
    k *= torch.linspace(0.1, 20, 640, device="cuda").bfloat16()[None, :, None, None]
    check_all(q, k, v, dout)
    check_all(q, k.flip(1).contiguous(), v, dout)


@pytest.mark.parametrize("d", [32, 64])
def test_rows_that_are_no_numbers_stay_alone(d):
    """A NaN or an infinity in a query makes its own row NaN, in a batch item's states its own item.  (Rows computed beside them are redone with another reference: the same up to the
    roundings that the bound counts.)"""
    q, k, v, dout = inputs(3, 6, 7, 2, 2, d, 100, seed=13)
    (want, _), (bound, _) = ref.forward(q, k, v)
    q[0, 2, 3, 1, 0] = float("nan")
    q[1, 0, 0, 0, 1] = float("inf")
    k[2, 70, 1, 0] = float("nan")
    got = run_both(q, k, v, dout, backward=False)[0]
    bad = torch.zeros(3, 6, 7, 2, dtype=torch.bool, device="cuda")
    bad[0, 2, 3, 1] = bad[1, 0, 0, 0] = True
    bad[2, :, :, 1] = True
    assert got[bad].isnan().all()
    ref.check("out", got[~bad], want[~bad], bound[~bad])


def test_keys_of_minus_infinity_weigh_nothing():
    """Infinite keys whose logits are minus infinity drop out of the softmax; a row that has no others is NaN."""
    q, k, v, _ = inputs(1, 4, 4, 1, 1, 32, 200, seed=14)
    q[..., 0] = 1.0
    k[..., 0] = 0.0
    k[0, 0:70, 0, 0] = -float("inf")
    out = rib.rib_cross_attn_fwd(q, k, v)[0]
    want = rib.rib_cross_attn_fwd(q, k[:, 70:].contiguous(), v[:, 70:].contiguous())[0]
    (exact, _), (bound, _) = ref.forward(q, k[:, 70:], v[:, 70:])
    ref.check("out", out, exact, bound)
    ref.check("out", want, exact, bound)
    k[..., 0] = -float("inf")
    assert rib.rib_cross_attn_fwd(q, k, v)[0].isnan().all()


def test_results_are_the_same_from_run_to_run():
    q, k, v, dout = inputs(2, 20, 30, 4, 2, 32, 500, seed=15)
    first, second = run_both(q, k, v, dout), run_both(q, k, v, dout)
    for a, b in zip((*first[:2], *first[2]), (*second[:2], *second[2])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("L", [1, 16, 64, 77, 130])
@pytest.mark.parametrize("heads,kv,d", [(6, 6, 32), (6, 3, 64), (3, 1, 20)])
def test_many_tiles_for_each_block_of_the_grid(L, heads, kv, d):
    """Items follow one another without a pause, some of them without keys."""
    q, k, v, dout = inputs(6, 64, 50, heads, kv, d, L, seed=L)
    check_all(q, k, v, dout)
    check_all(q, k, v, dout, torch.tensor([L, 0, (L + 1) // 2, 1, 0, L], dtype=torch.int32, device="cuda"))
