"""Attention to states whose values are large enough that a sum of weights times values overflows before it is normalised, though the result, a weighted mean, does not."""
import math

import pytest
import torch

import cross_util as ref
from paper_2603_06738_b200 import binding as rib

pytestmark = pytest.mark.gpu


def even_logits(B, H, W, heads, kv, d, L, least, most, seed):
    """Queries and keys whose logits are all 0 (keys have no channel 0, queries no other), and values of magnitudes from `least` to `most` of either sign."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.zeros(B, H, W, heads, d, device="cuda").bfloat16()
    q[..., 0] = 1.0
    k = torch.randn(B, L, kv, d, device="cuda", generator=g).bfloat16()
    k[..., 0] = 0.0
    sizes = torch.rand(B, L, kv, d, device="cuda", generator=g) * (most - least) + least
    return q, k, (sizes * torch.where(torch.rand(B, L, kv, d, device="cuda", generator=g) < 0.5, -1.0, 1.0)).bfloat16()


def check(q, k, v, lengths=None):
    out, lse = rib.rib_cross_attn_fwd(q, k, v, lengths=lengths)
    (want, want_lse), (bound, bound_lse) = ref.forward(q, k, v, lengths)
    assert torch.isfinite(want).all() and torch.isfinite(out.float()).all()
    ref.check("out", out, want, bound)
    ref.check("lse", lse, want_lse, bound_lse)


@pytest.mark.parametrize("above", [3.0, 6.0, 10.0, 13.0, 30.0])
@pytest.mark.parametrize("d", [20, 32, 64])
@pytest.mark.parametrize("B,H,W,L", [(2, 16, 16, 200), (1, 3, 5, 1000), (6, 64, 50, 300)])
def test_one_state_above_those_before_it(B, H, W, L, d, above):
    """Weights relative to the first states' logits are large, and so are the values: from 6 on their product passes 3.4e38."""
    q, k, v = even_logits(B, H, W, 2, 2, d, L, 1e36, 1.5e36, seed=L + d)
    k[:, 150, :, 0] = above * math.sqrt(d)
    check(q, k, v)


SHAPES = [(2, 9, 15, 2, 2, 1), (2, 9, 15, 2, 2, 16), (2, 9, 15, 2, 2, 100), (3, 16, 16, 4, 2, 128), (2, 16, 16, 2, 2, 200), (1, 3, 5, 2, 1, 5000), (6, 64, 50, 2, 2, 300), (1, 1, 1, 2, 2, 5),
          (1, 1, 1, 2, 2, 9000), (1, 1, 2, 3, 3, 700), (64, 1, 1, 6, 3, 1200), (1, 1, 1, 8, 2, 6000)]


@pytest.mark.parametrize("d", [8, 20, 32, 64])
@pytest.mark.parametrize("B,H,W,heads,kv,L", SHAPES)
def test_values_as_large_as_the_type_holds(B, H, W, heads, kv, L, d):
    """Values up to 3e38: two of them add up to infinity."""
    q, k, v = even_logits(B, H, W, heads, kv, d, L, 2e38, 3e38, seed=L + d)
    check(q, k, v)
    check(q, k, v.abs())
    lengths = torch.randint(1, L + 1, (B,), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(L))
    check(q, k, v.abs(), lengths)


@pytest.mark.parametrize("d", [32, 64])
@pytest.mark.parametrize("B,H,W,L", [(2, 16, 16, 200), (1, 3, 5, 2000), (1, 1, 1, 900), (2, 9, 15, 100)])
@pytest.mark.parametrize("above", [3.0, 5.0, 13.0, 60.0])
def test_such_values_and_states_above_others(B, H, W, L, d, above):
    q, k, v = even_logits(B, H, W, 2, 2, d, L, 2e38, 3e38, seed=L + d)
    k[:, 3 * L // 4:, :, 0] = above * math.sqrt(d)
    check(q, k, v)
    check(q, k, v.abs())


@pytest.mark.parametrize("L", [200, 5000])
def test_such_values_in_the_exact_form(L):
    before = rib.rib_set_path(rib.RIB_PATH_SM100_EXACT)
    try:
        q, k, v = even_logits(2, 8, 9, 2, 2, 32, L, 2e38, 3e38, seed=L)
        check(q, k, v.abs())
        k[:, L // 2:, :, 0] = 7.5 / math.log2(math.e) * math.sqrt(32)        # just below where the reference moves
        check(q, k, v.abs())
    finally:
        rib.rib_set_path(before)
