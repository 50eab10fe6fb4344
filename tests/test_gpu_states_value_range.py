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
