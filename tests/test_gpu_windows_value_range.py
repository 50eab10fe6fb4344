"""Windows in which one token's logit is a little above the others', with values that overflow when they are multiplied by its weight relative to those: the output, a weighted mean, does not.

The values are scaled by a power of two, so every weight, product and sum is the same but for its exponent, and the results are those of the unscaled values, scaled, but for items that the
exact form of the softmax has redone: P is rounded to bf16 in both, at most 2^-8 of every weight and of their sum each, and out once more: (2 + 2 + 2) 2^-8 max |v|, as the weights add
up to 1."""
import math

import pytest
import torch

from paper_2603_06738_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,W,M,s", [(64, 64, 32, 0), (128, 64, 32, 16), (32, 48, 16, 8), (40, 24, 16, 0), (41, 23, 16, 0), (32, 32, 8, 0), (12, 12, 6, 0)])
@pytest.mark.parametrize("d,r", [(32, 16), (32, 32), (16, 16)])
@pytest.mark.parametrize("above", [6.0, 9.0, 13.0])
def test_one_token_above_the_others(H, W, M, s, d, r, above):
    g = torch.Generator(device="cuda").manual_seed(5)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    q, k = torch.zeros(1, H, W, 2, d, device="cuda"), normal(1, H, W, 2, d)
    q[..., 0] = 1.0
    k[..., 0] = 0.0
    v = normal(1, H, W, 2, d)
    ys, xs = (torch.arange(n, device="cuda") for n in (H, W))
    late = ((ys + M - s) % M == M - 1)[:, None] & ((xs + M - s) % M == M - 1)[None, :]       # the last token of a window
    k[:, late, :, 0] = above * math.sqrt(d)
    v[:, late] = 3.0 * torch.where(v[:, late] < 0, -1.0, 1.0)
    q, k, v = (t.bfloat16() for t in (q, k, v))
    pq, pk = (torch.zeros(M * M, r, device="cuda").bfloat16() for _ in range(2))
    want, want_lse = binding.rib_window_attn_fwd_padded(q, k, v, pq, pk, M, s)
    scaled = (v.float() * 2.0 ** 119).bfloat16()          # 2e36: 3 x 2^119 x exp(6) = 8e38
    out, lse = binding.rib_window_attn_fwd_padded(q, k, scaled, pq, pk, M, s)
    assert torch.isfinite(out.float()).all()
    assert float((out.float() * 2.0 ** -119 - want.float()).abs().max()) <= 6 * 2.0 ** -8 * float(v.float().abs().max())
    assert float((lse - want_lse).abs().max()) <= 2.0 ** -8
