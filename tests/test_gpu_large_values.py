"""Values and logits that are large at the same time: the output is of the size of the values, whatever the weights are before they are normalised.

The values are scaled by a power of two, so every weight, product and sum is the same but for its exponent, and the results are those of the unscaled values,
scaled, except where the fast form of the softmax overflowed and the exact form has redone an item: P is rounded to bf16 in both, 2^-9 of every weight
and of their sum each, and out once more: (2 + 2 + 2) 2^-9 max |v|, as the weights add up to 1."""
import pytest
import torch

from paper_2603_06738_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,W,M,s,masked", [(64, 64, 32, 0, False), (32, 48, 16, 8, False), (32, 48, 16, 8, True), (40, 24, 16, 0, False), (41, 23, 16, 0, False), (32, 32, 8, 0, False),
                                            (12, 12, 6, 0, False)])
@pytest.mark.parametrize("r", [16, 32])
@pytest.mark.parametrize("q_scale", [1.0, 12.0, 14.0, 16.0])
def test_rank_r_layers(H, W, M, s, masked, r, q_scale):
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(1, H, W, 2, 32, generator=g).bfloat16().cuda() for _ in range(3))
    q = (q.float() * q_scale).bfloat16()
    pq, pk = ((torch.randn(M * M, r, generator=g) * 0.5).bfloat16().cuda() for _ in range(2))
    fwd = binding.rib_window_attn_fwd_masked if masked else binding.rib_window_attn_fwd_padded
    want, want_lse = fwd(q, k, v, pq, pk, M, s)
    bound = 6 * 2.0 ** -9 * float(v.float().abs().max())
    for exponent in (-60, 60, 90, 100):
        out, lse = fwd(q, k, (v.float() * 2.0 ** exponent).bfloat16(), pq, pk, M, s)
        assert float((out.float() * 2.0 ** -exponent - want.float()).abs().max()) <= bound, exponent
        assert float((lse - want_lse).abs().max()) <= 2.0 ** -8
