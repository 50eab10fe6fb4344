"""Maps of more than 2^31 pixels: the same rows of windows from top to bottom, so every row of windows has the results of the first, bit by bit."""
import pytest
import torch

from paper_2603_06738_b200 import binding

from test_gpu_bucketed import log_map, make

pytestmark = pytest.mark.gpu


def tall(t, H):
    """[1, rows, W, ...] repeated down to H rows."""
    out = torch.empty((1, H, *t.shape[2:]), dtype=t.dtype, device="cuda")
    out.view(H // t.shape[1], *t.shape[1:]).copy_(t.expand(H // t.shape[1], *t.shape[1:]))
    return out


def repeats(t, rows):
    """Is every row of windows of [1, H, W, ...] the first one, the last among them? (a strip at a time)"""
    first = t[0, :rows]
    return all(torch.equal(t[0, y:y + rows], first) for y in (t.shape[1] // rows // 2 * rows, t.shape[1] - 2 * rows, t.shape[1] - rows))


@pytest.mark.parametrize("M,d,rows,H,W", [(16, 8, 32, 46368, 46352), (7, 1, 7, 46347, 46347)])
def test_more_than_2_31_pixels(M, d, rows, H, W):
    """Forward; where the gradients fit as well (heads of one channel), backward."""
    assert H * W > 1 << 31 and H % rows == 0 and W % M == 0
    q, k, v, dout, bias, named = (t.cuda() for t in make(1, rows, W, 1, d, M, log_map(M), torch.float32, seed=36))
    want_out, want_lse = binding.rib_window_attn_fwd_bucketed(q, q, q, bias, named, M)
    big = tall(q, H)
    out, lse = binding.rib_window_attn_fwd_bucketed(big, big, big, bias, named, M)
    assert torch.equal(out[:, :rows], want_out) and torch.equal(lse[:, :, :rows], want_lse)
    assert repeats(out, rows) and repeats(lse.view(1, H, W), rows)
    if d > 1:
        return
    want = binding.rib_window_attn_bwd_bucketed(q, q, q, bias, named, want_out, want_lse, dout, M)
    grads = binding.rib_window_attn_bwd_bucketed(big, big, big, bias, named, out, lse, tall(dout, H), M)
    for got, ref in zip(grads[:3], want[:3]):
        assert torch.equal(got[:, :rows], ref) and repeats(got, rows)
    # copies of a sum: a block has fp32 sums of up to 4 x 10^4 windows x 49 pairs, each addition off by half a step of the partial sum, independently of one another:
    # (2 x 10^6) ^ 0.5 x 2^-24 = 8e-5 of partial sums, which are up to 2^3 times as large as the sum itself
    copies = H // rows
    assert float((grads[3] / copies - want[3]).norm()) <= 1e-3 * float(want[3].norm())
