"""Channels that the rotation leaves as they are, beside infinities and NaN: nothing of one of them reaches another, forward or backward."""
import pytest
import torch

from paper_2603_06738_b200 import binding as rib

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def rows(seed, *shape):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).bfloat16()


def same(x, y):
    return bool(((x == y) | (x.isnan() & y.isnan())).all())


def table_of(rot, H, W):
    return rib.rib_rope_table(rib.rib_rope_frequencies(rot), H, W, y0=3) if rot else None


@pytest.mark.parametrize("d,rot", [(32, 0), (64, 32), (48, 16), (24, 8), (24, 0), (40, 16), (20, 12), (18, 6), (30, 16), (33, 32), (63, 10), (5, 4), (3, 2), (1, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("what", [INF, -INF, NAN])
def test_without_a_norm_they_are_copied(d, rot, interleaved, what):
    B, H, W, heads, kv = 2, 5, 7, 3, 2
    q, k, gq, gk = rows(1, B, H, W, heads, d), rows(2, B, H, W, kv, d), rows(3, B, H, W, heads, d), rows(4, B, H, W, kv, d)
    for i, t in enumerate((q, k, gq, gk)):
        for c in range(rot, d):              # one channel of a token each, so that every place of a unit has its turn
            t.view(-1, t.shape[3], d)[(c + i) % (B * H * W), c % t.shape[3], c] = what
    table = table_of(rot, H, W)
    outs = rib.rib_qk_norm_rope_fwd(q, k, None, None, table, interleaved=interleaved)
    grads = rib.rib_qk_norm_rope_bwd(q, k, None, None, table, gq, gk, interleaved=interleaved)
    for got, src in zip((*outs, *grads[:2]), (q, k, gq, gk)):
        assert same(got[..., rot:], src[..., rot:])
        assert torch.isfinite(got[..., :rot].float()).all()


@pytest.mark.parametrize("d,rot", [(32, 0), (64, 32), (48, 16), (24, 8), (20, 12), (18, 6), (33, 32), (30, 16), (63, 10)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_with_a_norm_an_infinity_stays_in_its_channel(d, rot, interleaved):
    """x infinite in one channel: its root is infinite, so that channel is NaN and every other one 0.  Its gradient infinite: dw of that channel, and of no other, is infinite or NaN."""
    B, H, W, heads = 1, 4, 6, 2
    channels = [rot, d - 1, (rot + d) // 2]
    w = 1 + 0.1 * rows(5, heads, d).float()
    table = table_of(rot, H, W)
    for c in channels:
        x, g = rows(6, B, H, W, heads, d), rows(7, B, H, W, heads, d)
        x[0, 2, 3, 1, c] = INF
        out = rib.rib_qk_norm_rope_fwd(x, None, w, None, table, interleaved=interleaved)[0]
        row = out[0, 2, 3, 1].float()
        assert row[c].isnan() and int(row.isnan().sum()) == 1 and (row.nan_to_num(nan=0.0) == 0).all()
        x, g[0, 2, 3, 1, c] = rows(6, B, H, W, heads, d), INF
        dw = rib.rib_qk_norm_rope_bwd(x, None, w, None, table, g, None, interleaved=interleaved)[2]
        bad = ~torch.isfinite(dw)
        assert bad[1, c] and int(bad.sum()) == 1


@pytest.mark.parametrize("d,rot", [(32, 0), (64, 32), (48, 16), (24, 8), (20, 12), (18, 6), (33, 32), (30, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("what", [INF, NAN, 3e38])
def test_a_weight_that_is_no_finite_number_stays_in_its_channel(d, rot, interleaved, what):
    for c in (rot, d - 1, (rot + d) // 2):
        w = 1 + 0.1 * rows(5, 2, d).float()
        w[1, c] = what
        x = rows(6, 1, 4, 6, 2, d).abs() + 1.0
        x[..., c] = 8.0                                 # times its root more than 1.2: passes 3.4e38 too
        out = rib.rib_qk_norm_rope_fwd(x, None, w, None, table_of(rot, 4, 6), interleaved=interleaved)[0]
        bad = ~torch.isfinite(out.float())
        assert bad[:, :, :, 1, c].all() and int(bad.sum()) == 4 * 6
