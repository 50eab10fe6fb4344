"""The oracle of window attention with a bias by buckets and of the 8-bit checkpoints, held against independent statements of the same
(CPU only): torch's attention with an additive bias, autograd, differences, closed forms, planted mistakes."""
import numpy as np
import pytest
import torch

from oracle import rib_bias_oracle as orc
from oracle import rib_oracle

RNG = np.random.default_rng(5)


def draw(B, H, W, heads, d, M, buckets=None, shared=False):
    side = 2 * M - 1
    named = RNG.integers(0, 7, (side, side)) if buckets is None else buckets
    count = 7 if buckets is None else int(buckets.max()) + 1
    q, k, v, g = (RNG.standard_normal((B, H, W, heads, d)) for _ in range(4))
    return q, k, v, RNG.standard_normal(count) if shared else RNG.standard_normal((heads, count)), named, g


@pytest.mark.parametrize("H,W,M,s", [(8, 12, 4, 0), (8, 8, 4, 3), (4, 4, 4, 1), (7, 10, 4, 2), (3, 3, 5, 0), (1, 1, 1, 0)])
@pytest.mark.parametrize("shared", [False, True])
def test_equals_torch_attention_and_autograd(H, W, M, s, shared):
    q, k, v, bias, named, g = draw(2, H, W, 2, 5, M, shared=shared)
    nY, nX = -(-H // M), -(-W // M)
    t = {n: torch.tensor(a, requires_grad=True) for n, a in (("q", q), ("k", k), ("v", v), ("bias", bias))}

    def windows(a):          # the map extended, rolled and cut, by slices
        ext = torch.zeros(2, nY * M, nX * M, *a.shape[3:], dtype=torch.float64)
        ext[:, :H, :W] = a
        r = torch.roll(ext, (-s, -s), (1, 2)).reshape(2, nY, M, nX, M, *a.shape[3:]).permute(0, 1, 3, 5, 2, 4, 6)
        return r.reshape(2, nY * nX, a.shape[3], M * M, a.shape[4])

    def back(a):
        r = a.reshape(2, nY, nX, 2, M, M, -1).permute(0, 1, 4, 2, 5, 3, 6).reshape(2, nY * M, nX * M, 2, -1)
        return torch.roll(r, (s, s), (1, 2))[:, :H, :W]

    real = windows(torch.ones(2, H, W, 2, 1, dtype=torch.float64))[..., 0] > 0
    i = np.arange(M * M)
    u = torch.tensor(named[(i[None] // M - i[:, None] // M) + M - 1, (i[None] % M - i[:, None] % M) + M - 1])
    add = (t["bias"][u][None] if shared else t["bias"][:, u])[None, None] + torch.where(real, 0.0, -torch.inf)[..., None, :]
    out = back(torch.nn.functional.scaled_dot_product_attention(*(windows(t[n]) for n in ("q", "k", "v")), attn_mask=add.expand(2, nY * nX, 2, M * M, M * M)))
    got, lse = orc.fwd(q, k, v, bias, named, M, s)
    assert np.abs(got - out.detach().numpy()).max() < 1e-12 and np.isfinite(lse).all()
    out.backward(torch.tensor(g))
    for name, mine in zip(("q", "k", "v", "bias"), orc.bwd(q, k, v, bias, named, g, M, s)):
        assert np.abs(mine - t[name].grad.numpy()).max() < 1e-11, name


def test_equals_the_rank_r_oracle_where_the_tables_say_the_same():
    """A bias that depends on the offset only and the rank-r oracle with those logits: Pq, Pk chosen as one-hot rows and bias rows."""
    M, heads, d = 3, 1, 4
    n, side = M * M, 2 * M - 1
    named = np.arange(side * side).reshape(side, side)
    q, k, v, bias, _, g = draw(1, 6, 3, heads, d, M, buckets=named)
    i = np.arange(n)
    full = bias[0][named[(i[None] // M - i[:, None] // M) + M - 1, (i[None] % M - i[:, None] % M) + M - 1]]
    pq, pk = np.eye(n) * np.sqrt(n), full.T.copy()
    a, la = orc.fwd(q, k, v, bias, named, M, 1)
    b, lb = rib_oracle.fwd(q, k, v, pq, pk, M, 1)
    assert np.abs(a - b).max() < 1e-12 and np.abs(la - lb).max() < 1e-12


@pytest.mark.parametrize("masked", [False, True])
def test_gradients_against_differences(masked):
    M, s = 4, 2
    q, k, v, bias, named, g = draw(1, 8, 4, 2, 3, M)
    named = named.copy()
    named[0, :] = -1
    arrays = dict(q=q, k=k, v=v, bias=bias)
    grads = dict(zip(("q", "k", "v", "bias"), orc.bwd(q, k, v, bias, named, g, M, s, masked)))
    value = lambda: (orc.fwd(**arrays, buckets=named, window=M, shift=s, masked=masked)[0] * g).sum()  # noqa: E731
    for name, a in arrays.items():
        for at in RNG.choice(a.size, 6, replace=False):
            keep = a.flat[at]
            a.flat[at] = keep + 1e-5
            up = value()
            a.flat[at] = keep - 1e-5
            down = value()
            a.flat[at] = keep
            assert abs((up - down) / 2e-5 - grads[name].flat[at]) < 1e-7, name


def test_masked_parts_do_not_meet():
    q, k, v, bias, named, g = draw(1, 8, 8, 1, 3, 4)
    base, _ = orc.fwd(q, k, v, bias, named, 4, 2, masked=True)
    k2, v2 = k.copy(), v.copy()
    k2[:, 0], v2[:, 0] = 9.0, 9.0                   # row 0 came round the edge: of its windows only the rows 0 and 1 see it
    other, _ = orc.fwd(q, k2, v2, bias, named, 4, 2, masked=True)
    changed = np.abs(other - base).max((0, 2, 3, 4)) > 0
    assert changed.tolist() == [True, True] + [False] * 6
    plain, _ = orc.fwd(q, k2, v2, bias, named, 4, 2)
    assert (np.abs(plain - base).max((0, 2, 3, 4)) > 0)[6:].all()


def test_masked_offsets_and_rows_without_keys():
    M = 3
    named = np.full((5, 5), -1)
    named[2, 3] = 0                                 # only the neighbour to the right is attended to
    q, k, v, bias, _, g = draw(1, 3, 3, 1, 4, M, buckets=named)
    out, lse = orc.fwd(q, k, v, bias, named, M)
    assert np.array_equal(out[0, :, :2], v[0, :, 1:]) and (out[0, :, 2] == 0).all() and np.isneginf(lse[0, 0, :, 2]).all()
    dq, dk, dv, dbias = orc.bwd(q, k, v, bias, named, g, M)
    assert np.abs(dq).max() < 1e-12 and np.abs(dk).max() < 1e-12 and np.abs(dv[0, :, 1:] - g[0, :, :2]).max() < 1e-12
    assert (dv[0, :, 0] == 0).all() and np.abs(dbias).max() < 1e-12
    for low in (-np.inf, -3.4028234663852886e38, -1e30):
        both = np.zeros((5, 5), dtype=int)
        both[2, 3] = 1
        a, la = orc.fwd(q, k, v, np.array([[low, bias[0, 0]]]), both, M)
        assert np.array_equal(a, out) and np.array_equal(la, lse)


def test_a_shared_table_gets_the_sum_over_the_heads_and_every_row_of_ds_sums_to_zero():
    q, k, v, bias, named, g = draw(1, 4, 8, 3, 4, 4, shared=True)
    one = orc.bwd(q, k, v, bias, named, g, 4)[3]
    each = orc.bwd(q, k, v, np.tile(bias, (3, 1)), named, g, 4)[3]
    assert np.abs(one - each.sum(0)).max() < 1e-12
    assert np.abs(each.sum(1)).max() < 1e-10        # sum over all keys of dS is 0 for every query


@pytest.mark.parametrize("mistake", ["transposed map", "query minus key", "bias scaled by 1/sqrt(d)"])
def test_planted_mistakes_show(mistake):
    q, k, v, bias, named, g = draw(1, 8, 8, 2, 4, 4)
    out, _ = orc.fwd(q, k, v, bias, named, 4)
    if mistake == "transposed map":
        other = orc.fwd(q, k, v, bias, named.T, 4)[0]
    elif mistake == "query minus key":
        other = orc.fwd(q, k, v, bias, named[::-1, ::-1], 4)[0]
    else:
        other = orc.fwd(q, k, v, bias / 2, named, 4)[0]
    assert np.abs(out - other).max() > 1e-2


def test_checkpoints():
    x = RNG.standard_normal((50, 24)).astype(np.float32)
    x[3], x[4, 5], x[6, 0] = 0, np.inf, np.nan
    x[7] = 0
    x[7, 2] = -1e-40                                # a subnormal row
    x[8], x[8, 0] = np.arange(24) - 12.0, 127.0     # scale 1: whole numbers are kept
    codes, scale = orc.store(x)
    back = orc.restore(codes, scale)
    assert (back[3] == 0).all() and scale[3] == 0 and np.isnan(back[4]).all() and np.isnan(back[6]).all()
    assert codes.min() >= -127 and np.array_equal(np.abs(codes).max(-1)[9:], np.full(41, 127))
    assert np.abs(back[8] - x[8]).max() < 1e-5
    rest = [i for i in range(50) if i not in (4, 6, 7)]
    assert (np.abs(back - x)[rest] <= 0.5001 * scale[rest, None]).all()          # half a step
    assert abs(back[7, 2] + 1e-40) < 2e-42
