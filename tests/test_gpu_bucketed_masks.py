"""Keys that are not attended to, under a bias by buckets, whatever their finite logits and the other biases are.

Tolerances are those of tests/test_gpu_bucketed.py.  The large channels of a marked query and a marked key meet no others: every logit that counts is one of
ordinary inputs, so what holds for those holds here.  Where a channel is large the results are compared without it as well."""
import numpy as np
import pytest
import torch

from oracle import rib_bias_oracle as orc
from paper_2603_06738_b200 import binding

from parity_util import to_f64
from test_gpu_bucketed import close, log_map, make, sum_noise

pytestmark = pytest.mark.gpu

# B, H, W, heads, d, M, s: tcgen05 kernels (whole patches, an odd number of them, a map that cuts them, one large window), warp-level MMAs, any-shape
SHAPES = [(1, 32, 48, 2, 32, 16, 8), (1, 24, 40, 2, 32, 8, 0), (1, 48, 24, 2, 16, 24, 8), (1, 41, 53, 2, 32, 16, 0), (1, 64, 64, 1, 32, 64, 32),
          (1, 23, 31, 2, 20, 7, 3), (1, 20, 40, 2, 10, 20, 4)]


def places(size, M, s):
    """Shifted place of every row (or column) of the map."""
    return (np.arange(size) - s) % (-(-size // M) * M)


def marked(case, named, q_row, k_row):
    """Inputs of the case whose query at one token and key at another of its window hold q_row and k_row, channels that are 0 in all other rows; the offset
    of the two is not attended to.  Returns them, the head and the two tokens."""
    B, H, W, heads, d, M, s = case
    q, k, v, dout, bias, named = make(B, H, W, heads, d, M, named, torch.float32, seed=31)
    py, px = places(H, M, s), places(W, M, s)
    h, Y, X = heads - 1, int(np.where(py == 4)[0][0]), int(np.where(px == 5)[0][0])
    KY, KX = int(np.where(py == 2)[0][0]), int(np.where(px == 6)[0][0])
    width = len(q_row)
    q[..., :width] = 0
    k[..., :width] = 0
    q[0, Y, X, h] = 0
    k[0, KY, KX, h] = 0
    q[0, Y, X, h, :width] = torch.tensor(q_row)
    k[0, KY, KX, h, :width] = torch.tensor(k_row)
    assert q[0, Y, X, h, :width].tolist() == list(q_row) and k[0, KY, KX, h, :width].tolist() == list(k_row)
    named[2 - 4 + M - 1, 6 - 5 + M - 1] = -1
    return (q, k, v, dout, bias, named)


def run(inputs, M, s, path=binding.RIB_PATH_NONE):
    q, k, v, dout, bias, named = (t.cuda() for t in inputs)
    old = binding.rib_set_path(path)
    try:
        out, lse = binding.rib_window_attn_fwd_bucketed(q, k, v, bias, named, M, s)
        grads = binding.rib_window_attn_bwd_bucketed(q, k, v, bias, named, out, lse, dout, M, s)
    finally:
        binding.rib_set_path(old)
    torch.cuda.synchronize()
    assert binding.rib_query_status() == 0
    return out, lse, grads


def compare(inputs, M, s, out, lse, grads, width):
    q, k, v, dout, bias, named = inputs
    f = [to_f64(t) for t in (q, k, v, bias)] + [named.numpy()]
    ref_out, ref_lse = orc.fwd(*f, M, s)
    close("out", out, ref_out)
    close("lse", lse, ref_lse)
    *refs, norm = orc.bwd(*f, to_f64(dout), M, s, out=to_f64(out), lse=to_f64(lse), want_norm=True)
    for name, got, ref in zip(("dq", "dk", "dv", "dbias"), grads, refs):
        close(name, got, ref, noise=sum_noise(norm) if name == "dbias" else 0.0)
        if name in ("dq", "dk"):
            close(name + " without the large channels", got[..., width:], ref[..., width:])


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "x".join(map(str, c)))
@pytest.mark.parametrize("size", [2560.0, 2.0 ** 30])
def test_a_key_out_of_reach_with_a_large_logit(case, size):
    """The logit of the pair is 10^6 and more above the others of the row, and finite."""
    d, M, s = case[4:]
    inputs = marked(case, log_map(M), (size,), (size,))
    compare(inputs, M, s, *run(inputs, M, s), 1)


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "x".join(map(str, c)))
@pytest.mark.parametrize("k_row", [(4000.0, 43.0), (4000.0, 45.0), (3984.0, 2.0), (3.0e32, 0.0), (1.0e35, 0.0)])
def test_a_key_out_of_reach_whose_logit_meets_a_stand_in(case, k_row):
    """Rows attend to their own token and two others, so that one weight too many shows.  Logits of the pair around 10^6 (in log2 units), and large ones."""
    d, M, s = case[4:]
    named = np.full((2 * M - 1, 2 * M - 1), -1)
    named[M - 1, M - 1], named[M - 1, M], named[M - 2, M - 1] = 0, 1, 2
    k_row = torch.tensor(k_row).bfloat16().tolist()
    inputs = marked(case, named, (980.0, 24.0), k_row)
    compare(inputs, M, s, *run(inputs, M, s), 2)


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "x".join(map(str, c)))
@pytest.mark.parametrize("low", [-7e13, -6e13, -1e9, -1e7, -1e4])
def test_low_biases_beside_very_low_ones(case, low):
    """Half of the offsets have a bias of -40, the others one that leaves them no weight beside those."""
    B, H, W, heads, d, M, s = case
    named = (np.add.outer(np.arange(2 * M - 1) * 5, np.arange(2 * M - 1) * 3) % 7 < 3).astype(int)
    named[M - 1, M - 1] = 0
    q, k, v, dout, bias, named = inputs = make(B, H, W, heads, d, M, named, torch.float32, seed=35)
    bias[:, 0], bias[:, 1] = -40.0, low
    compare(inputs, M, s, *run(inputs, M, s), 0)


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "x".join(map(str, c)))
@pytest.mark.parametrize("low", [-1e6, -1e9, -9e29])
def test_rows_whose_biases_are_all_very_low(case, low):
    """A finite bias counts, however low: the offsets that have a bucket share `low`, others have none.

    lse is fp32, so probabilities recomputed from it carry |lse| 2^-24 of its last place, and with sqrt(d) <= 5.7 the tcgen05 kernels' accumulators a
    few units of 2^23.  At 10^6 that is, in log2 units: the accumulator's last place 0.5 and half of it, and the rounding of sqrt(d) 0.34, times log2(e) / sqrt(d) = 0.255:
    0.28; the rounding of that factor 0.17; of bias log2(e) 0.1: a probability is off by up to a factor of 2^0.55 < 1.5.  Beyond, nothing is left of the
    digits; a probability is still at most 1, so dv is at most the sum of |dO|, and the rest is finite."""
    B, H, W, heads, d, M, s = case
    named = np.where(np.add.outer(np.arange(2 * M - 1) * 5, np.arange(2 * M - 1) * 3) % 7 < 2, -1, 0)
    named[M - 1, M - 1] = 0
    q, k, v, dout, bias, named = inputs = make(B, H, W, heads, d, M, named, torch.float32, seed=32)
    bias.fill_(low)
    for path in (binding.RIB_PATH_NONE, binding.RIB_PATH_GENERIC):
        out, lse, grads = run(inputs, M, s, path)
        assert all(torch.isfinite(t.float()).all() for t in (out, lse, *grads))
        dq, dk, dv, dbias = (to_f64(t) for t in grads)
        assert (np.abs(dv) <= 1.01 * np.abs(to_f64(dout)).sum((0, 1, 2))).all()
        if low < -1e6:
            continue
        f = [to_f64(t) for t in (q, k, v, bias)] + [named.numpy()]
        given = dict(out=to_f64(out), lse=to_f64(lse))
        ref_dq, ref_dk, ref_dv, _, norm = orc.bwd(*f, to_f64(dout), M, s, **given, want_norm=True)
        _, _, reach, _ = orc.bwd(*f, np.abs(to_f64(dout)), M, s, **given)                 # P^T |dO|
        assert (np.abs(dv - ref_dv) <= 0.5 * reach + 2.0 ** -8 * np.abs(ref_dv) + 1e-6).all()
        for got, ref, other in ((dq, ref_dq, k), (dk, ref_dk, q)):
            assert np.linalg.norm(got - ref) <= 0.5 * norm * np.linalg.norm(to_f64(other)) / np.sqrt(d)


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "x".join(map(str, c)))
@pytest.mark.parametrize("path", [binding.RIB_PATH_NONE, binding.RIB_PATH_SM100_EXACT, binding.RIB_PATH_GENERIC])
@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
def test_a_key_with_an_infinite_channel(case, path, value):
    """The sign of a query's channel decides: a logit of plus infinity makes out and lse of the row NaN, one of minus infinity is a weight of 0, and the row is what a very
    low logit leaves of it.  Rows that do not attend to the key do not notice it.  Every path has the same rows."""
    B, H, W, heads, d, M, s = case
    named = log_map(M)
    named[np.add.outer(np.arange(2 * M - 1) * 5, np.arange(2 * M - 1) * 3) % 7 < 3] = -1
    named[M - 1, M - 1] = 0
    q, k, v, _, bias, named = make(B, H, W, heads, d, M, named, torch.float32, seed=37)
    q[..., 1] = torch.where(q[..., 1] == 0, 0.5, q[..., 1].float()).bfloat16()
    py, px = places(H, M, s), places(W, M, s)
    h, KY, KX = heads - 1, int(np.where(py == 2)[0][0]), int(np.where(px == 6)[0][0])
    far, bad = k.clone(), k.clone()
    bad[0, KY, KX, h, 1] = value
    far[0, KY, KX, h, 1] = float(np.sign(value)) * 1e30
    old = binding.rib_set_path(path)
    try:
        out, lse = binding.rib_window_attn_fwd_bucketed(*(t.cuda() for t in (q, bad, v, bias, named)), M, s)
    finally:
        binding.rib_set_path(old)
    ref_out, ref_lse = orc.fwd(*(to_f64(t) for t in (q, far, v, bias)), named.numpy(), M, s)
    lost = np.zeros((H, W, heads), dtype=bool)
    for Y in range(H):
        for X in range(W):
            dy, dx = 2 - py[Y], 6 - px[X]
            if py[Y] // M == 0 and px[X] // M == 0 and named[dy + M - 1, dx + M - 1] >= 0:
                lost[Y, X, h] = float(q[0, Y, X, h, 1]) * value > 0
    assert 0 < lost.sum() < M * M - 1
    got_out, got_lse = to_f64(out)[0], to_f64(lse)[0].transpose(1, 2, 0)
    assert np.array_equal(np.isnan(got_lse), lost) and np.array_equal(np.isnan(got_out).all(-1), lost) and np.array_equal(np.isnan(got_out).any(-1), lost)
    close("out", torch.from_numpy(got_out[~lost]), ref_out[0][~lost])
    close("lse", torch.from_numpy(got_lse[~lost]), ref_lse[0].transpose(1, 2, 0)[~lost])


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "x".join(map(str, c)))
@pytest.mark.parametrize("bias_level,v_scale", [(60.0, 2.0 ** 20), (60.0, 2.0 ** 60), (30.0, 2.0 ** 100), (-20.0, 2.0 ** 100), (0.0, 2.0 ** -60)])
def test_large_and_small_values_beside_large_biases(case, bias_level, v_scale):
    """A level that all biases share changes no weight, and the output is of the size of the values, whatever both are."""
    B, H, W, heads, d, M, s = case
    q, k, v, dout, bias, named = make(B, H, W, heads, d, M, log_map(M), torch.float32, seed=41)
    bias += bias_level
    out, lse, grads = run((q, k, (v.float() * v_scale).bfloat16(), dout, bias, named), M, s)
    inputs = (q, k, v, dout, bias, named)
    back = lambda t: t.float() / v_scale  # noqa: E731  (a power of two: exact)
    compare(inputs, M, s, back(out), lse, (back(grads[0]), back(grads[1]), grads[2], back(grads[3])), 0)


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "x".join(map(str, c)))
@pytest.mark.parametrize("huge", [1e24, 3e38])
@pytest.mark.parametrize("level", [0.0, -20.0])
def test_a_key_out_of_reach_with_a_huge_value(case, huge, level):
    """A finite value has no part in the rows that do not attend to its key; in all heads, every fifth token of the map has one."""
    B, H, W, heads, d, M, s = case
    named = np.full((2 * M - 1, 2 * M - 1), -1)
    named[M - 1, M - 1], named[M - 1, M], named[M - 2, M - 1] = 0, 1, 2          # itself, the token to the right and the one above
    q, k, v, _, bias, named = make(B, H, W, heads, d, M, named, torch.float32, seed=42)
    bias += level
    far = torch.arange(H)[:, None] * 2 + torch.arange(W)[None, :]
    marked = (far % 5 == 0)
    plain = v.clone()
    v[:, marked] = huge
    out, lse = binding.rib_window_attn_fwd_bucketed(*(t.cuda() for t in (q, k, v, bias, named)), M, s)
    ref, ref_lse = orc.fwd(*(to_f64(t) for t in (q, k, plain, bias)), named.numpy(), M, s)
    py, px = places(H, M, s), places(W, M, s)
    at = {(int(a), int(b)): (Y, X) for Y, a in enumerate(py) for X, b in enumerate(px)}
    clean = np.ones((H, W), dtype=bool)
    for (a, b), (Y, X) in at.items():
        for dy, dx in ((0, 0), (0, 1), (-1, 0)):
            other = at.get((a + dy, b + dx))
            if other is not None and (a + dy) // M == a // M and (b + dx) // M == b // M and marked[other]:
                clean[Y, X] = False
    assert 0.2 < clean.mean() < 0.9
    close("out", out[:, torch.from_numpy(clean)], ref[:, clean])
    close("lse", lse, ref_lse)


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "x".join(map(str, c)))
@pytest.mark.parametrize("which", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("checkpointed", [False, True])
def test_what_is_no_number_stays_in_its_window_and_head(case, which, value, checkpointed):
    """One row of one input: the gradients of the other windows and heads are those without it (sums of fp32 atomics in another order, rounded to bf16: 1e-3 as in
    tests/test_gpu_bucketed_calls.py), and so are the sums of the other heads' tables."""
    B, H, W, heads, d, M, s = case
    if which == "dout" and checkpointed:
        pytest.skip("dout is no checkpoint")
    q, k, v, dout, bias, named = (t.cuda() for t in make(B, H, W, heads, d, M, log_map(M), torch.float32, seed=43))

    def gradients(**bad):
        x = {**dict(q=q, k=k, v=v, dout=dout), **bad}
        out, lse = binding.rib_window_attn_fwd_bucketed(x["q"], x["k"], x["v"], bias, named, M, s)
        if not checkpointed:
            return binding.rib_window_attn_bwd_bucketed(x["q"], x["k"], x["v"], bias, named, out, lse, x["dout"], M, s)
        saved = [binding.rib_checkpoint_store(t) for t in (x["q"], x["k"], x["v"], out)]
        return binding.rib_window_attn_bwd_bucketed_checkpointed(*saved, bias, named, lse, x["dout"], M, s)

    clean = gradients()
    py, px = places(H, M, s), places(W, M, s)
    h, Y, X = heads - 1, int(np.where(py == 2)[0][0]), int(np.where(px == 5)[0][0])
    bad = dict(q=q, k=k, v=v, dout=dout)[which].clone()
    bad[0, Y, X, h, d // 2] = value
    got = gradients(**{which: bad})
    other = torch.ones(B, H, W, heads, dtype=torch.bool)
    rows, cols = torch.from_numpy(py // M == 0), torch.from_numpy(px // M == 0)
    other[0, :, :, h] = ~(rows[:, None] & cols[None, :])
    assert other.any() or heads * B == 1
    for a, b in zip(got[:3], clean[:3]):
        a, b = a.float().cpu()[other], b.float().cpu()[other]
        assert torch.isfinite(a).all() and float((a - b).norm()) <= 1e-3 * float(b.norm())
    a, b = got[3][:h], clean[3][:h]
    assert torch.isfinite(a).all() and float((a - b).norm()) <= 1e-5 * float(b.norm())
