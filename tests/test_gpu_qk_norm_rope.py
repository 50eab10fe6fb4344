"""Norms of queries and keys with the rotation by position, forward and backward, against 64 bits.

A result is rounded to bf16 once (at most U = 2^-8 of it); everything before that is fp32: sums of d squares or products, a reciprocal root, the table's entries and the
products of a rotation, each a few 2^-24 of the magnitudes that enter, counted by N = (d + 40) 2^-24.  Sums over tokens: n 2^-24 of the sum of magnitudes at most.
"""
import math

import pytest
import torch

from paper_2603_06738_b200 import binding as rib

pytestmark = pytest.mark.gpu
U = 2.0 ** -8
EPS = 1e-6


def angles(frequencies, H, W, y0, x0):
    f = frequencies.double()
    y = torch.arange(H, device="cuda", dtype=torch.float64) + y0
    x = torch.arange(W, device="cuda", dtype=torch.float64) + x0
    return (y[:, None, None] * f[0] + x[None, :, None] * f[1])[:, :, None]         # [H, W, 1, pairs]


def turned(z, angle, interleaved, magnitude=1.0):
    """The rotation, and the same of magnitudes (a bound of what its roundings see)."""
    pairs = angle.shape[-1]
    rot = 2 * pairs
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, pairs), slice(pairs, rot))
    out = z.clone()
    out[..., first] = magnitude * (z[..., first] * angle.cos() - z[..., second] * angle.sin())
    out[..., second] = magnitude * (z[..., first] * angle.sin() + z[..., second] * angle.cos())
    size = z.abs().clone()
    size[..., first] = abs(magnitude) * (z[..., first].abs() + z[..., second].abs())
    size[..., second] = size[..., first]
    return out, size


def forward(x, weight, angle, interleaved, magnitude=1.0):
    x = x.double()
    if weight is not None:
        x = x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * weight.double()
    if angle is None:
        return x, x.abs()
    return turned(x, angle, interleaved, magnitude)


def backward(x, weight, angle, interleaved, g, magnitude=1.0):
    """dx, dw and bounds of their errors."""
    d = x.shape[-1]
    n = (d + 40) * 2.0 ** -24
    x, g = x.double(), g.double()
    size = g.abs()
    if angle is not None:
        g, size = turned(g, -angle, interleaved, magnitude)
    if weight is None:
        return g, None, U * g.abs() + n * size, None
    root = (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
    unit, w = x / root, weight.double()
    rows = unit[..., 0].numel()
    dw, sw = g * unit, size * unit.abs()
    over = (0, 1, 2) if weight.dim() == 2 else (0, 1, 2, 3)
    gw = g * w
    dx = (gw - unit * (gw * unit).mean(-1, keepdim=True)) / root
    sx = (size * w.abs() + unit.abs() * (size * w.abs() * unit.abs()).mean(-1, keepdim=True)) / root
    sums = min(rows, 4096) * 2.0 ** -24      # a thread adds few rows, and blocks' sums are added in a tree; their number is the depth of neither
    return dx, dw.sum(over), U * dx.abs() + 2 * n * sx, (n + sums) * sw.sum(over)


def check(name, got, want, bound):
    off = ((got.double() - want).abs() - bound).max().item()
    assert off <= 0, f"{name}: {off:.3e} beyond the bound"


def projected(B, H, W, heads, kv, d, seed):
    """q and k as slices of the output of one projection, the way a layer has them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    qkv = (normal(B, H, W, heads + 2 * kv, d) * 2).bfloat16()
    return qkv, qkv[:, :, :, :heads], qkv[:, :, :, heads:heads + kv], normal


def check_both(B, H, W, heads, kv, d, rot, interleaved=False, per_head=False, normed=True, y0=0, x0=0, magnitude=1.0, seed=0, sequence=False):
    qkv, q, k, normal = projected(B, H, W, heads, kv, d, seed)
    weights = [(1 + 0.3 * normal(*((n, d) if per_head else (d,)))) if normed else None for n in (heads, kv)]
    table = angle = None
    if rot:
        frequencies = rib.rib_rope_frequencies(rot, sequence=sequence) + 0.01 * normal(2, rot // 2).abs()
        table = rib.rib_rope_table(frequencies, H, W, y0=y0, x0=x0, magnitude=magnitude)
        angle = angles(frequencies, H, W, y0, x0)
    outs = rib.rib_qk_norm_rope_fwd(q, k, *weights, table, interleaved=interleaved, eps=EPS)
    n = (d + 40) * 2.0 ** -24
    for name, got, x, w in zip("qk", outs, (q, k), weights):
        want, size = forward(x, w, angle, interleaved, magnitude)
        check(name, got, want, U * want.abs() + n * size)
    grads = [normal(*t.shape).bfloat16() for t in outs]
    into = torch.full_like(qkv, 7.0)
    dq, dk, dqw, dkw = rib.rib_qk_norm_rope_bwd(q, k, *weights, table, *grads, interleaved=interleaved, eps=EPS)
    rib.rib_qk_norm_rope_bwd(q, k, *weights, table, *grads, interleaved=interleaved, eps=EPS, dq=into[:, :, :, :heads], dk=into[:, :, :, heads:heads + kv])
    assert torch.equal(into[:, :, :, :heads], dq) and torch.equal(into[:, :, :, heads:heads + kv], dk)
    assert (into[:, :, :, heads + kv:] == 7.0).all()
    for name, dx, dw, x, w, g in zip("qk", (dq, dk), (dqw, dkw), (q, k), weights, grads):
        want, want_w, bound, bound_w = backward(x, w, angle, interleaved, g, magnitude)
        check("d" + name, dx, want, bound)
        if w is not None:
            check(f"d{name}_weight", dw, want_w, bound_w)


@pytest.mark.parametrize("d,rot", [(32, 32), (32, 16), (64, 64), (64, 32), (16, 16), (24, 16), (48, 16), (40, 32), (8, 0), (32, 0), (64, 0), (8, 8), (24, 12), (30, 30), (20, 20),
                                   (20, 12), (18, 6), (2, 2), (3, 2), (33, 32), (63, 10), (1, 0), (5, 4)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_widths_and_layouts(d, rot, interleaved):
    check_both(2, 5, 7, 3, 2, d, rot, interleaved=interleaved, seed=d)


@pytest.mark.parametrize("heads,kv", [(1, 1), (6, 6), (8, 2), (5, 1), (7, 7), (64, 8), (1, 12)])
@pytest.mark.parametrize("per_head", [False, True])
def test_heads(heads, kv, per_head):
    check_both(2, 6, 9, heads, kv, 32, 32, per_head=per_head, seed=heads)


@pytest.mark.parametrize("B,H,W", [(1, 1, 1), (1, 1, 37), (3, 50, 1), (2, 31, 33), (1, 128, 160), (5, 64, 64)])
def test_maps(B, H, W):
    check_both(B, H, W, 4, 4, 32, 32, seed=H)
    check_both(B, H, W, 3, 3, 20, 20, interleaved=True, seed=W)


def test_without_a_norm():
    check_both(2, 9, 10, 3, 3, 32, 16, normed=False)
    check_both(2, 9, 10, 3, 3, 30, 30, normed=False, interleaved=True)


@pytest.mark.parametrize("far", [100000, 2 ** 31, -(2 ** 33)])
def test_far_positions_keep_their_digits(far):
    check_both(1, 12, 13, 2, 2, 32, 32, y0=far, x0=far // 3, seed=4)


def test_magnitude():
    check_both(1, 12, 13, 2, 2, 32, 16, magnitude=1.7, seed=5)


def test_sequences():
    """States of an encoder as a map of one column."""
    check_both(2, 77, 1, 2, 2, 32, 32, sequence=True, seed=6)


def test_queries_alone():
    _, q, _, normal = projected(2, 5, 6, 3, 3, 32, 7)
    w = 1 + 0.2 * normal(32)
    table = rib.rib_rope_table(rib.rib_rope_frequencies(32), 5, 6)
    both = rib.rib_qk_norm_rope_fwd(q, q, w, w, table)
    alone, none = rib.rib_qk_norm_rope_fwd(q, None, w, None, table)
    assert none is None and torch.equal(alone, both[0]) and torch.equal(alone, both[1])
    g = normal(*q.shape).bfloat16()
    dq, dk, dqw, dkw = rib.rib_qk_norm_rope_bwd(q, None, w, None, table, g, None)
    full = rib.rib_qk_norm_rope_bwd(q, q, w, w, table, g, g)
    assert dk is None and dkw is None and torch.equal(dq, full[0])
    _, want, _, bound = backward(q, w, angles(rib.rib_rope_frequencies(32), 5, 6, 0, 0), False, g)
    check("dq_weight", dqw, want, bound)
    check("dq_weight", full[2], want, bound)


def test_one_weight_alone():
    _, q, k, normal = projected(2, 5, 6, 3, 3, 32, 8)
    w = 1 + 0.2 * normal(32)
    got_q, got_k = rib.rib_qk_norm_rope_fwd(q, k, w, None, None)
    want, _ = forward(q, w, None, False)
    check("q", got_q, want, U * want.abs() + 72 * 2.0 ** -24 * want.abs())
    assert torch.equal(got_k, k)


def test_rows_that_are_no_numbers_stay_alone():
    qkv, q, k, normal = projected(1, 8, 9, 4, 4, 32, 9)
    w = 1 + 0.2 * normal(32)
    table = rib.rib_rope_table(rib.rib_rope_frequencies(32), 8, 9)
    clean = rib.rib_qk_norm_rope_fwd(q, k, w, w, table)
    qkv[0, 2, 3, 1, 5] = float("nan")
    qkv[0, 4, 0, 5, 0] = float("inf")
    got = rib.rib_qk_norm_rope_fwd(q, k, w, w, table)
    bad = torch.zeros(2, 1, 8, 9, 4, dtype=torch.bool, device="cuda")
    bad[0, 0, 2, 3, 1] = bad[1, 0, 4, 0, 1] = True
    for i in range(2):
        assert torch.equal(got[i][~bad[i]], clean[i][~bad[i]])
        assert got[i][bad[i]].isnan().any()


def test_zero_rows():
    """A row of zeros stays one, and its gradient is w gz / sqrt(eps)."""
    x = torch.zeros(1, 2, 2, 1, 32, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(32, device="cuda")
    assert (rib.rib_qk_norm_rope_fwd(x, None, w)[0] == 0).all()
    g = torch.randn(1, 2, 2, 1, 32, device="cuda").bfloat16()
    dq, _, dw, _ = rib.rib_qk_norm_rope_bwd(x, None, w, None, None, g, None, eps=1e-4)
    check("dq", dq, g.double() * 100, U * g.double().abs() * 100 * 1.001)
    assert (dw == 0).all()


def test_gradients_against_differences():
    """The gradient's inner product with a direction against the difference of the operator along it, in a direction that bf16 holds exactly."""
    _, q, k, normal = projected(1, 4, 5, 2, 2, 32, 10)
    weights = [1 + 0.2 * normal(32) for _ in range(2)]
    frequencies = rib.rib_rope_frequencies(32)
    table, angle = rib.rib_rope_table(frequencies, 4, 5), angles(frequencies, 4, 5, 0, 0)
    grads = [normal(*t.shape).bfloat16() for t in (q, k)]
    dq, dk, dqw, dkw = rib.rib_qk_norm_rope_bwd(q, k, *weights, table, *grads)
    for x, w, g, dx, dw in ((q, weights[0], grads[0], dq, dqw), (k, weights[1], grads[1], dk, dkw)):
        along, along_w = normal(*x.shape).double(), normal(32).double()
        h = 1e-5
        value = lambda t: ((forward(x.double() + t * along, w.double() + t * along_w, angle, False)[0]) * g.double()).sum()  # noqa: E731
        slope = ((value(h) - value(-h)) / (2 * h)).item()
        got = ((dx.double() * along).sum() + (dw.double() * along_w).sum()).item()
        # dx is rounded to bf16: at most U of each term; the difference itself is off by h^2 and 2^-53 / h of values of the sum's size
        assert abs(got - slope) <= U * (dx.double() * along).abs().sum().item() + 1e-5 * (g.double().abs().sum().item())


def test_results_are_the_same_from_run_to_run():
    _, q, k, normal = projected(2, 60, 70, 6, 2, 32, 11)
    w = 1 + 0.2 * normal(32)
    table = rib.rib_rope_table(rib.rib_rope_frequencies(32), 60, 70)
    grads = [normal(*t.shape).bfloat16() for t in (q, k)]
    first, second = (rib.rib_qk_norm_rope_bwd(q, k, w, w, table, *grads) for _ in range(2))
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def test_scaled_frequencies():
    plain = rib.rib_rope_frequencies(32, device="cpu").double()
    linear = rib.rib_rope_frequencies(32, scaling="linear", scale=4.0, device="cpu").double()
    assert torch.allclose(linear, plain / 4)
    raised = rib.rib_rope_frequencies(32, scaling="base", scale=4.0, device="cpu").double()
    for axis in range(2):
        a, b = plain[axis][plain[axis] > 0], raised[axis][raised[axis] > 0]
        assert a[0] == b[0] == 1 and math.isclose(b[-1], a[-1] / 4, rel_tol=1e-6) and (b <= a).all()
    parts = rib.rib_rope_frequencies(64, base=10000.0, sequence=True, scaling="by_parts", scale=4.0, trained=1024, device="cpu").double()[0]
    whole = rib.rib_rope_frequencies(64, base=10000.0, sequence=True, device="cpu").double()[0]
    turns = 1024 * whole / (2 * math.pi)
    assert torch.allclose(parts[turns >= 32], whole[turns >= 32]) and torch.allclose(parts[turns <= 1], whole[turns <= 1] / 4)
    assert ((parts <= whole) & (parts >= whole / 4 * (1 - 1e-6))).all()


@pytest.mark.parametrize("d,rot", [(24, 24), (40, 40), (56, 24), (32, 8), (8, 8), (20, 8), (12, 8), (44, 40), (28, 24), (60, 56), (36, 0), (4, 0), (12, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("per_head", [False, True])
def test_words_of_four_channels(d, rot, interleaved, per_head):
    """Widths and rotated parts that are multiples of 4 and 8, not of 8 and 16."""
    check_both(2, 13, 17, 5, 3, d, rot, interleaved=interleaved, per_head=per_head, seed=d + rot)
    check_both(1, 64, 90, 2, 2, d, rot, interleaved=interleaved, per_head=per_head, seed=rot)
    check_both(2, 6, 5, 3, 1, d, rot, interleaved=interleaved, per_head=per_head, normed=False, seed=d)
