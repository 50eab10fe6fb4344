"""GPU parity of window attention with a learned bias by buckets (rib_window_attn_fwd_bucketed, rib_window_attn_bwd_bucketed) with the oracle
of that definition: every element, every head, at the sizes, maps and masks where it can go wrong.

Tolerances.  The inputs are bf16 and the arithmetic of the any-shape kernels fp32, so what is left is the rounding of the results to
bf16 (half a step, 2^-8 of a value; 2^-8 / sqrt(3) = 2.3e-3 in the mean of the worst case of a binade, 1.7e-3 over all).  The tcgen05 kernels
also round P and dS to bf16 before they are contracted: independent errors of the same size, which in a sum over n keys shrink with
sqrt(n) where the result does, so the two together stay below 1.5 x 2.3e-3 = 3.5e-3 in relative L2.  Bounds: 5e-3 in relative L2 and 1e-2 of the
largest value, those of the rank-r kernels.  lse is fp32: its error is that of ln of a sum of bf16-rounded terms, at most 2^-8.

The gradients are compared with the oracle's for the out and lse that the backward pass was given: D = rowsum(dO o out) of a rounded out is off
by up to 2^-8 of its terms, which is a property of that input and, where rows are all but one key each or a bucket's sum cancels, larger
than the gradients themselves.  dbias is a sum of many dS of both signs, which the tcgen05 kernels round to bf16 first: independent errors, so
in L2 2^-8 / sqrt(3) x |dS| in the mean; four times that is allowed beside the relative bound (`noise`), which counts where the sum of a bucket
cancels (one bucket for all keys: it is 0)."""
import numpy as np
import pytest
import torch

from oracle import rib_bias_oracle as orc
from paper_2603_06738_b200 import binding

from parity_util import to_f64

pytestmark = pytest.mark.gpu


def takes_tensor_cores(case):
    _, _, _, _, d, M, s, _ = case
    return d % 8 == 0 and d <= 32 and M % 8 == 0 and M <= 64 and s % 8 == 0


def log_map(M, steps=2):
    d = np.arange(1 - M, M)
    far = np.minimum(np.abs(d), steps + np.floor(np.log2(np.maximum(np.abs(d), 1) / steps) * 2).clip(0).astype(int))
    _, at = np.unique(np.sign(d) * far, return_inverse=True)
    return at[:, None] * (at.max() + 1) + at[None, :]


def own_map(M):
    return np.arange((2 * M - 1) ** 2).reshape(2 * M - 1, 2 * M - 1)


def reach_map(M, reach):
    d = np.abs(np.arange(1 - M, M))
    return np.where(np.maximum(d[:, None], d[None, :]) > reach, -1, log_map(M))


def make(B, H, W, heads, d, M, named, dtype=torch.bfloat16, shared=False, seed=0, q_scale=1.0, bias_scale=0.5):
    g = torch.Generator().manual_seed(seed)
    q, k, v, dout = (torch.randn(B, H, W, heads, d, generator=g).bfloat16() for _ in range(4))
    q = (q.float() * q_scale).bfloat16()
    count = max(1, int(named.max()) + 1)
    bias = (torch.randn(*((count,) if shared else (heads, count)), generator=g) * bias_scale).to(dtype)
    return q, k, v, dout, bias, torch.tensor(named, dtype=torch.int32)


def close(name, got, ref, rel_l2=5e-3, noise=0.0):
    got, ref = to_f64(got), np.asarray(ref)
    inf = np.isinf(ref)
    assert np.array_equal(np.isinf(got), inf) and not np.isnan(got).any(), name
    got, ref = got[~inf], ref[~inf]
    if ref.size == 0:
        return
    err, norm = np.abs(got - ref).max(), np.linalg.norm(ref)
    assert err <= 1e-2 * max(1.0, np.abs(ref).max()) + noise, (name, err)
    assert np.linalg.norm(got - ref) <= rel_l2 * norm + 1e-5 * np.sqrt(ref.size) + noise, (name, np.linalg.norm(got - ref) / norm)


def sum_noise(norm):
    return 4 * 2.0 ** -8 / 3 ** 0.5 * norm


def check(inputs, M, s, masked=False, path="auto", fast=None):
    q, k, v, dout, bias, named = inputs
    cuda = [t.cuda() for t in (q, k, v, bias, named)]
    binding.rib_set_path({"auto": binding.RIB_PATH_NONE, "exact": binding.RIB_PATH_SM100_EXACT, "generic": binding.RIB_PATH_GENERIC}[path])
    try:
        out, lse = binding.rib_window_attn_fwd_bucketed(*cuda, M, s, masked=masked)
        used = [binding.rib_last_path()]
        grads = binding.rib_window_attn_bwd_bucketed(*cuda, out, lse, dout.cuda(), M, s, masked=masked)
        used.append(binding.rib_last_path())
    finally:
        binding.rib_set_path(binding.RIB_PATH_NONE)
    torch.cuda.synchronize()
    assert binding.rib_query_status() == 0
    if fast is not None:
        want = binding.RIB_PATH_SM100 if fast and path != "generic" else binding.RIB_PATH_GENERIC
        assert used == [want, want]
    f = [to_f64(t) for t in (q, k, v, bias)] + [named.numpy()]
    ref_out, ref_lse = orc.fwd(*f, M, s, masked)
    close("out", out, ref_out)
    close("lse", lse, ref_lse)
    *refs, norm = orc.bwd(*f, to_f64(dout), M, s, masked, out=to_f64(out), lse=to_f64(lse), want_norm=True)
    for name, got, ref in zip(("dq", "dk", "dv", "dbias"), grads, refs):
        close(name, got, ref, noise=sum_noise(norm) if name == "dbias" else 0.0)
    assert grads[3].dtype == bias.dtype and grads[3].shape == bias.shape
    return out, lse, grads


# B, H, W, heads, d, window, shift, masked
SHAPES = [
    (1, 1, 1, 1, 1, 1, 0, False),               # one token
    (2, 3, 5, 2, 3, 4, 3, False),               # a map smaller than its window
    (1, 8, 12, 2, 16, 4, 1, True),
    (2, 50, 39, 3, 20, 7, 3, False),            # nothing even
    (1, 10, 10, 2, 64, 10, 5, False),           # the widest head
    (1, 12, 24, 1, 40, 12, 0, False),
    (1, 16, 16, 2, 8, 8, 0, False),             # shapes of the tcgen05 kernels from here on
    (1, 24, 40, 2, 24, 8, 0, False),
    (2, 32, 48, 2, 32, 16, 8, False),
    (1, 32, 32, 3, 16, 16, 8, True),
    (1, 48, 24, 2, 32, 24, 16, True),
    (1, 64, 64, 2, 32, 32, 16, False),
    (1, 64, 32, 2, 32, 32, 24, True),
    (1, 41, 53, 2, 32, 16, 0, False),           # ragged maps
    (1, 41, 53, 2, 24, 16, 8, False),
    (2, 33, 71, 1, 32, 32, 8, False),
    (1, 5, 90, 2, 32, 24, 0, False),
    (1, 96, 48, 1, 32, 48, 24, False),
    (1, 64, 64, 1, 32, 64, 32, False),
    (1, 70, 64, 1, 8, 64, 40, False),
]
MAPS = {"log": log_map, "own": own_map, "reach": lambda M: reach_map(M, max(1, M // 3))}


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "x".join(map(str, c)))
@pytest.mark.parametrize("path", ["auto", "exact", "generic"])
def test_every_element(case, path):
    B, H, W, heads, d, M, s, masked = case
    if path == "exact" and not takes_tensor_cores(case):
        pytest.skip("the exact softmax form is a form of the tcgen05 kernel")
    for seed, name in enumerate(MAPS):
        check(make(B, H, W, heads, d, M, MAPS[name](M), seed=seed), M, s, masked, path, takes_tensor_cores(case))


@pytest.mark.parametrize("M,d,s", [(5, 7, 2), (16, 32, 8)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shared", [False, True])
def test_table_types_and_shared_tables(M, d, s, dtype, shared):
    check(make(2, 2 * M, 3 * M, 3, d, M, log_map(M), dtype, shared, seed=9), M, s)


@pytest.mark.parametrize("M,d", [(5, 8), (16, 32), (24, 16)])
def test_rows_without_keys(M, d):
    """Only the right neighbour is attended to: the last column of every window has no key at all, others have one."""
    named = np.full((2 * M - 1, 2 * M - 1), -1)
    named[M - 1, M] = 0
    q, k, v, dout, bias, buckets = inputs = make(1, 2 * M, M, 2, d, M, named, seed=3)
    out, lse, (dq, dk, dv, dbias) = check(inputs, M, 0)
    assert (out[:, :, -1] == 0).all() and torch.isneginf(lse[..., -1]).all() and (dq[:, :, -1] == 0).all() and (dv[:, :, 0] == 0).all()
    # and none for anybody
    check((q, k, v, dout, bias, torch.full_like(buckets, -1)), M, 0)
    check((q, k, v, dout, bias, torch.full_like(buckets, 1)), M, 0)          # (one bucket: 1 is outside)


@pytest.mark.parametrize("low", [-float("inf"), -1e30, float(torch.finfo(torch.float32).min)])
@pytest.mark.parametrize("M,d", [(6, 10), (16, 32)])
def test_biases_that_mask(low, M, d):
    named = np.where(np.add.outer(np.arange(2 * M - 1), np.arange(2 * M - 1)) % 3 == 0, 1, 0)      # (no row loses all keys)
    q, k, v, dout, bias, buckets = make(1, M, 2 * M, 2, d, M, named, torch.float32, seed=4)
    bias[:, 1] = low
    inputs = (q, k, v, dout, bias, buckets)
    _, _, grads = check(inputs, M, 0)
    assert (grads[3][:, 1] == 0).all()
    bias[:, 0] = low                                                        # now every row has lost all
    out, lse, grads = check(inputs, M, 0)
    assert (out == 0).all() and torch.isneginf(lse).all() and all((t == 0).all() for t in grads)


@pytest.mark.parametrize("M,d,s", [(7, 16, 0), (16, 32, 8), (32, 32, 0)])
@pytest.mark.parametrize("q_scale,bias_scale", [(1.0, 30.0), (12.0, 0.5), (30.0, 60.0)])
def test_large_logits(M, d, s, q_scale, bias_scale):
    """Rows whose largest logits are far apart: logits and biases of tens to a hundred nat.  A logit of 100 is known to 2^-24 of itself, a
    weight to 1e-5."""
    check(make(1, M * 2, M, 2, d, M, log_map(M), torch.float32, seed=6, q_scale=q_scale, bias_scale=bias_scale), M, s)


def test_orientation():
    """A bias that is large for one offset only picks that neighbour: the key (dy, dx) away, not the one opposite."""
    M, dy, dx = 16, 3, -2
    bias = torch.zeros(1, (2 * M - 1) ** 2)
    bias[0, (dy + M - 1) * (2 * M - 1) + dx + M - 1] = 200.0
    q, k, v, _, _, named = make(1, M, M, 1, 32, M, own_map(M), seed=2)
    out, _ = binding.rib_window_attn_fwd_bucketed(q.cuda(), k.cuda(), v.cuda(), bias.cuda(), named.cuda(), M)
    assert torch.equal(out[0, : M - dy, -dx:].cpu(), v[0, dy:, : M + dx])


def test_strides_between_tables_and_untouched_elements():
    """The C call takes tables further apart than they are long; what lies between them is neither read nor written."""
    M, heads, d = 16, 3, 32
    q, k, v, dout, bias, named = make(1, 32, 16, heads, d, M, log_map(M), torch.float32, seed=7)
    count, stride = bias.shape[1], bias.shape[1] + 5
    wide = torch.full((heads, stride), float("nan"))
    wide[:, :count] = bias
    t = [x.cuda() for x in (q, k, v, wide, named, dout)]
    out, lse = torch.empty_like(t[0]), torch.empty(1, heads, 32, 16, device="cuda")
    lib, s = binding.library(), torch.cuda.current_stream().cuda_stream
    p = lambda x: x.data_ptr()  # noqa: E731
    assert lib.rib_window_attn_fwd_bucketed(p(t[0]), p(t[1]), p(t[2]), p(t[3]), 0, stride, p(t[4]), count, 1, 32, 16, heads, d, M, 8, 0, p(out), p(lse), s) == 0
    need = lib.rib_window_attn_bwd_bucketed_workspace(stride, count, 1, 32, 16, heads, d, M)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    grads, dwide = [torch.empty_like(t[0]) for _ in range(3)], torch.full_like(t[3], 7.0)
    assert lib.rib_window_attn_bwd_bucketed(p(t[0]), p(t[1]), p(t[2]), p(t[3]), 0, stride, p(t[4]), count, p(out), p(lse), p(t[5]), 1, 32, 16, heads, d, M, 8, 0,
                                            *[p(x) for x in grads], p(dwide), p(ws), need, s) == 0
    ref = binding.rib_window_attn_fwd_bucketed(*t[:3], bias.cuda(), t[4], M, 8)
    assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1]) and (dwide[:, count:] == 7.0).all()
    *refs, norm = orc.bwd(*(to_f64(x) for x in (q, k, v, bias)), named.numpy(), to_f64(dout), M, 8, out=to_f64(out), lse=to_f64(lse), want_norm=True)
    close("dbias", dwide[:, :count], refs[3], noise=sum_noise(norm))


def test_other_streams_graphs_and_repeats():
    """Captured and replayed on a stream of its own, with the inputs of the next replay, and twice in a row."""
    M = 16
    a, b = (make(2, 32, 32, 2, 32, M, log_map(M), seed=s) for s in (11, 12))
    hold = [t.cuda() for t in a]
    q, k, v, dout, bias, named = hold

    def step():
        out, lse = binding.rib_window_attn_fwd_bucketed(q, k, v, bias, named, M, 8)
        return (out, lse, *binding.rib_window_attn_bwd_bucketed(q, k, v, bias, named, out, lse, dout, M, 8))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want_a = [t.clone() for t in step()]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step()
    torch.cuda.current_stream().wait_stream(side)
    for inputs in (b, a):
        for t, x in zip(hold, inputs):
            t.copy_(x)
        for _ in range(2):
            graph.replay()
    torch.cuda.synchronize()
    for x, y in zip(got, want_a):
        close("replay", x, to_f64(y))
    assert torch.equal(got[0], want_a[0])


def test_a_training_loop_uses_them_together():
    """Forward, backward and a step of the table, ten times, the gradient of every step held against the oracle's.

    The steps are large, so that the rows become all but one key each and dP - D small beside dP and D.  Those are fp32 sums of d = 32 products
    each, off by at most 32 x 2^-24 |dO_i| |v_j|; with weights P_ij that add up to 1 over a row and errors that are independent
    between rows, dbias is off by up to 2 x 2^-19 max_j |v_j| |dO| in L2 (`noise`)."""
    M, heads, d = 16, 2, 32
    q, k, v, _, target, named = (t.cuda() for t in make(1, 32, 32, heads, d, M, log_map(M), torch.float32, seed=20, bias_scale=1.5))
    want, _ = binding.rib_window_attn_fwd_bucketed(q, k, v, target, named, M, 8)
    bias, longest = torch.zeros_like(target), v.float().norm(dim=-1).max().item()
    for _ in range(10):
        out, lse = binding.rib_window_attn_fwd_bucketed(q, k, v, bias, named, M, 8)
        dout = (out.float() - want.float()).bfloat16()
        grads = binding.rib_window_attn_bwd_bucketed(q, k, v, bias, named, out, lse, dout, M, 8)
        assert all(torch.isfinite(t.float()).all() for t in grads)
        *refs, norm = orc.bwd(*(to_f64(t) for t in (q, k, v, bias)), named.cpu().numpy(), to_f64(dout), M, 8, out=to_f64(out), lse=to_f64(lse), want_norm=True)
        close("dbias", grads[3], refs[3], noise=sum_noise(norm) + 2.0 ** -18 * longest * dout.float().norm().item())
        bias -= 2.0 * grads[3]
