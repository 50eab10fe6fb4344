"""How the calls of attention to states and of norms with rotation are made: natively and in Python, on other streams, captured into graphs, next to one another; the ends of their
buffers, far offsets, and the two forms of the softmax."""
import math

import pytest
import torch

import cross_util as ref
from paper_2603_06738_b200 import binding as rib
from test_gpu_marshal import both, same

pytestmark = pytest.mark.gpu


def make(seed=0, B=2, H=7, W=9, heads=4, kv=2, d=32, L=100, contexts=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()  # noqa: E731
    contexts = B if contexts is None else contexts
    return normal(B, H, W, heads, d), normal(contexts, L, kv, d), normal(contexts, L, kv, d), normal(B, H, W, heads, d)


def rope_inputs(seed=0, B=2, H=7, W=9, heads=4, kv=2, d=32, rot=32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = torch.randn(B, H, W, heads + 2 * kv, d, device="cuda", generator=g).bfloat16()
    weights = [1 + 0.2 * torch.randn(d, device="cuda", generator=g) for _ in range(2)]
    frequencies = rib.rib_rope_frequencies(rot)
    grads = [torch.randn(B, H, W, n, d, device="cuda", generator=g).bfloat16() for n in (heads, kv)]
    return qkv[:, :, :, :heads], qkv[:, :, :, heads:heads + kv], weights, frequencies, grads


# ------------------------------------------------------------------------------------------------- native and Python
def test_native_and_python_marshalling_agree(monkeypatch):
    q, k, v, dout = make()
    lengths = torch.tensor([30, 100], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for options in ({}, {"lengths": lengths}, {"want_lse": False}, {"stream": side}, {"workspace": torch.empty(1 << 20, dtype=torch.uint8, device="cuda")}):
        a, b = both(monkeypatch, lambda: rib.rib_cross_attn_fwd(q, k, v, **options))
        torch.cuda.synchronize()
        assert same(a, b)
    out, lse = rib.rib_cross_attn_fwd(q, k, v)
    for options in ({}, {"lengths": lengths}, {"stream": side}, {"workspace": torch.empty(1 << 22, dtype=torch.uint8, device="cuda")}):
        a, b = both(monkeypatch, lambda: rib.rib_cross_attn_bwd(q, k, v, out, lse, dout, **options))
        torch.cuda.synchronize()
        assert same(a, b)
    x, y, weights, frequencies, grads = rope_inputs()
    for options in ({}, {"y0": 5, "x0": -7, "magnitude": 1.5}, {"stream": side}):
        a, b = both(monkeypatch, lambda: rib.rib_rope_table(frequencies, 7, 9, **options))
        torch.cuda.synchronize()
        assert same(a, b)
    table = rib.rib_rope_table(frequencies, 7, 9)
    heads = [w.expand(n, 32).contiguous() for w, n in zip(weights, (4, 2))]
    for args in ((x, y, *weights, table), (x, y, *heads, table), (x, y, None, weights[1], table), (x, None, weights[0], None, table), (x, y, *weights, None)):
        for options in ({}, {"interleaved": True, "eps": 1e-3}, {"stream": side}):
            a, b = both(monkeypatch, lambda: rib.rib_qk_norm_rope_fwd(*args, **options))
            c, e = both(monkeypatch, lambda: rib.rib_qk_norm_rope_bwd(*args, grads[0], grads[1] if args[1] is not None else None, **options))
            torch.cuda.synchronize()
            assert same(a, b) and same(c, e)


def refusals():
    q, k, v, dout = make()
    out, lse = rib.rib_cross_attn_fwd(q, k, v)
    x, y, weights, frequencies, grads = rope_inputs()
    table = rib.rib_rope_table(frequencies, 7, 9)
    short = torch.tensor([1], dtype=torch.int32, device="cuda")
    many = make(L=300)
    results = rib.rib_cross_attn_fwd(*many[:3])
    return [
        lambda: rib.rib_cross_attn_fwd(q.float(), k, v),
        lambda: rib.rib_cross_attn_fwd(q.transpose(1, 2), k, v),
        lambda: rib.rib_cross_attn_fwd(q, k[:, :50], v[:, :50]),
        lambda: rib.rib_cross_attn_fwd(q, k, v[:, :99].contiguous()),
        lambda: rib.rib_cross_attn_fwd(q[..., :16].contiguous(), k, v),
        lambda: rib.rib_cross_attn_fwd(q[:, :, :, :3].contiguous(), k, v),
        lambda: rib.rib_cross_attn_fwd(torch.cat([q, q[:1]]), k, v),
        lambda: rib.rib_cross_attn_fwd(q, k[:, :0].contiguous(), v[:, :0].contiguous()),
        lambda: rib.rib_cross_attn_fwd(q, k, v, lengths=short),
        lambda: rib.rib_cross_attn_fwd(q, k, v, lengths=torch.tensor([1, 2], device="cuda")),
        lambda: rib.rib_cross_attn_fwd(q, k, v, lengths=torch.tensor([1, 2], dtype=torch.int32)),
        lambda: rib.rib_cross_attn_bwd(q, k, v, out, lse, dout[..., :16]),
        lambda: rib.rib_cross_attn_bwd(q, k, v, out, lse[:1], dout),
        lambda: rib.rib_cross_attn_bwd(*many[:3], *results, many[3], workspace=torch.empty(256, dtype=torch.uint8, device="cuda")),
        lambda: rib.rib_rope_table(frequencies.double(), 7, 9),
        lambda: rib.rib_rope_table(frequencies, 0, 9),
        lambda: rib.rib_rope_table(torch.zeros(2, 33, device="cuda"), 7, 9),
        lambda: rib.rib_qk_norm_rope_fwd(x.transpose(3, 4), y, *weights, table),
        lambda: rib.rib_qk_norm_rope_fwd(x[:, ::2], y[:, ::2], *weights, None),
        lambda: rib.rib_qk_norm_rope_fwd(x, y[:, :5], *weights, table),
        lambda: rib.rib_qk_norm_rope_fwd(x, y, weights[0][:16], weights[1], table),
        lambda: rib.rib_qk_norm_rope_fwd(x, y, weights[0], weights[1].expand(2, 32).contiguous(), table),
        lambda: rib.rib_qk_norm_rope_fwd(x, y, *weights, rib.rib_rope_table(frequencies, 9, 9)),
        lambda: rib.rib_qk_norm_rope_fwd(x, None, *weights, table),
        lambda: rib.rib_qk_norm_rope_fwd(x, y, *weights, table, eps=-1.0),
        lambda: rib.rib_qk_norm_rope_fwd(x[..., :16], y[..., :16], None, None, table),
        lambda: rib.rib_qk_norm_rope_bwd(x, y, *weights, table, grads[0], None),
        lambda: rib.rib_qk_norm_rope_bwd(x, y, *weights, table, grads[0], grads[1], dq=torch.empty_like(grads[1])),
    ]


def test_refusals_are_the_same_natively_and_in_python(monkeypatch):
    for i, call in enumerate(refusals()):
        a, b = both(monkeypatch, call)
        assert isinstance(a, tuple) and isinstance(a[0], type) and issubclass(a[0], (ValueError, rib.RibError)) and a == b, (i, a, b)
    torch.cuda.synchronize()
    assert rib.rib_query_status() == 0


# ----------------------------------------------------------------------------------------------- streams and graphs
def test_on_another_stream():
    q, k, v, dout = make(1, H=40, W=50, L=300)
    lengths = torch.tensor([300, 120], dtype=torch.int32, device="cuda")
    x, y, weights, frequencies, grads = rope_inputs(1, H=40, W=50)

    def everything(stream):
        out, lse = rib.rib_cross_attn_fwd(q, k, v, lengths=lengths, stream=stream)
        table = rib.rib_rope_table(frequencies, 40, 50, stream=stream)
        return (out, lse, *rib.rib_cross_attn_bwd(q, k, v, out, lse, dout, lengths=lengths, stream=stream), *rib.rib_qk_norm_rope_fwd(x, y, *weights, table, stream=stream),
                *rib.rib_qk_norm_rope_bwd(x, y, *weights, table, *grads, stream=stream))

    want = everything(None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = everything(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("B,H,W,heads,kv,d,L", [(2, 20, 30, 4, 2, 32, 200), (3, 1, 1, 2, 2, 64, 900), (1, 9, 11, 3, 3, 30, 70)])
def test_captured_and_replayed_with_other_inputs(B, H, W, heads, kv, d, L):
    """Two graphs that share their scratch, replayed one after the other, and again after the inputs have changed."""
    sets = [make(s, B, H, W, heads, kv, d, L) for s in (2, 3)]
    held = [t.clone() for t in sets[0]]
    lengths = torch.full((B,), L, dtype=torch.int32, device="cuda")
    sizes = (B, H, W, heads, kv, d, L, B)
    scratch = torch.empty(max(rib.rib_cross_attn_fwd_workspace(*sizes), rib.rib_cross_attn_bwd_workspace(*sizes), 256), dtype=torch.uint8, device="cuda")

    def step():
        q, k, v, dout = held
        out, lse = rib.rib_cross_attn_fwd(q, k, v, lengths=lengths, workspace=scratch)
        return (out, lse, *rib.rib_cross_attn_bwd(q, k, v, out, lse, dout, lengths=lengths, workspace=scratch))

    step()
    graphs, results = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            results.append(step())
        graphs.append(g)
    for chosen, cut in ((0, 0), (1, 3), (0, 1)):
        for t, new in zip(held, sets[chosen]):
            t.copy_(new)
        lengths.fill_(max(1, L - cut * 7))
        want = [t.clone() for t in step()]
        for g, got in zip(graphs, results):
            for t in got:
                t.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert rib.rib_query_status() == 0


def test_norms_captured_and_replayed():
    x, y, weights, frequencies, grads = rope_inputs(4)

    def step():
        table = rib.rib_rope_table(frequencies, 7, 9)
        return (*rib.rib_qk_norm_rope_fwd(x, y, *weights, table), *rib.rib_qk_norm_rope_bwd(x, y, *weights, table, *grads))

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    frequencies.mul_(1.1)
    weights[0].add_(0.3)
    g.replay()
    want = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_two_calls_at_once_on_two_streams():
    """Each with scratch of its own."""
    sets = [make(s, H=30, W=40, L=260) for s in (5, 6)]
    alone = [rib.rib_cross_attn_bwd(q, k, v, *rib.rib_cross_attn_fwd(q, k, v), dout) for q, k, v, dout in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(3):
        for i, (stream, (q, k, v, dout)) in enumerate(zip(streams, sets)):
            out, lse = rib.rib_cross_attn_fwd(q, k, v, stream=stream)
            got[i].append(rib.rib_cross_attn_bwd(q, k, v, out, lse, dout, stream=stream))
    torch.cuda.synchronize()
    for want, several in zip(alone, got):
        assert all(torch.equal(a, b) for one in several for a, b in zip(want, one))
    assert rib.rib_query_status() == 0


# -------------------------------------------------------------------------------------------------- ends of buffers
class Guarded:
    """A buffer between two stretches that nothing may write to."""
    EDGE = 4096

    def __init__(self, shape, dtype, extra=0):
        count = math.prod(shape) + extra
        self.size = count * torch.empty((), dtype=dtype).element_size()
        self.raw = torch.full((2 * self.EDGE + (self.size + 255) // 256 * 256,), 0xA5, dtype=torch.uint8, device="cuda")
        self.t = self.raw[self.EDGE:self.EDGE + self.size].view(dtype)[:math.prod(shape)].view(shape)

    def intact(self):
        return bool((self.raw[:self.EDGE] == 0xA5).all() and (self.raw[self.EDGE + self.size:] == 0xA5).all())


@pytest.mark.parametrize("B,H,W,heads,kv,d,L,contexts", [(2, 5, 7, 3, 1, 32, 70, 2), (3, 1, 1, 4, 4, 64, 700, 3), (2, 9, 13, 6, 2, 20, 33, 1), (1, 30, 40, 2, 2, 24, 129, 1), (2, 1, 3, 5, 5, 1, 17, 2)])
def test_nothing_is_written_beside_the_results(B, H, W, heads, kv, d, L, contexts):
    q, k, v, dout = make(7, B, H, W, heads, kv, d, L, contexts)
    lib = rib.library()
    sizes = (B, H, W, heads, kv, d, L, contexts)
    out, lse = Guarded(q.shape, torch.bfloat16), Guarded((B, heads, H, W), torch.float32)
    dq, dk, dv = Guarded(q.shape, torch.bfloat16), Guarded(k.shape, torch.bfloat16), Guarded(k.shape, torch.bfloat16)
    forward, backward = rib.rib_cross_attn_fwd_workspace(*sizes), rib.rib_cross_attn_bwd_workspace(*sizes)
    for lengths in (None, torch.randint(0, L + 1, (contexts,), dtype=torch.int32, device="cuda")):
        ws = Guarded((max(forward, 1),), torch.uint8)
        stream = torch.cuda.current_stream().cuda_stream
        ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        assert lib.rib_cross_attn_fwd(ptr(q), ptr(k), ptr(v), ptr(lengths), *sizes, ptr(out.t), ptr(lse.t), ptr(ws.t), forward, stream) == 0
        scratch = Guarded((backward,), torch.uint8)
        assert lib.rib_cross_attn_bwd(ptr(q), ptr(k), ptr(v), ptr(lengths), ptr(out.t), ptr(lse.t), ptr(dout), *sizes, ptr(dq.t), ptr(dk.t), ptr(dv.t), ptr(scratch.t), backward, stream) == 0
        torch.cuda.synchronize()
        assert all(x.intact() for x in (out, lse, dq, dk, dv, ws, scratch))
        want = rib.rib_cross_attn_fwd(q, k, v, lengths=lengths)
        assert torch.equal(out.t, want[0]) and torch.equal(lse.t, want[1])


@pytest.mark.parametrize("B,H,W,heads,kv,d,rot,per_head", [(2, 5, 7, 3, 1, 32, 32, False), (1, 1, 1, 1, 0, 64, 0, True), (2, 9, 11, 12, 12, 24, 16, True), (1, 17, 19, 5, 2, 30, 30, False), (1, 3, 5, 300, 7, 8, 8, True)])
def test_nothing_is_written_beside_the_norms_results(B, H, W, heads, kv, d, rot, per_head):
    lib = rib.library()
    g = torch.Generator(device="cuda").manual_seed(8)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x = normal(B, H, W, heads + kv, d).bfloat16()
    grads = [normal(B, H, W, n, d).bfloat16() for n in (heads, kv)]
    shapes = [((n, d) if per_head else (d,)) for n in (heads, kv)]
    weights = [1 + 0.1 * normal(*s) for s in shapes]
    table = Guarded((H + W, max(rot // 2, 1), 2), torch.float32)
    stream = torch.cuda.current_stream().cuda_stream
    if rot:
        f = rib.rib_rope_frequencies(rot)
        assert lib.rib_rope_table(f.data_ptr(), H, W, rot // 2, 3, 4, 1.0, table.t.data_ptr(), stream) == 0
    outs = [Guarded((B, H, W, n, d), torch.bfloat16) for n in (heads, kv)]
    dx = Guarded(x.shape, torch.bfloat16)
    dws = [Guarded(s, torch.float32) for s in shapes]
    ws = Guarded((rib.rib_qk_norm_rope_bwd_workspace(B, H, W, heads, kv, d, per_head),), torch.uint8)
    some = lambda t: t.data_ptr() if kv else None  # noqa: E731
    layer = (x.data_ptr(), (heads + kv) * d, x[:, :, :, heads:].data_ptr() if kv else None, (heads + kv) * d, weights[0].data_ptr(), some(weights[1]), int(per_head), table.t.data_ptr() if rot else None)
    sizes = (B, H, W, heads, kv, d, rot, 0, 1e-6)
    assert lib.rib_qk_norm_rope_fwd(*layer, *sizes, outs[0].t.data_ptr(), some(outs[1].t), stream) == 0
    assert lib.rib_qk_norm_rope_bwd(*layer, grads[0].data_ptr(), some(grads[1]), *sizes, dx.t.data_ptr(), (heads + kv) * d, dx.t[:, :, :, heads:].data_ptr() if kv else None, (heads + kv) * d,
                                    dws[0].t.data_ptr(), some(dws[1].t), ws.t.data_ptr(), ws.size, stream) == 0
    torch.cuda.synchronize()
    assert all(b.intact() for b in (table, *outs, dx, *dws, ws))
    assert torch.isfinite(dx.t.float()).all() and torch.isfinite(dws[0].t).all()


# ------------------------------------------------------------------------------------------------------ far offsets
@pytest.mark.parametrize("heads,kv,d,L", [(32, 32, 64, 1_100_000), (64, 16, 64, 2_200_000)])
def test_offsets_beyond_32_bits(heads, kv, d, L):
    """More than 2^31 elements of keys: on the plain pipes (a row to a group), and on the tensor cores (four), with gradients."""
    g = torch.Generator(device="cuda").manual_seed(9)
    k, v = (torch.empty(1, L, kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (k, v):
        for lo in range(0, L, 200_000):
            t[:, lo:lo + 200_000] = torch.randn(1, min(200_000, L - lo), kv, d, device="cuda", generator=g).bfloat16()
    k[0, -3:, -1] *= 6                                    # the last states of the last head matter
    q, dout = (torch.randn(1, 1, 1, heads, d, device="cuda", generator=g).bfloat16() for _ in range(2))
    assert k.numel() > 2 ** 31
    out, lse = rib.rib_cross_attn_fwd(q, k, v)
    few = kv - 1
    rows = slice(few * (heads // kv), heads)
    s = (q[0, 0, 0, rows].double() @ k[0, :, few].double().T) / math.sqrt(d)
    want_lse = torch.logsumexp(s, 1)
    p = torch.exp(s - want_lse[:, None])
    want = p @ v[0, :, few].double()
    x = ref.score_error(q, k[:, -3:], None)
    bound = ref.U * want.abs() + (ref.U + 2 * x + 2.0 ** -16) * (p @ v[0, :, few].double().abs())
    assert ((out[0, 0, 0, rows].double() - want).abs() <= bound).all()
    assert ((lse[0, rows, 0, 0].double() - want_lse).abs() <= x + 2.0 ** -16).all()
    if heads == kv:
        return
    dq, dk, dv = rib.rib_cross_attn_bwd(q, k, v, out, lse, dout)
    g64, last = dout[0, 0, 0, rows].double(), slice(L - 1000, L)
    weights = torch.exp(s - lse[0, rows, 0, 0].double()[:, None])
    ds = weights * (g64 @ v[0, :, few].double().T - (out[0, 0, 0, rows].double() * g64).sum(1, keepdim=True))
    want_v, want_k = weights[:, last].T @ g64, ds[:, last].T @ q[0, 0, 0, rows].double() / math.sqrt(d)
    assert ((dv[0, last, few].double() - want_v).abs() <= ref.U * want_v.abs() + (ref.U + 2 * x + 2.0 ** -16) * (weights[:, last].T @ g64.abs()) + 1e-30).all()
    loose = (weights * (g64.abs() @ v[0, :, few].double().abs().T + (out[0, 0, 0, rows].double() * g64).abs().sum(1, keepdim=True)))[:, last] * (d + 8) * 2.0 ** -24
    assert ((dk[0, last, few].double() - want_k).abs() <=
            ref.U * want_k.abs() + ((ds[:, last].abs() * (ref.U + 2 * x + 2.0 ** -16) + loose).T @ q[0, 0, 0, rows].double().abs()) / math.sqrt(d) + 1e-30).all()


def test_norms_of_far_tokens():
    """Tokens of a projection whose elements pass 2^31."""
    tokens, width = 1 << 20, 40
    qkv = torch.zeros(1, 1024, 1024, width, 64, dtype=torch.bfloat16, device="cuda")
    assert qkv.numel() > 2 ** 31
    qkv[0, -1, -3:] = torch.randn(3, width, 64, device="cuda").bfloat16()
    w = torch.ones(64, device="cuda")
    q, k = rib.rib_qk_norm_rope_fwd(qkv[:, :, :, :8], qkv[:, :, :, 38:], w, w)
    for got, x in ((q[0, -1, -3:], qkv[0, -1, -3:, :8].double()), (k[0, -1, -3:], qkv[0, -1, -3:, 38:].double())):
        want = x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()
        assert ((got.double() - want).abs() <= ref.U * want.abs() * 1.001).all()
    assert tokens == q[0, ..., 0, 0].numel() and (q[0, 0] == 0).all()


# ----------------------------------------------------------------------------------------------- the softmax's forms
@pytest.fixture
def exact_form():
    before = rib.rib_set_path(rib.RIB_PATH_SM100_EXACT)
    yield
    rib.rib_set_path(before)


@pytest.mark.parametrize("d", [32, 64, 20])
@pytest.mark.parametrize("L", [1, 40, 128, 300])
def test_the_exact_form(exact_form, d, L):
    q, k, v, _ = make(10, H=17, W=19, d=d, L=L)
    out, lse = rib.rib_cross_attn_fwd(q, k, v)
    (want, want_lse), (bound, bound_lse) = ref.forward(q, k, v)
    ref.check("out", out, want, bound)
    ref.check("lse", lse, want_lse, bound_lse)


@pytest.mark.parametrize("above", [10.0, 60.0, 200.0, 5000.0])
@pytest.mark.parametrize("d", [32, 64])
def test_scores_far_above_those_of_the_first_states(above, d):
    """Beyond the range of the fixed reference the item is redone; every row of some items, one row of others."""
    q, k, v, _ = make(11, B=2, H=24, W=25, heads=2, kv=2, d=d, L=400)
    q[..., 0] = 1.0
    k[..., 0] = 0.0
    k[0, 200:260, 0, 0] = above * math.sqrt(d)
    q[1] = 0
    q[1, 13, 7, 1] = k[1, 333, 1] * (above / 8)
    out, lse = rib.rib_cross_attn_fwd(q, k, v)
    (want, want_lse), (bound, bound_lse) = ref.forward(q, k, v)
    ref.check("out", out, want, bound)
    ref.check("lse", lse, want_lse, bound_lse)


@pytest.mark.parametrize("d", [32, 64])
def test_large_values_behind_large_weights(d):
    """Sums that overflow relative to the fixed reference though the output does not."""
    q, k, v, _ = make(12, H=16, W=16, d=d, L=200)
    q[..., 0] = 1.0
    k[..., 0] = 0.0
    k[:, 150:, :, 0] = 60.0 * math.sqrt(d)
    v *= 1e30
    out, lse = rib.rib_cross_attn_fwd(q, k, v)
    (want, want_lse), (bound, bound_lse) = ref.forward(q, k, v)
    assert torch.isfinite(out.float()).all()
    ref.check("out", out, want, bound)
    ref.check("lse", lse, want_lse, bound_lse)


# ------------------------------------------------------------------------------------------------------ a run of them
def test_a_block_of_a_model():
    """Norms and rotation, attention in windows, norms, attention to states, and the whole way back, as a layer does it; gradients against 64 bits through autograd.

    Roundings to bf16 on a way from the output's gradient to an input's: states attention 3 (P, dS, result), norms 1, windows 3, rotation 1, and of the forward values that enter
    there 6; each is at most U of what it rounds, in norm too, so 14 U bounds what they add up to if none is enlarged on its way."""
    B, H, W, heads, d, M, r, L = 2, 32, 32, 4, 32, 16, 16, 77
    g = torch.Generator(device="cuda").manual_seed(13)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    qkv, states, dout = normal(B, H, W, 3 * heads, d).bfloat16(), normal(B, L, 2 * heads, d).bfloat16(), normal(B, H, W, heads, d).bfloat16()
    pq, pk = (normal(M * M, r).mul(0.5).bfloat16() for _ in range(2))
    w = [1 + 0.2 * normal(d) for _ in range(4)]
    lengths = torch.tensor([77, 40], dtype=torch.int32, device="cuda")
    f = rib.rib_rope_frequencies(d)
    table = rib.rib_rope_table(f, H, W)
    q, k, v = qkv[:, :, :, :heads], qkv[:, :, :, heads:2 * heads], qkv[:, :, :, 2 * heads:].contiguous()
    keys, values = states[:, :, None, :heads], states[:, :, heads:].contiguous()

    q1, k1 = rib.rib_qk_norm_rope_fwd(q, k, w[0], w[1], table)
    a, lse_a = rib.rib_window_attn_fwd(q1, k1, v, pq, pk, M, 8)
    q2, _ = rib.rib_qk_norm_rope_fwd(a, None, w[2])
    k2, _ = rib.rib_qk_norm_rope_fwd(keys, None, w[3])                     # the states as a map of one column
    k2 = k2[:, :, 0]
    out, lse_o = rib.rib_cross_attn_fwd(q2, k2, values, lengths=lengths)
    dq2, dk2, dvalues = rib.rib_cross_attn_bwd(q2, k2, values, out, lse_o, dout, lengths=lengths)
    dkeys, _, dw3, _ = rib.rib_qk_norm_rope_bwd(keys, None, w[3], None, None, dk2[:, :, None], None)
    da, _, dw2, _ = rib.rib_qk_norm_rope_bwd(a, None, w[2], None, None, dq2, None)
    dq1, dk1, dv, dpq, dpk = rib.rib_window_attn_bwd(q1, k1, v, pq, pk, a, lse_a, da, M, 8)
    dqkv = torch.empty_like(qkv)
    _, _, dw0, dw1 = rib.rib_qk_norm_rope_bwd(q, k, w[0], w[1], table, dq1, dk1, dq=dqkv[:, :, :, :heads], dk=dqkv[:, :, :, heads:2 * heads])
    dqkv[:, :, :, 2 * heads:] = dv
    torch.cuda.synchronize()
    assert rib.rib_query_status() == 0

    leaves = [t.double().requires_grad_() for t in (qkv, states, *w, pq, pk)]
    X, S, W0, W1, W2, W3, PQ, PK = leaves
    norm = lambda x, weight: x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * weight  # noqa: E731
    y, x = torch.arange(H, device="cuda").double(), torch.arange(W, device="cuda").double()
    angle = (y[:, None, None] * f[0].double() + x[None, :, None] * f[1].double())[:, :, None]

    def turn(z):
        one, two = z[..., :d // 2], z[..., d // 2:]
        return torch.cat([one * angle.cos() - two * angle.sin(), two * angle.cos() + one * angle.sin()], -1)

    def windows(t):
        t = torch.roll(t, (-8, -8), (1, 2)).view(B, H // M, M, W // M, M, heads, d)
        return t.permute(0, 1, 3, 5, 2, 4, 6).reshape(B, H // M, W // M, heads, M * M, d)

    Q, K, V = turn(norm(X[:, :, :, :heads], W0)), turn(norm(X[:, :, :, heads:2 * heads], W1)), X[:, :, :, 2 * heads:]
    s = windows(Q) @ windows(K).transpose(-1, -2) / math.sqrt(d) + PQ @ PK.T / math.sqrt(r)
    A = (torch.softmax(s, -1) @ windows(V)).view(B, H // M, W // M, heads, M, M, d).permute(0, 1, 4, 2, 5, 3, 6).reshape(B, H, W, heads, d)
    A = torch.roll(A, (8, 8), (1, 2))
    Q2 = norm(A, W2).flatten(1, 2).transpose(1, 2)
    K2, V2 = norm(S[:, :, :heads], W3).transpose(1, 2), S[:, :, heads:].transpose(1, 2)
    s = (Q2 @ K2.transpose(-1, -2) / math.sqrt(d)).masked_fill((torch.arange(L, device="cuda") >= lengths[:, None])[:, None, None], -math.inf)
    O = (torch.softmax(s, -1) @ V2).transpose(1, 2).reshape(B, H, W, heads, d)
    O.backward(dout.double())
    dstates = torch.cat([dkeys[:, :, 0], dvalues], 2)
    for name, got, want in (("out", out, O.detach()), ("qkv", dqkv, X.grad), ("states", dstates, S.grad), ("w0", dw0, W0.grad), ("w1", dw1, W1.grad), ("w2", dw2, W2.grad), ("w3", dw3, W3.grad),
                            ("pq", dpq, PQ.grad), ("pk", dpk, PK.grad)):
        off = ((got.double() - want).norm() / want.norm()).item()
        assert off <= 14 * ref.U, f"{name}: {off:.3e}"
