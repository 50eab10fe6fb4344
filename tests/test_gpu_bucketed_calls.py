"""How the calls for a bias by buckets and for 8-bit checkpoints are made: with and without the native marshaller, with late inputs on a side stream,
old values in the results, two graphs that share a workspace, and tensors of more than 2^31 elements.

What is compared is compared bit by bit where the arithmetic has one order.  dq and dbias are sums of fp32 atomics, whose order may differ: their
difference is a few rounding steps of the sums, 2^-24 each, of terms that are larger than the result by a factor that stays below 2^6 for the
inputs here, and for what is rounded to bf16 behind it one step more of a few values: 1e-3 in relative L2 for those, 1e-5 for fp32."""
import ctypes

import pytest
import torch

from paper_2603_06738_b200 import binding

from test_gpu_bucketed import log_map, make
from test_gpu_checkpoints import kept
from test_gpu_marshal import both, same
from test_gpu_overtaking import LATE
from test_gpu_safety import Guarded

pytestmark = pytest.mark.gpu


def near(a, b):
    assert a.shape == b.shape and a.dtype == b.dtype and a.device == b.device
    assert float((a.float() - b.float()).norm()) <= (1e-5 if a.dtype == torch.float32 else 1e-3) * float(b.float().norm())


def agree(a, b, exact):
    for i, (x, y) in enumerate(zip(a, b, strict=True)):
        if i in exact:
            assert same(x, y), i
        else:
            near(x, y)


@pytest.mark.parametrize("M,d,s", [(16, 32, 8), (7, 20, 3), (20, 10, 4)])
@pytest.mark.parametrize("dtype,shared", [(torch.float32, False), (torch.bfloat16, True)])
def test_same_results_without_the_native_marshaller(monkeypatch, M, d, s, dtype, shared):
    assert binding._marshal is not None
    q, k, v, dout, bias, named = (t.cuda() for t in make(2, 33, 40, 2, d, M, log_map(M), dtype, shared=shared, seed=3))
    for options in ({}, {"want_lse": False}, {"stream": torch.cuda.Stream()}):
        torch.cuda.synchronize()
        a, b = both(monkeypatch, lambda: binding.rib_window_attn_fwd_bucketed(q, k, v, bias, named, M, s, **options))
        torch.cuda.synchronize()
        assert same(a, b)
    out, lse = binding.rib_window_attn_fwd_bucketed(q, k, v, bias, named, M, s)
    workspace = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    exact = {1, 2} if M != 20 else {0, 1, 2}
    for options in ({}, {"workspace": workspace}):
        agree(*both(monkeypatch, lambda: binding.rib_window_attn_bwd_bucketed(q, k, v, bias, named, out, lse, dout, M, s, **options)), exact)
    stored = both(monkeypatch, lambda: [binding.rib_checkpoint_store(t) for t in (q, k, v, out)])
    assert same(*stored)
    assert same(*both(monkeypatch, lambda: [binding.rib_checkpoint_restore(*x) for x in stored[0]]))
    for options in ({}, {"workspace": workspace}):
        agree(*both(monkeypatch, lambda: binding.rib_window_attn_bwd_bucketed_checkpointed(*stored[0], bias, named, lse, dout, M, s, **options)), exact)


@pytest.mark.parametrize("headwise", [False, True])
def test_same_results_of_a_rank_r_layer_without_the_native_marshaller(monkeypatch, headwise):
    g = torch.Generator().manual_seed(9)
    q, k, v, dout = (torch.randn(1, 32, 48, 2, 32, generator=g).bfloat16().cuda() for _ in range(4))
    pq, pk = (torch.randn(*((2,) if headwise else ()), 256, 16, generator=g).bfloat16().cuda() for _ in range(2))
    out, lse = binding.rib_window_attn_fwd_masked(q, k, v, pq, pk, 16, 8)
    saved = kept((q, k, v, out))
    workspace = torch.empty(1 << 25, dtype=torch.uint8, device="cuda")
    for options in ({}, {"workspace": workspace}):
        agree(*both(monkeypatch, lambda: binding.rib_window_attn_bwd_checkpointed(*saved, pq, pk, lse, dout, 16, 8, masked=True, **options)), {1, 2})


def refusals():
    q, k, v, dout, bias, named = (t.cuda() for t in make(1, 16, 16, 2, 16, 8, log_map(8), seed=4))
    out, lse = binding.rib_window_attn_fwd_bucketed(q, k, v, bias, named, 8)
    saved = kept((q, k, v, out))
    short = (saved[0][0], saved[0][1][:, :8])
    bwd, kb = binding.rib_window_attn_bwd_bucketed, binding.rib_window_attn_bwd_bucketed_checkpointed
    yield lambda: binding.rib_window_attn_fwd_bucketed(q, k.float(), v, bias, named, 8)
    yield lambda: binding.rib_window_attn_fwd_bucketed(q, k, v, bias.double(), named, 8)
    yield lambda: binding.rib_window_attn_fwd_bucketed(q, k, v, bias, named.long(), 8)
    yield lambda: binding.rib_window_attn_fwd_bucketed(q, k, v, bias, named[:3], 8)
    yield lambda: binding.rib_window_attn_fwd_bucketed(q, k, v, bias, named, 8, 8)
    yield lambda: binding.rib_window_attn_fwd_bucketed(q[:, :12], k[:, :12], v[:, :12], bias, named, 8, 4, masked=True)
    yield lambda: binding.rib_window_attn_fwd_bucketed(q, k, v, bias.cpu(), named, 8)
    yield lambda: bwd(q, k, v, bias, named, out, lse[:, :1], dout, 8)
    yield lambda: bwd(q, k, v, bias, named, out, lse, dout.transpose(1, 2), 8)
    yield lambda: bwd(q, k, v, bias, named, out, lse, dout, 8, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    yield lambda: kb(short, *saved[1:], bias, named, lse, dout, 8)
    yield lambda: kb(saved[0][0], *saved[1:], bias, named, lse, dout, 8)
    yield lambda: kb(*saved, bias, named, lse, dout, 8, 9)
    yield lambda: kb(*saved, bias, named, lse, dout, 8, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    yield lambda: binding.rib_window_attn_bwd_checkpointed(*saved, bias, bias, lse, dout, 8)


def test_same_refusals(monkeypatch):
    for i, call in enumerate(refusals()):
        a, b = both(monkeypatch, call)
        assert isinstance(a[0], type) and issubclass(a[0], Exception) and a == b, (i, a, b)


def layer(M, d, s, B=2, H=40, W=33, heads=2, masked=False, seed=5):
    """run(): the C calls into buffers that stay, from an output gradient that is copied in first; results."""
    q, k, v, given, bias, named = (t.cuda() for t in make(B, H, W, heads, d, M, log_map(M), torch.float32, seed=seed))
    lib, p, count, size = binding.library(), lambda t: t.data_ptr(), bias.shape[1], (B, H, W, heads, d, M)
    out, lse = torch.empty_like(q), torch.empty(B, heads, H, W, device="cuda")
    saved = kept((q, k, v, q))
    late, dout, results = torch.zeros_like(given), torch.zeros_like(given), [torch.empty_like(q) for _ in range(3)] + [torch.empty_like(bias)]
    need = lib.rib_window_attn_bwd_bucketed_checkpointed_workspace(count, count, *size)

    def run(workspace, checkpointed):
        dout.copy_(late)
        stream = torch.cuda.current_stream().cuda_stream
        rc = lib.rib_window_attn_fwd_bucketed(p(q), p(k), p(v), p(bias), 0, count, p(named), count, *size, s, int(masked), p(out), p(lse), stream)
        assert rc == 0
        grads = [p(t) for t in results]
        if checkpointed:
            for t, (codes, scales) in zip((q, k, v, out), saved):
                assert lib.rib_checkpoint_store(p(t), B * H * W * heads, d, p(codes), p(scales), stream) == 0
            array = (ctypes.c_void_p * 8)(*[p(t) for pair in saved for t in pair])
            rc = lib.rib_window_attn_bwd_bucketed_checkpointed(array, p(bias), 0, count, p(named), count, p(lse), p(dout), *size, s, int(masked), *grads, p(workspace), need, stream)
        else:
            rc = lib.rib_window_attn_bwd_bucketed(p(q), p(k), p(v), p(bias), 0, count, p(named), count, p(out), p(lse), p(dout), *size, s, int(masked), *grads, p(workspace), need, stream)
        assert rc == 0
    return run, need, late, given, results


@pytest.mark.parametrize("M,d,s", [(16, 32, 8), (16, 16, 0), (7, 20, 3), (20, 10, 4)])
@pytest.mark.parametrize("checkpointed", [False, True])
def test_late_inputs_and_old_values_on_a_side_stream(M, d, s, checkpointed):
    """The kernels behind the first of a backward pass start before it ends: they may read neither its old sums nor its old inputs."""
    run, need, late, given, results = layer(M, d, s)
    workspace = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    late.copy_(given)
    run(workspace, checkpointed)
    torch.cuda.synchronize()
    want = [t.clone() for t in results]
    side = torch.cuda.Stream()
    for _ in range(3):
        late.zero_()
        workspace.fill_(255)
        for t in results:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(LATE)
            late.copy_(given)
            run(workspace, checkpointed)
        torch.cuda.synchronize()
        agree(results, want, {1, 2})


@pytest.mark.parametrize("checkpointed", [False, True])
def test_two_graphs_share_a_workspace(checkpointed):
    """Two layers of different shapes, captured apart, replayed in turn on one stream with one workspace."""
    layers = [layer(16, 32, 8), layer(24, 16, 0, B=1, H=48, W=72, heads=3, seed=6), layer(7, 20, 3, seed=7)]
    workspace = torch.full((max(x[1] for x in layers),), 255, dtype=torch.uint8, device="cuda")
    wants, graphs = [], []
    for run, _, late, given, results in layers:
        late.copy_(given)
        run(workspace, checkpointed)
        torch.cuda.synchronize()
        wants.append([t.clone() for t in results])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(workspace, checkpointed)
        graphs.append(graph)
    for order in ((0, 1, 2), (2, 0, 1), (1, 1, 0)):
        for i in order:
            for t in layers[i][4]:
                t.fill_(float("nan"))
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in order:
            agree(layers[i][4], wants[i], {1, 2})


@pytest.mark.parametrize("M,d,s", [(16, 32, 8), (7, 20, 3)])
def test_more_than_2_31_elements(M, d, s):
    """One image many times over: every copy has the results of the first, those behind element 2^31 as well."""
    H, W, heads = 64, 48, 4
    one = H * W * heads * d
    B = (1 << 31) // one + 3
    q, k, v, dout, bias, named = (t.cuda() for t in make(1, H, W, heads, d, M, log_map(M), torch.float32, seed=8))
    want_out, want_lse = binding.rib_window_attn_fwd_bucketed(q, k, v, bias, named, M, s)
    want = binding.rib_window_attn_bwd_bucketed(q, k, v, bias, named, want_out, want_lse, dout, M, s)
    many = [t.expand(B, -1, -1, -1, -1).contiguous() for t in (q, k, v, dout)]
    out, lse = binding.rib_window_attn_fwd_bucketed(*many[:3], bias, named, M, s)
    assert out.numel() > 1 << 31 and all(torch.equal(out[b], want_out[0]) for b in (0, B // 2, B - 3, B - 2, B - 1)) and torch.equal(lse[B - 1], want_lse[0])
    dq, dk, dv, dbias = binding.rib_window_attn_bwd_bucketed(*many[:3], bias, named, out, lse, many[3], M, s)
    for b in (0, B // 2, B - 2, B - 1):
        agree((dq[b], dk[b], dv[b]), [t[0] for t in want[:3]], {1, 2})
    # B copies of a sum: fp32 sums of many equal terms, off by up to half a step per addition of a partial sum
    assert float((dbias / B - want[3]).norm()) <= 1e-3 * float(want[3].norm())
    del dq, dk, dv
    codes, scales = binding.rib_checkpoint_store(out)
    first = binding.rib_checkpoint_store(want_out)
    assert torch.equal(codes[B - 1], first[0][0]) and torch.equal(scales[B - 1], first[1][0])
    back = binding.rib_checkpoint_restore(codes, scales)
    assert torch.equal(back[B - 1], binding.rib_checkpoint_restore(*first)[0])


@pytest.mark.parametrize("M,d,s", [(16, 32, 8), (32, 32, 16), (7, 20, 3), (16, 32, 3), (20, 10, 4)])
@pytest.mark.parametrize("path", [binding.RIB_PATH_NONE, binding.RIB_PATH_GENERIC])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_no_numbers(M, d, s, path, value):
    """In q: that row of out and lse and no other.  In k, where half of the offsets are not attended to: the rows that attend to it and no others.  All
    paths have the same rows.  (A row of q against keys whose channels have both signs: infinities of both signs, so NaN.)

    The other rows of that window and head may come from the exact form of the softmax in place of the fast one.  P is rounded to bf16 in both, 2^-9 of
    every weight and of their sum each, and out once more, so the two differ by at most (2 + 2 + 2) 2^-9 max |v|, as the weights add up to 1."""
    B, H, W, heads = 1, 40, 33, 2
    q, k, v, _, bias, named = make(B, H, W, heads, d, M, log_map(M), torch.float32, seed=10)
    named = torch.where((torch.arange((2 * M - 1) ** 2).view(2 * M - 1, -1) * 7) % 5 < 2, -1, named).int()
    named[M - 1, M - 1] = 0
    old = binding.rib_set_path(path)
    try:
        clean, _ = binding.rib_window_attn_fwd_bucketed(*(t.cuda() for t in (q, k, v, bias, named)), M, s)
        y, x = 5, 9
        bad = q.clone()
        bad[0, y, x, 1, 2] = value
        out, lse = binding.rib_window_attn_fwd_bucketed(*(t.cuda() for t in (bad, k, v, bias, named)), M, s)
        hit = torch.zeros(B, H, W, heads, dtype=torch.bool)
        hit[0, y, x, 1] = True
        assert torch.equal(torch.isnan(out).all(-1).cpu(), hit) and torch.equal(torch.isnan(out).any(-1).cpu(), hit)
        assert torch.equal(torch.isnan(lse).cpu(), hit.permute(0, 3, 1, 2))
        others = [out, clean]
        bad = k.clone()
        bad[0, y, x, 1] = value                                    # (against q of both signs: infinities of both signs or NaN, per row one of them)
        out, _ = binding.rib_window_attn_fwd_bucketed(*(t.cuda() for t in (q, bad, v, bias, named)), M, s)
    finally:
        binding.rib_set_path(old)
    place = lambda at, size: ((at - s) % (-(-size // M) * M))  # noqa: E731  (in the shifted map)
    ky, kx = place(y, H), place(x, W)
    most = 6 * 2.0 ** -9 * float(v.float().abs().max())
    got, first, clean = out[0].float().cpu(), others[0][0].float().cpu(), others[1][0].float().cpu()
    for Y in range(H):
        for X in range(W):
            qy, qx = place(Y, H), place(X, W)
            near = qy // M == ky // M and qx // M == kx // M
            attends = near and named[ky - qy + M - 1, kx - qx + M - 1] >= 0
            bound = torch.tensor([0.0, most if near else 0.0])[:, None]
            if (Y, X) != (y, x):
                assert ((first[Y, X] - clean[Y, X]).abs() <= bound).all(), (Y, X)
            if not attends:
                assert ((got[Y, X] - clean[Y, X]).abs() <= bound).all(), (Y, X)
            elif value != value:
                assert torch.isnan(got[Y, X, 1]).all(), (Y, X)


# B, H, W, heads, d, M, s, masked: tcgen05 kernels (whole and cut patches, region mask, one short window), warp-level MMAs (every width of a load), any-shape
GUARDED = [(2, 32, 48, 2, 32, 16, 8, False), (1, 35, 41, 3, 16, 32, 8, False), (2, 32, 32, 2, 24, 16, 8, True), (1, 5, 9, 1, 8, 64, 0, False), (1, 72, 72, 2, 32, 64, 40, False),
           (2, 23, 31, 3, 20, 7, 3, False), (1, 24, 16, 2, 48, 8, 3, True), (1, 13, 17, 2, 33, 5, 2, False), (1, 20, 33, 2, 30, 12, 7, False), (1, 33, 18, 1, 64, 16, 5, False),
           (1, 21, 22, 2, 10, 18, 4, False), (3, 1, 1, 1, 1, 1, 0, False)]


@pytest.mark.parametrize("case", GUARDED, ids=lambda c: "x".join(map(str, c)))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_results_and_workspaces_stay_inside_their_buffers(case, dtype):
    B, H, W, heads, d, M, s, masked = case
    q, k, v, dout, bias, named = (t.cuda() for t in make(B, H, W, heads, d, M, log_map(M), dtype, seed=12))
    lib, p, count, size, kind = binding.library(), lambda t: t.data_ptr(), bias.shape[1], (B, H, W, heads, d, M), int(dtype == torch.bfloat16)
    g = Guarded()
    out, lse = g.tensor(q.shape, torch.bfloat16), g.tensor((B, heads, H, W), torch.float32)
    assert lib.rib_window_attn_fwd_bucketed(p(q), p(k), p(v), p(bias), kind, count, p(named), count, *size, s, int(masked), p(out), p(lse), None) == 0
    saved = [(g.tensor(q.shape, torch.int8, fill=99), g.tensor(q.shape[:4], torch.float32)) for _ in range(4)]
    for t, (codes, scales) in zip((q, k, v, out), saved):
        assert lib.rib_checkpoint_store(p(t), B * H * W * heads, d, p(codes), p(scales), None) == 0
    back = g.tensor(q.shape, torch.bfloat16)
    assert lib.rib_checkpoint_restore(p(saved[0][0]), p(saved[0][1]), B * H * W * heads, d, p(back), None) == 0
    torch.cuda.synchronize()
    g.check("forward and checkpoints")
    assert not any(torch.isnan(t.float()).any() for t in (out, lse, back, *(x[1] for x in saved)))
    array = (ctypes.c_void_p * 8)(*[p(t) for pair in saved for t in pair])
    for checkpointed in (False, True):
        g = Guarded()
        results = [g.tensor(q.shape, torch.bfloat16) for _ in range(3)] + [g.tensor(bias.shape, dtype)]
        need = getattr(lib, "rib_window_attn_bwd_bucketed" + ("_checkpointed" if checkpointed else "") + "_workspace")(count, count, *size)
        ws = g.tensor((need,), torch.uint8)
        tail = (*size, s, int(masked), *(p(t) for t in results), p(ws), need, None)
        if checkpointed:
            rc = lib.rib_window_attn_bwd_bucketed_checkpointed(array, p(bias), kind, count, p(named), count, p(lse), p(dout), *tail)
        else:
            rc = lib.rib_window_attn_bwd_bucketed(p(q), p(k), p(v), p(bias), kind, count, p(named), count, p(out), p(lse), p(dout), *tail)
        assert rc == 0
        torch.cuda.synchronize()
        assert binding.rib_query_status() == 0
        g.check("backward")
        assert not any(torch.isnan(t.float()).any() for t in results)
