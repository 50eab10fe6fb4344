"""Calls that are given a stream which is not the current one: the memory of their results and of what they allocate for themselves belongs to that stream, and
no tensor of a call is handed out again while the call still uses it.

The side stream is held up by a delay.  What the current stream frees and allocates meanwhile may not meet what the call works on."""
import pytest
import torch

from paper_2603_06738_b200 import binding as rib

from test_gpu_bucketed import log_map, make
from test_gpu_overtaking import LATE

pytestmark = pytest.mark.gpu

M, D, HEADS, SIDE = 16, 32, 2, 64


def tensors(x):
    if torch.is_tensor(x):
        return [x]
    return [t for y in x for t in tensors(y)] if isinstance(x, (tuple, list)) else []


def calls():
    """name -> (function, arguments, whether the sums' order may differ)."""
    q, k, v, dout, bias, named = (t.cuda() for t in make(2, SIDE, SIDE, HEADS, D, M, log_map(M), torch.float32, seed=33))
    g = torch.Generator(device="cuda").manual_seed(34)
    rand = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    pq, pk = rand(M * M, 16).bfloat16(), rand(M * M, 16).bfloat16()
    hq, hk = rand(HEADS, M * M, 16).bfloat16(), rand(HEADS, M * M, 16).bfloat16()
    out, lse = rib.rib_window_attn_fwd(q, k, v, pq, pk, M, 8)
    hout, hlse = rib.rib_window_attn_fwd_headwise(q, k, v, hq, hk, M, 8)
    mout, mlse = rib.rib_window_attn_fwd_masked(q, k, v, pq, pk, M, 8)
    bout, blse = rib.rib_window_attn_fwd_bucketed(q, k, v, bias, named, M, 8)
    kept = [rib.rib_checkpoint_store(t) for t in (q, k, v, out)]
    bkept = kept[:3] + [rib.rib_checkpoint_store(bout)]
    x, gate = rand(2, SIDE, SIDE, HEADS * D).bfloat16(), rand(2, SIDE, SIDE, HEADS * D).sigmoid().bfloat16()
    conv = [rand(*s) * 0.1 for s in ((HEADS * D, 3, 3), (HEADS * D,), (HEADS * D, HEADS * D), (HEADS * D,))]
    gen = [rand(*s) * 0.2 for s in ((42, 32), (32,), (32, 16), (32, 16))]
    two = lambda t: [t, t]  # noqa: E731
    return {
        "fwd": (rib.rib_window_attn_fwd, (q, k, v, pq, pk, M, 8)),
        "bwd": (rib.rib_window_attn_bwd, (q, k, v, pq, pk, out, lse, dout, M, 8)),
        "fwd_headwise": (rib.rib_window_attn_fwd_headwise, (q, k, v, hq, hk, M, 8)),
        "bwd_headwise": (rib.rib_window_attn_bwd_headwise, (q, k, v, hq, hk, hout, hlse, dout, M, 8)),
        "fwd_padded": (rib.rib_window_attn_fwd_padded, (q, k, v, pq, pk, M, 8)),
        "bwd_padded": (rib.rib_window_attn_bwd_padded, (q, k, v, pq, pk, out, lse, dout, M, 8)),
        "fwd_masked": (rib.rib_window_attn_fwd_masked, (q, k, v, pq, pk, M, 8)),
        "bwd_masked": (rib.rib_window_attn_bwd_masked, (q, k, v, pq, pk, mout, mlse, dout, M, 8)),
        "fwd_gated": (rib.rib_window_attn_fwd_gated, (q, k, v, pq, pk, gate, M, 8)),
        "cycle_fwd": (rib.rib_window_cycle_fwd, (two(q), two(k), two(v), two(pq), two(pk), [M, M], [0, 8])),
        "cycle_bwd": (rib.rib_window_cycle_bwd, (two(q), two(k), two(v), two(pq), two(pk), two(out), two(lse), two(dout), [M, M], [8, 8])),
        "fwd_bucketed": (rib.rib_window_attn_fwd_bucketed, (q, k, v, bias, named, M, 8)),
        "bwd_bucketed": (rib.rib_window_attn_bwd_bucketed, (q, k, v, bias, named, bout, blse, dout, M, 8)),
        "store": (rib.rib_checkpoint_store, (q,)),
        "restore": (rib.rib_checkpoint_restore, kept[0]),
        "bwd_checkpointed": (rib.rib_window_attn_bwd_checkpointed, (*kept, pq, pk, lse, dout, M, 8)),
        "bwd_bucketed_checkpointed": (rib.rib_window_attn_bwd_bucketed_checkpointed, (*bkept, bias, named, blse, dout, M, 8)),
        "cla_gate": (rib.rib_cla_gate, (x, *conv)),
        "cla_product": (rib.rib_cla_product, (out, gate)),
        "cla_product_bwd": (rib.rib_cla_product_bwd, (out, gate, dout)),
        "cla_gate_bwd": (rib.rib_cla_gate_bwd, (x, *conv, gate)),
        "generate": (rib.rib_generate_features, (*gen, M)),
        "generate_bwd": (rib.rib_generate_features_bwd, (*gen, pq.float(), pk.float(), M)),
    }


NAMES = ["fwd", "bwd", "fwd_headwise", "bwd_headwise", "fwd_padded", "bwd_padded", "fwd_masked", "bwd_masked", "fwd_gated", "cycle_fwd", "cycle_bwd", "fwd_bucketed", "bwd_bucketed",
         "store", "restore", "bwd_checkpointed", "bwd_bucketed_checkpointed", "cla_gate", "cla_product", "cla_product_bwd", "cla_gate_bwd", "generate", "generate_bwd"]


def copied(x):
    return x.clone() if torch.is_tensor(x) else type(x)(copied(y) for y in x) if isinstance(x, (tuple, list)) else x


def agree(got, want):
    """Equal but for the order of fp32 sums: a few steps of 2^-24 of partial sums, and where bf16 is behind them one step of a few values."""
    for x, y in zip(tensors(got), tensors(want), strict=True):
        assert x.shape == y.shape and x.dtype == y.dtype
        assert float((x.float() - y.float()).norm()) <= (1e-5 if x.dtype == torch.float32 else 1e-3) * float(y.float().norm())


@pytest.fixture(scope="module")
def table():
    return calls()


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("name", NAMES)
def test_nothing_of_a_call_is_handed_out_again_too_early(monkeypatch, table, name, native):
    """The arguments are dropped when the call has returned, and the current stream takes, and fills, as much memory of their sizes and of a workspace's as it can get
    while the side stream has not begun."""
    if not native:
        monkeypatch.setattr(rib, "_marshal", None)
    call, args = table[name]
    want = copied(call(*args))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    given = copied(args)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LATE)
    got = call(*given, stream=side)
    del given
    sizes = {t.numel() * t.element_size() for t in tensors(args) + tensors(want)} | {1 << n for n in range(9, 26)}
    taken = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for size in sizes for _ in range(4)]
    torch.cuda.synchronize()
    assert taken
    agree(got, want)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("name", NAMES)
def test_results_do_not_land_in_what_the_current_stream_still_reads(monkeypatch, table, name, native):
    """The current stream is the late one: it has yet to read memory that the program has given back to it."""
    if not native:
        monkeypatch.setattr(rib, "_marshal", None)
    call, args = table[name]
    want = copied(call(*args))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    sizes = sorted({t.numel() * t.element_size() for t in tensors(want)} | {1 << n for n in range(9, 26)})
    held = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for size in sizes for _ in range(4)]
    seen = [torch.zeros(t.numel(), dtype=torch.uint8, device="cuda") for t in held]
    torch.cuda.synchronize()
    torch.cuda._sleep(LATE)
    for to, t in zip(seen, held):
        to.copy_(t)
    del held, to, t
    got = call(*args, stream=side)
    torch.cuda.synchronize()
    assert all(bool((t == 7).all()) for t in seen)
    agree(got, want)
    # and what the current stream reads of the results, ordered behind the call, is theirs when they are dropped
    got = call(*args, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(LATE)
    read = copied(got)
    del got
    with torch.cuda.stream(side):
        taken = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for size in sizes for _ in range(4)]
    torch.cuda.synchronize()
    assert taken
    agree(read, want)


@pytest.mark.parametrize("name", ["bwd", "bwd_bucketed", "store", "generate"])
def test_a_stream_of_another_library(table, name):
    """Anything with a `cuda_stream` will do."""
    call, args = table[name]
    want = copied(call(*args))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = type("Other", (), {"cuda_stream": side.cuda_stream})()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LATE)
    got = call(*args, stream=other)
    assert not side.query()
    torch.cuda.synchronize()
    agree(got, want)


@pytest.mark.parametrize("name", ["bwd", "fwd_bucketed", "bwd_bucketed", "bwd_bucketed_checkpointed"])
def test_captured_on_a_branch(table, name):
    """A call on a second stream of a capture: the branch's memory is the graph's, and every replay has the results of the call."""
    call, args = table[name]
    want = copied(call(*args))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = call(*args, stream=side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(2):
        for t in tensors(got):
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        agree(got, want)


def test_a_stream_of_another_device_is_refused(table):
    """Before anything is launched."""
    call, args = table["store"]
    other = type("Other", (torch.cuda.Stream,), {"device": property(lambda self: torch.device("cuda:1")), "cuda_stream": 1 << 20})
    launches = rib.rib_kernel_launches()
    with pytest.raises(ValueError, match="cuda:1"):
        rib._beside(other(), call, *args)
    assert rib.rib_kernel_launches() == launches
