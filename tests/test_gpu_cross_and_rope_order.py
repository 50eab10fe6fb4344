"""The kernels for attention to states and for norms with rotation may start while what is before them on the stream still runs, and wait for its end before they read or write: behind fills, copies from the
host and kernels, eagerly and captured, call behind call without a pause."""
import pytest
import torch

from paper_2603_06738_b200 import binding as rib

pytestmark = pytest.mark.gpu


def normal(seed, *shape):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def attention(q, k, v, dout, lengths):
    out, lse = rib.rib_cross_attn_fwd(q, k, v, lengths=lengths)
    return (out, lse, *rib.rib_cross_attn_bwd(q, k, v, out, lse, dout, lengths=lengths))


@pytest.mark.parametrize("B,H,W,heads,kv,d,L", [(2, 40, 50, 4, 2, 32, 77), (2, 40, 50, 4, 2, 64, 300), (3, 1, 1, 2, 2, 32, 900), (2, 20, 30, 3, 3, 20, 90), (2, 20, 30, 3, 3, 30, 400)])
@pytest.mark.parametrize("captured", [False, True])
def test_attention_behind_what_writes_its_inputs(B, H, W, heads, kv, d, L, captured):
    shapes = [(B, H, W, heads, d), (B, L, kv, d), (B, L, kv, d), (B, H, W, heads, d)]
    news = [[normal(10 * s + i, *shape).bfloat16() for i, shape in enumerate(shapes)] for s in range(3)]
    cuts = [torch.tensor([max(1, (s + 1) * L // 4), L], dtype=torch.int32).repeat(2)[:B].contiguous().pin_memory() for s in range(3)]
    wants = [[t.clone() for t in attention(*new, cut.cuda())] for new, cut in zip(news, cuts)]
    held = [torch.zeros_like(t) for t in news[0]]
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    hosts = [[t.cpu().pin_memory() for t in new] for new in news]

    def everything():
        results = []
        for s in range(3):
            for t, new, host in zip(held, news[s], hosts[s]):
                if s == 0:
                    t.copy_(new)                          # a copy on the device
                elif s == 1:
                    t.copy_(host, non_blocking=True)      # from the host
                else:
                    t.zero_()
                    t.add_(new)                           # kernels
            if s == 2:
                lengths.zero_()
                lengths.add_(cuts[2].cuda(non_blocking=True) if not captured else on_card)
            else:
                lengths.copy_(cuts[s], non_blocking=True)
            results.append(attention(*held, lengths))
        for t in held:
            t.fill_(float("nan"))                         # a kernel behind must not overtake the reads
        lengths.fill_(-1)
        return results

    on_card = cuts[2].cuda()
    got = everything()
    if captured:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = everything()
        for result in got:
            for t in result:
                t.fill_(float("nan"))
        for _ in range(3):
            g.replay()
    torch.cuda.synchronize()
    assert rib.rib_query_status() == 0
    for want, result in zip(wants, got):
        assert all(torch.equal(a, b) for a, b in zip(want, result))


@pytest.mark.parametrize("d,rot,interleaved", [(32, 32, False), (64, 32, True), (30, 30, False), (24, 16, True)])
@pytest.mark.parametrize("captured", [False, True])
def test_norms_behind_what_writes_their_inputs(d, rot, interleaved, captured):
    B, H, W, heads = 2, 37, 41, 3
    news = [[normal(10 * s + i, B, H, W, heads, d).bfloat16() for i in range(4)] + [normal(10 * s + 5 + i, d) for i in range(2)] for s in range(2)]
    turns = [rib.rib_rope_frequencies(rot) * (1 + s) for s in range(2)]

    def step(q, k, dq, dk, wq, wk, frequencies):
        table = rib.rib_rope_table(frequencies, H, W)
        return (*rib.rib_qk_norm_rope_fwd(q, k, wq, wk, table, interleaved=interleaved), *rib.rib_qk_norm_rope_bwd(q, k, wq, wk, table, dq, dk, interleaved=interleaved))

    wants = [[t.clone() for t in step(*new, f)] for new, f in zip(news, turns)]
    held, frequencies = [torch.zeros_like(t) for t in news[0]], torch.zeros_like(turns[0])

    def everything():
        results = []
        for new, f in zip(news, turns):
            frequencies.copy_(f)
            for t, n in zip(held, new):
                t.copy_(n)
            results.append(step(*held, frequencies))
        for t in held:
            t.fill_(float("nan"))
        return results

    got = everything()
    if captured:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = everything()
        for _ in range(3):
            g.replay()
    torch.cuda.synchronize()
    for want, result in zip(wants, got):
        assert all(torch.equal(a, b) for a, b in zip(want, result))
