"""Norms of queries and keys with the rotation by position, and attention to a sequence of states: what the library is timed on there, and the
same operators in plain torch.

Kinds of case:
  attend      every token of a map attends to the states of an encoder, a text or a dictionary (L of them), forward only.
  train       the same in training: forward, and backward to q, k and v.
  positions   q and k of an attention layer, as they come out of one projection: each head normalised, then rotated by the token's place in the map.
  tune        the same in training: forward, and backward to q, k and the weights of the norms.

The states are k, v [B, L, kv_heads, d], or [1, L, kv_heads, d] (`shared`) when all maps of the batch attend to the same ones, such as a learned
dictionary; `heads / kv_heads` query heads share a head of keys and values.  With `ragged` every batch item has a length of its own, and what lies behind it
is padding that is not attended to.
A rotation turns the pairs of the first `rot` channels of a head, channels (2 i, 2 i + 1) (`interleaved`) or (i, i + rot / 2), by
y f_y[i] + x f_x[i]; `kept` says that the cosines and sines of the map's rows and columns are a table that the program made before, else they are
computed from the frequencies within the call (learned frequencies, or a new size of map).  `far` is the place of the map's first row and column
(a tile of a large image).
"""
import math

import torch

own = False


def listed():
    return [
        # the smallest call: one token and a text of 77 states
        dict(name="attend_1x1_L77", kind="attend", B=1, H=1, W=1, heads=2, kv_heads=2, d=32, L=77, shared=False, ragged=False),
        # serving: one token for each of 64 requests over long contexts of their own lengths
        dict(name="attend_1x1_b64_L4096", kind="attend", B=64, H=1, W=1, heads=6, kv_heads=6, d=32, L=4096, shared=False, ragged=True),
        # a 1280 x 720 output at x4 conditioned on a text
        dict(name="attend_180x320_L77", kind="attend", B=1, H=180, W=320, heads=6, kv_heads=6, d=32, L=77, shared=False, ragged=False),
        # the largest inference: one square map, the states of a second map of 32 x 32
        dict(name="attend_256x256_L1024", kind="attend", B=1, H=256, W=256, heads=6, kv_heads=6, d=32, L=1024, shared=False, ragged=False),
        # the training configuration of the benchmark with states of ragged lengths
        dict(name="train_96x96_L256_ragged", kind="train", B=16, H=96, W=96, heads=6, kv_heads=6, d=32, L=256, shared=False, ragged=True),
        # one learned dictionary for all maps of a batch
        dict(name="train_64x64_dictionary", kind="train", B=10, H=64, W=64, heads=6, kv_heads=6, d=32, L=128, shared=True, ragged=False),
        # wide heads, four query heads to a head of keys, long contexts
        dict(name="train_48x48_d64_grouped_L2048", kind="train", B=4, H=48, W=48, heads=8, kv_heads=2, d=64, L=2048, shared=False, ragged=True),
        # nothing even: an odd map, heads of 20 channels, 45 states
        dict(name="train_50x39_d20_L45", kind="train", B=2, H=50, W=39, heads=3, kv_heads=3, d=20, L=45, shared=False, ragged=True),
        # inference on one square map, the table of the map kept
        dict(name="positions_256x256", kind="positions", B=1, H=256, W=256, heads=6, kv_heads=6, d=32, rot=32, interleaved=False, per_head=False, kept=True, far=0),
        # a small odd tile far inside a large image, two thirds of the head rotated, the table made within the call
        dict(name="positions_37x53_d24", kind="positions", B=1, H=37, W=53, heads=3, kv_heads=3, d=24, rot=16, interleaved=True, per_head=False, kept=False, far=30000),
        # the training configuration of the benchmark, frequencies that change from step to step
        dict(name="tune_96x96_d32", kind="tune", B=16, H=96, W=96, heads=6, kv_heads=6, d=32, rot=32, interleaved=True, per_head=False, kept=False, far=0),
        # wide grouped heads, half of the head rotated, a weight for every head
        dict(name="tune_64x64_d64_grouped", kind="tune", B=4, H=64, W=64, heads=8, kv_heads=2, d=64, rot=32, interleaved=False, per_head=True, kept=True, far=0),
    ]


def _spread(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def _side(rng, lo, hi):
    return _spread(rng, lo, hi)


def draw(rng):
    while True:
        kind = rng.choices(["attend", "train", "positions", "tune"], weights=[4, 4, 2, 2])[0]
        heads = rng.choice([1, 2, 3, 4, 6, 6, 8, 12])
        kv_heads = rng.choice([heads] * 3 + [g for g in range(1, heads + 1) if heads % g == 0])
        d = rng.choice([8, 16, 20, 24, 30, 32, 32, 32, 40, 48, 64, 64])
        B = _spread(rng, 1, 16)
        if kind in ("positions", "tune"):
            rot = rng.choice([d, d // 2, d // 4]) // 2 * 2
            case = dict(kind=kind, B=B, H=_side(rng, 1, 256), W=_side(rng, 1, 256), heads=heads, kv_heads=kv_heads, d=d, rot=max(2, rot),
                        interleaved=rng.random() < 0.5, per_head=rng.random() < 0.3, kept=rng.random() < 0.5, far=rng.choice([0, 0, _spread(rng, 1, 50000)]))
            if work(case)["bytes"] <= _most("tune_96x96_d32", "bytes"):
                return case
            continue
        if kind == "attend" and rng.random() < 0.25:        # single tokens
            H = W = 1
            B, L = _spread(rng, 1, 64), _spread(rng, 1, 8192)
        else:
            H, W, L = _side(rng, 1, 256), _side(rng, 1, 256), _spread(rng, 1, 4096)
        case = dict(kind=kind, B=B, H=H, W=W, heads=heads, kv_heads=kv_heads, d=d, L=L, shared=rng.random() < 0.2, ragged=rng.random() < 0.4)
        if work(case)["flops"] <= _most("train_48x48_d64_grouped_L2048", "flops") and B * H * W * heads * L <= 6e8:
            return case


def _most(name, what):
    return work(next(c for c in listed() if c["name"] == name))[what]


# ------------------------------------------------------------------------------------------------------------- inputs
def _lengths(c):
    """Lengths of the contexts in no particular order: spread evenly up to L."""
    n = 1 if c["shared"] else c["B"]
    return [max(1, round(c["L"] * (i + 1) / n)) for i in range(n)] if c["ragged"] else [c["L"]] * n


def _frequencies(c, g):
    """[2, rot / 2] angles per row and per column: the first half of the pairs turns with the rows, the second with the columns, and where they
    are learned (not `kept`) every pair a little with the other axis too."""
    pairs = c["rot"] // 2
    i = torch.arange(pairs, device="cuda")
    rows = (pairs + 1) // 2
    along = torch.where(i < rows, i / rows, (i - rows) / max(1, pairs - rows))
    f = 100.0 ** -along.double()
    f = torch.stack([torch.where(i < rows, f, 0.0), torch.where(i < rows, 0.0, f)])
    if not c["kept"]:
        f = f + 0.02 * torch.randn(2, pairs, device="cuda", generator=g, dtype=torch.float64)
    return f.float().contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 6271 + 29)
    B, H, W, heads, kv, d = (case[k] for k in ("B", "H", "W", "heads", "kv_heads", "d"))
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    state = dict(case)
    if case["kind"] in ("attend", "train"):
        L, contexts = case["L"], 1 if case["shared"] else B
        state.update(q=normal(B, H, W, heads, d).bfloat16(), k=normal(contexts, L, kv, d).bfloat16(), v=normal(contexts, L, kv, d).bfloat16(), lengths=None)
        if case["ragged"]:
            order = torch.randperm(contexts, device="cuda", generator=g)
            state["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")[order].contiguous()
        if case["kind"] == "train":
            state["dout"] = normal(B, H, W, heads, d).bfloat16()
        return state
    # q, k (and v, which nothing here touches) beside each other in the output of one projection, some channels larger than others
    x = normal(B, H, W, heads + 2 * kv, d) * (0.5 + torch.rand(heads + 2 * kv, d, device="cuda", generator=g) * 2)
    state["qkv"] = x.bfloat16()
    shapes = ((heads, d), (kv, d)) if case["per_head"] else ((d,), (d,))
    state["q_weight"], state["k_weight"] = (1 + 0.2 * normal(*s) for s in shapes)
    state["frequencies"] = _frequencies(case, g)
    if case["kept"]:
        state["table"] = _table(state)
    if case["kind"] == "tune":
        state["dq"], state["dk"] = normal(B, H, W, heads, d).bfloat16(), normal(B, H, W, kv, d).bfloat16()
    return state


# -------------------------------------------------------------------------------------------------- plain operators
def _table(c):
    """[H + W, rot / 2, 2] cosines and sines of the map's rows, then of its columns; far angles in 64 bits."""
    f = c["frequencies"].double()
    y = torch.arange(c["far"], c["far"] + c["H"], device="cuda", dtype=torch.float64)
    x = torch.arange(c["far"], c["far"] + c["W"], device="cuda", dtype=torch.float64)
    angle = torch.cat([y[:, None] * f[0], x[:, None] * f[1]])
    return torch.stack([angle.cos(), angle.sin()], -1).float()


def _turns(c, table):
    """Cosine and sine of every token and pair, [H, W, 1, rot / 2]."""
    row, column = table[: c["H"], None, None], table[None, c["H"]:, None]
    return row[..., 0] * column[..., 0] - row[..., 1] * column[..., 1], row[..., 1] * column[..., 0] + row[..., 0] * column[..., 1]


def _rotate(z, c, cos, sin):
    rot = c["rot"]
    a, b = (z[..., 0:rot:2], z[..., 1:rot:2]) if c["interleaved"] else (z[..., : rot // 2], z[..., rot // 2: rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, z[..., rot:]], -1)


_EPS = 1e-6


def _split(c):
    q, k, _ = c["qkv"].split([c["heads"], c["kv_heads"], c["kv_heads"]], dim=3)
    return q, k


def _normed(x, weight):
    x = x.float()
    inverse = torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS)
    return x * inverse, inverse, weight


def _norm_gradients(x, weight, g, c, cos, sin):
    unit, inverse, _ = _normed(x, weight)
    g = _rotate(g.float(), c, cos, -sin)                 # the rotation back
    dweight = g * unit
    dweight = dweight.sum((0, 1, 2)) if c["per_head"] else dweight.sum((0, 1, 2, 3))
    g = g * weight
    return (inverse * (g - unit * (g * unit).mean(-1, keepdim=True))).bfloat16(), dweight


def _heads_first(x, c):
    """k or v as [contexts, kv_heads, 1, L, d]."""
    return x.float().permute(0, 2, 1, 3)[:, :, None]


def _queries(x, c):
    """[B, kv_heads, heads / kv_heads, tokens, d]."""
    return x.float().flatten(1, 2).permute(0, 2, 1, 3).unflatten(1, (c["kv_heads"], c["heads"] // c["kv_heads"]))


def _map(x, c):
    """The reverse."""
    return x.flatten(1, 2).permute(0, 2, 1, 3).reshape(c["B"], c["H"], c["W"], c["heads"], c["d"])


def _probabilities(c, q, k):
    s = q @ k.transpose(-1, -2) * (1 / math.sqrt(c["d"]))
    if c["lengths"] is not None:
        s.masked_fill_((torch.arange(c["L"], device="cuda") >= c["lengths"][:, None])[:, None, None, None], -math.inf)
    s = s.sub_(s.amax(-1, keepdim=True)).exp_()
    return s.div_(s.sum(-1, keepdim=True))


def run(c):
    if own:
        from paper_2603_06738_b200 import binding as rib
        if c["kind"] == "attend":
            return rib.rib_cross_attn_fwd(c["q"], c["k"], c["v"], lengths=c["lengths"], want_lse=False)[0]
        if c["kind"] == "train":
            out, lse = rib.rib_cross_attn_fwd(c["q"], c["k"], c["v"], lengths=c["lengths"])
            return (out, *rib.rib_cross_attn_bwd(c["q"], c["k"], c["v"], out, lse, c["dout"], lengths=c["lengths"]))
        table = c["table"] if c["kept"] else rib.rib_rope_table(c["frequencies"], c["H"], c["W"], y0=c["far"], x0=c["far"])
        layer = (*_split(c), c["q_weight"], c["k_weight"], table)
        q, k = rib.rib_qk_norm_rope_fwd(*layer, interleaved=c["interleaved"], eps=_EPS)
        if c["kind"] == "positions":
            return q, k
        return (q, k, *rib.rib_qk_norm_rope_bwd(*layer, c["dq"], c["dk"], interleaved=c["interleaved"], eps=_EPS))
    if c["kind"] in ("attend", "train"):
        q, k, v = _queries(c["q"], c), _heads_first(c["k"], c), _heads_first(c["v"], c)
        p = _probabilities(c, q, k)
        if c["lengths"] is not None:                        # what lies behind the last state is no number that counts
            v = v.masked_fill((torch.arange(c["L"], device="cuda") >= c["lengths"][:, None])[:, None, None, :, None], 0.0)
        out = p @ v
        if c["kind"] == "attend":
            return _map(out, c).bfloat16()
        g = _queries(c["dout"], c)
        over = (0, 2) if c["shared"] else (2,)
        dv = (p.transpose(-1, -2) @ g).sum(over, keepdim=True)
        ds = (g @ v.transpose(-1, -2)).sub_((out * g).sum(-1, keepdim=True)).mul_(p).mul_(1 / math.sqrt(c["d"]))
        dk = (ds.transpose(-1, -2) @ q).sum(over, keepdim=True)
        states = lambda t: t[:, :, 0].permute(0, 2, 1, 3).bfloat16().contiguous()  # noqa: E731
        return _map(out, c).bfloat16(), _map(ds @ k, c).bfloat16(), states(dk), states(dv)
    cos, sin = _turns(c, c["table"] if c["kept"] else _table(c))
    results = []
    for x, weight in zip(_split(c), (c["q_weight"], c["k_weight"])):
        unit, _, _ = _normed(x, weight)
        results.append(_rotate(unit * weight, c, cos, sin).bfloat16())
    if c["kind"] == "positions":
        return tuple(results)
    q, k = _split(c)
    dq, dq_weight = _norm_gradients(q, c["q_weight"], c["dq"], c, cos, sin)
    dk, dk_weight = _norm_gradients(k, c["k_weight"], c["dk"], c, cos, sin)
    return (*results, dq, dk, dq_weight, dk_weight)


# --------------------------------------------------------------------------------------------------------- the measure
def work(c):
    tokens = float(c["B"] * c["H"] * c["W"])
    d, heads, kv = c["d"], c["heads"], c["kv_heads"]
    if c["kind"] in ("attend", "train"):
        lengths = _lengths(c)
        queries = 2.0 * tokens * heads * d                  # bytes of q
        states = 2.0 * sum(lengths) * kv * d                # bytes of the keys that are attended to
        pairs = tokens * heads * (lengths[0] if c["shared"] else sum(lengths) / len(lengths))
        if c["kind"] == "attend":
            return {"bytes": 2 * queries + 2 * states, "flops": 4 * pairs * d}
        return {"bytes": 4 * queries + 4 * states, "flops": 14 * pairs * d}       # in: q, dout, k, v; out: out and four gradients' worth
    rows = tokens * (heads + kv) * d
    if c["kind"] == "positions":
        return {"bytes": 4 * rows, "flops": 8 * rows}
    return {"bytes": 8 * rows, "flops": 28 * rows}          # in: q, k and their gradients; out: q, k and two gradients


# ------------------------------------------------------------------------------------------------------------- 64 bits
def _exact_attention(c):
    B, H, W, heads, d = c["q"].shape
    contexts, L, kv, _ = c["k"].shape
    group, n, train = heads // kv, H * W, c["kind"] == "train"
    f = lambda t: t.double()  # noqa: E731
    out = torch.zeros(B, n, heads, d, dtype=torch.float64, device="cuda")
    dq = torch.zeros_like(out)
    dk, dv = (torch.zeros(contexts, L, kv, d, dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(B):
        at = b if contexts > 1 else 0
        here = L if c["lengths"] is None else int(c["lengths"][at])
        for h in range(heads):
            keys, values = f(c["k"][at, :here, h // group]), f(c["v"][at, :here, h // group])
            for lo in range(0, n, 16384):
                rows = slice(lo, min(n, lo + 16384))
                query = f(c["q"][b].reshape(n, heads, d)[rows, h])
                p = torch.softmax(torch.einsum("id,jd->ij", query, keys) / math.sqrt(d), 1)
                o = torch.einsum("ij,jd->id", p, values)
                out[b, rows, h] = o
                if not train:
                    continue
                go = f(c["dout"][b].reshape(n, heads, d)[rows, h])
                z = torch.einsum("id,jd->ij", go, values)
                z = p * (z - (p * z).sum(1, keepdim=True)) / math.sqrt(d)
                dq[b, rows, h] = torch.einsum("ij,jd->id", z, keys)
                dk[at, :here, h // group] += torch.einsum("ij,id->jd", z, query)
                dv[at, :here, h // group] += torch.einsum("ij,id->jd", p, go)
    shape = (B, H, W, heads, d)
    return (out.view(shape), dq.view(shape), dk, dv) if train else out.view(shape)


def _exact_positions(c):
    heads, kv, d, rot = c["heads"], c["kv_heads"], c["d"], c["rot"]
    y = torch.arange(c["H"], device="cuda").double() + c["far"]
    x = torch.arange(c["W"], device="cuda").double() + c["far"]
    f = c["frequencies"].double()
    # a rotation as a matrix for every token: [H, W, d, d]
    angle = y[:, None, None] * f[0] + x[None, :, None] * f[1]
    i = torch.arange(rot // 2, device="cuda")
    first, second = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + rot // 2)
    turn = torch.eye(d, dtype=torch.float64, device="cuda").repeat(c["H"], c["W"], 1, 1)
    turn[:, :, first, first] = angle.cos()
    turn[:, :, second, second] = angle.cos()
    turn[:, :, first, second] = -angle.sin()
    turn[:, :, second, first] = angle.sin()
    results, gradients, weights = [], [], []
    for name, lo, count in (("q", 0, heads), ("k", heads, kv)):
        part = c["qkv"][:, :, :, lo: lo + count].double()
        weight = c[name + "_weight"].double().expand(count, d)
        total = weight.new_zeros(count, d)
        values, slopes = torch.empty_like(part), torch.empty_like(part)
        for b in range(c["B"]):                             # (an item at a time: memory)
            p = part[b]
            size = (p.pow(2).sum(-1, keepdim=True) / d + _EPS).sqrt()
            unit = p / size
            values[b] = torch.einsum("yxij,yxhj->yxhi", turn, unit * weight)
            if c["kind"] == "tune":
                g = torch.einsum("yxij,yxhi->yxhj", turn, c["d" + name][b].double())
                total += (g * unit).sum((0, 1))
                g = g * weight
                slopes[b] = (g - unit * (g * unit).sum(-1, keepdim=True) / d) / size
        results.append(values)
        gradients.append(slopes)
        weights.append(total if c["per_head"] else total.sum(0))
    return tuple(results) if c["kind"] == "positions" else (*results, *gradients, *weights)


def exact(case, seed):
    c = prepare(case, seed)
    return _exact_attention(c) if case["kind"] in ("attend", "train") else _exact_positions(c)
