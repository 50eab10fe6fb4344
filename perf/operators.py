"""Window attention with a learned bias for relative positions, and 8-bit checkpoints of an attention layer's activations:
what the library is timed on there, and the same operators in plain torch.

Kinds of case:
  infer       one attention layer with a bias table, forward only, one map or frame.
  train       the same layer on a batch of training patches: forward, and backward to q, k, v and the table.
  store       q, k, v and the output of a layer put into 8 bits for its backward pass and fetched back.
  resume      the backward pass of a layer from such checkpoints: with the rank-r tables (`r` > 0) or with a bias table (`r` = 0).

A bias is looked up by bucket: an integer map over the (2 M - 1)^2 offsets (key minus query, rows then columns) of a window of side M
names the bucket of every offset; -1 is an offset whose keys are not attended to.  `steps` is the number of distances per axis that have a
bucket of their own before distances share one (0: every offset has its own bucket), `reach` the largest distance that is
attended to (0: all).
"""
import math

import torch

own = False


def listed():
    return [
        # the smallest call: one small map, two heads, launch and host latency are what counts
        dict(name="infer_64x64_h2_w16", kind="infer", B=1, H=64, W=64, heads=2, d=32, window=16, shift=0, masked=False, steps=0, reach=0),
        # inference on one square map, large windows
        dict(name="infer_256x256_w64_s32", kind="infer", B=1, H=256, W=256, heads=6, d=32, window=64, shift=32, masked=False, steps=8, reach=0),
        # a 1280 x 720 output at x4: rows that neither the window nor a patch of 8 divides; keys further than 20 away are left out
        dict(name="infer_180x320_w32_reach20", kind="infer", B=1, H=180, W=320, heads=6, d=32, window=32, shift=0, masked=False, steps=4, reach=20),
        # the smallest training step
        dict(name="train_64x64_h2_w16", kind="train", B=1, H=64, W=64, heads=2, d=32, window=16, shift=8, masked=False, steps=4, reach=0),
        # the training configuration of the benchmark: 16 patches of 96 x 96 in windows of 32, shifted by half a window
        dict(name="train_96x96_w32_s16", kind="train", B=16, H=96, W=96, heads=6, d=32, window=32, shift=16, masked=False, steps=0, reach=0),
        # 64 x 64 patches that are one window each: the longest rows
        dict(name="train_64x64_w64", kind="train", B=10, H=64, W=64, heads=6, d=32, window=64, shift=0, masked=False, steps=8, reach=0),
        # narrow heads in small shifted windows whose wrapped parts do not attend to each other
        dict(name="train_d16_w16_masked", kind="train", B=4, H=96, W=96, heads=12, d=16, window=16, shift=8, masked=True, steps=0, reach=0),
        # nothing even: an odd map, an odd window, heads of 20 channels
        dict(name="train_50x39_d20_w7", kind="train", B=2, H=50, W=39, heads=3, d=20, window=7, shift=3, masked=False, steps=2, reach=0),
        # checkpoints of one odd map
        dict(name="store_37x53_d24", kind="store", B=1, H=37, W=53, heads=3, d=24),
        # checkpoints of a layer of the benchmark's training configuration
        dict(name="store_96x96_d32", kind="store", B=16, H=96, W=96, heads=6, d=32),
        # the backward pass of that layer from its checkpoints, rank-16 tables
        dict(name="resume_96x96_w32_s16_r16", kind="resume", B=16, H=96, W=96, heads=6, d=32, window=32, shift=16, masked=False, r=16, steps=0, reach=0),
        # the same for a layer with a bias table, small windows of a small batch
        dict(name="resume_96x96_w16_bias", kind="resume", B=4, H=96, W=96, heads=6, d=32, window=16, shift=8, masked=False, r=0, steps=4, reach=0),
    ]


_MOST = 2.4e11            # flops of a drawn case: the largest listed one has about that


def _spread(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    while True:
        kind = rng.choices(["infer", "train", "store", "resume"], weights=[3, 4, 2, 2])[0]
        if kind == "store":
            return dict(kind=kind, B=_spread(rng, 1, 16), H=_spread(rng, 7, 128), W=_spread(rng, 7, 128), heads=rng.randint(1, 12), d=rng.choice([8, 16, 20, 24, 30, 32, 32, 48, 64]))
        odd = kind != "resume" and rng.random() < 0.15      # an odd window or head, which run small
        d = rng.choice([18, 20, 30, 40]) if odd else rng.choice([8, 16, 24, 32, 32, 32])
        M = rng.choice([5, 7, 10, 12]) if odd else rng.choice([8, 16, 16, 24, 32, 32, 48, 64])
        B = 1 if kind == "infer" else _spread(rng, 1, 16)
        masked = not odd and rng.random() < 0.25
        if masked or rng.random() < 0.4:                    # whole windows
            H, W = M * _spread(rng, 1, max(1, 256 // M)), M * _spread(rng, 1, max(1, 256 // M))
        else:
            H, W = _spread(rng, M, 64 if odd else 320), _spread(rng, M, 64 if odd else 320)
        if kind == "resume":                                # checkpoints are of training patches, in whole windows
            H, W = M * max(1, H // M), M * max(1, W // M)
        if odd:
            B, heads = min(B, 2), rng.randint(1, 3)
        else:
            heads = rng.choice([2, 3, 4, 6, 6, 12])
        r = rng.choice([0, 16]) if kind == "resume" and M % 16 == 0 else 0
        shift = rng.choice([0, rng.randrange(M)]) if odd else rng.choice([0, 8 * rng.randrange(M // 8)])
        case = dict(kind=kind, B=B, H=H, W=W, heads=heads, d=d, window=M, shift=shift, masked=masked and shift > 0, steps=rng.choice([0, 2, 4, 8]),
                    reach=rng.choice([0, 0, 0, max(3, M // 2)]))
        if kind == "resume":
            case["r"] = r
            if r:
                case.update(masked=False, steps=0, reach=0)
        padded = -(-H // M) * M * -(-W // M) * M
        if work(case)["flops"] <= _MOST and 4.0 * B * padded * M * M * heads <= 7e9:
            return case


# ------------------------------------------------------------------------------------------------------------- inputs
def _axis_buckets(M, steps, device):
    """Bucket of every distance 1 - M .. M - 1 along an axis, and their number: up to `steps` a bucket each, beyond that one per doubling."""
    d = torch.arange(1 - M, M, device=device)
    far = d.abs()
    if steps and steps < M:
        log = steps + torch.floor(torch.log2(far.clamp(min=1).double() / steps) * 2).long().clamp(min=0)
        far = torch.where(far < steps, far, log)
    _, at = torch.unique(torch.sign(d) * far, return_inverse=True)
    return at, int(at.max()) + 1


def _bucket_map(M, steps, reach, device):
    at, count = _axis_buckets(M, steps, device)
    grid = at[:, None] * count + at[None, :]
    if reach:
        d = torch.arange(1 - M, M, device=device).abs()
        grid = torch.where(torch.maximum(d[:, None], d[None, :]) > reach, -1, grid)
    return grid.to(torch.int32).contiguous(), count * count


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)
    B, H, W, heads, d = (case[k] for k in ("B", "H", "W", "heads", "d"))
    normal = lambda *shape, sd=1.0: torch.randn(*shape, device="cuda", generator=g) * sd  # noqa: E731
    image = lambda: normal(B, H, W, heads, d).bfloat16()  # noqa: E731
    state = dict(case, q=image(), k=image(), v=image())
    if case["kind"] == "store":
        state["out"] = image()
        return state
    M = case["window"]
    if case["kind"] != "infer":
        state["dout"] = image()
    if case.get("r"):
        state["pq"], state["pk"] = (normal(M * M, case["r"], sd=0.5).bfloat16() for _ in range(2))
    else:
        state["buckets"], count = _bucket_map(M, case["steps"], case["reach"], "cuda")
        state["bias"] = normal(heads, count, sd=0.5).bfloat16()
    if case["kind"] == "resume":
        # a layer that has run forward and kept its activations in 8 bits
        logits = _logits(state)
        windows = _split(state["v"].float(), state)
        out, lse = _softmax_values(logits, windows)
        state["lse"] = _join_rows(lse, state)
        out = _join(out, state).bfloat16()
        for name, x in (("q", state.pop("q")), ("k", state.pop("k")), ("v", state.pop("v")), ("out", out)):
            state[name + "8"], state[name + "_scale"] = _to_8_bits(x)
    return state


# -------------------------------------------------------------------------------------------------- plain operators
def _places(c, device):
    """[windows, tokens] pixel of every place of every window (-1: beyond the map), and the part of the map it comes from."""
    H, W, M, s = c["H"], c["W"], c["window"], c["shift"]
    nY, nX = -(-H // M), -(-W // M)
    y = torch.arange(nY * M, device=device)
    x = torch.arange(nX * M, device=device)
    Y, X = (y + s) % (nY * M), (x + s) % (nX * M)
    at = torch.where((Y < H)[:, None] & (X < W)[None, :], Y[:, None] * W + X[None, :], -1)
    part = 2 * (Y < y).long()[:, None] + (X < x).long()[None, :] if c["masked"] else torch.zeros_like(at)
    cut = lambda t: t.view(nY, M, nX, M).transpose(1, 2).reshape(nY * nX, M * M)  # noqa: E731
    return cut(at), cut(part)


def _split(x, c):
    """[B, H, W, heads, d] -> [B, windows, heads, tokens, d]; zeros where there is no token."""
    at, _ = _places(c, x.device)
    flat = torch.cat([x.flatten(1, 2), x.new_zeros(x.shape[0], 1, *x.shape[3:])], 1)
    return flat[:, at].transpose(2, 3)


def _join(y, c):
    """The reverse: [B, windows, heads, tokens, d] -> [B, H, W, heads, d]."""
    at, _ = _places(c, y.device)
    out = y.new_zeros(y.shape[0], c["H"] * c["W"] + 1, y.shape[2], y.shape[4])
    out[:, at.flatten()] = y.transpose(2, 3).flatten(1, 2)
    return out[:, :-1].view(y.shape[0], c["H"], c["W"], y.shape[2], y.shape[4])


def _join_rows(y, c):
    """[B, windows, heads, tokens] -> [B, heads, H, W]."""
    return _join(y[..., None], c)[..., 0].permute(0, 3, 1, 2).contiguous()


def _offsets(M, device):
    """[tokens, tokens] entry of the bucket map for (query, key)."""
    t = torch.arange(M, device=device)
    y, x = t.repeat_interleave(M), t.repeat(M)
    return (y[None, :] - y[:, None] + M - 1) * (2 * M - 1) + x[None, :] - x[:, None] + M - 1


def _logits(c, q=None, k=None):
    """[B, windows, heads, tokens, tokens] in 32 bits; minus infinity where a key is not attended to."""
    q, k = (c["q"] if q is None else q), (c["k"] if k is None else k)
    M, d = c["window"], c["d"]
    s = _split(q.float(), c) @ _split(k.float(), c).transpose(-1, -2) * (1 / math.sqrt(d))
    if "pq" in c:
        s += c["pq"].float() @ c["pk"].float().T * (1 / math.sqrt(c["r"]))
    else:
        bucket = c["buckets"].flatten().long()[_offsets(M, q.device)]
        s += torch.where(bucket < 0, -math.inf, c["bias"].float()[:, bucket.clamp(min=0)])
    at, part = _places(c, q.device)
    kept = (at >= 0)[:, None, :] & (part[:, :, None] == part[:, None, :])
    return s.masked_fill_(~kept[:, None], -math.inf)


def _softmax_values(s, v):
    """P V and the logarithm of the sum of exponentials of every row; a row without keys gives 0 and minus infinity."""
    most = s.amax(-1, keepdim=True)
    s = s.sub_(torch.where(most == -math.inf, 0.0, most)).exp_()
    total = s.sum(-1, keepdim=True)
    out = (s @ v) / torch.where(total == 0, 1.0, total)
    return out, (torch.where(most == -math.inf, 0.0, most) + total.log())[..., 0]


def _gradients(c, q, k, v, out, lse, dout):
    """dq, dk, dv and the gradient of the table(s), the probabilities recomputed from lse."""
    M, isd = c["window"], 1 / math.sqrt(c["d"])
    q, k, v, out, dout = (t.float() for t in (q, k, v, out, dout))
    p = _logits(c, q, k).sub_(torch.where(lse == -math.inf, 0.0, lse)[..., None]).exp_()
    g, vw = _split(dout, c), _split(v, c)
    dv = p.transpose(-1, -2) @ g
    mean = (_split(out, c) * g).sum(-1, keepdim=True)
    ds = (g @ vw.transpose(-1, -2)).sub_(mean).mul_(p)
    dq = ds @ _split(k, c) * isd
    dk = ds.transpose(-1, -2) @ _split(q, c) * isd
    grads = [_join(t, c).bfloat16() for t in (dq, dk, dv)]
    if "pq" in c:
        total, isr = ds.sum((0, 1, 2)), 1 / math.sqrt(c["r"])
        return (*grads, (total @ c["pk"].float() * isr).bfloat16(), (total.T @ c["pq"].float() * isr).bfloat16())
    bucket = c["buckets"].flatten().long()[_offsets(M, q.device)].flatten()
    dbias = torch.zeros(c["heads"], c["bias"].shape[1] + 1, dtype=torch.float64, device=q.device)
    dbias.index_add_(1, torch.where(bucket < 0, c["bias"].shape[1], bucket), ds.sum((0, 1), dtype=torch.float64).flatten(1))
    return (*grads, dbias[:, :-1].to(c["bias"].dtype))


def _to_8_bits(x):
    """Whole numbers -127 .. 127 and a scale for each row of the last dimension: its largest magnitude is 127."""
    x = x.float()
    scale = x.abs().amax(-1) * (1 / 127)
    return torch.round(x / torch.where(scale == 0, 1.0, scale)[..., None]).to(torch.int8), scale


def _from_8_bits(codes, scale):
    return codes.float() * scale[..., None]


def run(c):
    if own:
        from paper_2603_06738_b200 import binding as rib
        if c["kind"] == "store":
            return [rib.rib_checkpoint_restore(*rib.rib_checkpoint_store(c[name])) for name in ("q", "k", "v", "out")]
        if c["kind"] == "resume":
            saved = [(c[name + "8"], c[name + "_scale"]) for name in ("q", "k", "v", "out")]
            if c["r"]:
                *grads, dpq, dpk = rib.rib_window_attn_bwd_checkpointed(*saved, c["pq"], c["pk"], c["lse"], c["dout"], c["window"], c["shift"])
                return (*grads, dpq.bfloat16(), dpk.bfloat16())
            return rib.rib_window_attn_bwd_bucketed_checkpointed(*saved, c["bias"], c["buckets"], c["lse"], c["dout"], c["window"], c["shift"],
                                                                 masked=c["masked"])
        layer = (c["q"], c["k"], c["v"], c["bias"], c["buckets"])
        if c["kind"] == "infer":
            return rib.rib_window_attn_fwd_bucketed(*layer, c["window"], c["shift"], masked=c["masked"], want_lse=False)[0]
        out, lse = rib.rib_window_attn_fwd_bucketed(*layer, c["window"], c["shift"], masked=c["masked"])
        return (out, *rib.rib_window_attn_bwd_bucketed(*layer, out, lse, c["dout"], c["window"], c["shift"], masked=c["masked"]))
    if c["kind"] == "store":
        return [_from_8_bits(*_to_8_bits(c[name])).bfloat16() for name in ("q", "k", "v", "out")]
    if c["kind"] == "resume":
        q, k, v, out = (_from_8_bits(c[name + "8"], c[name + "_scale"]) for name in ("q", "k", "v", "out"))
        return _gradients(c, q, k, v, out, _split(c["lse"].permute(0, 2, 3, 1)[..., None], c)[..., 0], c["dout"])
    values, lse = _softmax_values(_logits(c), _split(c["v"].float(), c))
    if c["kind"] == "infer":
        return _join(values, c).bfloat16()
    out = _join(values, c)
    return (out.bfloat16(), *_gradients(c, c["q"], c["k"], c["v"], out, lse, c["dout"]))


# --------------------------------------------------------------------------------------------------------- the measure
def _pairs_of_tokens(c):
    """Query-key pairs that some head of some window has to look at."""
    H, W, M, s = c["H"], c["W"], c["window"], c["shift"]

    def axis(size):
        n = -(-size // M)
        here, wrapped = [0] * n, [0] * n            # tokens of a window, and those that came round the edge
        for i in range(n * M):
            at = (i + s) % (n * M)
            if at < size:
                (wrapped if at < i else here)[i // M] += 1
        return sum(a * a + b * b for a, b in zip(here, wrapped)) if c["masked"] else sum((a + b) ** 2 for a, b in zip(here, wrapped))

    return c["B"] * c["heads"] * axis(H) * axis(W)


def work(c):
    tokens = c["B"] * c["H"] * c["W"] * c["heads"]
    row = 2.0 * tokens * c["d"]                     # bytes of q
    if c["kind"] == "store":                        # bf16 read, 8 bits and a scale written; the same read, bf16 written
        return {"bytes": 4 * (2 * row + 2 * (row / 2 + 4 * tokens)), "flops": 4 * 3.0 * tokens * c["d"]}
    M, pairs = c["window"], _pairs_of_tokens(c)
    share = 1.0
    if c["reach"]:                                  # keys out of reach need not be looked at
        near = sum(max(0, M - a) * (1 if a == 0 else 2) for a in range(min(c["reach"], M - 1) + 1)) / M ** 2
        share = near * near
    pairs *= share
    if c.get("r"):
        table = 2.0 * M * M * c["r"] * 2
    else:
        count = _axis_buckets(M, c["steps"], "cpu")[1] ** 2
        table = 4.0 * (2 * M - 1) ** 2 + 2.0 * c["heads"] * count
    d, wide = c["d"], c["d"] + c.get("r", 0)
    forward, backward = 2.0 * pairs * (wide + d), 2.0 * pairs * (3 * wide + 2 * d)
    if c["kind"] == "infer":
        return {"bytes": 4 * row + table, "flops": forward}
    if c["kind"] == "train":                        # in: q, k, v, dout, table; out: out, dq, dk, dv, the table's gradient
        return {"bytes": 8 * row + 2 * table, "flops": forward + backward}
    return {"bytes": 4 * (row / 2 + 4 * tokens) + 4 * row + 4 * tokens + 2 * table, "flops": backward}


# ------------------------------------------------------------------------------------------------------------- 64 bits
def _exact_window(c, b, wy, wx):
    """Pixels of the tokens of one window and, for every two of them, whether they see each other and their place in the bucket map."""
    H, W, M, s = c["H"], c["W"], c["window"], c["shift"]
    nY, nX = -(-H // M), -(-W // M)
    rows, ys = zip(*[(Y, y) for y in range(M) for Y in [(wy * M + y + s) % (nY * M)] if Y < H]) if any((wy * M + y + s) % (nY * M) < H for y in range(M)) else ((), ())
    cols, xs = zip(*[(X, x) for x in range(M) for X in [(wx * M + x + s) % (nX * M)] if X < W]) if any((wx * M + x + s) % (nX * M) < W for x in range(M)) else ((), ())
    if not rows or not cols:
        return None
    t = lambda v: torch.tensor(v, device="cuda")  # noqa: E731
    rows, cols, ys, xs = t(rows), t(cols), t(ys), t(xs)
    n = len(rows) * len(cols)
    pixel = (rows[:, None] * W + cols[None, :]).reshape(n)
    y, x = ys[:, None].expand(len(ys), len(xs)).reshape(n), xs[None, :].expand(len(ys), len(xs)).reshape(n)
    seen = torch.ones(n, n, dtype=torch.bool, device="cuda")
    if c["masked"]:
        low, left = wy == nY - 1, wx == nX - 1
        label = (2 * (y >= M - s).long() if low and s else 0 * y) + ((x >= M - s).long() if left and s else 0 * x)
        seen = label[None, :] == label[:, None]
    return pixel, y * M + x, seen, (y[None, :] - y[:, None] + M - 1, x[None, :] - x[:, None] + M - 1)


def exact(case, seed):
    c = prepare(case, seed)
    f = lambda t: t.double()  # noqa: E731
    unpacked = lambda n: f(c[n + "8"]) * f(c[n + "_scale"])[..., None]  # noqa: E731
    if c["kind"] == "store":
        res = []
        for name in ("q", "k", "v", "out"):
            x = f(c[name])
            scale = x.abs().amax(-1, keepdim=True) / 127
            res.append(torch.round(x / torch.where(scale == 0, torch.ones_like(scale), scale)) * scale)
        return res
    resume, infer = c["kind"] == "resume", c["kind"] == "infer"
    q, k, v = (unpacked(n) if resume else f(c[n]) for n in ("q", "k", "v"))
    B, H, W, heads, d = q.shape
    M = c["window"]
    flat = lambda t: t.reshape(B, H * W, heads, -1)  # noqa: E731
    q, k, v = flat(q), flat(k), flat(v)
    out = torch.zeros_like(v)
    dq, dk, dv = (torch.zeros_like(v) for _ in range(3))
    g = None if infer else flat(f(c["dout"]))
    saved_out = flat(unpacked("out")) if resume else None
    saved_lse = f(c["lse"]).reshape(B, heads, H * W) if resume else None
    if c.get("r"):
        pq, pk = f(c["pq"]), f(c["pk"])
        tables = [torch.zeros_like(pq), torch.zeros_like(pk)]
    else:
        bias = torch.cat([f(c["bias"]), torch.full((heads, 1), -math.inf, dtype=torch.float64, device="cuda")], 1)
        tables = [torch.zeros_like(bias)]
    for wy in range(-(-H // M)):
        for wx in range(-(-W // M)):
            window = _exact_window(c, 0, wy, wx)
            if window is None:
                continue
            pixel, token, seen, (oy, ox) = window
            if not c.get("r"):
                named = c["buckets"][oy, ox].long()
                named = torch.where(named < 0, bias.shape[1] - 1, named)
            for b in range(B):
                take = lambda t: t[b, pixel].transpose(0, 1)  # noqa: E731  [heads, tokens, d]
                qw, kw, vw = take(q), take(k), take(v)
                z = torch.einsum("hid,hjd->hij", qw, kw) / math.sqrt(d)
                z = z + (torch.einsum("ir,jr->ij", pq[token], pk[token]) / math.sqrt(c["r"]) if c.get("r") else bias[:, named])
                z = torch.where(seen, z, torch.full_like(z, -math.inf))
                if resume:
                    p = torch.exp(z - saved_lse[b][:, pixel][..., None])
                    o = take(saved_out)
                else:
                    p = torch.softmax(z, -1)
                    p = torch.nan_to_num(p, nan=0.0)
                    o = torch.einsum("hij,hjd->hid", p, vw)
                    out[b, pixel] = o.transpose(0, 1)
                if infer:
                    continue
                gw = take(g)
                dz = p * (torch.einsum("hid,hjd->hij", gw, vw) - (gw * o).sum(-1, keepdim=True))
                dq[b, pixel] = torch.einsum("hij,hjd->ihd", dz, kw) / math.sqrt(d)
                dk[b, pixel] = torch.einsum("hij,hid->jhd", dz, qw) / math.sqrt(d)
                dv[b, pixel] = torch.einsum("hij,hid->jhd", p, gw)
                if c.get("r"):
                    both = dz.sum(0)
                    tables[0].index_add_(0, token, both @ pk[token] / math.sqrt(c["r"]))
                    tables[1].index_add_(0, token, both.T @ pq[token] / math.sqrt(c["r"]))
                else:
                    tables[0].index_add_(1, named.reshape(-1), dz.reshape(heads, -1))
    shape = (B, H, W, heads, d)
    if infer:
        return out.view(shape)
    grads = [t.view(shape) for t in (dq, dk, dv)]
    grads += tables if c.get("r") else [tables[0][:, :-1].contiguous()]
    return tuple(grads) if resume else (out.view(shape), *grads)
