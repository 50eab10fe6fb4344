"""Attention of a map's tokens to states in 64 bits, written out, and how far the kernels may be from it.

A rounding to bf16 is off by at most U = 2^-8 of the value.  The kernels round P and dS once each before they enter a product and the results once more; logits, sums and
statistics are fp32, whose roundings are counted by X: the exponent x = logit - reference is off by a few 2^-24 of the largest logit, the sums of d products by d 2^-24 of the
sum of their magnitudes, and the exponential itself by 2^-22.
"""
import math

import torch

U = 2.0 ** -8


def heads_of(x, group):
    """Keys or values [contexts, L, kv_heads, d] for every query head, [contexts, heads, L, d] in 64 bits."""
    return x.double().permute(0, 2, 1, 3).repeat_interleave(group, 1)


def rows_of(x):
    """[B, H, W, heads, d] -> [B, heads, tokens, d] in 64 bits."""
    return x.double().flatten(1, 2).permute(0, 2, 1, 3)


def as_map(x, like):
    return x.permute(0, 2, 1, 3).reshape(like.shape)


def as_states(x, like):
    """Gradients for every query head and map, summed over those that share states: [contexts, L, kv_heads, d]."""
    contexts, L, kv, d = like.shape
    B, heads = x.shape[:2]
    x = x.view(B, kv, heads // kv, L, d).sum(2)
    return (x.sum(0, keepdim=True) if contexts == 1 else x).permute(0, 2, 1, 3)


def lengths_of(k, lengths):
    contexts, L = k.shape[:2]
    return torch.full((contexts,), L, device=k.device) if lengths is None else lengths.long().clamp(0, L)


def cleaned(x, lengths):
    """States behind a length as zeros: what they hold does not count."""
    there = torch.arange(x.shape[1], device=x.device) < lengths_of(x, lengths)[:, None]
    return torch.where(there[:, :, None, None], x, torch.zeros_like(x)), there


def logits(q, k, lengths):
    group = q.shape[3] // k.shape[2]
    k, there = cleaned(k, lengths)
    s = rows_of(q) @ heads_of(k, group).transpose(-1, -2) / math.sqrt(q.shape[-1])
    return s.masked_fill(~there[:, None, None, :], -math.inf)


def forward(q, k, v, lengths=None):
    """out [B, H, W, heads, d], lse [B, heads, H, W] and the bounds of their errors."""
    B, H, W, heads, d = q.shape
    s = logits(q, k, lengths)
    group = heads // k.shape[2]
    values = heads_of(cleaned(v, lengths)[0], group)
    some = (s > -math.inf).any(-1, keepdim=True)
    lse = torch.logsumexp(s, -1, keepdim=True)
    p = torch.where(some, torch.exp(s - torch.where(some, lse, 0.0)), 0.0)
    out = p @ values
    x = score_error(q, k, lengths)
    bound = U * out.abs() + (U + 2 * x) * 1.01 * (p @ values.abs())
    return (as_map(out, q), lse[..., 0].view(B, heads, H, W)), (as_map(bound, q) + 1e-30, x + 2.0 ** -20)


def score_error(q, k, lengths):
    """How far a logit may be off, and with it the logarithm of a weight."""
    d = q.shape[-1]
    k = cleaned(k, lengths)[0]
    most = (rows_of(q).norm(dim=-1).max() * k.double().norm(dim=-1).max() / math.sqrt(d)).item()
    return (d + 16) * 2.0 ** -24 * most + 2.0 ** -20


def backward(q, k, v, out, lse, dout, lengths=None):
    """dq, dk, dv for the given out and lse, and the bounds of their errors."""
    heads, d = q.shape[3:]
    group = heads // k.shape[2]
    s = logits(q, k, lengths)
    keys, values = (heads_of(cleaned(t, lengths)[0], group) for t in (k, v))
    rows, g = rows_of(q), rows_of(dout)
    flat = lse.double().flatten(2)[..., None]
    p = torch.where(s > -math.inf, torch.exp(s - torch.where(flat > -math.inf, flat, 0.0)), 0.0)
    mean = (rows_of(out) * g).sum(-1, keepdim=True)
    dp = g @ values.transpose(-1, -2)
    ds = p * (dp - mean)
    isd = 1 / math.sqrt(d)
    dq, dk, dv = ds @ keys * isd, ds.transpose(-1, -2) @ rows * isd, p.transpose(-1, -2) @ g
    x = score_error(q, k, lengths)
    # fp32 sums of d products: dP and D
    loose = p * ((g.abs() @ values.abs().transpose(-1, -2)) + (rows_of(out) * g).abs().sum(-1, keepdim=True)) * (d + 8) * 2.0 ** -24
    es = ds.abs() * (U + 2 * x) * 1.01 + loose * 1.01
    n = 2.0 ** -20                                          # sums over rows or keys, in fp32
    bq = U * dq.abs() + (es + n * ds.abs()) @ keys.abs() * isd
    bk = as_states((es + n * ds.abs()).transpose(-1, -2) @ rows.abs() * isd, k)
    bv = as_states((p * (U + 2 * x + n) * 1.01).transpose(-1, -2) @ g.abs(), v)
    dk, dv = as_states(dk, k), as_states(dv, v)
    return (as_map(dq, q), dk, dv), (as_map(bq, q) + 1e-30, bk + U * dk.abs() + 1e-30, bv + U * dv.abs() + 1e-30)


def check(name, got, want, bound):
    got = got.double()
    assert got.shape == want.shape, name
    assert torch.equal(got.isnan(), want.isnan()), f"{name}: {int(got.isnan().sum())} NaN, expected {int(want.isnan().sum())}"
    off = ((got - want).abs() - bound).nan_to_num(nan=0.0, posinf=0.0)
    worst = off.max().item()
    assert worst <= 0, f"{name}: {worst:.3e} beyond the bound, largest value {want.abs().nan_to_num(0, 0, 0).max().item():.3e}"
    infinite = want.isinf()
    assert torch.equal(got[infinite], want[infinite]), f"{name}: infinities"
