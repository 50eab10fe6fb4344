"""CPU oracle for window attention with a learned bias by buckets of the relative position, and for activation checkpoints in 8 bits.

TEST INFRASTRUCTURE ONLY.  Plain numpy in float64, one window and head at a time; it shares no code with the CUDA path nor with the other
oracles.  Definition: with (y, x) the place of a token inside its window of side M, u = buckets[y_j - y_i + M - 1, x_j - x_i + M - 1],

    S_ij = q_i . k_j / sqrt(d) + bias[h, u]     (minus infinity where u is no bucket, the bias is -1e30 or less, j is no token or, with
                                                 `masked`, i and j lie in parts of the window that come from different sides of the map)
    P = SoftMax(S),  out = P V,  lse = ln sum_j exp S_ij;   a row without any key: out = 0, lse = -inf, no gradient
    dS = P o (dO V^T - rowsum(dO o out)),  dq = dS K / sqrt(d),  dk = dS^T Q / sqrt(d),  dv = P^T dO,  dbias[h, u] = sum of dS_ij over u(i, j) = u.

Maps that are no multiples of the window are extended to multiples; places beyond the map are no tokens.
"""
from __future__ import annotations

import numpy as np


def _windows(H, W, M, s, masked):
    """For every window: rows, columns (image), places (y, x) and part labels of its tokens."""
    nY, nX = -(-H // M), -(-W // M)
    if masked and (H % M or W % M):
        raise ValueError("the mask is defined on maps that are multiples of the window")
    for wy in range(nY):
        for wx in range(nX):
            tokens = []
            for y in range(M):
                for x in range(M):
                    py, px = wy * M + y + s, wx * M + x + s
                    Y, X = py % (nY * M), px % (nX * M)
                    if Y < H and X < W:
                        tokens.append((Y, X, y, x, (2 * (py >= nY * M) + (px >= nX * M)) if masked else 0))
            if tokens:
                yield [np.array(c) for c in zip(*tokens)]


def _bias(table, buckets, M, y, x):
    u = buckets[y[None, :] - y[:, None] + M - 1, x[None, :] - x[:, None] + M - 1]
    named = (u >= 0) & (u < table.shape[0])
    b = np.where(named, table[np.where(named, u, 0)], -np.inf)
    return u, np.where(b <= -1e30, -np.inf, b)


def _table(bias, h):
    return bias if bias.ndim == 1 else bias[h]


def fwd(q, k, v, bias, buckets, window, shift=0, masked=False):
    """out [B,H,W,heads,d], lse [B,heads,H,W]; bias [heads, buckets] or [buckets]."""
    q, k, v, bias = (np.asarray(a, dtype=np.float64) for a in (q, k, v, bias))
    B, H, W, heads, d = q.shape
    out, lse = np.full(q.shape, np.nan), np.full((B, heads, H, W), np.nan)
    for Y, X, y, x, part in _windows(H, W, window, shift, masked):
        for h in range(heads):
            _, add = _bias(_table(bias, h), buckets, window, y, x)
            add = np.where(part[:, None] == part[None, :], add, -np.inf)
            for b in range(B):
                s = q[b, Y, X, h] @ k[b, Y, X, h].T / np.sqrt(d) + add
                top = s.max(1, keepdims=True)
                e = np.exp(s - np.where(np.isinf(top), 0.0, top))
                total = e.sum(1, keepdims=True)
                out[b, Y, X, h] = e @ v[b, Y, X, h] / np.where(total == 0, 1.0, total)
                with np.errstate(divide="ignore"):
                    lse[b, h, Y, X] = (np.where(np.isinf(top), 0.0, top) + np.log(total))[:, 0]
    return out, lse


def bwd(q, k, v, bias, buckets, dout, window, shift=0, masked=False, out=None, lse=None, want_norm=False):
    """dq, dk, dv and dbias (and the 2-norm of all dS); out and lse are computed here unless those of a forward pass on other inputs are given."""
    q, k, v, bias, dout = (np.asarray(a, dtype=np.float64) for a in (q, k, v, bias, dout))
    if out is None:
        out, lse = fwd(q, k, v, bias, buckets, window, shift, masked)
    out, lse = np.asarray(out, dtype=np.float64), np.asarray(lse, dtype=np.float64)
    B, H, W, heads, d = q.shape
    dq, dk, dv, dbias = np.full(q.shape, np.nan), np.full(q.shape, np.nan), np.full(q.shape, np.nan), np.zeros(bias.shape)
    squares = 0.0
    for Y, X, y, x, part in _windows(H, W, window, shift, masked):
        for h in range(heads):
            u, add = _bias(_table(bias, h), buckets, window, y, x)
            add = np.where(part[:, None] == part[None, :], add, -np.inf)
            seen = ~np.isinf(add)
            for b in range(B):
                qw, kw, vw, g = (t[b, Y, X, h] for t in (q, k, v, dout))
                l = lse[b, h, Y, X][:, None]
                p = np.where(seen, np.exp(np.where(seen, qw @ kw.T / np.sqrt(d) + add - np.where(np.isinf(l), 0.0, l), 0.0)), 0.0)
                ds = p * (g @ vw.T - (g * out[b, Y, X, h]).sum(1, keepdims=True))
                dq[b, Y, X, h] = ds @ kw / np.sqrt(d)
                dk[b, Y, X, h] = ds.T @ qw / np.sqrt(d)
                dv[b, Y, X, h] = p.T @ g
                np.add.at(_table(dbias, h), u[seen], ds[seen])
                squares += (ds * ds).sum()
    return (dq, dk, dv, dbias, np.sqrt(squares)) if want_norm else (dq, dk, dv, dbias)


def store(x):
    """Codes (whole numbers) and scales of the rows of x, with the scale and the quotient rounded to float32 as the definition says."""
    x = np.asarray(x, dtype=np.float32)
    scale = (np.abs(x).max(-1) * np.float32(1 / 127)).astype(np.float32)
    with np.errstate(invalid="ignore"):
        bad = ~np.isfinite(x).all(-1)
        safe = np.where((scale == 0) | bad, np.float32(1), scale)
        codes = np.where(((scale == 0) | bad)[..., None], 0, np.rint(x / safe[..., None])).astype(np.int8)
    return codes, np.where(bad, np.float32(np.nan), scale)


def restore(codes, scale):
    return np.asarray(codes, dtype=np.float64) * np.asarray(scale, dtype=np.float64)[..., None]
