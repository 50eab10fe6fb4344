"""8-bit checkpoints on the GPU: the codes and scales bit by bit, and the backward passes from checkpoints against the oracles on the restored values.

Tolerances of the gradients: those of the backward passes themselves (5e-3 in relative L2), and beside it the rounding of the restored q, k, v and out
to bf16, 2^-9 / sqrt(3) = 1.1e-3 of every value in the mean.  dq is a sum of dS_ij k_j with dS = P (dP - D): the errors of dP (v) and D (out) are
independent of those of k and do not cancel as dP - D does; with N(0, 1) inputs |dP| + |D| is at most twice |dP - D| in the mean, so the four of them
add up to about sqrt(1 + 1 + 4 + 4) x 1.1e-3 = 3.6e-3, and with the 3.5e-3 of the pass itself to 5e-3.  Bound: 8e-3."""
import numpy as np
import pytest
import torch

from oracle import rib_bias_oracle as orc
from oracle import rib_oracle
from paper_2603_06738_b200 import binding

from parity_util import to_f64
from test_gpu_bucketed import log_map, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(1,), (64,), (3, 1), (5, 7), (1000, 8), (37, 16), (257, 20), (1, 37, 53, 3, 24), (333, 30), (2, 9, 11, 2, 32), (129, 33), (70, 48), (65, 64), (2, 8, 8, 2, 32)])
def test_codes_scales_and_values_bit_by_bit(shape):
    g = torch.Generator().manual_seed(1)
    x = (torch.randn(shape, generator=g) * torch.exp(4 * torch.randn(*shape[:-1], 1, generator=g))).bfloat16()
    rows = x.view(-1, shape[-1])
    if rows.shape[0] > 60:
        rows[3], rows[5, 0], rows[7, -1], rows[11] = 0, float("inf"), float("nan"), 1e-40
        rows[13], rows[14, 0] = -3.0, -float("inf")
        rows[17], rows[17, 0] = 3.3e38, -3.3e38
    codes, scales = binding.rib_checkpoint_store(x.cuda())
    back = binding.rib_checkpoint_restore(codes, scales)
    want_codes, want_scales = orc.store(x.float().numpy())
    assert np.array_equal(codes.cpu().numpy(), want_codes)
    assert np.array_equal(scales.cpu().numpy(), want_scales, equal_nan=True)
    want = (torch.tensor(want_codes).float() * torch.tensor(want_scales)[..., None]).bfloat16()
    assert torch.equal(torch.isnan(back.cpu()), torch.isnan(want)) and torch.equal(back.cpu().nan_to_num(), want.nan_to_num())


@pytest.mark.parametrize("d", [64, 63])
@pytest.mark.parametrize("exponent", [-120, -100, -93, -1, 0, 127])
def test_codes_of_every_pair_of_mantissas(d, exponent):
    """Every bf16 mantissa as a row's maximum beside every bf16 value down to 2^-9 of it (smaller ones have code 0): the codes are those of the division."""
    most = torch.arange(128, 256, dtype=torch.float64) * 2.0 ** (exponent - 7)
    parts = torch.cat([torch.arange(128, 256, dtype=torch.float64) * 2.0 ** (exponent - 7 - e) for e in range(10)])
    parts = torch.nn.functional.pad(parts, (0, -len(parts) % (d - 1))).view(-1, d - 1)
    x = torch.cat([most[:, None, None].expand(-1, len(parts), 1), torch.minimum(parts[None], most[:, None, None])], 2).reshape(-1, d).bfloat16()
    x[1::2] = -x[1::2]
    codes, scales = binding.rib_checkpoint_store(x.cuda())
    want_codes, want_scales = orc.store(x.float().numpy())
    assert np.array_equal(codes.cpu().numpy(), want_codes) and np.array_equal(scales.cpu().numpy(), want_scales)


def test_empty_and_refused():
    codes, scales = binding.rib_checkpoint_store(torch.empty(0, 32, dtype=torch.bfloat16, device="cuda"))
    assert codes.shape == (0, 32) and scales.shape == (0,) and binding.rib_checkpoint_restore(codes, scales).shape == (0, 32)
    x = torch.zeros(4, 32, dtype=torch.bfloat16, device="cuda")
    for bad in (x.float(), x.t(), torch.zeros(4, 65, dtype=torch.bfloat16, device="cuda")):
        with pytest.raises((ValueError, binding.RibError)):
            binding.rib_checkpoint_store(bad)
    with pytest.raises(ValueError):
        binding.rib_checkpoint_restore(torch.zeros(4, 32, dtype=torch.int8, device="cuda"), torch.zeros(5, device="cuda"))


def kept(tensors):
    return [binding.rib_checkpoint_store(t) for t in tensors]


def near(name, got, ref, bound=8e-3):
    got = to_f64(got)
    assert np.isfinite(got).all(), name
    assert np.linalg.norm(got - ref) <= bound * np.linalg.norm(ref), (name, np.linalg.norm(got - ref) / np.linalg.norm(ref))
    assert np.abs(got - ref).max() <= 2e-2 * max(1.0, np.abs(ref).max()), name


# B, H, W, heads, d, window, shift, masked
@pytest.mark.parametrize("case", [(1, 6, 9, 2, 10, 3, 1, False), (2, 32, 32, 2, 32, 16, 8, False), (1, 48, 48, 3, 16, 16, 8, True), (1, 40, 24, 2, 24, 8, 0, False),
                                  (1, 64, 64, 2, 32, 32, 16, False), (1, 35, 41, 1, 32, 16, 8, False)], ids=lambda c: "x".join(map(str, c)))
def test_backward_of_a_bias_layer_from_checkpoints(case):
    B, H, W, heads, d, M, s, masked = case
    q, k, v, dout, bias, named = (t.cuda() for t in make(B, H, W, heads, d, M, log_map(M), seed=31))
    out, lse = binding.rib_window_attn_fwd_bucketed(q, k, v, bias, named, M, s, masked=masked)
    saved = kept((q, k, v, out))
    grads = binding.rib_window_attn_bwd_bucketed_checkpointed(*saved, bias, named, lse, dout, M, s, masked=masked)
    torch.cuda.synchronize()
    assert binding.rib_query_status() == 0
    values = [orc.restore(c.cpu().numpy(), sc.cpu().numpy()) for c, sc in saved]
    ref = orc.bwd(*values[:3], to_f64(bias), named.cpu().numpy(), to_f64(dout), M, s, masked, out=values[3], lse=to_f64(lse))
    for name, got, want in zip(("dq", "dk", "dv", "dbias"), grads, ref):
        near(name, got, want)
    # the same call on the restored tensors does the same arithmetic
    plain = binding.rib_window_attn_bwd_bucketed(*(binding.rib_checkpoint_restore(*x) for x in saved[:3]), bias, named, binding.rib_checkpoint_restore(*saved[3]),
                                                 lse, dout, M, s, masked=masked)
    assert torch.equal(plain[2], grads[2]) and torch.equal(plain[1], grads[1])


# B, H, W, heads, d, r, window, shift, masked, headwise
@pytest.mark.parametrize("case", [(1, 8, 8, 2, 6, 5, 4, 1, False, False), (2, 32, 32, 2, 32, 16, 16, 8, False, False), (1, 64, 32, 2, 32, 16, 32, 16, False, True),
                                  (1, 32, 32, 2, 32, 16, 16, 8, True, False), (1, 16, 16, 2, 32, 16, 8, 0, False, False), (1, 40, 24, 2, 32, 16, 16, 0, False, False),
                                  (1, 32, 32, 2, 30, 18, 16, 0, False, False)], ids=lambda c: "x".join(map(str, c)))
def test_backward_of_a_rank_r_layer_from_checkpoints(case):
    B, H, W, heads, d, r, M, s, masked, headwise = case
    g = torch.Generator().manual_seed(41)
    q, k, v, dout = (torch.randn(B, H, W, heads, d, generator=g).bfloat16().cuda() for _ in range(4))
    pq, pk = ((torch.randn(*((heads,) if headwise else ()), M * M, r, generator=g) * 0.5).bfloat16().cuda() for _ in range(2))
    divides = H % M == 0 and W % M == 0
    fwd = binding.rib_window_attn_fwd_masked if masked else binding.rib_window_attn_fwd_padded
    bwd = binding.rib_window_attn_bwd_masked if masked else binding.rib_window_attn_bwd_padded
    out, lse = fwd(q, k, v, pq, pk, M, s)
    saved = kept((q, k, v, out))
    grads = binding.rib_window_attn_bwd_checkpointed(*saved, pq, pk, lse, dout, M, s, masked=masked)
    back = [binding.rib_checkpoint_restore(*x) for x in saved]
    plain = bwd(*back[:3], pq, pk, back[3], lse, dout, M, s)
    torch.cuda.synchronize()
    assert binding.rib_query_status() == 0
    for a, b in zip(grads[:3], plain[:3]):
        near("same arithmetic", a, to_f64(b), 2e-3)          # (sums in another order, rounded to bf16)
    for a, b in zip(grads[3:], plain[3:]):
        near("same arithmetic", a, to_f64(b), 1e-4)
    if divides and not masked:
        # P and dS from the values and the lse that were kept
        values = [orc.restore(c.cpu().numpy(), sc.cpu().numpy()) for c, sc in saved]
        ref = gradients(*values, to_f64(pq), to_f64(pk), to_f64(lse), to_f64(dout), M, s)
        for name, got, want in zip(("dq", "dk", "dv", "dpq", "dpk"), grads, ref):
            near(name, got, want)


def gradients(q, k, v, out, pq, pk, lse, dout, M, s):
    """Chain rule of Eq. 6 from given values, lse and out, in float64."""
    B, H, W, heads, d = q.shape
    r = pq.shape[-1]
    res = [np.zeros_like(q) for _ in range(3)] + [np.zeros_like(pq), np.zeros_like(pk)]
    y, x = np.divmod(np.arange(M * M), M)
    for b in range(B):
        for wy in range(H // M):
            for wx in range(W // M):
                Y, X = (wy * M + y + s) % H, (wx * M + x + s) % W
                for h in range(heads):
                    a, c = (pq[h], pk[h]) if pq.ndim == 3 else (pq, pk)
                    qw, kw, vw, ow, g = (t[b, Y, X, h] for t in (q, k, v, out, dout))
                    p = np.exp(qw @ kw.T / np.sqrt(d) + a @ c.T / np.sqrt(r) - lse[b, h, Y, X][:, None])
                    ds = p * (g @ vw.T - (g * ow).sum(1, keepdims=True))
                    res[0][b, Y, X, h], res[1][b, Y, X, h], res[2][b, Y, X, h] = ds @ kw / np.sqrt(d), ds.T @ qw / np.sqrt(d), p.T @ g
                    for t, value in ((res[3], ds @ c / np.sqrt(r)), (res[4], ds.T @ a / np.sqrt(r))):
                        if t.ndim == 3:
                            t[h] += value
                        else:
                            t += value
    return res


def test_the_helper_agrees_with_the_oracle():
    rng = np.random.default_rng(3)
    q, k, v, g = (rng.standard_normal((1, 8, 4, 2, 3)) for _ in range(4))
    pq, pk = rng.standard_normal((2, 16, 5))
    out, lse = rib_oracle.fwd(q, k, v, pq, pk, 4, 1)
    for a, b in zip(gradients(q, k, v, out, pq, pk, lse, g, 4, 1), rib_oracle.bwd(q, k, v, pq, pk, g, 4, 1)):
        assert np.abs(a - b).max() < 1e-12
