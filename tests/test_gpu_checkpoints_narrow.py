"""The backward passes from checkpoints of layers with narrow heads, against the oracles on the values code x scale, not rounded to bf16.

Bound: that of the backward passes from the tensors themselves, 5e-3 in relative L2.  With one rounding to bf16 of q, k and v before they are used, heads of 8 and 16 channels
pass it: a logit is a sum of few products then, and the largest logits, which carry the weight, have the largest errors."""
import ctypes

import pytest
import torch

from oracle import rib_bias_oracle as orc
from paper_2603_06738_b200 import binding

from parity_util import to_f64
from test_gpu_bucketed import log_map, make
from test_gpu_checkpoints import gradients, kept, near
from test_gpu_safety import Guarded

pytestmark = pytest.mark.gpu


# B, H, W, heads, d, window, shift, masked
@pytest.mark.parametrize("case", [(2, 16, 24, 3, 8, 8, 0, False), (1, 48, 32, 3, 8, 16, 8, True), (1, 48, 48, 3, 8, 48, 0, False), (2, 64, 64, 2, 8, 64, 32, False), (1, 35, 41, 3, 8, 32, 8, False),
                                  (2, 32, 48, 3, 16, 16, 8, False), (1, 48, 48, 3, 16, 48, 0, False), (2, 64, 64, 2, 16, 64, 32, False), (1, 41, 35, 3, 16, 24, 8, False)],
                         ids=lambda c: "x".join(map(str, c)))
def test_bias_layer(case):
    B, H, W, heads, d, M, s, masked = case
    q, k, v, dout, bias, named = (t.cuda() for t in make(B, H, W, heads, d, M, log_map(M), seed=38))
    out, lse = binding.rib_window_attn_fwd_bucketed(q, k, v, bias, named, M, s, masked=masked)
    saved = kept((q, k, v, out))
    grads = binding.rib_window_attn_bwd_bucketed_checkpointed(*saved, bias, named, lse, dout, M, s, masked=masked)
    torch.cuda.synchronize()
    assert binding.rib_query_status() == 0 and binding.rib_last_path() == binding.RIB_PATH_SM100
    values = [orc.restore(c.cpu().numpy(), sc.cpu().numpy()) for c, sc in saved]
    ref = orc.bwd(*values[:3], to_f64(bias), named.cpu().numpy(), to_f64(dout), M, s, masked, out=values[3], lse=to_f64(lse))
    for name, got, want in zip(("dq", "dk", "dv", "dbias"), grads, ref):
        near(name, got, want, 5e-3)


# B, H, W, heads, d, r, window, shift, headwise
@pytest.mark.parametrize("case", [(2, 32, 48, 3, 8, 16, 16, 8, False), (1, 64, 64, 2, 8, 16, 32, 16, True), (1, 96, 48, 3, 8, 8, 48, 24, False), (1, 64, 64, 2, 8, 32, 64, 0, False),
                                  (2, 32, 48, 3, 16, 24, 16, 8, False), (2, 32, 48, 3, 8, 16, 8, 0, False), (2, 32, 48, 3, 16, 24, 8, 0, False), (2, 64, 64, 2, 16, 16, 32, 16, False), (2, 64, 64, 2, 16, 16, 64, 32, False)], ids=lambda c: "x".join(map(str, c)))
def test_rank_r_layer(case):
    B, H, W, heads, d, r, M, s, headwise = case
    g = torch.Generator().manual_seed(39)
    q, k, v, dout = (torch.randn(B, H, W, heads, d, generator=g).bfloat16().cuda() for _ in range(4))
    pq, pk = ((torch.randn(*((heads,) if headwise else ()), M * M, r, generator=g) * 0.5).bfloat16().cuda() for _ in range(2))
    out, lse = binding.rib_window_attn_fwd_padded(q, k, v, pq, pk, M, s)
    saved = kept((q, k, v, out))
    grads = binding.rib_window_attn_bwd_checkpointed(*saved, pq, pk, lse, dout, M, s)
    torch.cuda.synchronize()
    assert binding.rib_query_status() == 0 and binding.rib_last_path() == binding.RIB_PATH_SM100
    values = [orc.restore(c.cpu().numpy(), sc.cpu().numpy()) for c, sc in saved]
    ref = gradients(*values, to_f64(pq), to_f64(pk), to_f64(lse), to_f64(dout), M, s)
    for name, got, want in zip(("dq", "dk", "dv", "dpq", "dpk"), grads, ref):
        near(name, got, want, 5e-3)


# B, H, W, heads, d, r, window, shift
@pytest.mark.parametrize("case", [(2, 32, 48, 3, 8, 16, 16, 8), (1, 64, 32, 2, 16, 32, 32, 16), (2, 32, 48, 3, 8, 16, 8, 0), (1, 40, 56, 3, 16, 16, 16, 8), (1, 24, 40, 2, 8, 8, 48, 0), (1, 9, 7, 2, 16, 8, 4, 1)],
                         ids=lambda c: "x".join(map(str, c)))
def test_results_and_workspaces_stay_inside_their_buffers(case):
    B, H, W, heads, d, r, M, s = case
    g = torch.Generator().manual_seed(40)
    q, k, v, dout = (torch.randn(B, H, W, heads, d, generator=g).bfloat16().cuda() for _ in range(4))
    pq, pk = ((torch.randn(M * M, r, generator=g) * 0.5).bfloat16().cuda() for _ in range(2))
    out, lse = binding.rib_window_attn_fwd_padded(q, k, v, pq, pk, M, s)
    saved = kept((q, k, v, out))
    lib, p = binding.library(), lambda t: t.data_ptr()  # noqa: E731
    guarded = Guarded()
    results = [guarded.tensor(q.shape, torch.bfloat16) for _ in range(3)] + [guarded.tensor(pq.shape, torch.float32) for _ in range(2)]
    need = lib.rib_window_attn_bwd_checkpointed_workspace(0, B, H, W, heads, d, r, M)
    ws = guarded.tensor((need,), torch.uint8)
    array = (ctypes.c_void_p * 8)(*[p(t) for pair in saved for t in pair])
    args = [array, p(pq), p(pk), 0, p(lse), p(dout), B, H, W, heads, d, r, M, s, 0, *(p(t) for t in results), p(ws)]
    assert lib.rib_window_attn_bwd_checkpointed(*args, need - 1, None) == -5
    assert lib.rib_window_attn_bwd_checkpointed(*args, need, None) == 0
    torch.cuda.synchronize()
    assert binding.rib_query_status() == 0
    guarded.check("backward from checkpoints")
    for a, b in zip(results, binding.rib_window_attn_bwd_checkpointed(*saved, pq, pk, lse, dout, M, s)):
        assert not torch.isnan(a.float()).any() and float((a.float() - b.float()).norm()) <= 1e-3 * float(b.float().norm())
