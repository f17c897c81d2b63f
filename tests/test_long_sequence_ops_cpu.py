"""Refusals of the calls for long sequences (checked on the host before any CUDA
call), and the reference definitions against brute force. CPU only."""
import ctypes
import math

import numpy as np
import pytest
import torch

import sublayer_reference as ref
from paper_2609_10018_gb300 import binding
from test_abi_cpu import lib  # noqa: F401  (builds the library where it is stale)

P = 1 << 20  # any 16-byte aligned address: refused before it is used


def _quantize(lib, **kw):
    a = dict(x=P, x_type=binding.BF16, ldx=256, q=P, ldq=256, scale=P, lds=8, rows=8, cols=200) | kw
    return lib.elasto_op_quantize_fp8(None, *a.values())


@pytest.mark.parametrize("kw", [dict(x=None), dict(q=None), dict(scale=None), dict(rows=0), dict(cols=0), dict(cols=-1),
                                dict(ldx=199), dict(ldq=199), dict(lds=7), dict(x_type=3), dict(x_type=-1),
                                dict(x=P + 1), dict(scale=P + 2), dict(x=P + 2, x_type=binding.F32)])
def test_quantize_refusals(lib, kw):  # noqa: F811
    assert _quantize(lib, **kw) == binding.ERR_INVALID_ARG
    assert "elasto_op_quantize_fp8" in binding.elasto_last_error()


def test_quantize_too_many_blocks(lib):  # noqa: F811
    assert _quantize(lib, rows=1 << 30, lds=1 << 30, cols=1000, ldx=1000, ldq=1000) == binding.ERR_UNSUPPORTED


def _gemm(lib, **kw):
    a = dict(A=P, lda=256, a_scale=P, lds=8, W=P, ldw=256, w_scale=P, bias=P, out=P, ldo=40, M=8, N=40, K=250,
             epilogue=binding.EPI_BIAS_BF16, status=None) | kw
    return lib.elasto_op_gemm_fp8(None, *a.values())


@pytest.mark.parametrize("kw", [dict(A=None), dict(a_scale=None), dict(W=None), dict(w_scale=None), dict(out=None),
                                dict(M=0), dict(N=0), dict(K=0), dict(lda=240), dict(ldw=240), dict(lds=7), dict(ldo=39),
                                dict(lda=264), dict(ldw=264), dict(A=P + 8), dict(W=P + 8), dict(out=P + 1),
                                dict(a_scale=P + 2), dict(bias=P + 1), dict(epilogue=binding.EPI_BIAS_RELU_BF16),
                                dict(epilogue=-1), dict(epilogue=9), dict(out=P + 2, epilogue=binding.EPI_BIAS_F32)])
def test_gemm_fp8_refusals(lib, kw):  # noqa: F811
    assert _gemm(lib, **kw) == binding.ERR_INVALID_ARG
    assert "elasto_op_gemm_fp8" in binding.elasto_last_error()


def _rope(lib, **kw):
    a = dict(dtype=binding.BF16, rows=4, heads_q=2, heads_k=1, head_dim=64, rot_dim=64, eps=1e-6, q=P, q_row=256, q_head=64,
             k=P, k_row=256, k_head=64, v=P, v_row=256, v_head=64, q_out=2 * P, q_out_row=128, q_out_head=64, k_out=2 * P,
             k_out_row=64, k_out_head=64, v_out=2 * P, v_out_row=64, v_out_head=64, cos_sin=P, positions=P, n_positions=9) | kw
    return lib.elasto_op_qk_norm_rope(None, ctypes.byref(binding.QkNormRope(**a)), None)


@pytest.mark.parametrize("kw", [dict(dtype=binding.F32), dict(dtype=7), dict(rows=0), dict(heads_q=0, heads_k=0),
                                dict(heads_q=-1), dict(heads_q=70000), dict(eps=-1e-6), dict(eps=math.nan), dict(q=None),
                                dict(q_out=None), dict(k=None), dict(k_out=None), dict(v=None), dict(v_out=None),
                                dict(q=P + 8), dict(k_row=250), dict(v_out_head=60), dict(q_head=-64), dict(cos_sin=None),
                                dict(positions=None), dict(n_positions=0), dict(cos_sin=P + 4), dict(positions=P + 2),
                                dict(q_gain=P + 4), dict(k_gain=P + 8), dict(slots=P, n_slots=0), dict(slots=P + 1, n_slots=4),
                                dict(k_out=P, k_out_row=256, slots=P, n_slots=4), dict(q_out=P)])
def test_qk_norm_rope_refusals(lib, kw):  # noqa: F811
    assert _rope(lib, **kw) == binding.ERR_INVALID_ARG
    assert "elasto_op_qk_norm_rope" in binding.elasto_last_error()


@pytest.mark.parametrize("kw", [dict(head_dim=60), dict(head_dim=264), dict(rot_dim=24), dict(rot_dim=80), dict(rot_dim=-16)])
def test_qk_norm_rope_unsupported(lib, kw):  # noqa: F811
    assert _rope(lib, **kw) == binding.ERR_UNSUPPORTED


def test_qk_norm_rope_null(lib):  # noqa: F811
    assert lib.elasto_op_qk_norm_rope(None, None, None) == binding.ERR_INVALID_ARG


def _attention(lib, **kw):
    a = dict(dtype=binding.BF16, batch=2, heads=4, heads_kv=2, head_dim=64, causal=1, window=8, sinks=1, scale=0.125,
             max_queries=5, q_rows=10, q=P, q_row=256, q_head=64, out=2 * P, out_row=256, out_head=64, max_keys=9, kv_rows=12,
             k=P, k_batch=2048, k_row=128, k_head=64, v=P, v_batch=2048, v_row=128, v_head=64) | kw
    return lib.elasto_op_window_attention(None, ctypes.byref(binding.WindowAttention(**a)), None)


@pytest.mark.parametrize("kw", [dict(dtype=binding.F32), dict(batch=0), dict(heads=0), dict(heads_kv=0), dict(heads_kv=3),
                                dict(max_queries=0), dict(max_keys=0), dict(max_keys=13), dict(kv_rows=0), dict(q_rows=9),
                                dict(q_rows=0), dict(q_rows=(1 << 30) + 1), dict(kv_rows=(1 << 30) + 1), dict(sinks=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
                                dict(scale=math.inf), dict(q=None), dict(out=None), dict(k=None), dict(v=None), dict(q=P + 8),
                                dict(out_row=250), dict(k_batch=1), dict(v_head=-8), dict(kv_start=P, kv_len=P),
                                dict(q_start=P + 1), dict(kv_start=P + 2), dict(kv_len=P + 3)])
def test_window_attention_refusals(lib, kw):  # noqa: F811
    assert _attention(lib, **kw) == binding.ERR_INVALID_ARG
    assert "elasto_op_window_attention" in binding.elasto_last_error()


@pytest.mark.parametrize("kw", [dict(head_dim=60), dict(head_dim=136), dict(head_dim=0)])
def test_window_attention_unsupported(lib, kw):  # noqa: F811
    assert _attention(lib, **kw) == binding.ERR_UNSUPPORTED


def test_window_attention_null(lib):  # noqa: F811
    assert lib.elasto_op_window_attention(None, None, None) == binding.ERR_INVALID_ARG


@pytest.mark.parametrize("nq,nk,causal,window,sinks", [(5, 9, True, 2, 1), (9, 5, True, 2, 1), (7, 7, False, 1, 2),
                                                       (4, 4, False, -1, 0), (3, 8, True, -1, 0), (6, 6, True, 0, 0)])
def test_reference_attention_brute_force(nq, nk, causal, window, sinks):
    """The matrix form against sums over the visible keys, one query at a time."""
    g = torch.Generator().manual_seed(nq * 31 + nk)
    q, k, v = (torch.randn((n, h, 4), generator=g, dtype=torch.float64) for n, h in ((nq, 4), (nk, 2), (nk, 2)))
    got, _ = ref.attention(q, k, v, 0.7, causal, window, sinks)
    for i in range(nq):
        p = nk - nq + i
        for h in range(4):
            num, den = np.zeros(4), 0.0
            for j in range(nk):
                near = window < 0 or abs(j - p) <= window
                seen = (j <= p and (near or j < sinks)) if causal else (near or j < sinks or p < sinks)
                if p >= 0 and seen:
                    e = math.exp(0.7 * float(q[i, h] @ k[j, h // 2]))
                    num, den = num + e * v[j, h // 2].numpy(), den + e
            want = num / den if den else np.zeros(4)
            assert np.max(np.abs(got[i, h].numpy() - want)) <= 1e-12


def test_reference_rotation_keeps_length():
    g = torch.Generator().manual_seed(3)
    x = torch.randn((5, 2, 32), generator=g, dtype=torch.float64)
    angle = torch.randn((5, 16), generator=g, dtype=torch.float64)
    for interleaved in (False, True):
        y = ref.norm_rope(x, None, angle.cos(), angle.sin(), 0.0, interleaved)
        assert torch.allclose((y * y).mean(2), torch.ones(5, 2, dtype=torch.float64), atol=1e-12)
