"""Refusals of the operators of a transformer block (checked on the host before any CUDA call), and their reference
definitions against torch's own. CPU only."""
import ctypes
import math

import pytest
import torch

import block_reference as block
from paper_2609_10018_gb300 import binding
from test_abi_cpu import lib  # noqa: F401  (builds the library where it is stale)

P = 1 << 20  # any 32-byte aligned address: refused before it is used


def _residual(lib, **kw):
    a = dict(rows=4, cols=40, eps=1e-6, x_factor=1.0, x_type=binding.F32, x=P, x_row=40, x_out=2 * P, x_out_row=40, y_type=binding.BF16,
             y=3 * P, y_row=40, post_norm=binding.NORM_RMS, post_gain=4 * P, y_scale=5 * P, pre_norm=binding.NORM_LAYER, pre_gain=6 * P,
             pre_bias=7 * P, groups=2, group=8 * P, mod_type=binding.BF16, mod_row=120, gate=9 * P, shift=10 * P, scale=11 * P,
             z_type=binding.E4M3, z=12 * P, z_row=40, z_scale=13 * P, z_scale_row=4) | kw
    return lib.elasto_op_residual_norm(None, ctypes.byref(binding.ResidualNorm(**a)), None)


@pytest.mark.parametrize("kw", [dict(rows=0), dict(rows=-1), dict(cols=0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf),
                                dict(x_factor=math.nan), dict(x_factor=math.inf), dict(x_factor=-math.inf), dict(x=None), dict(x_type=3),
                                dict(x_type=-1), dict(x=P + 2), dict(x_row=39), dict(y_type=binding.E4M3), dict(y=P + 1), dict(y_row=39),
                                dict(x_out=None, z=None), dict(x_out=2 * P + 2), dict(x_out_row=39), dict(z_type=4), dict(z_type=-1),
                                dict(z_type=binding.BF16, z=12 * P + 1), dict(z_row=39), dict(z_scale=None), dict(z_scale=13 * P + 2),
                                dict(z_scale_row=3), dict(post_norm=3), dict(post_norm=-1), dict(pre_norm=3), dict(post_gain=P + 1),
                                dict(post_bias=P + 2), dict(y_scale=P + 3), dict(pre_gain=P + 1), dict(pre_bias=P + 1), dict(groups=-1),
                                dict(groups=0), dict(group=P + 1), dict(mod_type=binding.E4M3), dict(mod_row=39), dict(gate=P + 1),
                                dict(shift=P + 1), dict(scale=P + 1), dict(mod_type=binding.F32, scale=P + 2),
                                dict(x_out=P, x_out_row=48), dict(z=P), dict(z=3 * P), dict(z_scale=P), dict(x_out=3 * P), dict(z=2 * P),
                                dict(z_scale=12 * P), dict(z_scale=2 * P), dict(z=9 * P), dict(z=8 * P), dict(x_out=6 * P)])
def test_residual_norm_refusals(lib, kw):  # noqa: F811
    assert _residual(lib, **kw) == binding.ERR_INVALID_ARG
    assert "elasto_op_residual_norm" in binding.elasto_last_error()


def test_residual_norm_too_wide(lib):  # noqa: F811
    wide = dict(cols=16385, x_row=16385, x_out_row=16385, y_row=16385, z_row=16385, mod_row=16385)
    assert _residual(lib, **wide) == binding.ERR_UNSUPPORTED
    assert lib.elasto_op_residual_norm(None, None, None) == binding.ERR_INVALID_ARG


def _axes(values):
    return (ctypes.c_uint8 * len(values))(*values)


def _rope(lib, axis_of=(0,) * 16 + (1,) * 16, **kw):
    a = dict(dtype=binding.BF16, rows=4, heads_q=2, heads_k=1, head_dim=64, rot_dim=64, pairing=binding.PAIRS_HALF, norm=1, eps=1e-6,
             q=P, q_row=256, q_head=64, k=P, k_row=256, k_head=64, v=P, v_row=256, v_head=64, q_out=2 * P, q_out_row=128, q_out_head=64,
             k_out=2 * P, k_out_row=64, k_out_head=64, v_out=2 * P, v_out_row=64, v_out_head=64, cos_sin=P, n_positions=9, axes=2,
             axis_of=_axes(axis_of) if axis_of else None, positions=P, positions_row=2, positions_axis=1) | kw
    return lib.elasto_op_qk_norm_rope_axes(None, ctypes.byref(binding.QkNormRopeAxes(**a)), None)


@pytest.mark.parametrize("kw", [dict(dtype=binding.F32), dict(rows=0), dict(heads_q=0, heads_k=0), dict(heads_q=70000), dict(eps=-1e-6),
                                dict(q=None), dict(k_out=None), dict(v=None), dict(q=P + 8), dict(k_row=250), dict(q_head=-64),
                                dict(cos_sin=None), dict(positions=None), dict(n_positions=0), dict(cos_sin=P + 4), dict(positions=P + 2),
                                dict(q_gain=P + 4), dict(slots=P, n_slots=0), dict(k_out=P, k_out_row=256, slots=P, n_slots=4), dict(q_out=P),
                                dict(pairing=3), dict(pairing=-1), dict(norm=2), dict(norm=-1), dict(axes=0), dict(axes=5),
                                dict(axis_of=None), dict(axis_of=(0,) * 31 + (2,)), dict(axis_of=(255,) + (0,) * 31), dict(positions_row=-1),
                                dict(positions_axis=-1), dict(pairing=2, axis_of=(0,) * 12 + (1,) * 20),
                                dict(pairing=2, axis_of=(0,) * 8 + (1,) * 16 + (0,) * 8), dict(pairing=2, axis_of=(0, 1) * 16)])
def test_rope_axes_refusals(lib, kw):  # noqa: F811
    assert _rope(lib, **kw) == binding.ERR_INVALID_ARG
    assert "elasto_op_qk_norm_rope_axes" in binding.elasto_last_error()


@pytest.mark.parametrize("kw", [dict(head_dim=60), dict(head_dim=264), dict(rot_dim=24), dict(rot_dim=80), dict(rot_dim=-16)])
def test_rope_axes_unsupported(lib, kw):  # noqa: F811
    assert _rope(lib, **kw) == binding.ERR_UNSUPPORTED
    assert lib.elasto_op_qk_norm_rope_axes(None, None, None) == binding.ERR_INVALID_ARG


def test_reference_norms():
    g = torch.Generator().manual_seed(1)
    v, gain, bias = torch.randn((5, 37), generator=g, dtype=torch.float64), torch.randn(37, generator=g), torch.randn(37, generator=g)
    got = block.norm(v, block.LAYER, gain, bias, 1e-5)[0]
    assert torch.allclose(got, torch.nn.functional.layer_norm(v, (37,), gain.double(), bias.double(), 1e-5), atol=1e-12)
    got = block.norm(v, block.RMS, gain, None, 1e-5)[0]
    assert torch.allclose(got, torch.nn.functional.rms_norm(v, (37,), gain.double(), 1e-5), atol=1e-12)


@pytest.mark.parametrize("pairing", [block.HALF, block.NEIGHBOURS, block.AXIS])
def test_reference_rotation_by_axes(pairing):
    """Lengths stay; scores of rotated heads depend on the differences of the positions on each axis alone."""
    g = torch.Generator().manual_seed(2)
    axis_of, inv = [0] * 8 + [1] * 16, 100.0 ** -torch.rand(24, generator=g, dtype=torch.float64)
    angle = torch.arange(40, dtype=torch.float64)[:, None] * inv
    table = torch.cat([angle.cos(), angle.sin()], 1)
    q, k = torch.randn((1, 1, 56), generator=g, dtype=torch.float64), torch.randn((1, 1, 56), generator=g, dtype=torch.float64)
    turn = lambda x, *p: block.rope_axes(x, None, table, torch.tensor([p]), axis_of, pairing, False, 0.0)  # noqa: E731
    assert math.isclose(float(turn(q, 3, 9).norm()), float(q.norm()), rel_tol=1e-12)
    a = (turn(q, 3, 9) * turn(k, 7, 2)).sum()
    b = (turn(q, 13, 29) * turn(k, 17, 22)).sum()
    c = (turn(q, 13, 29) * turn(k, 16, 22)).sum()
    assert abs(a - b) <= 1e-12 * abs(a) + 1e-12 and abs(a - c) > 1e-6
    channels = sorted(c for pair in block.channels(axis_of, pairing) for c in pair)
    assert channels == list(range(48))


def _prefix(lib, call="elasto_op_prefix_attention", **kw):
    a = dict(dtype=binding.BF16, batch=2, heads=4, heads_kv=2, head_dim=64, scale=0.125, max_queries=5, q_rows=10, q=P, q_row=256,
             q_head=64, out=2 * P, out_row=256, out_head=64, prefixes=2, seq_start=3 * P, max_prefix=9, prefix_rows=12, prefix_k=4 * P,
             prefix_k_batch=2048, prefix_k_row=128, prefix_k_head=64, prefix_v=5 * P, prefix_v_batch=2048, prefix_v_row=128, prefix_v_head=64,
             max_keys=9, kv_rows=12, k=6 * P, k_batch=2048, k_row=128, k_head=64, v=7 * P, v_batch=2048, v_row=128, v_head=64,
             workspace=8 * P, workspace_bytes=1 << 30) | kw
    return lib.elasto_op_prefix_attention(None, ctypes.byref(binding.PrefixAttention(**a)), None)


SIZES = [dict(dtype=binding.F32), dict(batch=0), dict(heads=0), dict(heads_kv=0), dict(heads_kv=3), dict(max_queries=0), dict(max_prefix=0),
         dict(max_prefix=13), dict(max_keys=-1), dict(max_keys=13), dict(kv_rows=0), dict(q_rows=0), dict(q_rows=(1 << 30) + 1),
         dict(prefix_rows=0), dict(prefix_rows=(1 << 30) + 1), dict(kv_rows=(1 << 30) + 1), dict(prefixes=0), dict(seq_start=None)]


@pytest.mark.parametrize("kw", SIZES + [
    dict(q_rows=9), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=2.4e38), dict(q=None), dict(out=None),
    dict(prefix_k=None), dict(prefix_v=None), dict(k=None), dict(v=None), dict(q=P + 8), dict(out_row=250), dict(prefix_k_row=1),
    dict(prefix_v_batch=4), dict(prefix_k_head=-8), dict(k_batch=1), dict(v_head=-8), dict(kv_start=P, kv_len=P), dict(q_start=P + 1),
    dict(seq_start=P + 2), dict(prefix_len=P + 1), dict(kv_start=P + 2), dict(kv_len=P + 3), dict(workspace=None), dict(workspace=8 * P + 8),
    dict(out=P), dict(out=4 * P), dict(out=5 * P), dict(out=6 * P), dict(out=7 * P), dict(workspace=P), dict(workspace=2 * P),
    dict(workspace=4 * P), dict(workspace=7 * P)])
def test_prefix_attention_refusals(lib, kw):  # noqa: F811
    assert _prefix(lib, **kw) == binding.ERR_INVALID_ARG
    assert "elasto_op_prefix_attention" in binding.elasto_last_error()


@pytest.mark.parametrize("kw", [dict(head_dim=60), dict(head_dim=136), dict(head_dim=0)])
def test_prefix_attention_unsupported(lib, kw):  # noqa: F811
    assert _prefix(lib, **kw) == binding.ERR_UNSUPPORTED
    assert lib.elasto_op_prefix_attention(None, None, None) == binding.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", SIZES)
def test_prefix_workspace_refusals(lib, kw):  # noqa: F811
    a = dict(dtype=binding.BF16, batch=2, heads=4, heads_kv=2, head_dim=64, max_queries=5, q_rows=10, prefixes=2, seq_start=P, max_prefix=9,
             prefix_rows=12, max_keys=9, kv_rows=12) | kw
    n = ctypes.c_size_t()
    assert lib.elasto_op_prefix_attention_workspace(ctypes.byref(binding.PrefixAttention(**a)), ctypes.byref(n)) == binding.ERR_INVALID_ARG
    assert "elasto_op_prefix_attention_workspace" in binding.elasto_last_error()
    assert lib.elasto_op_prefix_attention_workspace(None, ctypes.byref(n)) == binding.ERR_INVALID_ARG


@pytest.mark.parametrize("nq,nk,p", [(1, 5, 7), (4, 4, 3), (6, 2, 5), (3, 0, 4), (2, 1, 0)])
def test_reference_prefix_attention(nq, nk, p):
    """Behind a prefix whose keys are the first of one sequence: torch's own attention with that mask."""
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn((n, h, 8), generator=g, dtype=torch.float64) for n, h in ((nq, 4), (nk, 2), (nk, 2)))
    pk, pv = torch.randn((p, 2, 8), generator=g, dtype=torch.float64), torch.randn((p, 2, 8), generator=g, dtype=torch.float64)
    got, _ = block.prefix_attention(q, k, v, pk, pv, 0.5)
    j = torch.arange(p + nk)
    seen = j[None] <= (p + nk - nq + torch.arange(nq))[:, None]
    seen[:, :p] = True
    kk, vv = torch.cat([pk, k]).repeat_interleave(2, 1), torch.cat([pv, v]).repeat_interleave(2, 1)
    rows = seen.any(1)
    want = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1)[:, rows], kk.transpose(0, 1), vv.transpose(0, 1), seen[rows], scale=0.5)
    assert torch.allclose(got[rows], want.transpose(0, 1), atol=1e-12)
    assert (got[~rows] == 0).all()
