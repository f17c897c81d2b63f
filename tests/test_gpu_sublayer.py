"""The calls for long sequences together, as one attention sublayer uses them: e4m3 rows -> QKV product ->
norms and rotation (keys and values into a cache) -> windowed attention -> e4m3 rows -> output product."""
import math

import pytest
import torch

import sublayer_reference as ref
from helpers import stream_handle
from paper_2609_10018_gb300 import binding

pytestmark = pytest.mark.gpu
D_MODEL, HEADS, HEADS_KV, D, WINDOW, SINKS, CAP = 256, 4, 2, 64, 30, 2, 128


class Sublayer:
    """Weights and buffers of a user's program; lens: tokens already in each sequence's cache."""

    def __init__(self, batch):
        g = torch.Generator().manual_seed(5)
        self.batch, cols = batch, (HEADS + 2 * HEADS_KV) * D
        self.w = {n: torch.randn(s, generator=g) / math.sqrt(s[1]) for n, s in (("qkv", (cols, D_MODEL)), ("out", (D_MODEL, HEADS * D)))}
        self.codes, self.scales = {}, {}
        for n, w in self.w.items():
            q, s = ref.quantize(w)  # [n, k] with a scale a row; take one for each 128 rows
            s = s.t().reshape(ref.blocks(w.shape[0]), 128, -1).amax(1)
            self.codes[n] = (w / s.repeat_interleave(128, 0).repeat_interleave(128, 1)).to(torch.float8_e4m3fn).cuda()
            self.scales[n] = s.contiguous().cuda()
        inv = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
        angle = torch.arange(CAP, dtype=torch.float64)[:, None] * inv
        self.table = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
        self.gain = (1 + 0.2 * torch.randn(D, generator=g)).cuda()
        self.k = torch.zeros((batch, CAP, HEADS_KV, D), dtype=torch.bfloat16, device="cuda")
        self.v = torch.zeros_like(self.k)

    def project(self, name, x, out, epilogue):
        rows, cols = x.shape
        q = torch.empty((rows, cols), dtype=torch.uint8, device="cuda")
        scale = torch.empty((cols // 128, rows), device="cuda")
        s, w = stream_handle(), self.codes[name]
        binding.elasto_op_quantize_fp8(s, x.data_ptr(), binding.F32 if x.dtype == torch.float32 else binding.BF16, cols,
                                       q.data_ptr(), cols, scale.data_ptr(), rows, rows, cols)
        binding.elasto_op_gemm_fp8(s, q.data_ptr(), cols, scale.data_ptr(), rows, w.data_ptr(), cols, self.scales[name].data_ptr(),
                                   None, out.data_ptr(), out.shape[1], rows, w.shape[0], cols, epilogue)

    def step(self, x, counts, before):
        """x fp32 [sum(counts), D_MODEL], updated in place: counts[b] new tokens of sequence b behind before[b] cached."""
        rows = x.shape[0]
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        positions = i32([before[b] + i for b in range(self.batch) for i in range(counts[b])])
        slots = i32([b * CAP + before[b] + i for b in range(self.batch) for i in range(counts[b])])
        q_start = i32([sum(counts[:b]) for b in range(self.batch + 1)])
        kv_len = i32([a + c for a, c in zip(before, counts)])
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        cols = (HEADS + 2 * HEADS_KV) * D
        qkv = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
        o = torch.empty((rows, HEADS * D), dtype=torch.bfloat16, device="cuda")
        self.project("qkv", x, qkv, binding.EPI_BIAS_BF16)
        at, cache = qkv.data_ptr(), dict(row=HEADS_KV * D)
        binding.elasto_op_qk_norm_rope(stream_handle(), binding.QkNormRope(
            dtype=binding.BF16, rows=rows, heads_q=HEADS, heads_k=HEADS_KV, head_dim=D, rot_dim=D, eps=1e-6,
            q=at, q_row=cols, q_head=D, k=at + 2 * HEADS * D, k_row=cols, k_head=D,
            v=at + 2 * (HEADS + HEADS_KV) * D, v_row=cols, v_head=D, q_out=at, q_out_row=cols, q_out_head=D,
            k_out=self.k.data_ptr(), k_out_row=cache["row"], k_out_head=D, v_out=self.v.data_ptr(), v_out_row=cache["row"],
            v_out_head=D, q_gain=self.gain.data_ptr(), k_gain=self.gain.data_ptr(), cos_sin=self.table.data_ptr(),
            positions=positions.data_ptr(), n_positions=CAP, slots=slots.data_ptr(), n_slots=self.batch * CAP), st.data_ptr())
        binding.elasto_op_window_attention(stream_handle(), binding.WindowAttention(
            dtype=binding.BF16, batch=self.batch, heads=HEADS, heads_kv=HEADS_KV, head_dim=D, causal=1, window=WINDOW, sinks=SINKS,
            scale=1 / math.sqrt(D), max_queries=max(counts), q_rows=rows, q_start=q_start.data_ptr(), q=at, q_row=cols, q_head=D,
            out=o.data_ptr(), out_row=HEADS * D, out_head=D, max_keys=CAP, kv_rows=CAP, kv_len=kv_len.data_ptr(),
            k=self.k.data_ptr(), k_batch=CAP * HEADS_KV * D, k_row=HEADS_KV * D, k_head=D,
            v=self.v.data_ptr(), v_batch=CAP * HEADS_KV * D, v_row=HEADS_KV * D, v_head=D), st.data_ptr())
        self.project("out", o, x, binding.EPI_BIAS_RESID_F32)
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        return x


def _reference(sub, x):
    """One whole sequence in 64 bits with the dequantised weights; activations are not rounded."""
    w = {n: sub.codes[n].cpu().double() * sub.scales[n].cpu().double().repeat_interleave(128, 0).repeat_interleave(128, 1)
         for n in sub.w}
    n = x.shape[0]
    qkv = (x.double() @ w["qkv"].t()).view(n, -1, D)
    t = sub.table[:n].cpu()
    gain = sub.gain.cpu()
    q = ref.norm_rope(qkv[:, :HEADS], gain, t[:, :D // 2], t[:, D // 2:], 1e-6, False)
    k = ref.norm_rope(qkv[:, HEADS:HEADS + HEADS_KV], gain, t[:, :D // 2], t[:, D // 2:], 1e-6, False)
    o, _ = ref.attention(q, k, qkv[:, HEADS + HEADS_KV:], 1 / math.sqrt(D), True, WINDOW, SINKS)
    return x.double() + o.reshape(n, -1) @ w["out"].t()


def test_sublayer_prefill_then_single_tokens():
    """Prefill of ragged sequences, then their tokens one at a time through the cache: the same rows as the
    whole sequences at once. Against 64 bits: two roundings to e4m3 (2^-4 a value, independent, so about
    2^-4 / sqrt(3) of the added term's norm each, and the scores' change of the same order): within
    a fifth of its norm."""
    g = torch.Generator().manual_seed(8)
    lens = [50, 77]
    x = [torch.randn((n, D_MODEL), generator=g) for n in lens]
    whole = Sublayer(2)
    at_once = whole.step(torch.cat(x).cuda(), lens, [0, 0]).cpu()
    steps = Sublayer(2)
    first = [30, 57]
    got = steps.step(torch.cat([a[:f] for a, f in zip(x, first)]).cuda(), first, [0, 0]).cpu()
    rows = [list(got[:30]), list(got[30:])]
    for t in range(20):
        y = steps.step(torch.stack([a[f + t] for a, f in zip(x, first)]).cuda(), [1, 1], [f + t for f in first]).cpu()
        for b in range(2):
            rows[b].append(y[b])
    step_by_step = torch.cat([torch.stack(r) for r in rows])
    # the cache holds the same values; the attention's sums may differ by fp32 roundings, which move a
    # bf16 rounding, and that one of e4m3, at most here and there
    x_all = torch.cat(x)
    added = (at_once - x_all).norm()
    assert (step_by_step - at_once).norm() <= 2.0 ** -6 * added
    want = torch.cat([_reference(whole, a) for a in x])
    assert (at_once.double() - want).norm() <= 0.2 * (want - x_all.double()).norm()
