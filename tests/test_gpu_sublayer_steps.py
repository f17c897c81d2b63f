"""The attention sublayer of test_gpu_sublayer.py with buffers of its own: every step against its definition on the
inputs that it got, and the whole captured into graphs and replayed."""
import math

import pytest
import torch

import sublayer_reference as ref
from helpers import stream_handle
from paper_2609_10018_gb300 import binding
from test_gpu_sublayer import CAP, D, D_MODEL, HEADS, HEADS_KV, SINKS, WINDOW, Sublayer

pytestmark = pytest.mark.gpu
COLS = (HEADS + 2 * HEADS_KV) * D


class Prepared(Sublayer):
    """Calls for up to `rows` tokens on buffers that stay; rows past the last sequence have the slot -1."""

    def __init__(self, batch, rows, caches=None):
        super().__init__(batch)
        if caches:
            self.k, self.v = caches.k, caches.v
        dev = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
        self.rows, self.max_q = rows, 1 if rows == batch else rows
        self.x, self.qkv = dev(rows, D_MODEL, dtype=torch.float32), dev(rows, COLS, dtype=torch.bfloat16)
        self.o = dev(rows, HEADS * D, dtype=torch.bfloat16)
        self.x8, self.xs = dev(rows, D_MODEL, dtype=torch.uint8), dev(D_MODEL // 128, rows, dtype=torch.float32)
        self.o8, self.os = dev(rows, HEADS * D, dtype=torch.uint8), dev(HEADS * D // 128, rows, dtype=torch.float32)
        self.positions, self.slots, self.q_start, self.kv_len, self.status = dev(rows), dev(rows), dev(batch + 1), dev(batch), dev(1)

    def tables(self, counts, before):
        """(positions, slots, q_start, kv_len) of counts[b] tokens behind before[b] cached."""
        pad = self.rows - sum(counts)
        pos = [before[b] + i for b in range(self.batch) for i in range(counts[b])]
        slot = [b * CAP + before[b] + i for b in range(self.batch) for i in range(counts[b])]
        t = [pos + [0] * pad, slot + [-1] * pad, [sum(counts[:b]) for b in range(self.batch + 1)], [a + c for a, c in zip(before, counts)]]
        return [torch.tensor(v, dtype=torch.int32).cuda() for v in t]

    def set(self, x, tables):
        """From device memory, in stream order."""
        self.x.copy_(x)
        for d, t in zip((self.positions, self.slots, self.q_start, self.kv_len), tables):
            d.copy_(t)

    def steps(self):
        s, at, n = stream_handle(), self.qkv.data_ptr(), self.rows
        w = {n: (c.data_ptr(), self.scales[n].data_ptr()) for n, c in self.codes.items()}
        yield "x8", lambda: binding.elasto_op_quantize_fp8(s, self.x.data_ptr(), binding.F32, D_MODEL, self.x8.data_ptr(), D_MODEL,
                                                           self.xs.data_ptr(), n, n, D_MODEL)
        yield "qkv", lambda: binding.elasto_op_gemm_fp8(s, self.x8.data_ptr(), D_MODEL, self.xs.data_ptr(), n, w["qkv"][0], D_MODEL,
                                                        w["qkv"][1], None, at, COLS, n, COLS, D_MODEL, binding.EPI_BIAS_BF16,
                                                        self.status.data_ptr())
        yield "rope", lambda: binding.elasto_op_qk_norm_rope(s, binding.QkNormRope(
            dtype=binding.BF16, rows=n, heads_q=HEADS, heads_k=HEADS_KV, head_dim=D, rot_dim=D, eps=1e-6,
            q=at, q_row=COLS, q_head=D, k=at + 2 * HEADS * D, k_row=COLS, k_head=D, v=at + 2 * (HEADS + HEADS_KV) * D, v_row=COLS, v_head=D,
            q_out=at, q_out_row=COLS, q_out_head=D, k_out=self.k.data_ptr(), k_out_row=HEADS_KV * D, k_out_head=D,
            v_out=self.v.data_ptr(), v_out_row=HEADS_KV * D, v_out_head=D, q_gain=self.gain.data_ptr(), k_gain=self.gain.data_ptr(),
            cos_sin=self.table.data_ptr(), positions=self.positions.data_ptr(), n_positions=CAP, slots=self.slots.data_ptr(),
            n_slots=self.batch * CAP), self.status.data_ptr())
        yield "o", lambda: binding.elasto_op_window_attention(s, binding.WindowAttention(
            dtype=binding.BF16, batch=self.batch, heads=HEADS, heads_kv=HEADS_KV, head_dim=D, causal=1, window=WINDOW, sinks=SINKS,
            scale=1 / math.sqrt(D), max_queries=self.max_q, q_rows=n, q_start=self.q_start.data_ptr(), q=at, q_row=COLS, q_head=D,
            out=self.o.data_ptr(), out_row=HEADS * D, out_head=D, max_keys=CAP, kv_rows=CAP, kv_len=self.kv_len.data_ptr(),
            k=self.k.data_ptr(), k_batch=CAP * HEADS_KV * D, k_row=HEADS_KV * D, k_head=D,
            v=self.v.data_ptr(), v_batch=CAP * HEADS_KV * D, v_row=HEADS_KV * D, v_head=D), self.status.data_ptr())
        yield "o8", lambda: binding.elasto_op_quantize_fp8(s, self.o.data_ptr(), binding.BF16, HEADS * D, self.o8.data_ptr(), HEADS * D,
                                                           self.os.data_ptr(), n, n, HEADS * D)
        yield "x", lambda: binding.elasto_op_gemm_fp8(s, self.o8.data_ptr(), HEADS * D, self.os.data_ptr(), n, w["out"][0], HEADS * D,
                                                      w["out"][1], None, self.x.data_ptr(), D_MODEL, n, D_MODEL, HEADS * D,
                                                      binding.EPI_BIAS_RESID_F32, self.status.data_ptr())

    def run(self):
        for _, call in self.steps():
            call()

    def capture(self):
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            self.run()
        return graph


def _random(rows, seed):
    return torch.randn((rows, D_MODEL), generator=torch.Generator().manual_seed(seed))


def _close(got, want, tol):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (bad.nonzero()[:4].tolist(), float((got.double() - want).abs().max()))


def _check_product(sub, name, codes, scales, got, start=None):
    """The bound of test_gpu_gemm_fp8.py: one rounding for each product, three for each block."""
    f8 = lambda t: t.cpu().view(torch.float8_e4m3fn)  # noqa: E731
    acc, mag = ref.gemm_fp8(f8(codes), scales.cpu(), f8(sub.codes[name].view(torch.uint8)), sub.scales[name].cpu(), codes.shape[1])
    if start is not None:
        acc, mag = acc + start.double(), mag + start.double().abs()
    k, u = codes.shape[1], ref.half_step(got.dtype)
    tol = (k + 3 * ref.blocks(k) + 4) * 2.0 ** -24 * mag
    _close(got.cpu(), acc, tol * (1 + u) + u * acc.abs() if got.dtype == torch.bfloat16 else tol)


def _check_steps(sub, x, counts, before):
    """One pass, each step's result against 64 bits of what it read."""
    n = sum(counts)
    sub.o.fill_(0.0)
    sub.set(x.cuda(), sub.tables(counts, before))
    got = {}
    for name, call in sub.steps():
        call()
        got[name] = {t: getattr(sub, t).clone() for t in ("x8", "xs", "qkv", "k", "v", "o", "o8", "os", "x")}
    assert int(sub.status.item()) == 0
    codes, scales = ref.quantize(x)
    assert torch.equal(got["x8"]["x8"].cpu(), codes.view(torch.uint8)) and torch.equal(got["x8"]["xs"].cpu(), scales)
    _check_product(sub, "qkv", got["x8"]["x8"], got["x8"]["xs"], got["qkv"]["qkv"])
    u = ref.half_step(torch.bfloat16)
    qkv, turned = got["qkv"]["qkv"].cpu()[:n].view(n, -1, D), got["rope"]["qkv"].cpu()[:n].view(n, -1, D)
    angles = sub.table.cpu()[sub.positions.cpu()[:n].long()]
    want = ref.norm_rope(qkv[:, :HEADS + HEADS_KV], sub.gain.cpu(), angles[:, :D // 2], angles[:, D // 2:], 1e-6, False)
    slots = sub.slots.cpu()[:n].long()
    k, v = (got["rope"][t].view(-1, HEADS_KV, D).cpu() for t in "kv")
    # fp32 throughout: D products and sums of the norm, the root (2 ulp), six more operations; then one rounding
    tol = u * want.abs() + (D / 2 + 10) * 2.0 ** -24 * (want.abs() + 8.0)
    _close(turned[:, :HEADS], want[:, :HEADS], tol[:, :HEADS])
    _close(k[slots], want[:, HEADS:], tol[:, HEADS:])
    assert torch.equal(v[slots], qkv[:, HEADS + HEADS_KV:])
    row = 0
    for b, c in enumerate(counts):
        q, nk = turned[row:row + c, :HEADS], before[b] + c
        keys, values = (got["rope"][t][b, :nk].cpu() for t in "kv")
        want, mean = ref.attention(q, keys, values, 1 / math.sqrt(D), True, WINDOW, SINKS)
        _close(got["o"]["o"][row:row + c].cpu().view(c, HEADS, D), want, u * want.abs() + (1.01 * u + 5e-4) * mean + 2.0 ** -24)
        row += c
    codes, scales = ref.quantize(got["o"]["o"].cpu())
    assert torch.equal(got["o8"]["o8"].cpu(), codes.view(torch.uint8)) and torch.equal(got["o8"]["os"].cpu(), scales)
    _check_product(sub, "out", got["o8"]["o8"], got["o8"]["os"], got["x"]["x"], x)


def test_every_step_against_its_definition():
    prompt = Prepared(2, 127)
    _check_steps(prompt, _random(127, 3), [50, 77], [0, 0])
    token = Prepared(2, 2, prompt)
    for t in range(3):
        _check_steps(token, _random(2, 4 + t), [1, 1], [50 + t, 77 + t])
    _check_steps(prompt, _random(127, 8), [20, 40], [53, 80])  # a chunk behind the cache, and rows of no sequence


def test_captured_chain_replayed():
    """A prompt's graph and a single token's, replayed one behind the other without waiting, on new tokens, lengths and
    slots: the bits of the same calls made one by one."""
    rows, plan = 130, []
    for r, counts in enumerate([[50, 77], [100, 30], [1, 64]]):
        plan.append((rows, _random(rows, 20 + r), counts, [0, 0]))
        for t in range(6):
            plan.append((2, _random(2, 40 + 10 * r + t), [1, 1], [c + t for c in counts]))

    def outputs(captured):
        prompt = Prepared(2, rows)
        token = Prepared(2, 2, prompt)
        subs = {rows: prompt, 2: token}
        inputs = [(n, x.cuda(), subs[n].tables(counts, before)) for n, x, counts, before in plan]
        graphs = {}
        if captured:  # with tables of rows of no sequence
            for n, sub in subs.items():
                sub.set(torch.zeros_like(sub.x), sub.tables([0, 0], [0, 0]))
                graphs[n] = sub.capture()
        results = []
        for n, x, tables in inputs:
            sub = subs[n]
            sub.o.fill_(0.0)
            sub.set(x, tables)
            graphs[n].replay() if captured else sub.run()
            results.append((sub.x.clone(), sub.o.clone()))
        torch.cuda.synchronize()
        assert int(prompt.status.item()) == 0 and int(token.status.item()) == 0
        return [t.cpu() for pair in results for t in pair] + [prompt.k.cpu(), prompt.v.cpu()]

    eager = outputs(False)
    for got, want in zip(outputs(True), eager):
        assert torch.equal(got, want)
    for (n, x, counts, _), got in zip(plan, eager[::2]):
        assert got.isfinite().all() and not torch.equal(got[:sum(counts)], x[:sum(counts)])
