"""elasto_op_qk_norm_rope against its 64-bit definition."""
import pytest
import torch

import sublayer_reference as ref
from helpers import stream_handle
from paper_2609_10018_gb300 import binding

pytestmark = pytest.mark.gpu
EPS = 1e-6


def _table(n, rot, g):
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))
    angle = torch.arange(n, dtype=torch.float64)[:, None] * inv
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _tol(want, x_norm, dtype):
    """One rounding to the type; before it, in fp32: the sum of squares (256 terms at most, relative 2^-16),
    rsqrt, gain and rotation, within 2^-14 of the head's largest channel."""
    return ref.half_step(dtype) * want.abs() + 2.0 ** -14 * x_norm + torch.finfo(dtype).tiny * 2.0 ** -8


class Case:
    def __init__(self, rows, hq, hk, d, rot, interleaved=False, dtype=torch.bfloat16, gains=True, layout="packed", seed=0):
        g = torch.Generator().manual_seed(seed + rows * 31 + d)
        self.n, self.rows, self.hq, self.hk, self.d, self.rot, self.interleaved, self.dtype = 50, rows, hq, hk, d, rot, interleaved, dtype
        self.x = (torch.randn((rows, hq + 2 * hk, d), generator=g) * 2).to(dtype)
        self.gq = torch.randn(d, generator=g) if gains else None
        self.gk = torch.randn(d, generator=g) if gains else None
        self.table = _table(self.n, rot, g)
        self.pos = torch.randint(0, self.n, (rows,), generator=g, dtype=torch.int32)
        self.layout = layout

    def want(self):
        half = self.rot // 2
        t = self.table[self.pos.long()]
        q, k, v = self.x.split([self.hq, self.hk, self.hk], 1)
        f = lambda y, gain: ref.norm_rope(y, gain, t[:, :half], t[:, half:], EPS, self.interleaved)  # noqa: E731
        return f(q, self.gq), f(k, self.gk), v

    def args(self, d, **kw):
        """d: device tensors x, q_out, k_out, v_out (may be None), table, pos, gq, gk."""
        row, hd = d["x"].stride(0), d["x"].stride(1)
        at = lambda h: d["x"].data_ptr() + 2 * h * hd  # noqa: E731
        ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        a = dict(dtype=binding.BF16 if self.dtype == torch.bfloat16 else binding.F16, rows=self.rows, heads_q=self.hq,
                 heads_k=self.hk, head_dim=self.d, rot_dim=self.rot, interleaved=int(self.interleaved), eps=EPS,
                 q=at(0), q_row=row, q_head=hd, k=at(self.hq), k_row=row, k_head=hd,
                 q_gain=ptr(d["gq"]), k_gain=ptr(d["gk"]), cos_sin=ptr(d["table"]), positions=ptr(d["pos"]), n_positions=self.n)
        for name in ("q_out", "k_out", "v_out"):
            t = d.get(name)
            if t is not None:
                a |= {name: t.data_ptr(), name + "_row": t.stride(0), name + "_head": t.stride(1)}
        if d.get("v_out") is not None:
            a |= dict(v=at(self.hq + self.hk), v_row=row, v_head=hd)
        return binding.QkNormRope(**(a | kw))

    def device(self, v=True):
        d = {n: None if t is None else t.cuda() for n, t in (("x", self.x), ("gq", self.gq), ("gk", self.gk),
                                                             ("table", self.table), ("pos", self.pos))}
        d["q_out"] = torch.zeros((self.rows, self.hq, self.d), dtype=self.dtype, device="cuda")
        d["k_out"] = torch.zeros((self.rows, self.hk, self.d), dtype=self.dtype, device="cuda")
        d["v_out"] = torch.zeros((self.rows, self.hk, self.d), dtype=self.dtype, device="cuda") if v else None
        return d

    def near(self, got, want):
        big = want.abs().amax(2, keepdim=True)
        err = (got.cpu().double() - want).abs()
        assert (err <= _tol(want, big, self.dtype)).all(), float((err - _tol(want, big, self.dtype)).max())


def _run(args):
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.elasto_op_qk_norm_rope(stream_handle(), args, st.data_ptr())
    return int(st.item())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,hq,hk,d,rot", [(1, 1, 1, 16, 16), (3, 2, 1, 8, 0), (7, 3, 3, 64, 64), (5, 12, 12, 64, 32), (4, 5, 2, 80, 80),
                                              (9, 4, 4, 96, 48), (2, 32, 8, 128, 128), (6, 7, 1, 256, 256), (3, 3, 1, 256, 64),
                                              (11, 1, 0, 24, 16), (4, 0, 3, 40, 32), (700, 6, 2, 64, 64), (5000, 2, 1, 32, 32)])
def test_sizes(rows, hq, hk, d, rot, interleaved, dtype):
    c = Case(rows, hq, hk, d, rot, interleaved, dtype)
    t = c.device(v=hk > 0)
    assert _run(c.args(t)) == 0
    q, k, v = c.want()
    c.near(t["q_out"], q)
    c.near(t["k_out"], k)
    if hk:
        assert torch.equal(t["v_out"].cpu(), v)


def test_no_gains_and_no_values():
    c = Case(13, 4, 2, 64, 64, gains=False)
    t = c.device(v=False)
    assert _run(c.args(t)) == 0
    q, k, _ = c.want()
    c.near(t["q_out"], q)
    c.near(t["k_out"], k)


def test_in_place():
    """On the product's own columns: the same bits as into other buffers, the values untouched."""
    c = Case(50, 6, 2, 64, 64)
    t = c.device(v=False)
    assert _run(c.args(t)) == 0
    other = t["q_out"].clone(), t["k_out"].clone()
    x = t["x"]
    t["q_out"], t["k_out"] = x[:, :6], x[:, 6:8]
    assert _run(c.args(t)) == 0
    assert torch.equal(x[:, :6], other[0]) and torch.equal(x[:, 6:8], other[1])
    assert torch.equal(x[:, 8:].cpu(), c.x[:, 8:])


def test_heads_apart():
    """The [head][q | k | v] columns of a shared packed projection, one more column between rows."""
    c = Case(20, 3, 3, 64, 64)
    q, k, v = c.x.split(3, 1)
    both = torch.zeros((20, 3 * 3 * 64 + 8), dtype=c.dtype, device="cuda")
    both[:, :576] = torch.stack([q, k, v], 2).reshape(20, -1).cuda()
    t = c.device()
    at = both.data_ptr()
    strides = {n + f: s for n in "qkv" for f, s in (("_row", 584), ("_head", 192))}
    assert _run(c.args(t, q=at, k=at + 128, v=at + 256, **strides)) == 0
    wq, wk, wv = c.want()
    c.near(t["q_out"], wq)
    c.near(t["k_out"], wk)
    assert torch.equal(t["v_out"].cpu(), wv)


def test_cache_slots():
    """Keys and values at their slots; -1 stores neither, its query is still turned; other rows stay."""
    c = Case(9, 4, 2, 128, 128)
    t = c.device()
    slots = torch.tensor([5, 19, -1, 0, 7, 3, -1, 11, 2], dtype=torch.int32)
    for n in ("k_out", "v_out"):
        t[n] = torch.full((20, 2, 128), 9.0, dtype=c.dtype, device="cuda")
    ds = slots.cuda()
    assert _run(c.args(t, slots=ds.data_ptr(), n_slots=20)) == 0
    q, k, v = c.want()
    c.near(t["q_out"], q)
    stored = slots >= 0
    c.near(t["k_out"][slots[stored].long().cuda()], k[stored])
    assert torch.equal(t["v_out"].cpu()[slots[stored].long()], v[stored])
    rest = [r for r in range(20) if r not in slots.tolist()]
    assert (t["k_out"].cpu()[rest] == 9.0).all() and (t["v_out"].cpu()[rest] == 9.0).all()


@pytest.mark.parametrize("what", ["position", "slot"])
def test_bad_index_leaves_its_row_out(what):
    c = Case(6, 2, 1, 64, 64)
    t = c.device()
    slots = torch.arange(6, dtype=torch.int32)
    if what == "position":
        c.pos[2], c.pos[4] = -1, c.n
    else:
        slots[2], slots[4] = 6, 2 ** 31 - 1
    t["pos"] = c.pos.cuda()
    for n in ("q_out", "k_out", "v_out"):
        t[n].fill_(9.0)
    ds = slots.cuda()
    assert _run(c.args(t, slots=ds.data_ptr(), n_slots=6)) == binding.ERR_INVALID_ARG
    good = [0, 1, 3, 5]
    c.pos.clamp_(0, c.n - 1)
    q, k, v = c.want()
    c.near(t["q_out"][good], q[good])
    c.near(t["k_out"][good], k[good])
    for n in ("q_out", "k_out", "v_out"):
        assert (t[n].cpu()[[2, 4]] == 9.0).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,hq,hk,d,rot", [(20003, 5, 2, 64, 64), (9999, 3, 3, 128, 64), (19999, 1, 1, 40, 32), (40001, 2, 1, 32, 0),
                                              (160001, 1, 1, 8, 0), (80002, 3, 0, 16, 16)])
def test_several_rows_a_warp(rows, hq, hk, d, rot, interleaved):
    """Many rows, the last warps' short of some; every 7th is left out by its slot, and some have bad positions."""
    c = Case(rows, hq, hk, d, rot, interleaved)
    slots = torch.arange(rows, dtype=torch.int32).flip(0)
    slots[::7] = -1
    bad = torch.zeros(rows, dtype=torch.bool)
    if rot:
        bad[[0, 5, rows // 2, rows - 1]] = True
        c.pos[bad] = c.n
    t = c.device(v=hk > 0)
    for n in ("q_out", "k_out", "v_out"):
        if t[n] is not None:
            t[n].fill_(9.0)
    ds = slots.cuda()
    assert _run(c.args(t, slots=ds.data_ptr(), n_slots=rows)) == (binding.ERR_INVALID_ARG if rot else 0)
    c.pos.clamp_(0, c.n - 1)
    q, k, v = c.want()
    got = t["q_out"].cpu()
    c.near(got[~bad], q[~bad])
    assert (got[bad] == 9.0).all()
    if hk:
        there = ~bad & (slots >= 0)
        at = slots[there].long()
        c.near(t["k_out"].cpu()[at], k[there])
        assert torch.equal(t["v_out"].cpu()[at], v[there])
        rest = torch.ones(rows, dtype=torch.bool)
        rest[at] = False
        assert (t["k_out"].cpu()[rest] == 9.0).all() and (t["v_out"].cpu()[rest] == 9.0).all()


def test_zero_and_tiny_rows():
    """A head of zeros gives zeros, one of subnormals stays finite."""
    c = Case(3, 2, 1, 64, 64)
    c.x[0] = 0
    c.x[1] = 1e-39
    t = c.device()
    assert _run(c.args(t)) == 0
    q, k, _ = c.want()
    assert (t["q_out"].cpu()[0] == 0).all() and torch.isfinite(t["q_out"]).all()
    c.near(t["q_out"][1:], q[1:])
    c.near(t["k_out"], k)


def test_graph_replay_reads_new_positions():
    c = Case(8, 2, 1, 64, 64)
    t = c.device()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.elasto_op_qk_norm_rope(torch.cuda.current_stream().cuda_stream, c.args(t), 0)
    for shift in (1, 2):
        c.pos = (c.pos + shift) % c.n
        t["pos"].copy_(c.pos)
        graph.replay()
        torch.cuda.synchronize()
        c.near(t["q_out"], c.want()[0])
