"""elasto_op_qk_norm_rope_axes against its 64-bit definition."""
import ctypes

import pytest
import torch

import block_reference as block
import sublayer_reference as ref
from helpers import stream_handle
from paper_2609_10018_gb300 import binding
from test_gpu_qk_norm_rope import _tol

pytestmark = pytest.mark.gpu
EPS = 1e-6
HALF, NEIGHBOURS, AXIS = block.HALF, block.NEIGHBOURS, block.AXIS


class Case:
    def __init__(self, rows, hq, hk, d, axis_of, pairing, norm=True, dtype=torch.bfloat16, gains=True, n=60, axes=3, by_axis=True, seed=0):
        g = torch.Generator().manual_seed(seed + rows * 31 + d)
        self.rows, self.hq, self.hk, self.d, self.axis_of, self.pairing, self.norm, self.dtype = rows, hq, hk, d, axis_of, pairing, norm, dtype
        self.n, self.axes, self.by_axis = n, axes, by_axis
        self.x = (torch.randn((rows, hq + 2 * hk, d), generator=g) * 2).to(dtype)
        self.gq = torch.randn(d, generator=g) if gains else None
        self.gk = torch.randn(d, generator=g) if gains else None
        inv = 10000.0 ** -torch.rand(len(axis_of), generator=g, dtype=torch.float64)
        angle = torch.arange(n, dtype=torch.float64)[:, None] * inv
        self.table = torch.cat([angle.cos(), angle.sin()], 1).float()
        self.pos = torch.randint(0, n, (rows, axes), generator=g, dtype=torch.int32)

    def want(self):
        q, k, v = self.x.split([self.hq, self.hk, self.hk], 1)
        f = lambda y, gain: block.rope_axes(y, gain, self.table, self.pos, self.axis_of, self.pairing, self.norm, EPS)  # noqa: E731
        return f(q, self.gq), f(k, self.gk), v

    def device(self, v=True, cache=0):
        d = {n: None if t is None else t.cuda() for n, t in (("x", self.x), ("gq", self.gq), ("gk", self.gk), ("table", self.table))}
        d["pos"] = (self.pos.t() if self.by_axis else self.pos).contiguous().cuda()
        d["q_out"] = torch.zeros((self.rows, self.hq, self.d), dtype=self.dtype, device="cuda")
        d["k_out"] = torch.zeros((cache or self.rows, self.hk, self.d), dtype=self.dtype, device="cuda")
        d["v_out"] = torch.zeros((cache or self.rows, self.hk, self.d), dtype=self.dtype, device="cuda") if v else None
        return d

    def args(self, d, **kw):
        row, hd = d["x"].stride(0), d["x"].stride(1)
        at = lambda h: d["x"].data_ptr() + 2 * h * hd  # noqa: E731
        ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        a = dict(dtype=binding.BF16 if self.dtype == torch.bfloat16 else binding.F16, rows=self.rows, heads_q=self.hq, heads_k=self.hk,
                 head_dim=self.d, rot_dim=2 * len(self.axis_of), pairing=self.pairing, norm=int(self.norm), eps=EPS,
                 q=at(0), q_row=row, q_head=hd, k=at(self.hq), k_row=row, k_head=hd, q_gain=ptr(d["gq"]), k_gain=ptr(d["gk"]),
                 cos_sin=ptr(d["table"]), n_positions=self.n, axes=self.axes, axis_of=(ctypes.c_uint8 * len(self.axis_of))(*self.axis_of),
                 positions=ptr(d["pos"]), positions_row=1 if self.by_axis else self.axes, positions_axis=self.rows if self.by_axis else 1)
        for name in ("q_out", "k_out", "v_out"):
            t = d.get(name)
            if t is not None:
                a |= {name: t.data_ptr(), name + "_row": t.stride(0), name + "_head": t.stride(1)}
        if d.get("v_out") is not None:
            a |= dict(v=at(self.hq + self.hk), v_row=row, v_head=hd)
        return binding.QkNormRopeAxes(**(a | kw))

    def near(self, got, want):
        # (the tolerance of the one-axis call; without the norm the largest channel is the head's own)
        big = want.abs().amax(2, keepdim=True)
        err = (got.cpu().double() - want).abs() - _tol(want, big, self.dtype)
        assert (err <= 0).all(), float(err.max())


def _run(args):
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.elasto_op_qk_norm_rope_axes(stream_handle(), args, st.data_ptr())
    return int(st.item())


def runs(*n):
    return [a for a, k in enumerate(n) for _ in range(k)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("rows,hq,hk,d,axis_of,pairing", [
    (1, 1, 1, 16, runs(8), HALF), (7, 3, 3, 64, runs(8, 16, 8), AXIS), (7, 3, 3, 64, runs(0, 16, 16), AXIS), (9, 2, 1, 64, runs(32), AXIS),
    (5, 4, 2, 128, runs(16, 24, 24), HALF), (5, 4, 2, 128, runs(22, 21, 21), NEIGHBOURS), (5, 4, 2, 128, runs(22, 21, 21), HALF),
    (6, 2, 2, 128, [j % 3 for j in range(64)], HALF), (6, 2, 2, 128, [j % 3 for j in range(64)], NEIGHBOURS),
    (4, 12, 12, 80, runs(8, 16, 16), AXIS), (4, 5, 2, 80, runs(3, 5), HALF), (4, 5, 2, 80, runs(3, 5), NEIGHBOURS),
    (3, 2, 1, 256, runs(64, 32, 32), AXIS), (3, 2, 1, 256, runs(1, 126, 1), HALF), (3, 2, 1, 256, runs(1, 126, 1), NEIGHBOURS),
    (3, 2, 1, 8, [], HALF), (11, 4, 0, 24, runs(8), AXIS), (4, 0, 3, 40, runs(4, 4, 8), NEIGHBOURS), (3, 1, 1, 48, [2, 0, 1] * 8, HALF),
    (900, 6, 2, 64, runs(8, 12, 12), HALF), (11000, 2, 1, 32, runs(0, 8, 8), AXIS), (11000, 1, 1, 32, [1, 0, 2, 0] * 4, NEIGHBOURS)])
def test_sizes(rows, hq, hk, d, axis_of, pairing, norm, dtype):
    c = Case(rows, hq, hk, d, axis_of, pairing, norm, dtype, by_axis=rows % 2 == 0)
    t = c.device(v=hk > 0)
    assert _run(c.args(t)) == 0
    q, k, v = c.want()
    c.near(t["q_out"], q)
    c.near(t["k_out"], k)
    if hk:
        assert torch.equal(t["v_out"].cpu(), v)


@pytest.mark.parametrize("interleaved", [False, True])
def test_one_axis_gives_the_bits_of_the_call_for_one(interleaved):
    c = Case(70, 6, 2, 128, runs(48), NEIGHBOURS if interleaved else HALF, axes=1)
    t = c.device()
    assert _run(c.args(t)) == 0
    mine = t["q_out"].clone(), t["k_out"].clone()
    row, hd, at = t["x"].stride(0), t["x"].stride(1), t["x"].data_ptr()
    binding.elasto_op_qk_norm_rope(stream_handle(), binding.QkNormRope(
        dtype=binding.BF16, rows=70, heads_q=6, heads_k=2, head_dim=128, rot_dim=96, interleaved=int(interleaved), eps=EPS,
        q=at, q_row=row, q_head=hd, k=at + 12 * hd, k_row=row, k_head=hd, q_out=t["q_out"].data_ptr(), q_out_row=768, q_out_head=128,
        k_out=t["k_out"].data_ptr(), k_out_row=256, k_out_head=128, q_gain=t["gq"].data_ptr(), k_gain=t["gk"].data_ptr(),
        cos_sin=t["table"].data_ptr(), positions=t["pos"].data_ptr(), n_positions=c.n))
    assert torch.equal(mine[0], t["q_out"]) and torch.equal(mine[1], t["k_out"])


@pytest.mark.parametrize("rows,hq,hk", [(5, 4, 2), (12000, 2, 1)])
def test_positions_and_slots_outside(rows, hq, hk):
    """Rows with a position outside on any axis, or a slot past the cache, are left out; a negative slot stores no keys."""
    c = Case(rows, hq, hk, 64, runs(8, 16, 8), AXIS)
    cache = rows + 4
    slots = torch.randperm(cache, generator=torch.Generator().manual_seed(5))[:rows].to(torch.int32)
    c.pos[1, 2], c.pos[2, 0] = c.n, -1
    slots[3], slots[4] = cache, -7
    t = c.device(cache=cache)
    t["q_out"].fill_(5), t["k_out"].fill_(6), t["v_out"].fill_(7)
    st = _run(c.args(t, slots=(dev := slots.cuda()).data_ptr(), n_slots=cache))
    assert st == binding.ERR_INVALID_ARG and dev is not None
    c.pos[1, 2] = c.pos[2, 0] = 0
    q, k, v = c.want()
    good = torch.tensor([r for r in range(rows) if r not in (1, 2, 3)])
    c.near(t["q_out"][good.cuda()], q[good])
    assert (t["q_out"][1:4] == 5).all()
    stored = torch.tensor([r for r in range(rows) if r not in (1, 2, 3, 4)])
    at = slots[stored].long()
    c.near(t["k_out"][at.cuda()], k[stored])
    assert torch.equal(t["v_out"].cpu()[at], v[stored])
    other = torch.ones(cache, dtype=torch.bool)
    other[at] = False
    assert (t["k_out"].cpu()[other] == 6).all() and (t["v_out"].cpu()[other] == 7).all()


def test_axes_that_turn_nothing_are_checked_too():
    """A position of every axis that the call has must be in the table."""
    c = Case(6, 2, 1, 64, runs(0, 16, 16), HALF)
    c.pos[2, 0] = 99
    t = c.device()
    t["q_out"].fill_(5)
    assert _run(c.args(t)) == binding.ERR_INVALID_ARG
    assert (t["q_out"][2] == 5).all() and not (t["q_out"][3] == 5).all()


@pytest.mark.parametrize("pairing", [HALF, NEIGHBOURS, AXIS])
def test_infinities_without_a_norm(pairing):
    """Channels that do not turn keep their bits, and an infinite one reaches its own pair at most."""
    c = Case(4, 2, 1, 64, runs(8, 8), pairing, norm=False, gains=False)
    c.x[1, 0, 50], c.x[2, 1, 3] = float("inf"), float("nan")
    t = c.device()
    assert _run(c.args(t)) == 0
    got = t["q_out"].cpu()
    assert torch.equal(got[..., 32:], c.x[:, :2, 32:])
    partner = dict(block.channels(c.axis_of, pairing))
    partner |= {b: a for a, b in partner.items()}
    bad = torch.zeros(64, dtype=torch.bool)
    bad[3] = bad[partner[3]] = True
    assert torch.isnan(got[2, 1][bad]).all() and torch.isfinite(got[2, 1][~bad]).all()
    assert torch.isfinite(got[[0, 3]]).all()


def test_in_place():
    c = Case(50, 6, 2, 64, runs(8, 12, 12), HALF)
    t = c.device(v=False)
    assert _run(c.args(t)) == 0
    other = t["q_out"].clone(), t["k_out"].clone()
    x = t["x"]
    t["q_out"], t["k_out"] = x[:, :6], x[:, 6:8]
    assert _run(c.args(t)) == 0
    assert torch.equal(x[:, :6], other[0]) and torch.equal(x[:, 6:8], other[1])
    assert torch.equal(x[:, 8:].cpu(), c.x[:, 8:])


def test_captured():
    """The axes' order is read during the call: the host's array may go before the graph runs."""
    c = Case(40, 4, 4, 128, runs(22, 21, 21), NEIGHBOURS)
    t = c.device()
    assert _run(c.args(t)) == 0
    want = t["q_out"].clone(), t["k_out"].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.elasto_op_qk_norm_rope_axes(stream_handle(), c.args(t))
    t["q_out"].zero_(), t["k_out"].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(t["q_out"], want[0]) and torch.equal(t["k_out"], want[1])
