"""elasto_op_window_attention against its 64-bit definition."""
import math

import pytest
import torch

import sublayer_reference as ref
from helpers import stream_handle
from paper_2609_10018_gb300 import binding

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


class Case:
    """Sequences of the given lengths; packed, or in caches of `room` rows more than the longest."""

    def __init__(self, nq, nk, heads=2, heads_kv=2, d=64, causal=True, window=-1, sinks=0, packed=True, dtype=torch.bfloat16,
                 room=0, tail=0, seed=0, gap=0):
        g = torch.Generator().manual_seed(seed + 1000 * sum(nq) + sum(nk) + d)
        self.nq, self.nk, self.h, self.hk, self.d = list(nq), list(nk), heads, heads_kv, d
        self.causal, self.window, self.sinks, self.packed, self.dtype = causal, window, sinks, packed, dtype
        self.scale = 1 / math.sqrt(d)
        rand = lambda *s: torch.randn(s, generator=g).to(dtype)  # noqa: E731
        self.cap = max(max(nk), 1) + room
        self.q = rand(sum(nq) + tail, heads, d + gap)[..., :d]
        shape = (sum(nk) + room + 1, heads_kv) if packed else (len(nk), self.cap, heads_kv)
        self.k, self.v = rand(*shape, d + gap)[..., :d], rand(*shape, d + gap)[..., :d]
        self.max_q, self.max_k = max(max(nq), 1), max(max(nk), 1)

    def sequence(self, b):
        q0 = sum(self.nq[:b])
        q = self.q[q0:q0 + self.nq[b]]
        if self.packed:
            k0 = sum(self.nk[:b])
            return q, self.k[k0:k0 + self.nk[b]], self.v[k0:k0 + self.nk[b]]
        return q, self.k[b, :self.nk[b]], self.v[b, :self.nk[b]]

    def starts(self, n):
        return torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device="cuda")

    def device(self):
        dev = lambda t: torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda").copy_(t)  # noqa: E731
        self.dq, self.dk, self.dv = dev(self.q), dev(self.k), dev(self.v)
        self.out = torch.full((self.q.shape[0], self.h, self.d), 9.0, dtype=self.dtype, device="cuda")
        self.q_start = self.starts(self.nq)
        self.kv_start = self.starts(self.nk)
        self.kv_len = torch.tensor(self.nk, dtype=torch.int32, device="cuda")
        return self

    def args(self, **kw):
        q, k, v, out = self.dq, self.dk, self.dv, self.out
        a = dict(dtype=binding.BF16 if self.dtype == torch.bfloat16 else binding.F16, batch=len(self.nq), heads=self.h,
                 heads_kv=self.hk, head_dim=self.d, causal=int(self.causal), window=self.window, sinks=self.sinks,
                 scale=self.scale, max_queries=self.max_q, q_rows=q.shape[0], q_start=self.q_start.data_ptr(),
                 q=q.data_ptr(), q_row=q.stride(0), q_head=q.stride(1),
                 out=out.data_ptr(), out_row=out.stride(0), out_head=out.stride(1),
                 max_keys=self.max_k, kv_rows=k.shape[0] if self.packed else self.cap,
                 kv_start=self.kv_start.data_ptr() if self.packed else None,
                 kv_len=None if self.packed else self.kv_len.data_ptr(),
                 k=k.data_ptr(), k_batch=0 if self.packed else k.stride(0), k_row=k.stride(-3), k_head=k.stride(-2),
                 v=v.data_ptr(), v_batch=0 if self.packed else v.stride(0), v_row=v.stride(-3), v_head=v.stride(-2))
        return binding.WindowAttention(**(a | kw))

    def run(self, **kw):
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        binding.elasto_op_window_attention(stream_handle(), self.args(**kw), st.data_ptr())
        assert int(st.item()) == 0
        return self.out.cpu()

    def want(self, b):
        q, k, v = self.sequence(b)
        return ref.attention(q, k, v, self.scale, self.causal, self.window, self.sinks)

    def check(self, got=None):
        """Probabilities and the result are rounded to the type (half a step of each term, and of the
        result); fp32 scores of |q . k| scale <= 32 are off by less than 2^-24 * 128 * 32, which is 2.5e-4
        of a probability, and as much again comes from the sum of up to 2^12 of them."""
        got = self.device().run() if got is None else got
        u = ref.half_step(self.dtype)
        for b in range(len(self.nq)):
            want, mean = self.want(b)
            q0 = sum(self.nq[:b])
            g = got[q0:q0 + self.nq[b]].double()
            fine = want.isfinite()
            assert torch.equal(fine, g.isfinite()), "sequence %d" % b
            tol = u * want.abs() + (1.01 * u + 5e-4) * mean + 2.0 ** -24
            bad = ~(((g - want).abs() <= tol) | ~fine)
            assert not bad.any(), (b, bad.nonzero()[:4].tolist(), float((g - want).abs()[fine].max()))
        assert (got[sum(self.nq):] == 9.0).all()  # rows of no sequence


LENGTHS = [1, 2, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511, 640]


@pytest.mark.parametrize("n", LENGTHS)
@pytest.mark.parametrize("causal,window,sinks", [(True, -1, 0), (True, 40, 3), (False, -1, 0), (False, 50, 1), (True, 0, 0),
                                                 (False, 0, 2), (True, 200, 130)])
def test_whole_sequences(n, causal, window, sinks):
    Case([n], [n], causal=causal, window=window, sinks=sinks, tail=3).check()


@pytest.mark.parametrize("d", [8, 16, 40, 64, 72, 80, 96, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,heads_kv", [(1, 1), (4, 1), (6, 2), (3, 3), (14, 2)])
def test_heads_and_types(d, dtype, heads, heads_kv):
    Case([150, 33], [150, 33], heads, heads_kv, d, window=60, sinks=2, dtype=dtype).check()
    Case([1, 1, 1], [150, 33, 1], heads, heads_kv, d, window=60, sinks=2, dtype=dtype, packed=False, room=5).check()


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("causal", [True, False])
def test_ragged_lengths(packed, causal):
    """Empty sequences, queries without keys, more queries than keys (the first see nothing)."""
    Case([5, 0, 130, 1, 7, 300, 3, 64], [9, 4, 130, 200, 0, 290, 1, 700], 4, 2, causal=causal, window=70, sinks=2, packed=packed,
         room=9, tail=5).check()


@pytest.mark.parametrize("nq", [2, 3, 5, 16, 31, 64, 100])
@pytest.mark.parametrize("heads,heads_kv,d", [(8, 2, 128), (5, 1, 64), (16, 1, 64), (34, 2, 64), (2, 2, 128)])
def test_chunks_behind_a_cache(nq, heads, heads_kv, d):
    Case([nq, max(1, nq - 1)], [517, 300], heads, heads_kv, d, window=129, sinks=5, packed=False, room=30).check()
    Case([nq], [400], heads, heads_kv, d, packed=False).check()


@pytest.mark.parametrize("nq,nk,heads,heads_kv,d", [(2, 5000, 1, 1, 64), (33, 3001, 8, 2, 128), (7, 2049, 6, 1, 96), (128, 4100, 2, 2, 64),
                                                    (300, 1300, 2, 1, 128), (16, 1024, 24, 1, 40)])
def test_few_queries_many_keys(nq, nk, heads, heads_kv, d):
    """Items that several CTAs share."""
    Case([nq], [nk], heads, heads_kv, d, packed=False, room=3, tail=2).check()
    Case([nq, max(1, nq // 2), 1], [nk, nk // 3, 1], heads, heads_kv, d, window=nk // 2, sinks=70, packed=False).check()
    Case([nq, 0, nq], [nk - 5, 9, nq // 2], heads, heads_kv, d, window=900, sinks=3, packed=False, dtype=torch.float16).check()
    Case([nq], [nk], heads, heads_kv, d, causal=False, window=700, sinks=0).check()


@pytest.mark.parametrize("at", [0, 700, 1999])
def test_bad_value_with_few_queries(at):
    c = Case([20], [2000], 2, 1, 64, window=1400, sinks=1, packed=False)
    c.v[0, at, 0, 5], c.v[0, 650, 0, 7] = INF, -INF
    c.v[0, 1990, 0, 9] = NAN
    c.check()


@pytest.mark.parametrize("nk", [1, 2, 15, 16, 17, 63, 64, 65, 128, 200, 513, 1000, 2047])
@pytest.mark.parametrize("window,sinks", [(-1, 0), (0, 0), (0, 3), (63, 4), (500, 0), (100, 300)])
def test_single_tokens(nk, window, sinks):
    Case([1], [nk], 8, 2, 64, window=window, sinks=sinks, packed=False, room=7).check()
    Case([1, 1, 0, 1], [nk, max(1, nk // 3), 5, 0], 3, 3, 128, window=window, sinks=sinks, packed=False, room=70, tail=2).check()


@pytest.mark.parametrize("heads,heads_kv", [(1, 1), (7, 1), (16, 1), (24, 1), (40, 1), (64, 2), (33, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_single_tokens_head_groups(heads, heads_kv, causal):
    Case([1, 1], [300, 77], heads, heads_kv, 64, causal=causal, window=90, sinks=2, packed=False).check()
    Case([1, 1], [300, 77], heads, heads_kv, 96, causal=causal, window=90, sinks=2).check()


@pytest.mark.parametrize("batch,nk,heads,heads_kv", [(1, 9000, 2, 1), (3, 5000, 4, 4), (40, 600, 8, 8), (1, 20000, 8, 1)])
def test_single_tokens_long(batch, nk, heads, heads_kv):
    lens = [max(1, nk - 331 * i) for i in range(batch)]
    Case([1] * batch, lens, heads, heads_kv, 64, packed=False).check()
    Case([1] * batch, lens, heads, heads_kv, 128, window=4000, sinks=4, packed=False).check()


def test_many_short_sequences():
    n = [1 + (7 * i) % 20 for i in range(300)]
    Case(n, n, 2, 1, 32, window=6, sinks=1, dtype=torch.float16).check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,causal,window,sinks", [(257, True, 100, 0), (257, False, 100, 0), (700, False, 20, 1), (129, True, -1, 3),
                                                   (513, True, 30, 40)])
def test_many_items_with_uneven_tiles(n, causal, window, sinks, d):
    """More work items than SMs, one of whose two tiles has few rows, none, or far fewer keys than the other."""
    lens = [n - (i % 3) for i in range(48)]
    Case(lens, lens, 4, 4, d, causal=causal, window=window, sinks=sinks).check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window,sinks", [(255, 1), (224, 32), (300, 33), (199, 64), (130, 96), (160, 97), (270, 4), (31, 5)])
@pytest.mark.parametrize("heads,heads_kv,batch", [(2, 2, 1), (8, 2, 1), (8, 8, 12)])
def test_first_keys_far_from_the_window(causal, window, sinks, heads, heads_kv, batch):
    """The first keys stand alone or in front of the window's, with every remainder of its length."""
    lens = [730 - 41 * i for i in range(batch)]
    Case(lens, lens, heads, heads_kv, 64, causal=causal, window=window, sinks=sinks).check()


@pytest.mark.parametrize("nq,nk", [(700, 700), (650, 652), (640, 740), (700, 650), (700, 300), (129, 1000)])
@pytest.mark.parametrize("sinks", [1, 3, 60, 150])
@pytest.mark.parametrize("heads,heads_kv,batch,d", [(2, 2, 1, 64), (6, 6, 9, 64), (12, 3, 14, 128), (14, 2, 3, 96)])
def test_queries_that_see_everything(nq, nk, sinks, heads, heads_kv, batch, d):
    """Both directions: the first queries see all keys, the others a window; keys and queries of different numbers."""
    nq, nk = [nq - 9 * i for i in range(batch)], [nk - 9 * i for i in range(batch)]
    nq[-1] = nk[-1] = max(1, nk[-1] // 7)  # a short one among them
    Case(nq, nk, heads, heads_kv, d, causal=False, window=25, sinks=sinks, packed=batch % 2 == 1).check()


@pytest.mark.parametrize("value", [NAN, INF])
@pytest.mark.parametrize("at", [0, 2, 5, 130, 500, 639, 640, 676])
@pytest.mark.parametrize("causal", [True, False])
def test_bad_value_in_many_items(value, at, causal):
    """As below, where the first keys share a tile with the window's and queries that see everything share their keys."""
    c = Case([677] * 7, [677] * 7, 6, 6, 64, causal=causal, window=40, sinks=3)
    c.v[2 * 677 + at, 1, 5] = value
    c.check()


@pytest.mark.parametrize("causal", [True, False])
def test_hidden_keys_beside_the_first(causal):
    """NaN in keys and values right behind the first ones, which share a load with them."""
    c = Case([300] * 3, [900] * 3, 8, 8, 128, causal=causal, window=40, sinks=3)
    for b in range(3):
        c.k[900 * b + 3:900 * b + 500] = NAN
        c.v[900 * b + 3:900 * b + 500] = NAN
    c.check()


def test_long_sequence():
    Case([2900], [2900], 2, 1, 128, window=300, sinks=4).check()
    Case([1500], [1500], 1, 1, 64, causal=False, window=100, sinks=1).check()
    Case([1300], [2800], 3, 1, 64).check()


@pytest.mark.parametrize("nq,nk", [(200, 200), (1, 300), (3, 300)])
@pytest.mark.parametrize("value", [NAN, INF])
def test_hidden_garbage(nq, nk, value):
    """NaN and infinities where no query looks: past the lengths, behind the window, in the neighbours."""
    c = Case([nq, nq], [nk, nk - 40], 4, 2, 64, window=50, sinks=2, packed=False, room=90)
    low = max(2, nk - nq - 50)  # the first key in the window of the first query
    for b, n in enumerate(c.nk):
        lo = max(2, n - nq - 50)
        for t in (c.k, c.v):
            t[b, n:] = value
            t[b, 2:lo] = value
    assert low >= 2
    c.check()
    c = Case([nq, nq], [nk, nk], 2, 2, 128, window=50, sinks=0)
    c.k[2 * nk:], c.v[2 * nk:] = value, value
    c.check()


@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("at", [0, 77, 150, 199])
def test_bad_value_reaches_only_who_sees_it(value, d, causal, at):
    """One NaN or infinite value: the queries that see its key get it, the others do not."""
    c = Case([200], [200], 4, 2, d, causal=causal, window=30, sinks=1)
    c.v[at, 1, 5] = value
    got = c.device().run()
    want, _ = c.want(0)
    fine = want.isfinite()
    assert (~fine).any() and torch.equal(got.isfinite(), fine)
    c.check(got)
    if not math.isnan(value):
        assert torch.equal(got.double()[~fine], want[~fine])


@pytest.mark.parametrize("causal", [True, False])
def test_bad_key_reaches_only_who_sees_it(causal):
    c = Case([200], [200], 4, 2, 64, causal=causal, window=30, sinks=1)
    c.k[120, 0, 3] = NAN
    got = c.device().run()
    seen = ref.visible(200, 200, causal, 30, 1)[:, 120]
    assert got[seen][:, :2].isnan().all() and got[~seen].isfinite().all() and got[:, 2:].isfinite().all()


def test_large_scores():
    """Scores far apart: a softmax that is all on one key, and equal scores."""
    c = Case([130], [130], 2, 1, 64, window=-1)
    c.q.mul_(0)
    c.check()
    c = Case([130], [130], 2, 1, 64, window=40, sinks=1)
    c.k.mul_(0)
    c.k[:, :, 0] = (torch.arange(c.k.shape[0]) % 50)[:, None].to(c.dtype) * 4
    c.q.mul_(0)
    c.q[:, :, 0] = 16.0
    c.check()
    c.q.neg_()
    c.check()


def test_lengths_past_the_limits_are_cut():
    """Lengths on the device past what the host said: cut, nothing outside is touched."""
    c = Case([60], [90], 2, 1, 64, packed=False, room=10, tail=4).device()
    c.kv_len.fill_(5000)
    got = c.run()
    full = Case([60], [90], 2, 1, 64, packed=False, room=10, tail=4)
    full.check(got)
    c.kv_len.fill_(-7)
    assert (c.run()[:60] == 0).all()
    c.q_start.copy_(torch.tensor([-5, 1 << 30]))  # 64 rows, of which max_queries are computed
    c.kv_len.fill_(90)
    c.out.fill_(9.0)
    got = c.run()
    assert torch.equal(got[:60], full.device().run()[:60]) and (got[60:] == 9.0).all()


def test_equal_lengths_without_device_tables():
    c = Case([40, 40, 40], [70, 70, 70], 4, 2, 64, window=25, packed=False, room=3).device()
    a = c.run()
    c.out.fill_(9.0)
    assert torch.equal(c.run(q_start=None, kv_len=None), a)
    c.check(a)


def test_strides():
    """q, k and v as columns of one product's output, and wider rows than the heads take."""
    c = Case([100, 60], [100, 60], 4, 2, 64, window=33, sinks=1)
    qkv = torch.zeros((161, 8 * 64 + 24), dtype=c.dtype, device="cuda")
    parts = [qkv[:, 64 * a:64 * b].unflatten(1, (-1, 64)) for a, b in ((0, 4), (4, 6), (6, 8))]
    c.device()
    for part, t in zip(parts, (c.q, c.k, c.v)):
        part[:t.shape[0]].copy_(t)
    c.dq, c.dk, c.dv = parts[0][:160], parts[1], parts[2]
    c.check(c.run())
    Case([70], [70], 3, 1, 40, window=20, gap=24).check()
    Case([1, 1], [70, 50], 3, 1, 40, window=20, gap=24, packed=False).check()


def test_one_query_in_both_forms():
    """A single token through the single-token form and as one row of the general one."""
    c = Case([1, 1], [400, 222], 8, 2, 128, window=150, sinks=3, packed=False)
    one = c.device().run()
    c.check(one)
    c.out.fill_(9.0)
    c.check(c.run(max_queries=2))


def test_cache_past_32_bits():
    """A cache whose last rows are more than 2^31 values (4 GiB) from its start."""
    rows, d = 70000, 64
    heads_kv = 512  # 70000 * 512 * 64 = 2.3e9 values; two heads hold data
    k = torch.zeros((rows, heads_kv, d), dtype=torch.float16, device="cuda")
    v = torch.zeros((rows, heads_kv, d), dtype=torch.float16, device="cuda")
    for nq in (1, 5):
        c = Case([nq], [rows], 1, 1, d, window=300, sinks=4, packed=False, dtype=torch.float16)
        c.device()
        k[:, 511], v[:, 511] = c.dk[0, :, 0], c.dv[0, :, 0]
        got = c.run(k=k[:, 511:].data_ptr(), v=v[:, 511:].data_ptr(), k_row=heads_kv * d, v_row=heads_kv * d)
        c.check(got)


@pytest.mark.parametrize("nq", [1, 150])
def test_same_result_every_call_and_streams(nq):
    """The same bits again, on two streams at once, and from a replayed graph with new lengths."""
    c = Case([nq, nq], [400, 333], 8, 2, 64, window=200, sinks=2, packed=False).device()
    first = c.run()
    other = torch.zeros_like(c.out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for s, o in zip(streams, (c.out, other)):
            binding.elasto_op_window_attention(s.cuda_stream, c.args(out=o.data_ptr()), 0)
    torch.cuda.synchronize()
    assert torch.equal(c.out.cpu(), first) and torch.equal(other.cpu(), first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.elasto_op_window_attention(torch.cuda.current_stream().cuda_stream, c.args(), 0)
    c.nk = [350, 160]
    c.kv_len.copy_(torch.tensor(c.nk))
    graph.replay()
    torch.cuda.synchronize()
    c.check(c.out.cpu())


@pytest.mark.parametrize("causal,sinks", [(False, 2), (True, 3)])
def test_graph_replay_reads_new_lengths(causal, sinks):
    """Captured with full lengths, replayed with shorter ones; calls on two streams beside it."""
    c = Case([700] * 9, [700] * 9, 6, 6, 64, causal=causal, window=25, sinks=sinks)
    c.check()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        binding.elasto_op_window_attention(stream_handle(), c.args(), st.data_ptr())
    lens = [700, 1, 0, 333, 128, 699, 2, 257, 64]
    c.nq = c.nk = lens
    c.q_start.copy_(c.starts(lens))
    c.kv_start.copy_(c.starts(lens))
    c.out.fill_(9.0)
    graph.replay()
    torch.cuda.synchronize()
    got = c.out.cpu()
    c.check(got)
    outs, streams = [torch.full_like(c.out, 9.0) for _ in range(4)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        binding.elasto_op_window_attention(streams[i % 2].cuda_stream, c.args(out=out.data_ptr()), st.data_ptr())
    torch.cuda.synchronize()
    assert all(torch.equal(out.cpu(), got) for out in outs) and int(st.item()) == 0
