"""elasto_op_prefix_attention against its 64-bit definition."""
import math

import pytest
import torch

import block_reference as block
import sublayer_reference as ref
from helpers import stream_handle
from paper_2609_10018_gb300 import binding

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
BF16, F16 = torch.bfloat16, torch.float16


class Case:
    """prefixes: (keys, sequences) of each; nq, nk: queries and own keys of each sequence. `before`: sequences of no prefix
    in front; own keys packed, or in caches of `room` rows more than the longest. What is behind the lengths is NaN."""

    def __init__(self, prefixes, nq, nk, heads=4, heads_kv=2, d=64, dtype=BF16, packed=False, room=3, tail=0, gap=0, before=0, seed=0):
        g = torch.Generator().manual_seed(seed + 1000 * sum(nq) + sum(nk) + d)
        self.lens, self.nq, self.nk, self.h, self.hk, self.d = [p for p, _ in prefixes], list(nq), list(nk), heads, heads_kv, d
        self.dtype, self.packed, self.scale, self.before = dtype, packed, 1 / math.sqrt(d), before
        self.seq = [before + sum(n for _, n in prefixes[:i]) for i in range(len(prefixes) + 1)]
        rand = lambda *s: torch.randn(s, generator=g).to(dtype)[..., :d]  # noqa: E731
        self.rows = max(max(self.lens), 1) + room
        self.pk, self.pv = rand(len(prefixes), self.rows, heads_kv, d + gap), rand(len(prefixes), self.rows, heads_kv, d + gap)
        for i, n in enumerate(self.lens):
            self.pk[i, n:], self.pv[i, n:] = NAN, NAN
        self.q = rand(sum(nq) + tail, heads, d + gap)
        self.cap = max(max(nk), 1) + room
        shape = (sum(nk) + room + 1, heads_kv, d + gap) if packed else (len(nk), self.cap, heads_kv, d + gap)
        self.k, self.v = rand(*shape), rand(*shape)
        if packed:
            self.k[sum(nk):], self.v[sum(nk):] = NAN, NAN
        else:
            for i, n in enumerate(nk):
                self.k[i, n:], self.v[i, n:] = NAN, NAN

    def prefix_of(self, b):
        for i in range(len(self.lens)):
            if self.seq[i] <= b < self.seq[i + 1]:
                return i, self.lens[i]
        return 0, 0

    def sequence(self, b):
        q0, k0, (i, n) = sum(self.nq[:b]), sum(self.nk[:b]), self.prefix_of(b)
        own = (slice(k0, k0 + self.nk[b]),) if self.packed else (b, slice(0, self.nk[b]))
        return self.q[q0:q0 + self.nq[b]], self.k[own], self.v[own], self.pk[i, :n], self.pv[i, :n]

    def starts(self, n):
        return torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device="cuda")

    def device(self):
        dev = lambda t: torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda").copy_(t)  # noqa: E731
        self.t = {n: dev(getattr(self, n)) for n in ("q", "k", "v", "pk", "pv")}
        self.out = torch.full((self.q.shape[0], self.h, self.d), 9.0, dtype=self.dtype, device="cuda")
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.t |= {"q_start": self.starts(self.nq), "kv_start": self.starts(self.nk), "kv_len": ints(self.nk), "prefix_len": ints(self.lens),
                   "seq_start": ints(self.seq)}
        return self

    def args(self, workspace=True, **kw):
        t, out = self.t, self.out
        a = dict(dtype=binding.BF16 if self.dtype == BF16 else binding.F16, batch=len(self.nq), heads=self.h, heads_kv=self.hk,
                 head_dim=self.d, scale=self.scale, max_queries=max(max(self.nq), 1), q_rows=t["q"].shape[0],
                 q_start=t["q_start"].data_ptr(), q=t["q"].data_ptr(), q_row=t["q"].stride(0), q_head=t["q"].stride(1),
                 out=out.data_ptr(), out_row=out.stride(0), out_head=out.stride(1),
                 prefixes=len(self.lens), seq_start=t["seq_start"].data_ptr(), max_prefix=max(max(self.lens), 1), prefix_rows=self.rows,
                 prefix_len=t["prefix_len"].data_ptr(), max_keys=max(max(self.nk), 1), kv_rows=t["k"].shape[0] if self.packed else self.cap,
                 kv_start=t["kv_start"].data_ptr() if self.packed else None, kv_len=None if self.packed else t["kv_len"].data_ptr())
        for n, x, packed in (("prefix_k", "pk", False), ("prefix_v", "pv", False), ("k", "k", self.packed), ("v", "v", self.packed)):
            a |= {n: t[x].data_ptr(), n + "_batch": 0 if packed else t[x].stride(0), n + "_row": t[x].stride(-3), n + "_head": t[x].stride(-2)}
        args = binding.PrefixAttention(**(a | kw))
        if workspace:
            n = binding.elasto_op_prefix_attention_workspace(args)
            self.workspace = torch.full((n + 64,), 255, dtype=torch.uint8, device="cuda")  # (NaN)
            args.workspace, args.workspace_bytes = self.workspace.data_ptr(), n
        return args

    def run(self, **kw):
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        binding.elasto_op_prefix_attention(stream_handle(), self.args(**kw), st.data_ptr())
        assert int(st.item()) == 0
        assert (self.workspace[-64:] == 255).all()
        return self.out.cpu()

    def check(self, got=None):
        """Probabilities and the result are rounded to the type (half a step of each term, and of the
        result); fp32 scores of |q . k| scale <= 32 are off by less than 2^-24 * 128 * 32, which is 2.5e-4
        of a probability, and as much again comes from the sum of up to 2^12 of them and from the joins (2^-21 each)."""
        got = self.device().run() if got is None else got
        u = ref.half_step(self.dtype)
        for b in range(len(self.nq)):
            q, k, v, pk, pv = self.sequence(b)
            want, mean = block.prefix_attention(q, k, v, pk, pv, self.scale)
            q0 = sum(self.nq[:b])
            g = got[q0:q0 + self.nq[b]].double()
            fine = want.isfinite()
            assert torch.equal(fine, g.isfinite()), "sequence %d" % b
            tol = u * want.abs() + (1.01 * u + 5e-4) * mean + 2.0 ** -24
            bad = ~(((g - want).abs() <= tol) | ~fine)
            assert not bad.any(), (b, bad.nonzero()[:4].tolist(), float((g - want).abs()[fine].max()))
        assert (got[sum(self.nq):] == 9.0).all()  # rows of no sequence
        return got


@pytest.mark.parametrize("prefix", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 143, 255, 256, 257, 300, 640, 1000])
def test_prefix_lengths(prefix):
    Case([(prefix, 3)], [1, 1, 1], [1, 17, 64], tail=2).check()


@pytest.mark.parametrize("own", [0, 1, 2, 15, 16, 17, 63, 64, 65, 128, 129, 300])
def test_own_lengths(own):
    Case([(130, 2)], [1, 1], [own, 5]).check()
    Case([(130, 2)], [3, 1], [own, 5]).check()
    Case([(130, 2)], [40, 2], [own, 5]).check()


@pytest.mark.parametrize("d", [8, 16, 40, 64, 72, 80, 96, 128])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,heads_kv", [(1, 1), (4, 1), (6, 2), (3, 3), (14, 2), (34, 1), (40, 1)])
def test_heads_and_types(d, dtype, heads, heads_kv):
    Case([(200, 3)], [1, 1, 1], [30, 70, 1], heads, heads_kv, d, dtype, gap=8).check()
    Case([(200, 2)], [9, 4], [30, 70], heads, heads_kv, d, dtype, packed=True).check()


@pytest.mark.parametrize("queries", [2, 3, 4, 5, 16, 31, 64, 65, 100])
@pytest.mark.parametrize("heads,heads_kv,d", [(8, 2, 128), (5, 1, 64), (28, 4, 128)])
def test_several_queries(queries, heads, heads_kv, d):
    """Drafts and prompts: their own keys are causal, the prefix is not."""
    Case([(150, 3)], [queries, 1, max(1, queries - 1)], [queries, 40, queries + 70], heads, heads_kv, d).check()


@pytest.mark.parametrize("packed", [True, False])
def test_ragged(packed):
    """Empty sequences, sequences without own keys, more queries than own keys (the first see the prefix alone)."""
    Case([(70, 8)], [5, 0, 13, 1, 7, 30, 3, 6], [9, 4, 13, 90, 0, 29, 1, 0], 4, 2, packed=packed, tail=5).check()


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("single", [True, False])
def test_several_prefixes(packed, single):
    """Prefixes without keys, without sequences; sequences of no prefix in front and behind, some of which see nothing."""
    prefixes = [(130, 2), (0, 2), (300, 0), (17, 3), (129, 1), (256, 1)]
    n = 2 + sum(k for _, k in prefixes) + 2
    nq = [1] * n if single else [1, 2, 3, 1, 5, 1, 2, 4, 1, 9, 1, 2, 1]
    nk = [3, 0, 40, 7, 5, 0, 66, 4, 0, 9, 130, 0, 5]
    Case(prefixes, nq, nk, 6, 2, 64, packed=packed, before=2, tail=1).check()


def test_many_prefixes():
    """More than a warp looks through at once."""
    r = [(20 + 13 * i % 50, 1 + i % 2) for i in range(70)]
    n = sum(k for _, k in r)
    Case(r, [1] * n, [1 + i % 7 for i in range(n)], 2, 1, 32).check()


@pytest.mark.parametrize("prefix,batch,heads,heads_kv,d", [(5000, 1, 2, 1, 64), (4100, 3, 8, 2, 128), (3001, 2, 6, 1, 96), (2049, 40, 4, 1, 128),
                                                           (2500, 70, 4, 2, 64)])
def test_long_prefixes(prefix, batch, heads, heads_kv, d):
    """Keys shared out over many CTAs, one or two tiles of rows an item."""
    c = Case([(prefix, batch)], [1] * batch, [1 + 37 * i % 150 for i in range(batch)], heads, heads_kv, d)
    c.check()
    c.lens[0] = prefix // 3 + 1  # the plan stays that of the longest
    got = c.device().run(max_prefix=prefix, prefix_len=c.t["prefix_len"].data_ptr())
    c.check(got)


def test_long_own_caches():
    """Few sequences with long caches: their keys are shared out over a cluster."""
    Case([(200, 2)], [1, 1], [3000, 1777], 8, 2, 128).check()
    Case([(200, 2)], [5, 3], [3000, 1777], 8, 2, 64).check()


def test_without_own_keys():
    c = Case([(300, 3)], [1, 1, 2], [0, 0, 0]).device()
    c.check(c.run(max_keys=0, k=None, v=None, kv_rows=0, kv_len=None))
    c.check(c.device().run())


def test_without_starts():
    """The same number of queries each, full lengths, one prefix of all."""
    c = Case([(130, 3)], [2, 2, 2], [33, 33, 33], room=0).device()
    c.check(c.run(q_start=None, seq_start=None, prefix_len=None, kv_len=None))


@pytest.mark.parametrize("queries", [1, 4, 30])
def test_visible_values_that_are_not_finite(queries):
    """In the prefix and in own keys, to the queries that see them and no others: the sum of what is not finite, even
    where the probability has rounded to 0."""
    c = Case([(200, 2), (150, 1)], [queries] * 3, [queries + 3, queries, 40 + queries], 4, 2, 64)
    c.pv[0, 150, 0, 5], c.pv[0, 7, 1, 9], c.pv[0, 8, 1, 9] = INF, INF, -INF
    c.v[2, 12, 0, 3], c.v[2, 39 + queries, 1, 4], c.v[0, queries + 2, 1, 60] = -INF, NAN, INF
    c.k[2, 12] *= 200  # (a score far below or above the others)
    got = c.check()
    at = [sum(c.nq[:b]) for b in range(4)]
    assert (got[:at[2], :2, 5] == INF).all() and got[:at[2], 2:, 9].isnan().all()
    assert (got[at[2]:, :2, 3] == -INF).all() and got[at[3] - 1, 2:, 4].isnan().all()
    assert (got[at[1] - 1, 2:, 60] == INF).all()


def test_tiny_probabilities_of_infinities():
    c = Case([(300, 1)], [1], [20], 1, 1, 64, F16)
    c.q[:] = 4.0
    c.pk[0, :300], c.k[0, :20] = 1.0, 1.0
    c.pk[0, 100], c.k[0, 3] = -8.0, -8.0  # e^-288 of the others' probability
    c.pv[0, 100, 0, 3], c.v[0, 3, 0, 4] = INF, -INF
    got = c.device().run()
    assert got[0, 0, 3] == INF and got[0, 0, 4] == -INF and torch.isfinite(got[0, 0, 5:]).all()


def test_scores_that_are_not_finite():
    """A NaN score, or +infinity: NaN. -infinity: a probability of 0. All of them: NaN."""
    c = Case([(140, 4)], [1] * 4, [3] * 4, 1, 1, 64, F16)
    c.k[1, 2, 0, 0], c.k[2, 0, 0, 0] = NAN, -INF
    c.q[2:, 0, 0] = c.q[2:, 0, 0].abs() + 1
    got = c.device().run()
    assert torch.isfinite(got[0]).all() and got[1].isnan().all() and torch.isfinite(got[2]).all() and torch.isfinite(got[3]).all()
    c.pk[0, 139, 0, 0] = -INF
    got = c.device().run()
    assert torch.isfinite(got[2:]).all()


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F16, 128), (BF16, 40)])
@pytest.mark.parametrize("form,queries,heads,heads_kv,room", [("few", 1, 4, 2, 0), ("few", 4, 4, 2, 0), ("few", 5, 28, 4, 0), ("many", 1, 4, 2, 7000),
                                                              ("many", 4, 4, 2, 7000), ("inside", 4, 32 * 52, 52, 0)])
def test_infinite_values_behind_scores_of_minus_infinity(form, queries, heads, heads_kv, room, dtype, d):
    """A part of the keys without a finite score has no weight, but an infinite or NaN value in it is one that the query sees. In the
    joins of few and of many rows, and where the kernel of the own keys joins (tests/test_prefix_plan.py has the sizes)."""
    c = Case([(140, 2), (60, 1)], [queries] * 3, [queries, queries + 2, 20], heads, heads_kv, d, dtype, tail=room)
    c.q[:, :, 0] = c.q[:, :, 0].abs() + 1
    c.k[0, :queries, 0, 0] = -INF  # all own keys of the first sequence, for the first key head,
    c.pk[0, 128:140, 0, 0] = -INF  # those of a whole tile,
    c.pk[1, :60, 0, 0] = -INF      # and of a whole prefix
    finite = c.check(c.device().run(max_queries=max(queries, room)))
    c.v[0, 0, 0, 5], c.v[0, queries - 1, 0, 6] = INF, -INF
    c.pv[0, 130, 0, 7], c.pv[0, 139, 0, 4] = INF, NAN
    c.pv[1, 59, 0, 3] = -INF
    got = c.device().run(max_queries=max(queries, room))
    n, first = queries, slice(0, heads // heads_kv)
    assert (got[:n, first, 5] == INF).all() and (got[n - 1, first, 6] == -INF).all()
    assert torch.isfinite(got[:n - 1, first, 6]).all()  # (hidden)
    assert (got[:2 * n, first, 7] == INF).all() and got[:2 * n, first, 4].isnan().all()
    assert (got[2 * n:3 * n, first, 3] == -INF).all()
    # all others as with finite values there
    got[:n, first, 5], got[n - 1, first, 6] = finite[:n, first, 5], finite[n - 1, first, 6]
    got[:2 * n, first, 7], got[:2 * n, first, 4] = finite[:2 * n, first, 7], finite[:2 * n, first, 4]
    got[2 * n:3 * n, first, 3] = finite[2 * n:3 * n, first, 3]
    assert torch.equal(got, finite)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F16, 64), (BF16, 40)])
def test_prompts_whose_prefixes_fill_the_chip(dtype, d):
    """Items of the prefixes for every SM: the kernel of the own keys joins its rows itself. Prefixes without keys,
    sequences without a prefix, without own keys, with values that are not finite."""
    prefixes = [(200, 2), (0, 1), (128, 1), (17, 1), (129, 1), (64, 1), (150, 1), (199, 1)]
    n = 1 + sum(k for _, k in prefixes) + 1
    nq, nk = [7, 9, 8, 5, 9, 8, 7, 6, 9, 9, 4], [9, 9, 30, 0, 60, 3, 7, 33, 16, 17, 4]
    assert len(nq) == n and sum(nq) > 8 * 8
    c = Case(prefixes, nq, nk, 16 * 13, 13, d, dtype, before=1, tail=2)
    c.pv[0, 150, 0, 5], c.pv[0, 7, 1, 9], c.pv[0, 8, 1, 9] = INF, INF, -INF
    c.v[4, 59, 2, 3], c.v[4, 52, 3, 7], c.v[0, 8, 1, 1] = -INF, NAN, INF
    got = c.check()
    assert torch.equal(c.device().run().view(torch.int16), got.view(torch.int16))  # (bits: there are NaN)
    at = [sum(nq[:b]) for b in range(n + 1)]
    assert (got[at[1]:at[3], :16, 5] == INF).all() and got[at[1]:at[3], 16:32, 9].isnan().all()
    assert (got[at[5] - 1, 32:48, 3] == -INF).all() and torch.isfinite(got[at[4]:at[5] - 1, 32:48, 3]).all()
    assert got[at[5] - 2:at[5], 48:64, 7].isnan().all()


def test_large_bf16_values():
    """Sums of values near the end of bf16's range do not overflow before the division."""
    c = Case([(600, 2)], [1, 1], [70, 5], 2, 1, 64)
    c.pv[0, :600], c.v[0, :70], c.v[1, :5] = 3e38, 3e38, 3e38
    got = c.device().run()
    assert torch.isfinite(got).all() and ((got.double() - 3e38).abs() <= 2e-2 * 3e38).all()


def test_lengths_past_the_limits_are_cut():
    c = Case([(130, 2)], [1, 3], [20, 9], tail=4).device()
    want = c.run().clone()
    c.device()
    args = c.args()
    c.t["prefix_len"].fill_(2 ** 31 - 1)
    c.t["q_start"][2] = 2 ** 31 - 1  # (cut to max_queries)
    c.t["kv_len"][0] = 2 ** 31 - 1
    c.t["seq_start"][1] = 99
    c.t["pk"][0, 130:], c.t["pv"][0, 130:] = NAN, NAN
    args.max_prefix, args.max_keys = 130, 20
    binding.elasto_op_prefix_attention(stream_handle(), args)
    assert torch.equal(c.out.cpu(), want)
    c.t["prefix_len"].fill_(-5), c.t["kv_len"].fill_(-9)
    c.t["q_start"][2] = 4
    binding.elasto_op_prefix_attention(stream_handle(), args)
    assert (c.out[:4] == 0).all()  # nothing visible


def test_a_prefix_of_one_sequence_is_its_own_cache():
    """The result of windowed attention over the concatenated keys, within the roundings of P."""
    c = Case([(500, 1)], [12], [77], 8, 2, 128)
    got = c.device().run().double()
    k, v = torch.cat([c.pk[0, :500], c.k[0, :77]]).cuda(), torch.cat([c.pv[0, :500], c.v[0, :77]]).cuda()
    out = torch.empty_like(c.out)
    binding.elasto_op_window_attention(stream_handle(), binding.WindowAttention(
        dtype=binding.BF16, batch=1, heads=8, heads_kv=2, head_dim=128, causal=1, window=-1, sinks=0, scale=c.scale, max_queries=12,
        q_rows=12, q=c.t["q"].data_ptr(), q_row=c.t["q"].stride(0), q_head=c.t["q"].stride(1), out=out.data_ptr(), out_row=out.stride(0),
        out_head=out.stride(1), max_keys=577, kv_rows=577, k=k.data_ptr(), k_batch=k.numel(), k_row=k.stride(0), k_head=k.stride(1),
        v=v.data_ptr(), v_batch=v.numel(), v_row=v.stride(0), v_head=v.stride(1)))
    # (each is within 3 half steps of the weighted mean of |v| <= 1.2 here)
    assert (got - out.cpu().double()).abs().max() <= 6 * 2.0 ** -9 * 2 * 1.2


@pytest.mark.parametrize("queries", [1, 20])
def test_same_bits_again_captured_and_on_another_stream(queries):
    c = Case([(1500, 6), (700, 3)], [queries] * 9, [queries + 11 * i for i in range(9)], 8, 2, 128).device()
    want = c.run().clone()
    args = c.args()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        binding.elasto_op_prefix_attention(stream_handle(), args)
        binding.elasto_op_prefix_attention(stream_handle(), args)  # (one workspace, one after the other)
    for _ in range(3):
        c.out.fill_(9), c.workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out.cpu(), want)
    # other lengths, the same graph
    c.nk, c.lens = [n // 2 + 1 for n in c.nk], [333, 700]
    if queries == 1:
        c.t["kv_len"].copy_(torch.tensor(c.nk, dtype=torch.int32))
        c.t["prefix_len"].copy_(torch.tensor(c.lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        c.check(c.out.cpu())


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F16, 128), (BF16, 64), (F16, 40)])
@pytest.mark.parametrize("most", [600, 3400])
@pytest.mark.parametrize("packed", [True, False])
def test_room_for_many_queries(dtype, d, most, packed):
    """Blocks of 64 rows, and from 40000 rows on their join: sequences that are short, empty, longer than a block, with own
    keys of several tiles and of several CTAs, behind prefixes with and without keys and behind none."""
    for longest in (130, 1100):  # (one CTA for a block's keys; two and more)
        c = Case([(200, 2), (0, 1), (300, 1)], [70, 1, 0, 33, 9, 65], [longest, 30, 5, 33, 0, 64], 4, 2, d, dtype, packed=packed, before=1,
                 tail=most - 178)
        c.pv[0, 150, 0, 5], c.pv[0, 7, 1, 9], c.pv[0, 8, 1, 9] = INF, INF, -INF
        flat = c.v[sum(c.nk[:3]):] if packed else c.v[3]
        flat[32, 0, 3], flat[5, 1, 4] = -INF, NAN  # (the last of 33 queries sees both, the sixth and later the second)
        got = c.check(c.device().run(max_queries=most))
        assert (got[70, :2, 5] == INF).all() and got[70, 2:, 9].isnan().all()
        assert (got[103, :2, 3] == -INF).all() and torch.isfinite(got[71:103, :2]).all()
        assert torch.isfinite(got[71:76, 2:]).all() and got[76:104, 2:, 4].isnan().all()
        assert torch.equal(c.device().run(max_queries=most).view(torch.int16), got.view(torch.int16))


@pytest.mark.parametrize("d", [128, 72, 8])
def test_join_of_many_rows_and_parts(d):
    """Room for 128 queries in each of 320 sequences, 150 rows: parts of many CTAs, joined 64 rows at a time."""
    nq = [(3 * i) % 4 % 3 for i in range(320)]
    while sum(nq) > 128:
        nq[nq.index(max(nq))] -= 1
    c = Case([(20000, 150), (1900, 170)], nq, [11 * i % 70 for i in range(320)], 1, 1, d, tail=150 - sum(nq))
    c.check(c.device().run(max_queries=128))
    c.check(c.device().run(max_queries=150, q_rows=150))


@pytest.mark.parametrize("most", [3, 600, 7000])
def test_without_own_keys_and_room(most):
    c = Case([(300, 3)], [1, 3, 2], [0, 0, 0], tail=most)
    c.check(c.device().run(max_queries=most, max_keys=0, k=None, v=None, kv_rows=0, kv_len=None))


@pytest.mark.parametrize("most", [1, 100, 7000])
def test_all_sequences_empty(most):
    Case([(300, 2)], [0, 0], [5, 9], tail=most).check()
    c = Case([(300, 2)], [0, 0], [5, 9], tail=most)
    c.check(c.device().run(max_queries=most))


def test_more_rows_than_the_sequences_have():
    """q_rows is what the buffers hold, far more than max_queries allows for."""
    c = Case([(300, 2)], [1, 1], [9, 30], 4, 1, 64, tail=700)
    c.check()


def test_offsets_past_32_bits():
    """A prefix's and a cache's rows so far apart that their offsets pass 2^32 values."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    c = Case([(130, 1)], [1], [70], 1, 1, 64, room=0)
    c.device()
    row = (1 << 25) + 8
    for n, rows in (("pk", 130), ("pv", 130), ("k", 70), ("v", 70)):
        if n in ("pk", "k"):
            whole = torch.empty((rows - 1) * row + 64, dtype=BF16, device="cuda")
            view = whole.as_strided((1, rows, 1, 64), (0, row, 64, 1))
            view.copy_(getattr(c, n))
            c.t[n] = view
    c.check(c.run())


def test_a_workspace_that_is_too_small():
    c = Case([(300, 2)], [1, 1], [9, 30]).device()
    args = c.args()
    args.workspace_bytes -= 1
    with pytest.raises(binding.ElastoError) as e:
        binding.elasto_op_prefix_attention(stream_handle(), args)
    assert e.value.status == binding.ERR_INVALID_ARG and "workspace" in str(e.value)


@pytest.mark.parametrize("d,most", [(64, 70), (128, 600), (40, 2000), (128, 2 ** 31 - 1)])
@pytest.mark.parametrize("nq,nk", [([1], [1]), ([7, 3], [7, 3]), ([40, 1, 20], [30, 0, 20])])
def test_packed_keys_fewer_than_the_limit(d, most, nq, nk):
    """max_keys is a limit: packed sequences may have fewer rows altogether."""
    c = Case([(200, len(nq))], nq, nk, 4, 2, d, packed=True, room=0)
    assert c.k.shape[0] < most
    c.check(c.device().run(max_keys=most))
    with pytest.raises(binding.ElastoError) as e:  # of a cache there are as many
        c.device().run(max_keys=most, kv_start=None, kv_len=c.t["kv_len"].data_ptr())
    assert e.value.status == binding.ERR_INVALID_ARG


def test_sizes_past_any_workspace():
    """Sizes whose workspace no memory holds (and 64 bits of bytes neither) are refused, not reckoned modulo 2^64."""
    c = Case([(300, 1)], [1], [9]).device()
    args = c.args()
    args.q_rows, args.heads, args.heads_kv, args.head_dim = 1 << 30, 1 << 20, 1, 128
    for call in (lambda: binding.elasto_op_prefix_attention_workspace(args), lambda: binding.elasto_op_prefix_attention(stream_handle(), args)):
        with pytest.raises(binding.ElastoError) as e:
            call()
        assert e.value.status == binding.ERR_UNSUPPORTED
