"""elasto_op_window_attention: what the bits of its result may depend on, and visible values that are not finite."""
import pytest
import torch

from helpers import stream_handle
from paper_2609_10018_gb300 import binding
from test_gpu_window_attention import Case

pytestmark = pytest.mark.gpu


def _growing(c):
    """Scores that grow along the keys, so that running maxima move in every tile, with noise between the rows."""
    n = c.k.shape[-3]
    c.k.mul_(0.5)
    c.k[..., 0] = (torch.linspace(-8, 8, n)[:, None] if c.packed else torch.linspace(-8, 8, n)[None, :, None]).to(c.dtype)
    c.q[..., 0] = 8.0
    return c


def _fill_shared_memory(value):
    """A product whose operand tiles leave `value` (an e4m3 code) in the shared memory of every SM."""
    m, n, k = 4096, 4096, 1024
    a, w = (torch.full((r, k), value, dtype=torch.uint8, device="cuda") for r in (m, n))
    sa, sw = torch.ones((k // 128, m), device="cuda"), torch.ones((n // 128, k // 128), device="cuda")
    out = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    binding.elasto_op_gemm_fp8(stream_handle(), a.data_ptr(), k, sa.data_ptr(), m, w.data_ptr(), k, sw.data_ptr(), None,
                               out.data_ptr(), n, m, n, k, binding.EPI_BIAS_BF16)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("group", [3, 5, 6, 7])
@pytest.mark.parametrize("nq,nk,d", [(900, 900, 128), (640, 1500, 64), (40, 1200, 64)])
def test_bits_do_not_depend_on_shared_memory(nq, nk, d, group, dtype):
    """Groups of heads that leave rows of a tile of 128 without a query: what an earlier kernel left there is not seen."""
    c = _growing(Case([nq], [nk], 2 * group, 2, d, dtype=dtype)).device()
    _fill_shared_memory(0x00)
    first = c.run()
    for code in (0x7E, 0xFE, 0x38, 0x7B):  # +-448, 1, 352: as 16-bit pairs, values of very different sizes
        _fill_shared_memory(code)
        c.out.fill_(9.0)
        assert torch.equal(c.run(), first), hex(code)
    c.check(first)


@pytest.mark.parametrize("heads,heads_kv", [(2, 2), (6, 2), (8, 1)])
@pytest.mark.parametrize("nq", [20, 130, 700])
def test_bits_do_not_depend_on_the_next_sequence(nq, heads, heads_kv):
    """A tile's rows past a sequence's last query hold the next sequence's queries: they change nothing."""
    c = _growing(Case([nq, nq], [900, 900], heads, heads_kv, 64)).device()
    first = c.run()[:nq]
    for factor in (-1.0, 16.0, float("nan")):
        c.dq[nq:] = (c.q[nq:].float() * factor).to(c.dtype).cuda()
        c.out.fill_(9.0)
        assert torch.equal(c.run()[:nq], first), factor


INF = float("inf")


def _improbable(c, key, value, channel, head=0):
    """`value` at a key whose score is 240 below all others, so that its probability rounds to 0 in 16 and in 32 bits."""
    c.q[..., 0], c.k[..., 0] = 32.0, 0.0
    c.q[..., 1:].mul_(0.25)
    k, v = (c.k, c.v) if c.packed else (c.k[0], c.v[0])
    k[key, head, 0] = -7.5 * c.d ** 0.5
    v[key, head, channel] = value


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("value", [INF, -INF])
@pytest.mark.parametrize("at", [5, 130, 300, 511, 600])
def test_improbable_infinity_seen_in_part_by_one_tile(at, value, dtype):
    """Causal, two tiles of queries an item: the key tile of the first one's diagonal is whole for the second."""
    n, b = 677, 3
    c = Case([n] * 7, [n] * 7, 6, 6, 64, dtype=dtype)
    _improbable(c, b * n + at, value, 9, 2)
    c.device()
    first = c.run()
    c.check(first)
    rows = first[b * n:(b + 1) * n, 2, 9]
    sharers = [r for r in range(at, n) if r // 256 == at // 256]  # queries of the item whose diagonal tile holds the key
    assert (rows[sharers].float() == value).all()
    for _ in range(5):
        c.out.fill_(9.0)
        assert torch.equal(c.run().view(torch.int16), first.view(torch.int16))


def _check_not_finite(c):
    """Values that are not finite as the definition has them; the others within the usual bound."""
    got = c.device().run()
    c.check(got)
    for b in range(len(c.nq)):
        want, _ = c.want(b)
        g = got[sum(c.nq[:b]):sum(c.nq[:b + 1])].double()
        odd = ~want.isfinite()
        assert odd.any() or b > 0
        assert torch.equal(g[odd].isnan(), want[odd].isnan())
        assert torch.equal(g[odd].nan_to_num(nan=0.0), want[odd].nan_to_num(nan=0.0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("at", [0, 40, 333, 640])
@pytest.mark.parametrize("nq,nk,heads,kw", [
    ([677], [677], 2, dict()),                                                         # a tile an item
    ([677] * 7, [677] * 7, 6, dict(window=500, sinks=2)),                              # two tiles an item
    ([677] * 5, [677] * 5, 6, dict(causal=False, window=40, sinks=3)),                 # queries that see everything
    ([20], [2000], 2, dict(packed=False)),                                             # keys shared out over a cluster
    ([20, 3], [1999, 700], 2, dict(packed=False, window=1500, sinks=1)),
], ids=["one", "two", "wide", "split", "split_window"])
def test_improbable_infinity(nq, nk, heads, kw, at, d, dtype):
    """An infinite value behind a probability that rounds to 0 reaches who sees it, in every form and tile; with its
    opposite in the same channel NaN; a query of NaN stays NaN."""
    c = Case(nq, nk, heads, heads, d, dtype=dtype, **kw)
    _improbable(c, at, INF, 9, 1)
    _improbable(c, at + 9, -INF, 40, 1)
    (c.v if c.packed else c.v[0])[at + 11, 1, 40] = INF
    c.q[5, 1] = float("nan")
    _check_not_finite(c)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("at", [0, 40, 333, 2040])
@pytest.mark.parametrize("nk,kw", [(2100, dict(packed=False, room=3)), (2100, dict(window=2070, sinks=2)), (2052, dict(packed=False, window=20, sinks=400))],
                         ids=["all", "window", "sinks"])
def test_improbable_infinity_single_token(nk, kw, at, d, dtype):
    """As test_improbable_infinity, for the form of single tokens; three query heads share each key head."""
    c = Case([1], [nk], 6, 2, d, dtype=dtype, **kw)
    _improbable(c, at, INF, 9, 1)
    _improbable(c, at + 9, -INF, 40, 1)
    (c.v if c.packed else c.v[0])[at + 11, 1, 40] = INF
    (c.v if c.packed else c.v[0])[nk - 1, 0, 7] = float("nan")
    c.q[0, 5] = float("nan")
    _check_not_finite(c)


def test_infinity_hidden_from_a_single_token():
    """Not found by the search for visible ones either."""
    c = Case([1], [500], 2, 1, 64, window=100, sinks=3, packed=False, room=8)
    _improbable(c, 450, INF, 9)
    c.v[0, 3:399, 0, 9], c.v[0, 500:, 0, 9] = -INF, -INF
    _check_not_finite(c)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_large_finite_values_are_not_taken_for_infinities(dtype):
    """The type's largest value, seen by all with probability 1 / 2 and 1."""
    for nq, nk, packed in ((300, 300, True), (20, 2000, False)):
        c = Case([nq], [nk], 2, 2, 64, dtype=dtype, packed=packed)
        c.q.zero_()
        c.v.zero_()
        v = c.v if packed else c.v[0]
        v[:2, 0, 3], v[:, 1, 5] = torch.finfo(dtype).max / 512, -torch.finfo(dtype).max / 512
        c.check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("nq,nk,heads,kw", [([300] * 4, [300] * 4, 4, dict()), ([677] * 7, [677] * 7, 6, dict(window=500, sinks=2)),
                                            ([677] * 5, [677] * 5, 6, dict(causal=False, window=40, sinks=3)),
                                            ([20], [2000], 2, dict(packed=False)), ([1, 1], [1999, 70], 2, dict(packed=False))],
                         ids=["one", "two", "wide", "split", "single"])
def test_values_near_the_end_of_the_type(nq, nk, heads, kw, dtype):
    """Weighted means of values of half the type's largest, whose sums are past fp32's for bf16; scores that grow
    along the keys."""
    c = _growing(Case(nq, nk, heads, heads, 64, dtype=dtype, **kw))
    c.v.copy_((c.v.float().clamp(-4, 4) / 8 * torch.finfo(dtype).max).to(dtype))
    c.v[..., 3] = torch.finfo(dtype).max / 2
    c.check()


@pytest.mark.parametrize("share", [0.002, 0.3])
@pytest.mark.parametrize("nq,nk,heads,heads_kv,kw", [([300], [300], 6, 2, dict(window=40, sinks=5)), ([260] * 5, [300] * 5, 8, 8, dict(window=100)),
                                                     ([300], [300], 6, 2, dict(causal=False, window=30, sinks=9)),
                                                     ([400] * 4, [400] * 4, 10, 10, dict(causal=False, window=20, sinks=3)),
                                                     ([40], [1100], 5, 1, dict(packed=False, window=600, sinks=3)),
                                                     ([1, 1], [700, 90], 4, 2, dict(packed=False, window=300, sinks=3)),
                                                     ([90], [70], 4, 2, dict(window=30, sinks=3))],
                         ids=["grouped", "two", "both", "wide", "split", "single", "no_keys_first"])
def test_many_values_that_are_not_finite(nq, nk, heads, heads_kv, kw, share):
    """NaN and infinities of either sign all over the values: each row and channel gets the sum of those it sees."""
    c = Case(nq, nk, heads, heads_kv, 72, dtype=torch.float16, **kw)
    g = torch.Generator().manual_seed(5)
    kind = torch.rand(c.v.shape, generator=g)
    for i, value in enumerate((INF, -INF, float("nan"))):
        c.v[(kind >= i * share / 3) & (kind < (i + 1) * share / 3) & (torch.arange(72) % (3 if i == 2 else 1) == 0)] = value
    _check_not_finite(c)
