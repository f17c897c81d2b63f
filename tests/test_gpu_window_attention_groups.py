"""elasto_op_window_attention: many query heads to a key head, and sizes between the forms."""
import pytest
import torch

from test_gpu_window_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,heads_kv", [(33, 1), (40, 1), (67, 1), (130, 2)])
@pytest.mark.parametrize("nq,nk,kw", [(2, 700, dict(window=300, sinks=3)), (50, 50, dict(causal=False, window=7, sinks=2)), (130, 260, dict(window=33)),
                                      (5, 3000, dict(packed=False))])
def test_more_than_32_heads_a_key_head(heads, heads_kv, nq, nk, kw):
    """The group's heads are cut into equal parts, of which the last may be short."""
    Case([nq, max(1, nq // 2)], [nk, nk - 7], heads, heads_kv, 64, tail=2, room=4, **kw).check()
    Case([nq], [nk], heads, heads_kv, 24, dtype=torch.float16, **kw).check()


@pytest.mark.parametrize("nq", [1, 2, 3, 4, 5, 127, 128, 129, 255, 256, 257])
@pytest.mark.parametrize("causal", [True, False])
def test_bigger_batches_of_short_chunks(nq, causal):
    """Tiles cut at every place, two an item, in caches with rows to spare."""
    n = [max(1, nq - i % 3) for i in range(40)]
    Case(n, [v + 60 + i for i, v in enumerate(n)], 10, 2, 128, causal=causal, window=50, sinks=2, packed=False, room=3).check()


@pytest.mark.parametrize("nq,nk,window,sinks", [(300, 300, 1 << 30, 0), (300, 300, 2 ** 31 - 1, 2 ** 31 - 1), (1, 300, 2 ** 31 - 1, 2 ** 31 - 1),
                                                (300, 300, 0, 2 ** 31 - 1), (40, 2000, 2 ** 31 - 1, 7), (300, 500, -2 ** 31, 0)])
@pytest.mark.parametrize("causal", [True, False])
def test_limits_past_the_keys(nq, nk, window, sinks, causal):
    """Windows and first keys of any size mean all keys."""
    Case([nq], [nk], 4, 2, 64, causal=causal, window=window, sinks=sinks).check()


def _heads_first(t):
    """The same values with the heads' axis outside the rows'."""
    return t.transpose(-3, -2).contiguous().transpose(-3, -2)


@pytest.mark.parametrize("nq,nk", [(1, 300), (20, 2000), (300, 300)])
@pytest.mark.parametrize("packed", [True, False])
def test_heads_outside_rows(nq, nk, packed):
    """q, k, v and out stored head by head."""
    c = Case([nq, max(1, nq - 1)], [nk, nk - 5], 6, 2, 64, window=150, sinks=2, packed=packed, room=3, tail=2).device()
    plain = c.run()
    c.dq, c.dk, c.dv, c.out = (_heads_first(t) for t in (c.dq, c.dk, c.dv, torch.full_like(c.out, 9.0)))
    assert c.dk.stride(-2) > c.dk.stride(-3)
    c.check(c.run())
    assert torch.equal(c.out.cpu(), plain)


@pytest.mark.parametrize("nq", [1, 20, 300])
def test_one_cache_for_all_sequences(nq):
    """A batch stride of 0: every sequence reads the same keys, of its own length."""
    c = Case([nq] * 3, [400, 333, 400], 4, 2, 64, window=200, sinks=1, packed=False)
    c.k[:], c.v[:] = c.k[:1].clone(), c.v[:1].clone()
    c.device()
    plain = c.run()
    c.out.fill_(9.0)
    assert torch.equal(c.run(k_batch=0, v_batch=0), plain)
    c.check(plain)
