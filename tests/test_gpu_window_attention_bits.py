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
