"""elasto_op_gemm_fp8 in each of its forms: which one a size gets, and that one against the 64-bit sum."""
import pytest
import torch

from paper_2609_10018_gb300 import binding
from test_gpu_gemm_fp8 import BF16, F32, GELU, RESID, _call, _check, _problem

pytestmark = pytest.mark.gpu
PAIR = (256, 256, 1, 0)

# More tiles of 256 x 256 than half the SMs' pairs; the second and third with a second round of tiles.
PAIRS = [(2304, 2048, 384), (2200, 2001, 392), (2900, 2500, 200), (2817, 2504, 130), (18701, 251, 777)]


def _tile(M, N, K, want):
    assert binding.elasto_op_gemm_fp8_tile(M, N, K).fields() == want


@pytest.mark.parametrize("M,N,K", PAIRS)
@pytest.mark.parametrize("epi", [BF16, GELU, RESID, F32])
def test_pairs(M, N, K, epi):
    _tile(M, N, K, PAIR)
    _check(M, N, K, epi)


@pytest.mark.parametrize("M,N,K", [(2304, 2048, 384), (2200, 2001, 392), (2817, 2504, 130)])
@pytest.mark.parametrize("epi", [BF16, GELU, RESID, F32])
@pytest.mark.parametrize("extra,pad,bias", [(1, 8, False), (2, 6, True)])
def test_pairs_strides_and_no_bias(M, N, K, epi, extra, pad, bias):
    _tile(M, N, K, PAIR)
    _check(M, N, K, epi, extra, pad, bias)


@pytest.mark.parametrize("M,N,K", [(2304, 2048, 384), (2200, 2001, 392), (2900, 2500, 200)])
@pytest.mark.parametrize("epi", [BF16, GELU, RESID, F32])
def test_pairs_same_bits_wherever_out_starts(M, N, K, epi):
    """Repeated calls, and out at an offset that no wide store fits: tiles by TMA, by words and value by value."""
    _tile(M, N, K, PAIR)
    a, sa, w, sw, b = (t.cuda() for t in _problem(M, N, K, 17))
    dtype = torch.float32 if epi in (RESID, F32) else torch.bfloat16
    start = torch.randn((M, N), generator=torch.Generator().manual_seed(3)).to(dtype).cuda()

    def result(offset):
        store = torch.zeros(M * N + 16, dtype=dtype, device="cuda")
        out = store[offset:offset + M * N].view(M, N)
        out.copy_(start)
        st = _call(a, sa, w, sw, b, out, N, M, N, K, epi)
        assert int(st.item()) == 0 and (store[:offset] == 0).all() and (store[offset + M * N:] == 0).all()
        return out.cpu()

    first = result(0)
    for offset in (0, 1, 2, 7):
        assert torch.equal(result(offset), first), offset


@pytest.mark.parametrize("M,N,K,want", [(50, 25000, 256, (128, 64, 0, 0)), (5000, 1032, 777, (128, 128, 0, 0)),
                                        (5000, 1160, 100, (128, 64, 0, 0)), (2817, 2504, 130, PAIR), (2900, 2500, 200, PAIR)])
@pytest.mark.parametrize("epi", [BF16, GELU, RESID, F32])
def test_staging_of_the_tile_before(M, N, K, want, epi):
    """Several tiles a CTA that have one staging piece, or an odd number in the last columns: the next tile's first piece
    is not written before that one's store has read it."""
    _tile(M, N, K, want)
    _check(M, N, K, epi)
    a, sa, w, sw, b = (t.cuda() for t in _problem(M, N, K, 23))
    dtype = torch.float32 if epi in (RESID, F32) else torch.bfloat16
    outs = [torch.ones((M, N), dtype=dtype, device="cuda") for _ in range(6)]
    for o in outs:
        _call(a, sa, w, sw, b, o, N, M, N, K, epi)
    assert all(torch.equal(o, outs[0]) for o in outs)


@pytest.mark.parametrize("M,N,K,want", [(2200, 2001, 392, PAIR), (2200, 2041, 392, PAIR), (18701, 251, 777, PAIR), (5000, 1027, 777, (128, 128, 0, 0)),
                                        (5000, 1131, 100, (128, 64, 0, 0)), (300, 97, 260, (128, 64, 0, 0)), (300, 70, 260, (128, 64, 0, 0))])
@pytest.mark.parametrize("epi", [BF16, GELU, RESID, F32])
def test_columns_behind_the_last_are_left_alone(M, N, K, want, epi):
    """Rows that start on 16 bytes and end inside 16 bytes: what lies behind them is another tensor's."""
    _tile(M, N, K, want)
    unit = 4 if epi in (RESID, F32) else 8
    _check(M, N, K, epi, pad=-N % unit)
    _check(M, N, K, epi, pad=-N % unit + unit)


@pytest.mark.parametrize("M,N,K,rows,split", [
    (7, 9999, 100, 16, 1), (16, 300, 392, 16, 2), (7, 100, 1000, 16, 4), (13, 130, 2100, 16, 8),
    (27, 20001, 100, 32, 1), (32, 9999, 392, 32, 2), (27, 131, 1000, 32, 4), (17, 300, 2100, 32, 8),
    (50, 40001, 100, 64, 1), (50, 9999, 1500, 64, 2), (64, 100, 1500, 64, 4), (33, 300, 2100, 64, 8),
    (300, 33987, 100, 128, 1), (90, 2484, 4000, 128, 4), (150, 1292, 4000, 128, 4), (90, 301, 2500, 128, 8), (150, 100, 2500, 128, 8)])
@pytest.mark.parametrize("epi", [BF16, GELU, RESID, F32])
def test_few_rows(M, N, K, rows, split, epi):
    """Each height of a tile, with its blocks of K shared out over 1 to 8 CTAs; outputs of any row stride."""
    _tile(M, N, K, (rows, 128, 0, split))
    _check(M, N, K, epi)
    if N < 2500:
        _check(M, N, K, epi, extra=1, pad=5, bias=False)


@pytest.mark.parametrize("M,N,K", [(50, 100, 2000), (90, 301, 2500), (27, 131, 1000), (7, 100, 392)])
def test_few_rows_same_bits(M, N, K):
    a, sa, w, sw, b = (t.cuda() for t in _problem(M, N, K, 19))
    outs = [torch.empty((M, N + 3 * i), device="cuda") for i in range(4)]
    for o in outs:
        _call(a, sa, w, sw, b, o, o.shape[1], M, N, K, F32)
    assert all(torch.equal(o[:, :N], outs[0]) for o in outs)
