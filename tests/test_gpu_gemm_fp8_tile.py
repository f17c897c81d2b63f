"""elasto_op_gemm_fp8_tile: which form of the e4m3 product a size gets."""
import ctypes

import pytest

from paper_2609_10018_gb300 import binding

pytestmark = pytest.mark.gpu
PAIR = (256, 256, 1, 0)


def _tile(M, N, K, want):
    assert binding.elasto_op_gemm_fp8_tile(M, N, K).fields() == want


@pytest.mark.parametrize("M,N,K,want", [(300, 400, 1500, (128, 64, 0, 0)), (2560, 2304, 256, (128, 128, 0, 0)), (5000, 1030, 777, (128, 128, 0, 0)),
                                        (8192, 8192, 4096, PAIR),
                                        (50432, 2304, 768, PAIR), (8, 4096, 4096, (16, 128, 0, 8))])
def test_tiles_of_sizes(M, N, K, want):
    _tile(M, N, K, want)


def test_tile_refusals():
    t = binding.Fp8Tile()
    for args in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (-1, 1, 1)):
        assert binding.lib().elasto_op_gemm_fp8_tile(*args, ctypes.byref(t)) == binding.ERR_INVALID_ARG
    assert binding.lib().elasto_op_gemm_fp8_tile(1, 1, 1, None) == binding.ERR_INVALID_ARG
    assert binding.lib().elasto_op_gemm_fp8_tile(2 ** 31 - 1, 1, 1, ctypes.byref(t)) == binding.ERR_UNSUPPORTED
