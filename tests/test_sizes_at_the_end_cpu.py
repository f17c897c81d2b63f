"""Sizes and numbers at the ends of their types in the calls for long sequences: refused on the host. CPU only."""
import pytest

from paper_2609_10018_gb300 import binding
from test_abi_cpu import lib  # noqa: F401  (builds the library where it is stale)
from test_long_sequence_ops_cpu import _attention, _gemm, _quantize


@pytest.mark.parametrize("scale", [2.4e38, 2.9e38])
def test_scale_times_log2_e_past_fp32(lib, scale):  # noqa: F811
    """Scores are held in units of log2: the factor itself would be infinite, and every result NaN."""
    assert _attention(lib, scale=scale) == binding.ERR_INVALID_ARG
    assert "elasto_op_window_attention: sinks or scale" in binding.elasto_last_error()


@pytest.mark.parametrize("cols", [2 ** 31 - 127, 2 ** 31 - 1])
def test_quantize_last_block_past_an_int(lib, cols):  # noqa: F811
    assert _quantize(lib, cols=cols, ldx=2 ** 32, ldq=2 ** 32) == binding.ERR_UNSUPPORTED
    assert "columns" in binding.elasto_last_error()


@pytest.mark.parametrize("kw", [dict(M=2 ** 31 - 255, lds=2 ** 31), dict(M=2 ** 31 - 1, lds=2 ** 31), dict(N=2 ** 31 - 255, ldo=2 ** 31),
                                dict(N=2 ** 31 - 1, ldo=2 ** 31)])
def test_gemm_fp8_last_tile_past_an_int(lib, kw):  # noqa: F811
    assert _gemm(lib, **kw) == binding.ERR_UNSUPPORTED
    assert "2^31" in binding.elasto_last_error()
