"""Refusals on the host by the calls for long sequences: sizes and numbers at the ends of their types, outputs that
are inputs. CPU only."""
import pytest

from paper_2609_10018_gb300 import binding
from test_abi_cpu import lib  # noqa: F401  (builds the library where it is stale)
from test_long_sequence_ops_cpu import P, _attention, _gemm, _quantize


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


@pytest.mark.parametrize("kw", [dict(q=P, scale=3 * P), dict(q=2 * P, scale=P), dict(q=2 * P, scale=2 * P)])
def test_quantize_in_place(lib, kw):  # noqa: F811
    """A block's codes would be written where another's values have not been read."""
    assert _quantize(lib, **kw) == binding.ERR_INVALID_ARG
    assert "an output that is" in binding.elasto_last_error()


@pytest.mark.parametrize("of", ["A", "a_scale", "W", "w_scale", "bias"])
def test_gemm_fp8_into_an_input(lib, of):  # noqa: F811
    kw = dict(A=2 * P, a_scale=3 * P, W=4 * P, w_scale=5 * P, bias=6 * P)
    assert _gemm(lib, **kw | {of: P}) == binding.ERR_INVALID_ARG
    assert "one of the inputs" in binding.elasto_last_error()
