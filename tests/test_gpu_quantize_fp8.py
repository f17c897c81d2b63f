"""elasto_op_quantize_fp8 against its definition in fp32 operations: equal bit for bit."""
import pytest
import torch

import sublayer_reference as ref
from helpers import stream_handle
from paper_2609_10018_gb300 import binding

pytestmark = pytest.mark.gpu
TYPE = {"bf16": binding.BF16, "f16": binding.F16, "f32": binding.F32}


def _call(x, q, scale, kind, rows, cols, stream=None):
    binding.elasto_op_quantize_fp8(stream or stream_handle(), x.data_ptr(), TYPE[kind], x.stride(0), q.data_ptr(), q.stride(0),
                                   scale.data_ptr(), scale.stride(0), rows, cols)


def _check(x, kind, pad_x=0, pad_q=0, pad_s=0, offset=0):
    rows, cols = x.shape
    store = torch.full((rows * (cols + pad_x) + offset,), 7.0, dtype=x.dtype, device="cuda")
    xd = store[offset:].view(rows, cols + pad_x)
    xd[:, :cols] = x.cuda()
    q = torch.full((rows, cols + pad_q), 0x2A, dtype=torch.uint8, device="cuda")
    scale = torch.full((ref.blocks(cols), rows + pad_s), -3.0, device="cuda")
    _call(xd, q, scale, kind, rows, cols)
    want_q, want_s = ref.quantize(x)
    got_q, got_s = q.cpu(), scale.cpu()
    assert torch.equal(got_s[:, :rows].isnan(), want_s.isnan())
    assert torch.equal(got_s[:, :rows].nan_to_num(5.0), want_s.nan_to_num(5.0))
    a, b = got_q[:, :cols].contiguous().view(torch.float8_e4m3fn).float(), want_q.float()
    assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(5.0), b.nan_to_num(5.0))
    assert (got_q[:, cols:] == 0x2A).all() and (got_s[:, rows:] == -3.0).all()  # the rest is left as it was


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 129), (17, 8), (5, 1000), (64, 768), (257, 127), (2, 4096), (1000, 136)])
def test_sizes(kind, rows, cols):
    g = torch.Generator().manual_seed(rows * 10007 + cols)
    x = torch.randn((rows, cols), generator=g) * torch.exp(2 * torch.randn((1, cols), generator=g))
    _check(x.to(ref.DTYPES[kind]), kind)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("pad_x,pad_q,pad_s,offset", [(8, 8, 0, 0), (3, 0, 5, 0), (0, 5, 0, 0), (8, 8, 1, 1), (8, 16, 3, 8)])
def test_strides_and_alignment(kind, pad_x, pad_q, pad_s, offset):
    g = torch.Generator().manual_seed(pad_x + 10 * pad_q + 100 * offset)
    _check(torch.randn((37, 264), generator=g).to(ref.DTYPES[kind]), kind, pad_x, pad_q, pad_s, offset)


def test_extreme_values():
    """Zeros, subnormals, the types' largest, infinities and NaN, each in a block of its own."""
    x = torch.zeros((9, 256))
    x[1, 3] = 1e-42
    x[2] = torch.finfo(torch.float32).max
    x[3, 100], x[3, 130] = float("inf"), 1.0
    x[4, 5], x[4, 200] = float("nan"), 2.0
    x[5, :128] = 2.0 ** -100
    x[6, ::2] = -448.0
    x[7] = torch.linspace(-1, 1, 256)
    x[8, 0], x[8, 1] = float("-inf"), float("nan")
    _check(x, "f32")
    _check(x.bfloat16(), "bf16")
    y = x.clone()
    y[2] = 65504.0
    _check(y.half(), "f16")


def test_rounding_ties():
    """Values half way between two e4m3 numbers go to the even one."""
    x = torch.zeros((1, 128))
    x[0, 0] = 448.0  # scale 1
    x[0, 1:8] = torch.tensor([17.0, 19.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, 432.0])
    _check(x, "f32")


def test_stream_and_graph():
    """On another stream than the current one, and captured: the replay reads new inputs."""
    x = torch.randn((50, 300), device="cuda").bfloat16()
    q, scale = torch.zeros((50, 304), dtype=torch.uint8, device="cuda"), torch.zeros((3, 50), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _call(x, q, scale, "bf16", 50, 300, torch.cuda.current_stream().cuda_stream)
    for seed in (1, 2):
        fresh = torch.randn((50, 300), generator=torch.Generator().manual_seed(seed)).bfloat16()
        x.copy_(fresh)
        graph.replay()
        torch.cuda.synchronize()
        want_q, want_s = ref.quantize(fresh)
        assert torch.equal(scale.cpu(), want_s)
        assert torch.equal(q[:, :300].cpu().contiguous(), want_q.view(torch.uint8))
