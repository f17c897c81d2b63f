"""elasto_op_gemm_fp8 against the 64-bit sum of its definition."""
import pytest
import torch

import sublayer_reference as ref
from helpers import stream_handle
from paper_2609_10018_gb300 import binding

pytestmark = pytest.mark.gpu
BF16, GELU, RESID, F32 = (binding.EPI_BIAS_BF16, binding.EPI_BIAS_GELU_BF16, binding.EPI_BIAS_RESID_F32, binding.EPI_BIAS_F32)


def _codes(rows, cols, ld, g):
    """Random e4m3 rows of all magnitudes; 0x7F (NaN) past the columns."""
    x = torch.randn((rows, cols), generator=g) * 60
    store = torch.full((rows, ld), 0x7F, dtype=torch.uint8)
    store[:, :cols] = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return store


def _problem(M, N, K, seed, extra=0):
    g = torch.Generator().manual_seed(seed)
    ld = -(-K // 16) * 16 + 16 * extra
    a, w = _codes(M, K, ld, g), _codes(N, K, ld, g)
    sa = torch.rand((ref.blocks(K), M + 3 * extra), generator=g) * 0.02 + 1e-3
    sw = torch.rand((ref.blocks(N), ref.blocks(K)), generator=g) * 2e-3 + 1e-4
    return a, sa, w, sw, torch.randn(N, generator=g)


def _call(a, sa, w, sw, bias, out, ldo, M, N, K, epi, stream=None):
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.elasto_op_gemm_fp8(stream or stream_handle(), a.data_ptr(), a.stride(0), sa.data_ptr(), sa.stride(0), w.data_ptr(),
                               w.stride(0), sw.data_ptr(), None if bias is None else bias.data_ptr(), out.data_ptr(), ldo, M, N,
                               K, epi, st.data_ptr())
    return st


def _bound(mag, K):
    """fp32 sums of K products and a scaled addition (two roundings) for each block, in any order:
    every operation rounds by at most 2^-24 of a partial sum, which the sum of magnitudes bounds."""
    return (K + 3 * ref.blocks(K) + 4) * 2.0 ** -24 * mag


def _check(M, N, K, epi, extra=0, pad=0, bias=True):
    a, sa, w, sw, b = _problem(M, N, K, M * 7 + N * 3 + K, extra)
    acc, mag = ref.gemm_fp8(a.view(torch.float8_e4m3fn), sa[:, :M], w.view(torch.float8_e4m3fn), sw, K)
    want = acc + b.double() if bias else acc
    mag = mag + b.double().abs() if bias else mag
    dtype = torch.float32 if epi in (RESID, F32) else torch.bfloat16
    out = torch.randn((M, N + pad), generator=torch.Generator().manual_seed(1)).to(dtype)
    before = out.clone()
    if epi == RESID:
        want, mag = want + out[:, :N].double(), mag + out[:, :N].double().abs()
    tol = _bound(mag, K)
    if epi == GELU:  # slope at most 1.13; the approximation is off by 2.52e-5 at most
        want, tol = torch.nn.functional.gelu(want), 1.13 * tol + 2.6e-5
    if dtype == torch.bfloat16:
        tol = tol * (1 + ref.half_step(dtype)) + ref.half_step(dtype) * want.abs()
    d = [t.cuda() for t in (a, sa, w, sw, b)]
    do = out.cuda()
    st = _call(*d[:4], d[4] if bias else None, do, N + pad, M, N, K, epi)
    got = do.cpu()
    assert int(st.item()) == 0
    err = (got[:, :N].double() - want).abs()
    assert (err <= tol).all(), (float((err - tol).max()), float((err / mag).max()))
    assert torch.equal(got[:, N:], before[:, N:])


SIZES = [(1, 1, 1), (1, 64, 128), (2, 100, 16), (3, 257, 300), (8, 512, 1024), (16, 130, 129), (17, 96, 2000), (33, 1000, 256),
         (64, 129, 640), (65, 300, 500), (127, 128, 128), (128, 128, 256), (129, 255, 384), (200, 576, 392), (300, 64, 4096),
         (513, 1030, 777), (1000, 200, 136), (1, 2048, 4000), (5, 3000, 900)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("epi", [BF16, F32])
def test_sizes(M, N, K, epi):
    _check(M, N, K, epi)


@pytest.mark.parametrize("M,N,K", [(2560, 2304, 256), (2500, 2101, 392), (5000, 1100, 136), (257, 20000, 130)])
@pytest.mark.parametrize("epi", [BF16, GELU, RESID, F32])
def test_large_outputs(M, N, K, epi):
    """Enough tiles for CTA pairs; whole, ragged and odd."""
    _check(M, N, K, epi)


@pytest.mark.parametrize("M,N,K", [(1, 64, 128), (12, 257, 300), (129, 255, 384), (513, 1030, 777), (300, 512, 1152)])
@pytest.mark.parametrize("epi", [GELU, RESID])
def test_gelu_and_residual(M, N, K, epi):
    _check(M, N, K, epi)


@pytest.mark.parametrize("M,N,K", [(4, 100, 200), (40, 136, 200), (130, 136, 300), (260, 264, 520)])
@pytest.mark.parametrize("epi", [BF16, GELU, RESID, F32])
@pytest.mark.parametrize("extra,pad", [(1, 0), (2, 7), (1, 8)])
def test_strides(M, N, K, epi, extra, pad):
    _check(M, N, K, epi, extra, pad)


@pytest.mark.parametrize("M", [3, 200])
def test_no_bias_and_unaligned_output(M):
    _check(M, 192, 256, BF16, bias=False)
    a, sa, w, sw, b = (t.cuda() for t in _problem(M, 192, 256, 5))
    aligned = torch.empty((M, 192), dtype=torch.bfloat16, device="cuda")
    shifted = torch.empty(M * 192 + 1, dtype=torch.bfloat16, device="cuda")[1:]
    _call(a, sa, w, sw, b, aligned, 192, M, 192, 256, BF16)
    _call(a, sa, w, sw, b, shifted, 192, M, 192, 256, BF16)
    assert torch.equal(aligned.view(-1), shifted)


@pytest.mark.parametrize("M,N,K", [(6, 400, 1500), (300, 400, 1500)])
def test_same_result_every_call(M, N, K):
    """Nothing in the order of sums depends on the launch."""
    a, sa, w, sw, b = (t.cuda() for t in _problem(M, N, K, 11))
    outs = [torch.empty((M, N), device="cuda") for _ in range(3)]
    for o in outs:
        _call(a, sa, w, sw, b, o, N, M, N, K, F32)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_scales_of_zero_infinity_and_nan():
    """A scale reaches its own row or block of columns, and no other."""
    M, N, K = 140, 300, 260
    a, sa, w, sw, b = _problem(M, N, K, 13)
    sa[1, 7], sw[2, 0], sa[0, 9] = float("nan"), 0.0, float("inf")
    want, mag = ref.gemm_fp8(a.view(torch.float8_e4m3fn), sa, w.view(torch.float8_e4m3fn), sw, K)
    want = want + b.double()
    out = torch.empty((M, N), device="cuda")
    _call(*(t.cuda() for t in (a, sa, w, sw, b)), out, N, M, N, K, F32)
    got = out.cpu().double()
    rows = [r for r in range(M) if r not in (7, 9)]
    assert (((got - want).abs() <= _bound(mag + b.double().abs(), K))[rows]).all()
    assert got[7].isnan().all() and not got[9].isfinite().any()


def test_streams_at_once_and_graphs():
    """Two streams at once; two captured graphs replayed together read their new inputs."""
    problems = [_problem(70, 260, 500, s) for s in (1, 2)]
    dev = [[t.cuda() for t in p] for p in problems]
    outs = [torch.zeros((70, 260), device="cuda") for _ in dev]
    streams = [torch.cuda.Stream() for _ in dev]
    torch.cuda.synchronize()
    graphs = []
    for p, o, s in zip(dev, outs, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            _call(*p, o, 260, 70, 260, 500, F32, torch.cuda.current_stream().cuda_stream)
        graphs.append(graph)
    for seed in (21, 22):
        fresh = [_problem(70, 260, 500, seed + 10 * i) for i in range(2)]
        for p, f in zip(dev, fresh):
            for t, n in zip(p, f):
                t.copy_(n)
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for f, o in zip(fresh, outs):
            want, mag = ref.gemm_fp8(f[0].view(torch.float8_e4m3fn), f[1], f[2].view(torch.float8_e4m3fn), f[3], 500)
            err = (o.cpu().double() - want - f[4].double()).abs()
            assert (err <= _bound(mag + f[4].double().abs(), 500)).all()
