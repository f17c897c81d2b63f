"""elasto_op_residual_norm against its 64-bit definition."""
import pytest
import torch

import block_reference as block
import sublayer_reference as ref
from helpers import stream_handle
from paper_2609_10018_gb300 import binding

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
CODES = {F32: binding.F32, BF16: binding.BF16, F16: binding.F16, torch.float8_e4m3fn: binding.E4M3}
NONE, RMS, LAYER = block.NONE, block.RMS, block.LAYER


def _at(shape, dtype, pad=0, offset=0):
    """A view [rows, cols] whose rows are cols + pad apart and start `offset` values behind an aligned address."""
    rows, cols = shape
    whole = torch.zeros(rows * (cols + pad) + offset + 64, dtype=dtype, device="cuda")
    return whole[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


class Case:
    def __init__(self, rows, cols, x=F32, y=BF16, z=BF16, post=NONE, pre=LAYER, affine=True, y_scale=False, mod=None, groups=0,
                 factor=1.0, pad=0, offset=0, seed=0, eps=1e-6):
        g = torch.Generator().manual_seed(seed + 31 * rows + cols)
        rand = lambda *s: torch.randn(s, generator=g)  # noqa: E731
        self.rows, self.cols, self.z_type, self.groups, self.factor, self.eps, self.mod = rows, cols, z, groups, factor, eps, mod
        self.x = (2 * rand(rows, cols) + 0.3).to(x)
        self.y = None if y is None else (rand(rows, cols) * torch.exp(0.5 * rand(cols)) - 0.2).to(y)
        self.post, self.pre = post, pre
        self.v = {n: None for n in ("post_gain", "post_bias", "y_scale", "pre_gain", "pre_bias")}
        if affine:
            for n in ("post", "pre"):
                if getattr(self, n) != NONE:
                    self.v[n + "_gain"] = 1 + 0.2 * rand(cols)
                if getattr(self, n) == LAYER:
                    self.v[n + "_bias"] = 0.2 * rand(cols)
        if y_scale:
            self.v["y_scale"] = 0.3 * rand(cols)
        self.tables = {n: rand(groups, cols).mul(0.4).to(mod) if mod else None for n in ("gate", "shift", "scale")}
        self.group = torch.randint(0, groups, (rows,), generator=g, dtype=torch.int32) if mod else None
        self.pad, self.offset = pad, offset

    def device(self, in_place=False):
        d = {}
        for n, t in (("x", self.x), ("y", self.y)):
            if t is not None:
                d[n] = _at(t.shape, t.dtype, self.pad, self.offset)
                d[n].copy_(t)
        d["x_out"] = d["x"] if in_place else _at(self.x.shape, self.x.dtype, self.pad, self.offset)
        d["z"] = _at(self.x.shape, self.z_type if self.z_type != torch.float8_e4m3fn else torch.uint8, self.pad, self.offset)
        d["z_scale"] = torch.zeros((ref.blocks(self.cols), self.rows + 3), device="cuda")
        d |= {n: None if t is None else t.cuda() for n, t in (self.v | self.tables).items()}
        d["group"] = None if self.group is None else self.group.cuda()
        return d

    def args(self, d, **kw):
        a = dict(rows=self.rows, cols=self.cols, eps=self.eps, x_factor=self.factor, x_type=CODES[self.x.dtype],
                 post_norm=self.post, pre_norm=self.pre, groups=self.groups, z_type=CODES[self.z_type])
        for n in ("x", "y", "x_out", "z", "z_scale"):
            if d.get(n) is not None:
                a |= {n: d[n].data_ptr(), n + "_row": d[n].stride(0)}
        if self.y is not None:
            a["y_type"] = CODES[self.y.dtype]
        for n in list(self.v) + list(self.tables) + ["group"]:
            if d.get(n) is not None:
                a[n] = d[n].data_ptr()
        if self.mod:
            a |= dict(mod_type=CODES[self.mod], mod_row=self.cols)
        return binding.ResidualNorm(**(a | kw))

    def want(self):
        return block.residual_norm(self.x, self.y, self.factor, self.post, pre=self.pre, eps=self.eps, **self.v, **self.tables,
                                   group=None if self.group is None else self.group.long())

    def check(self, d, rows=slice(None)):
        s, z, ds, dz = (t[rows] for t in self.want())
        got = d["x_out"].cpu()[rows]
        assert ((got.double() - s).abs() <= ds + ref.half_step(got.dtype) * (s.abs() + ds) + _tiny(got.dtype)).all()
        if self.z_type != torch.float8_e4m3fn:
            got = d["z"].cpu()[rows]
            err = (got.double() - z).abs() - (dz + ref.half_step(got.dtype) * (z.abs() + dz) + _tiny(got.dtype))
            assert (err <= 0).all(), float(err.max())
            return
        codes = d["z"].cpu()[rows].contiguous().view(torch.float8_e4m3fn).double()
        for b in range(ref.blocks(self.cols)):
            cols = slice(128 * b, min(self.cols, 128 * b + 128))
            top = z[:, cols].abs().amax(1).clamp_min(ref.MIN_AMAX)
            scale = d["z_scale"][b, :self.rows].cpu()[rows].double()
            assert ((scale - top / 448).abs() <= dz[:, cols].amax(1) / 448 + 2.0 ** -22 * scale).all()
            want = z[:, cols] / scale[:, None]
            # (448 / a is rounded, and the product with it: 2^-22 of a value)
            err = (codes[:, cols] - want).abs() - (dz[:, cols] / scale[:, None] + 2.0 ** -22 * want.abs())
            assert (err <= block.e4m3_half_step(want) * (1 + 2.0 ** -10)).all()


def _tiny(dtype):
    """Half a step of subnormals."""
    return torch.finfo(dtype).tiny * torch.finfo(dtype).eps / 2


def _run(args):
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.elasto_op_residual_norm(stream_handle(), args, st.data_ptr())
    return int(st.item())


@pytest.mark.parametrize("z", [BF16, torch.float8_e4m3fn])
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 1)])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (5, 7), (2, 8), (9, 64), (4, 100), (7, 127), (3, 128), (2, 129), (130, 192), (5, 255),
                                       (6, 257), (33, 768), (2, 769), (3, 1000), (5, 1536), (1, 2047), (2, 4096), (3, 5000), (1, 6145),
                                       (1, 8192), (2, 12289), (1, 16384)])
def test_sizes(rows, cols, pad, offset, z):
    c = Case(rows, cols, z=z, post=RMS, pre=LAYER, y_scale=True, pad=pad, offset=offset)
    d = c.device()
    assert _run(c.args(d)) == 0
    c.check(d)


@pytest.mark.parametrize("cols", [200, 333, 2064])
@pytest.mark.parametrize("x,y,z", [(F32, F32, F32), (BF16, BF16, BF16), (F16, F16, F16), (F32, F16, F16), (BF16, F32, F32), (F16, BF16, F32),
                                   (BF16, F16, torch.float8_e4m3fn), (F32, BF16, torch.float8_e4m3fn)])
def test_types(x, y, z, cols):
    c = Case(19, cols, x, y, z, post=LAYER, pre=RMS, mod=BF16, groups=4)
    d = c.device()
    assert _run(c.args(d)) == 0
    c.check(d)


@pytest.mark.parametrize("cols", [96, 1031])
@pytest.mark.parametrize("mod", [None, F32, BF16, F16])
@pytest.mark.parametrize("post,pre", [(NONE, NONE), (NONE, RMS), (RMS, NONE), (LAYER, LAYER), (RMS, RMS)])
def test_norms_and_tables(post, pre, mod, cols):
    for affine in (False, True):
        c = Case(21, cols, F32, F32, F32, post, pre, affine, y_scale=affine, mod=mod, groups=5 if mod else 0, factor=0.75)
        d = c.device()
        assert _run(c.args(d)) == 0
        c.check(d)


def test_one_table_for_all_rows():
    c = Case(10, 320, mod=BF16, groups=1)
    d = c.device()
    assert _run(c.args(d)) == 0
    other = d["z"].clone()
    assert _run(c.args(d, group=None)) == 0
    assert torch.equal(other, d["z"])
    c.check(d)


@pytest.mark.parametrize("cols", [768, 1155])
def test_in_place_and_single_outputs(cols):
    c = Case(50, cols, post=RMS)
    d = c.device()
    assert _run(c.args(d)) == 0
    both = d["x_out"].clone(), d["z"].clone()
    d["z"].zero_()
    assert _run(c.args(d, x_out=None)) == 0
    assert torch.equal(d["z"], both[1])
    d["x_out"].zero_()
    assert _run(c.args(d, z=None)) == 0
    assert torch.equal(d["x_out"], both[0])
    d = c.device(in_place=True)
    assert _run(c.args(d)) == 0
    assert torch.equal(d["x"], both[0]) and torch.equal(d["z"], both[1])


def test_without_a_block():
    """The norm alone, of a factor times the stream."""
    c = Case(11, 384, y=None, pre=LAYER, factor=2.0)
    d = c.device()
    assert _run(c.args(d)) == 0
    c.check(d)


@pytest.mark.parametrize("cols,z", [(64, BF16), (67, F32), (640, torch.float8_e4m3fn)])
def test_groups_outside_are_left_out(cols, z):
    c = Case(40, cols, z=z, mod=F32, groups=3)
    bad = [0, 17, 39]
    for b, v in zip(bad, (-1, 3, 2 ** 31 - 1)):
        c.group[b] = v
    d = c.device()
    d["x_out"].fill_(7), d["z"].fill_(9), d["z_scale"].fill_(11)
    assert _run(c.args(d)) == binding.ERR_INVALID_ARG
    good = torch.tensor([r for r in range(40) if r not in bad])
    for b in bad:
        c.group[b] = 0
    c.check(d, good)
    assert (d["x_out"][bad] == 7).all() and (d["z"][bad] == 9).all()
    if z == torch.float8_e4m3fn:
        assert (d["z_scale"][:, bad] == 11).all()
    assert (d["z_scale"][:, 40:] == 11).all()


def test_values_that_are_not_finite_stay_in_their_rows():
    c = Case(8, 256, post=RMS)
    d = c.device()
    assert _run(c.args(d)) == 0
    clean = d["x_out"].clone(), d["z"].clone()
    d["x"][3, 7], d["y"][5, 200] = float("nan"), float("inf")
    assert _run(c.args(d)) == 0
    same = [0, 1, 2, 4, 6, 7]
    assert torch.equal(d["x_out"][same], clean[0][same]) and torch.equal(d["z"][same], clean[1][same])
    assert torch.isnan(d["z"][3]).all() and torch.isnan(d["x_out"][5, 200])


@pytest.mark.parametrize("cols", [256, 250])
def test_e4m3_rows_of_zeros_nan_and_infinities(cols):
    """As elasto_op_quantize_fp8: a block of zeros has the smallest scale, a NaN takes its block."""
    c = Case(4, cols, y=None, z=torch.float8_e4m3fn, pre=NONE)
    c.x[0] = 0
    c.x[1, 3] = float("nan")
    c.x[2, 130] = float("inf")
    d = c.device()
    assert _run(c.args(d)) == 0
    q, scale = ref.quantize(c.x)
    assert torch.equal(d["z"].cpu(), q.view(torch.uint8)) or torch.equal(
        torch.nan_to_num(d["z"].cpu().contiguous().view(torch.float8_e4m3fn).float(), nan=-1.0), torch.nan_to_num(q.float(), nan=-1.0))
    got = d["z_scale"][:, :4].cpu()
    assert torch.equal(torch.nan_to_num(got, nan=-1.0), torch.nan_to_num(scale, nan=-1.0))


def test_e4m3_rows_are_those_of_the_quantiser():
    """Without a norm: the bytes of elasto_op_quantize_fp8 on the stream, and nothing past the columns."""
    for cols in (768, 700, 131):
        c = Case(60, cols, z=torch.float8_e4m3fn, pre=NONE, pad=5)
        d = c.device()
        d["z"]._base.fill_(77)
        assert _run(c.args(d)) == 0
        q = torch.zeros((60, cols), dtype=torch.uint8, device="cuda")
        scale = torch.zeros((ref.blocks(cols), 60), device="cuda")
        binding.elasto_op_quantize_fp8(stream_handle(), d["x_out"].data_ptr(), binding.F32, d["x_out"].stride(0), q.data_ptr(), cols,
                                       scale.data_ptr(), 60, 60, cols)
        assert torch.equal(q, d["z"]) and torch.equal(scale, d["z_scale"][:, :60])
        assert (d["z"]._base.view(-1)[:60 * (cols + 5)].view(60, cols + 5)[:, cols:] == 77).all()


@pytest.mark.parametrize("cols,pad", [(8, 0), (100, 1), (200, 0), (384, 0), (1031, 3), (1536, 0), (6200, 0), (6201, 0)])
@pytest.mark.parametrize("eps", [0.0, 1e-38])
@pytest.mark.parametrize("post,pre,z", [(NONE, RMS, F32), (NONE, LAYER, F32), (RMS, LAYER, BF16), (LAYER, NONE, F32), (NONE, RMS, torch.float8_e4m3fn)])
def test_small_rows(post, pre, z, eps, cols, pad):
    """Rows whose squares are subnormal or 0 in fp32, beside rows of ordinary size: normed like these where eps leaves them."""
    c = Case(23, cols, F32, F32, z, post, pre, pad=pad, offset=pad, eps=eps)
    size = torch.tensor([1.0, 1e-17, 1e-18, 3e-19, 1e-19, 3e-20, 1e-20, 1e-21, 1e-22, 1e-23, 1e-24, 1e-27, 1e-30, 1e-34, 1.0, 1e3, 1e-26, 1e-10])
    size = torch.cat([size, 1e-25 * torch.ones(c.rows - len(size))])[:, None]
    c.x *= size
    c.y *= size
    d = c.device()
    assert _run(c.args(d)) == 0
    c.check(d)


def test_same_bits_captured_and_on_another_stream():
    c = Case(300, 1536, BF16, BF16, BF16, LAYER, LAYER, mod=BF16, groups=7)
    d = c.device()
    assert _run(c.args(d)) == 0
    want = d["x_out"].clone(), d["z"].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        binding.elasto_op_residual_norm(stream_handle(), c.args(d))
    d["x_out"].zero_(), d["z"].zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(d["x_out"], want[0]) and torch.equal(d["z"], want[1])


def test_offsets_past_32_bits():
    """Rows so far apart that an element's offset passes 2^32."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    rows, cols, row = 3, 64, (1 << 31) + 16
    whole = torch.empty((rows - 1) * row + cols, dtype=BF16, device="cuda")
    view = whole.as_strided((rows, cols), (row, 1))
    c = Case(rows, cols, BF16, None, BF16, pre=RMS)
    view.copy_(c.x)
    d = c.device()
    d["x"] = d["x_out"] = view
    assert _run(c.args(d)) == 0
    c.check(d)


@pytest.mark.parametrize("x,y,z,mod", [(F32, BF16, BF16, BF16), (BF16, F32, torch.float8_e4m3fn, F32), (BF16, BF16, F32, None)])
@pytest.mark.parametrize("rows,cols,pad", [(60000, 104, 0), (60000, 100, 0), (30000, 256, 0), (30000, 257, 1), (9000, 1536, 0), (9000, 1535, 0),
                                           (9000, 1536, 3), (3000, 5000, 0), (3000, 4999, 2), (700, 8192, 0), (700, 8191, 0)])
def test_many_rows_through_the_ring(rows, cols, pad, x, y, z, mod):
    """Several times as many rows as the rings of all SMs hold (152 CTAs of up to 24 teams with up to four stages each): a stage
    is copied into again and again, with another alignment and another group's tables each time. In place, and the same
    bits beside."""
    c = Case(rows, cols, x, y, z, RMS, LAYER, affine=mod is not None, y_scale=True, mod=mod, groups=7 if mod else 0, pad=pad, offset=pad)
    d = c.device(in_place=True)
    assert _run(c.args(d)) == 0
    c.check(d)
    e = c.device()
    assert _run(c.args(e)) == 0
    assert torch.equal(d["x"], e["x_out"]) and torch.equal(d["z"], e["z"]) and torch.equal(d["z_scale"], e["z_scale"])
