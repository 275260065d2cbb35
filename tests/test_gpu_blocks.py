"""Block codes on the GPU against their definition: every code and scale exactly, every value within its rounding."""
import pytest
import torch

from oracle import blocks as O
from paper_2511_11664_amd import binding as B

pytestmark = pytest.mark.gpu

DTYPES = (torch.float32, torch.float16, torch.bfloat16)
CODE = {torch.float32: B.F32, torch.float16: B.F16, torch.bfloat16: B.BF16}
SHAPES = [(1, 1), (1, 128), (3, 129), (5, 127), (128, 128), (130, 257), (257, 136), (70, 1000), (2, 4096)]
FILL = 0xA5


def tensor(rows, cols, dtype, seed=0):
    """Magnitudes over some powers of two, whole blocks of zeros, single large channels."""
    g = torch.Generator().manual_seed(1000 * rows + cols + seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-6, 5, (rows, cols), generator=g).float())
    x[:, cols // 2] *= 40
    x[rows // 2] *= torch.rand(cols, generator=g) < 0.1
    if rows > 2:
        x[1] = 0
    return x.to(dtype)


def values(codes, fmt):
    return O.decode8(codes.cpu(), fmt)


def scale_values(scales):
    s = scales.cpu()
    return torch.exp2(s.double() - 127) if s.dtype == torch.uint8 else s.double()


def same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=1e300), torch.nan_to_num(b, nan=1e300))


def memory(rows, cols, ld, dtype, offset=0):
    """A strided matrix inside filled memory, and the memory."""
    n = rows * ld + offset + 64
    whole = torch.full((n * torch.empty(0, dtype=dtype).element_size(),), FILL, dtype=torch.uint8, device="cuda").view(dtype)
    return whole.as_strided((rows, cols), (ld, 1), offset), whole


def untouched(whole, view):
    """Nothing outside the view was written."""
    mask = torch.ones(whole.numel(), dtype=torch.bool, device="cuda")
    mask.as_strided(view.shape, view.stride(), view.storage_offset()).zero_()
    size = whole.element_size()
    return bool((whole.view(torch.uint8).view(-1, size)[mask] == FILL).all())


def quantize(x, fmt, e8m0, tile, transpose, ld=None, off=0, x_ld=None, x_off=0):
    """The codes and scales of a CPU matrix through the entry point, in memory of the given strides."""
    rows, cols = reversed(x.shape) if transpose else x.shape
    xd, _ = memory(*x.shape, x_ld or x.shape[1], x.dtype, x_off)
    xd.copy_(x)
    nb, nr = -(-cols // 128), -(-rows // 128) if tile else rows
    code, code_mem = memory(rows, cols, ld or -(-cols // 16) * 16, torch.uint8, off)
    scale, scale_mem = memory(nr, nb, nb + (3 if ld else 0), torch.uint8 if e8m0 else torch.float32, 1 if ld else 0)
    b = B.make_blocks(rows, cols, code.stride(0), scale.stride(0), fmt, int(e8m0), int(tile))
    assert B.rans_block_quantize(xd, xd.stride(0), CODE[x.dtype], transpose, code, scale, b) == 0
    torch.cuda.synchronize()
    assert untouched(code_mem, code) and untouched(scale_mem, scale)
    return code, scale, b


@pytest.mark.parametrize("transpose", (False, True))
@pytest.mark.parametrize("tile", (False, True))
@pytest.mark.parametrize("e8m0", (False, True))
@pytest.mark.parametrize("fmt", (0, 1))
@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize(dtype, fmt, e8m0, tile, transpose):
    for rows, cols in SHAPES:
        x = tensor(rows, cols, dtype)
        want, s = O.quantize(x.t() if transpose else x, fmt, e8m0, tile)
        for strides in ({}, dict(ld=(rows if transpose else cols) + 5, off=3, x_ld=cols + 3, x_off=1)):
            code, scale, _ = quantize(x, fmt, e8m0, tile, transpose, **strides)
            assert same(scale_values(scale), s), (rows, cols, strides)
            assert same(values(code, fmt), want), (rows, cols, strides)


@pytest.mark.parametrize("e8m0", (False, True))
@pytest.mark.parametrize("fmt", (0, 1))
def test_quantize_is_within_half_a_step(fmt, e8m0):
    """|code s - x| <= half a step of the format at code, (1/2) 2^-mbits of its value or of the smallest normal one, times s;
    the reciprocal and the product with it add 2^-22 of x."""
    x = tensor(64, 512, torch.float32, 5)
    code, scale, _ = quantize(x, fmt, e8m0, False, False)
    s = O.spread(scale_values(scale), 64, 512, False)
    got = values(code, fmt)
    step = 2.0 ** -(3, 2)[fmt] * torch.clamp(got.abs(), min=2.0 ** (-6, -14)[fmt])
    assert ((got * s - x.double()).abs() <= s * step / 2 + 2.0 ** -22 * x.double().abs()).all()


@pytest.mark.parametrize("transpose", (False, True))
@pytest.mark.parametrize("tile", (False, True))
@pytest.mark.parametrize("e8m0", (False, True))
@pytest.mark.parametrize("fmt", (0, 1))
def test_quantize_special_values(fmt, e8m0, tile, transpose):
    """NaN and infinities beside finite numbers, a block of nothing else, the largest and the smallest numbers, -0."""
    x = torch.zeros(6, 700)
    g = torch.Generator().manual_seed(1)
    x[:, :512] = torch.randn(6, 512, generator=g)
    x[0, 5], x[0, 130], x[1, 131], x[2, 640], x[3, 300] = float("nan"), float("inf"), float("-inf"), float("nan"), -0.0
    x[4, :128] = float("inf")
    x[5, :128] = torch.randn(128, generator=g) * 2.0 ** -140
    x[5, 128:256] = torch.randn(128, generator=g).clamp(-1, 1) * 3.4e38
    x[5, 256:384] = 2.0 ** -149
    x[5, 384:512] = torch.randn(128, generator=g) * 1e-30
    want, s = O.quantize(x.t() if transpose else x, fmt, e8m0, tile)
    code, scale, _ = quantize(x, fmt, e8m0, tile, transpose)
    assert same(scale_values(scale), s)
    assert same(values(code, fmt), want)


@pytest.mark.parametrize("fmt", (0, 1))
def test_power_of_two_scales_at_their_border(fmt):
    """Largest values at v 2^e and one binary32 number to both sides of it."""
    v = torch.tensor([O.VMAX[fmt] * 2.0 ** e for e in (-120, -9, 0, 7)])
    rows = torch.cat([v, torch.nextafter(v, v * 2), torch.nextafter(v, v * 0)])
    x = rows[:, None] * torch.cat([torch.ones(1, 1), torch.rand(1, 127, generator=torch.Generator().manual_seed(3))], 1)
    want, s = O.quantize(x, fmt, True, False)
    code, scale, _ = quantize(x, fmt, True, False, False)
    assert same(scale_values(scale), s) and same(values(code, fmt), want)


@pytest.mark.parametrize("tile", (False, True))
@pytest.mark.parametrize("e8m0", (False, True))
@pytest.mark.parametrize("fmt", (0, 1))
@pytest.mark.parametrize("dtype", DTYPES)
def test_dequantize(dtype, fmt, e8m0, tile):
    """The binary32 product of code and scale, rounded once more: all codes, NaN scales, odd strides."""
    g = torch.Generator().manual_seed(fmt + 2 * e8m0)
    for rows, cols in SHAPES:
        c = torch.randint(0, 256, (rows, cols), generator=g, dtype=torch.uint8)
        nr, nb = -(-rows // 128) if tile else rows, -(-cols // 128)
        s = torch.randint(118, 133, (nr, nb), generator=g, dtype=torch.uint8) if e8m0 else torch.rand(nr, nb, generator=g) * 0.01
        if nb > 1:
            s[0, 1] = 255 if e8m0 else float("nan")
        if nb > 2:
            s[0, 2] = 0
        want = (O.decode8(c, fmt) * O.spread(torch.where(s == 255, torch.nan, torch.exp2(s.double() - 127)) if e8m0 else s.double(), rows, cols, tile)).float().to(dtype)
        for ld, off, x_ld, x_off in ((-(-cols // 16) * 16, 0, cols, 0), (cols + 5, 3, cols + 3, 1)):
            code, _ = memory(rows, cols, ld, torch.uint8, off)
            code.copy_(c)
            out, whole = memory(rows, cols, x_ld, dtype, x_off)
            b = B.make_blocks(rows, cols, ld, nb, fmt, int(e8m0), int(tile))
            assert B.rans_block_dequantize(code, s.cuda(), b, CODE[dtype], out, x_ld) == 0
            torch.cuda.synchronize()
            assert same(out.cpu().double(), want.double()) and untouched(whole, out)


def test_block_matrix_round_trip():
    x = tensor(200, 1000, torch.bfloat16).cuda()
    m = B.BlockMatrix(200, 1000, scale_type=B.SCALE_E8M0).quantize(x)
    y = m.dequantize(torch.empty_like(x))
    t = B.BlockMatrix(1000, 200, scale_type=B.SCALE_E8M0, block=B.BLOCK_TILE).quantize(x, transpose=True)
    z = B.BlockMatrix(200, 1000, scale_type=B.SCALE_E8M0, block=B.BLOCK_TILE).quantize(x)
    assert ((y - x).abs() <= x.abs() * 2.0 ** -4 + x.abs().amax(1, keepdim=True) * 2.0 ** -17).all()
    assert torch.equal(t.code[:, :200].t(), z.code[:, :1000])  # tiles of the transpose are the transposed tiles
    with pytest.raises(B.RansError):
        m.quantize(x.t())


def test_offsets_beyond_32_bits():
    """Rows more than 2^32 codes, and bytes of the tensor, apart."""
    ld, cols = (1 << 32) - 16, 200
    x = tensor(2, cols, torch.bfloat16)
    code = torch.empty(ld + cols, dtype=torch.uint8, device="cuda").as_strided((2, cols), (ld, 1))
    xd = torch.empty(ld + cols, dtype=torch.bfloat16, device="cuda").as_strided((2, cols), (ld, 1))
    xd.copy_(x)
    scale = torch.empty(2, 2, device="cuda")
    b = B.make_blocks(2, cols, ld, 2)
    assert B.rans_block_quantize(xd, ld, B.BF16, False, code, scale, b) == 0
    want, s = O.quantize(x, 0, False, False)
    assert same(scale.cpu().double(), s) and same(values(code, 0), want)
    xd.zero_()
    assert B.rans_block_dequantize(code, scale, b, B.BF16, xd, ld) == 0
    assert same(xd.cpu().double(), (want * O.spread(s, 2, cols, False)).float().to(torch.bfloat16).double())


def test_many_short_rows():
    """More rows than a grid's second dimension holds."""
    rows = (1 << 23) + 300
    x = (torch.arange(rows, device="cuda") % 251 + 1).to(torch.float32)[:, None].contiguous()
    for transpose in (False, True):
        m = B.BlockMatrix(1, rows, block=B.BLOCK_TILE) if transpose else B.BlockMatrix(rows, 1, block=B.BLOCK_TILE)
        m.quantize(x, transpose)
        nb = -(-rows // 128)
        top = torch.nn.functional.pad(x[:, 0], (0, nb * 128 - rows)).view(nb, 128).amax(1)
        top = top / torch.full_like(top, 448)  # torch multiplies by the reciprocal of a plain number
        assert torch.equal(m.scale.reshape(-1)[:nb] if transpose else m.scale[:, 0], top)
        got = (m.code[0, :rows] if transpose else m.code[:, 0]).contiguous().view(torch.float8_e4m3fn).float()
        assert torch.equal(got, (x[:, 0] * (1 / top).repeat_interleave(128)[:rows]).to(torch.float8_e4m3fn).float())


def test_rows_of_more_than_two_to_the_28():
    """A launch holds fewer rows of these than a tile."""
    cols = (1 << 28) + 200
    for tile in (False, True):
        x = (torch.arange(cols, device="cuda") % 255 - 127).to(torch.bfloat16).repeat(2, 1)
        x[1] *= 2
        m = B.BlockMatrix(2, cols, scale_type=B.SCALE_E8M0, block=B.BLOCK_TILE if tile else B.BLOCK_ROW).quantize(x)
        y = m.dequantize(torch.empty_like(x))
        # half a step of four bits at the value, or of the smallest codes at the block's scale, at most 1 / 128 here
        assert ((y.float() - x.float()).abs() <= x.float().abs() / 16 + 1 / 128).all()
