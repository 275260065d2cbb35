"""Every kernel of the product of two coded matrices - few rows, each tile with fetches and at any alignment, K in parts - with
every kind of scales and pair of formats, against 64 bits; each case says which kernel it runs.

Binary32 results, relative to S = |A| |B|^T: (128 + K / 128 + 4) 2^-23, as a block's 128 products, the blocks and the scales' product
are rounded.  Sixteen-bit results: the 8-bit instruction adds groups of eight products and cuts off what lies 2^-13 below the
largest of them, 7 * 2^-13 S at most, and half a step of the type.  That is the worst there can be; the sums of random products
are off by far less, which the norms show: |C - AB| as a norm is the rounding's and the sums' together."""
import math

import pytest
import torch

from paper_2511_11664_amd import binding as B

pytestmark = pytest.mark.gpu

F8 = (torch.float8_e4m3fn, torch.float8_e5m2)
OUT = {torch.float32: B.F32, torch.float16: B.F16, torch.bfloat16: B.BF16}
SCALES = {"tile": (B.SCALE_F32, B.BLOCK_TILE), "row": (B.SCALE_F32, B.BLOCK_ROW), "powers of two": (B.SCALE_E8M0, B.BLOCK_TILE),
          "powers of two, rows": (B.SCALE_E8M0, B.BLOCK_ROW)}
FORMATS = ((0, 0), (1, 0), (0, 1), (1, 1))  # forward, input and weight gradient, and the ones that no path has


def coded(x, fmt, scale_type, block, off=None):
    """Codes of a matrix by torch: (codes, scales, layout, values in 64 bits).  off: rows of codes end on end, from that address on."""
    rows, cols = x.shape
    nr, nb = -(-rows // 128) if block else rows, -(-cols // 128)
    g = torch.Generator(device="cuda").manual_seed(rows * 7 + cols)
    if scale_type:
        s = torch.randint(121, 124, (nr, nb), generator=g, device="cuda", dtype=torch.uint8)
        sv = torch.exp2(s.double() - 127)
    else:
        s = 0.01 + 0.05 * torch.rand(nr, nb, generator=g, device="cuda")
        sv = s.double()
    c = (x * 2.0 ** (4, 3)[fmt]).clamp(-400, 400).to(F8[fmt])
    ld, lds = (-(-cols // 16) * 16, -(-nb // 4) * 4) if off is None else (cols, nb)
    off = off or 0
    code = torch.full((rows * ld + off + 16,), 0x7f, dtype=torch.uint8, device="cuda").as_strided((rows, cols), (ld, 1), off)  # NaN beside the codes
    code.copy_(c.view(torch.uint8))
    scale = torch.full((nr * lds,), 255 if scale_type else float("nan"), dtype=s.dtype, device="cuda").as_strided((nr, nb), (lds, 1))
    scale.copy_(s)
    if block:
        sv = sv.repeat_interleave(128, 0)[:rows]
    return code, scale, B.make_blocks(rows, cols, ld, lds, fmt, scale_type, block), c.double() * sv.repeat_interleave(128, 1)[:, :cols]


def operands(m, n, k, scales, formats, off=None):
    st, block = SCALES[scales]
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    a, b = (torch.randn(r, k, generator=g, device="cuda") for r in (m, n))
    return coded(a, formats[0], st, B.BLOCK_ROW, off), coded(b, formats[1], st, block, off)


def run(a, b, out, ld_c, launched_kernels):
    m, n = a[2].rows, b[2].rows
    whole = torch.full((m * ld_c + 16,), 99.0, dtype=out, device="cuda")
    c = whole.as_strided((m, n), (ld_c, 1))
    size = B.rans_matmul_workspace_bytes(a[2], b[2])[1]
    ws = B.workspace(size) if size else None
    rc = []
    names = launched_kernels(lambda: rc.append(B.rans_block_matmul(*a[:3], *b[:3], OUT[out], c, ld_c, ws)))
    assert rc == [0]
    mask = torch.ones(whole.numel(), dtype=torch.bool, device="cuda")
    mask.as_strided((m, n), (ld_c, 1)).zero_()
    assert (whole[mask] == 99).all()
    return c, names


def check(c, a, b, what):
    out, k = c.dtype, a[2].cols
    bt = b[3].t().contiguous()
    want, total = a[3] @ bt, a[3].abs() @ bt.abs()
    f = torch.finfo(out)
    rounding = want.abs() * f.eps / 2 + f.smallest_normal * f.eps / 2
    tol = (128 + k / 128 + 4) * 2.0 ** -23 * total if out == torch.float32 else 7 * 2.0 ** -13 * total + 1.01 * rounding
    d = (c.double() - want).abs()
    assert want.abs().max() < f.max / 2 and (d <= tol).all(), (what, d.max().item(), (d > tol).sum().item())
    # the norms: 1e-4 of the result's for sums of 16-bit results, 2^-20 for those of binary32
    sums = 2.0 ** -20 if out == torch.float32 else 1e-4
    nearest = (want.to(out).double() - want).norm() if out != torch.float32 else 0.0
    assert d.norm() <= math.hypot(nearest, sums * want.norm()), (what, (d.norm() / want.norm()).item())


def case(m, n, k, out, scales, formats, name, launched_kernels, off=None, extra=0):
    a, b = operands(m, n, k, scales, formats, off)
    c, names = run(a, b, out, n + extra, launched_kernels)
    what = (m, n, k, str(out), scales, formats)
    assert names == set(name), (what, names)
    check(c, a, b, what)


@pytest.mark.parametrize("formats", FORMATS)
@pytest.mark.parametrize("scales", tuple(SCALES))
@pytest.mark.parametrize("out", tuple(OUT))
def test_few_rows(out, scales, formats, launched_kernels):
    """Two to 32 rows: one and two groups of 16, whole ones and some cut off; a short last block, rows that start anywhere."""
    for i, (m, n, k) in enumerate(((2, 1000, 4096), (4, 1003, 4100), (13, 2048, 4133), (16, 1003, 2500), (17, 1000, 4096), (24, 2040, 4099), (32, 1003, 3990))):
        case(m, n, k, out, scales, formats, ["k_block_matmul_few"], launched_kernels, off=(None, None, 3)[i % 3], extra=i % 2)


@pytest.mark.parametrize("formats", ((0, 0), (1, 0)))
@pytest.mark.parametrize("scales", ("tile", "powers of two", "powers of two, rows"))
@pytest.mark.parametrize("out", (torch.float16, torch.bfloat16))
def test_256_tiles(out, scales, formats, launched_kernels):
    """Whole tiles and such cut off on both sides; less than a block, an odd and an even number of whole ones, with and without a
    short one behind them."""
    for m, n, k, extra in ((3900, 4000, 300, 3), (4096, 4096, 512, 0), (3841, 4095, 641, 1), (4096, 3841, 100, 0), (4000, 4090, 384, 2), (4096, 4096, 128, 0)):
        case(m, n, k, out, scales, formats, ["k_block_matmul_256"], launched_kernels, extra=extra)


@pytest.mark.parametrize("formats", FORMATS)
@pytest.mark.parametrize("scales", tuple(SCALES))
@pytest.mark.parametrize("out", tuple(OUT))
def test_128_tiles(out, scales, formats, launched_kernels):
    """Two stages, four where each tile has a compute unit to itself, and any alignment."""
    least = 0 if out == torch.float32 else 1024  # blocks from which on four stages pay
    for m, n, k, extra in ((2050, 2060, 300, 1), (2176, 2048, 512, 0)):
        case(m, n, k, out, scales, formats, ["k_block_matmul_128"], launched_kernels, extra=extra)
    for m, n, k, extra in ((1000, 3990, 45 + least, 1), (1024, 4096, 128 + least, 0), (1000, 4000, 640 + least, 2), (1020, 4090, 513 + least, 3)):
        name = "k_block_matmul_deep" if k >= max(least, 128) else "k_block_matmul_128"
        case(m, n, k, out, scales, formats, [name], launched_kernels, extra=extra)
    for m, n, k, extra in ((2050, 2060, 300, 1), (2048, 2100, 515, 0)):
        case(m, n, k, out, scales, formats, ["k_block_matmul_any_128"], launched_kernels, off=1, extra=extra)


@pytest.mark.parametrize("formats", FORMATS)
@pytest.mark.parametrize("scales", tuple(SCALES))
@pytest.mark.parametrize("out", tuple(OUT))
def test_64_tiles_and_parts(out, scales, formats, launched_kernels):
    sums, tiles = ["k_block_matmul_sum"], ["k_block_matmul_128" if formats[1] and out != torch.float32 else "k_block_matmul"]
    for m, n, k in ((100, 257, 1001), (64, 130, 512), (33, 65, 2300)):
        case(m, n, k, out, scales, formats, ["k_block_matmul_deep" if tiles[0][-1] == "8" and k >= 1024 else tiles[0]], launched_kernels, extra=1)
        case(m, n, k, out, scales, formats, ["k_block_matmul_any"], launched_kernels, off=5)
    for m, n, k in ((64, 64, 4096), (100, 257, 4400), (48, 130, 16385)):
        name = "k_block_matmul_deep" if tiles[0][-1] == "8" else tiles[0]
        case(m, n, k, out, scales, formats, sums + [name], launched_kernels)
        case(m, n, k, out, scales, formats, sums + ["k_block_matmul_any"], launched_kernels, off=5, extra=1)
