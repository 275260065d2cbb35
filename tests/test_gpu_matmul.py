"""The product of two coded matrices on the GPU against 64 bits.

Tolerances, relative to S = |A| |B|^T with the scales in it.  Binary32 results: a block's 128 products are added with at most
128 errors of 2^-23, the two scales' product is rounded once, and every block's sum is added with one more:
(128 + K / 128 + 4) 2^-23 S.  Sixteen-bit results: the 8-bit instruction adds groups of eight products and cuts off what lies
2^-13 below the largest of them, 7 * 2^-13 of it at most, so of S; half a step of the type of the result on top."""
import math

import pytest
import torch

from oracle import blocks as O
from paper_2511_11664_amd import binding as B

pytestmark = pytest.mark.gpu

OUT = {torch.float32: B.F32, torch.float16: B.F16, torch.bfloat16: B.BF16}
SHAPES = [(1, 1, 1), (1, 16, 128), (1, 300, 4096), (2, 130, 129), (3, 77, 1000), (8, 256, 512), (15, 96, 144), (16, 1000, 384), (17, 33, 127), (31, 128, 260),
          (33, 65, 640), (64, 384, 256), (65, 129, 96), (100, 257, 1001), (128, 128, 128), (129, 300, 272), (256, 512, 1024), (257, 255, 520), (300, 130, 2100), (520, 768, 384)]


def half_step(v, dtype):
    f = torch.finfo(dtype)
    return v.abs() * f.eps / 2 + f.smallest_normal * f.eps / 2


def coded(rows, cols, fmt, e8m0, tile, seed, tight=False, off=0):
    """Random codes without NaN and infinities and random scales, on the GPU; their values in 64 bits."""
    g = torch.Generator().manual_seed(seed)
    c = (torch.randn(rows, cols, generator=g) * 2.0 ** (5, 9)[fmt]).to((torch.float8_e4m3fn, torch.float8_e5m2)[fmt]).view(torch.uint8)
    nr, nb = -(-rows // 128) if tile else rows, -(-cols // 128)
    s = torch.randint(120, 126, (nr, nb), generator=g, dtype=torch.uint8) if e8m0 else 0.01 + 0.05 * torch.rand(nr, nb, generator=g)
    ld, lds = (cols, nb) if tight else (-(-cols // 16) * 16, -(-nb // 4) * 4)
    code = torch.full((rows * ld + off + 16,), 0x7f, dtype=torch.uint8, device="cuda").as_strided((rows, cols), (ld, 1), off)  # NaN beside the codes
    code.copy_(c)
    scale = torch.full((nr * lds,), 255 if e8m0 else float("nan"), dtype=s.dtype, device="cuda").as_strided((nr, nb), (lds, 1))
    scale.copy_(s)
    sv = torch.exp2(s.double() - 127) if e8m0 else s.double()
    return code, scale, B.make_blocks(rows, cols, ld, lds, fmt, int(e8m0), int(tile)), O.decode8(c, fmt) * O.spread(sv, rows, cols, tile)


def product(a, b, out, ld_c=None):
    m, n = a[2].rows, b[2].rows
    ld_c = ld_c or n
    whole = torch.full((m * ld_c + 16,), 99.0, dtype=out, device="cuda")
    c = whole.as_strided((m, n), (ld_c, 1))
    rc, size = B.rans_matmul_workspace_bytes(a[2], b[2])
    assert rc == 0
    ws = B.workspace(size) if size else None
    assert B.rans_block_matmul(*a[:3], *b[:3], OUT[out], c, ld_c, ws) == 0
    torch.cuda.synchronize()
    mask = torch.ones(whole.numel(), dtype=torch.bool, device="cuda")
    mask.as_strided((m, n), (ld_c, 1)).zero_()
    assert (whole[mask] == 99).all()
    return c


def check(c, a, b, out, what=None):
    want, total = O.matmul(a[3], b[3])
    k = a[2].cols
    if out == torch.float32:
        tol = (128 + k / 128 + 4) * 2.0 ** -23 * total
    else:
        tol = 7 * 2.0 ** -13 * total + half_step(want, out) * 1.01
    got = c.cpu().double()
    d = (got - want).abs()
    # Half a step behind the type's largest value (65504 + 16 in binary16) rounding to nearest gives infinity, of the value's sign.
    top = torch.finfo(out).max + 2.0 ** math.floor(math.log2(torch.finfo(out).max)) * torch.finfo(out).eps / 2
    d[got.isinf() & (got.sign() == want.sign()) & (want.abs() + tol >= top)] = 0
    assert (d <= tol).all(), (what, d.max().item(), (d > tol).sum().item())


@pytest.mark.parametrize("tile", (False, True))
@pytest.mark.parametrize("e8m0", (False, True))
@pytest.mark.parametrize("out", tuple(OUT))
def test_matmul(out, e8m0, tile):
    for i, (m, n, k) in enumerate(SHAPES):
        a = coded(m, k, 0, e8m0, False, 3 * i, tight=i % 4 == 3)
        b = coded(n, k, 0, e8m0, tile, 3 * i + 1, tight=i % 4 == 3)
        check(product(a, b, out, n + (0, 4, 3)[i % 3]), a, b, out, (m, n, k))


@pytest.mark.parametrize("scales", ((False, True), (False, False), (True, True)))
@pytest.mark.parametrize("out", tuple(OUT))
def test_matmul_large(out, scales):
    """Sizes that take the 128 x 128 tiles, with two and with four stages, and the 256 x 256 ones; whole ones and some cut off."""
    for i, (m, n, k) in enumerate([(1000, 2050, 400), (1024, 2048, 1100), (1000, 2050, 1601), (3900, 4100, 300)]):
        a = coded(m, k, 0, scales[0], False, 3 * i, tight=i == 2)
        b = coded(n, k, 0, scales[0], scales[1], 3 * i + 1)
        check(product(a, b, out, n + (0, 4, 3)[i % 3]), a, b, out, (m, n, k))
    for k in (512, 1100):
        a, b = coded(129, k, 1, scales[0], False, 9), coded(260, k, 1, scales[0], scales[1], 10)
        if out != torch.float16:  # whose range the products of E5M2 pass
            check(product(a, b, out), a, b, out, ("e5m2", k))


@pytest.mark.parametrize("formats", ((0, 1), (1, 0), (1, 1)))
@pytest.mark.parametrize("out", (torch.float32, torch.bfloat16))
def test_matmul_formats(out, formats):
    for i, (m, n, k) in enumerate([(1, 40, 300), (5, 130, 384), (40, 40, 136), (129, 200, 257), (300, 260, 512)]):
        for e8m0, tile in ((False, True), (True, False)):
            a, b = coded(m, k, formats[0], e8m0, False, i), coded(n, k, formats[1], e8m0, tile, i + 50)
            check(product(a, b, out), a, b, out, (m, n, k, e8m0))


@pytest.mark.parametrize("off", (1, 4, 8))
def test_matmul_of_misaligned_codes(off):
    for m, n, k in ((1, 50, 300), (20, 70, 260), (140, 150, 400)):
        for out in (torch.float32, torch.float16):
            a, b = coded(m, k, 0, False, False, 1, tight=True, off=off), coded(n, k, 0, False, True, 2, off=off)
            check(product(a, b, out), a, b, out, (m, n, k))


@pytest.mark.parametrize("out", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("m", (1, 40, 300))
def test_matmul_rows_are_independent_of_their_neighbours(m, out):
    """NaN and infinity in one row of A, one of B, one scale: their own rows and columns alone; the others keep their bits."""
    a, b = coded(m, 512, 0, False, False, 8), coded(200, 512, 1, False, True, 9)
    clean = product(a, b, out).clone()
    b[0][7, 300] = 0x7c                      # infinity
    b[0][150, 511] = 0x7f                    # NaN
    bad = torch.zeros_like(clean, dtype=torch.bool)
    bad[:, 7] = bad[:, 150] = True
    if m > 2:
        a[0][2, 0] = 0xff
        a[1][m - 1, 3] = float("nan")
        bad[2] = bad[m - 1] = True
    got = product(a, b, out)
    assert torch.equal(got[~bad], clean[~bad])
    assert not torch.isfinite(got[bad]).any()


def test_matmul_nan_power_of_two_scale():
    for m in (1, 40, 300):
        for out in (torch.float32, torch.bfloat16):
            a, b = coded(m, 256, 0, True, False, 8), coded(130, 256, 0, True, False, 9)
            a[1][m - 1, 1] = 255
            b[1][3, 0] = 255
            got = product(a, b, out)
            assert got[m - 1].isnan().all() and got[:, 3].isnan().all()
            if m > 1:
                assert torch.isfinite(got[0, :3]).all()


def test_matmul_power_of_two_scales_far_from_one():
    """2^-100 by 2^90, and products beyond the type's range."""
    for m in (1, 40, 300):
        for out in (torch.float32, torch.bfloat16):
            a, b = coded(m, 384, 0, True, False, 4), coded(140, 384, 0, True, True, 5)
            a[1].sub_(100)
            b[1].add_(90)
            av, bv = a[3] * 2.0 ** -100, b[3] * 2.0 ** 90
            check(product(a, b, out), (*a[:3], av), (*b[:3], bv), out, m)
            a[1].fill_(250)
            b[1].fill_(250)
            assert not torch.isfinite(product(a, b, out)).any()


@pytest.mark.parametrize("out", tuple(OUT))
def test_matmul_of_nothing(out):
    """No columns: zeros.  No rows: nothing written."""
    e = torch.empty(0, dtype=torch.uint8, device="cuda")
    for m, n in ((3, 5), (200, 300)):
        a, b = (e, e.float(), B.make_blocks(m, 0, 0, 0), None), (e, e.float(), B.make_blocks(n, 0, 0, 0), None)
        assert (product(a, b, out) == 0).all()
    a = (e, e.float(), B.make_blocks(0, 128), None)
    b = coded(5, 128, 0, False, False, 0)
    c = torch.full((3, 5), 2.0, dtype=out, device="cuda")
    assert B.rans_block_matmul(*a[:3], *b[:3], OUT[out], c, 5, None) == 0
    assert (c == 2).all()


@pytest.mark.parametrize("out", (torch.float32, torch.bfloat16))
def test_matmul_long_sums(out):
    for m, n, k in ((1, 64, 40000), (2, 20, 16384), (70, 100, 16500), (300, 270, 11231)):
        a, b = coded(m, k, 1, False, False, k), coded(n, k, 0, False, False, k + 1)
        check(product(a, b, out), a, b, out, (m, n, k))


def test_matmul_offsets_beyond_32_bits():
    ld = (1 << 31) + 64
    for m in (3, 40, 130):
        a, b = coded(m, 300, 0, False, False, 1), coded(3, 300, 0, False, False, 2)
        far = torch.empty(2 * ld + 304, dtype=torch.uint8, device="cuda").as_strided((3, 300), (ld, 1))
        far.copy_(b[0])
        c_ld = 1 << 31
        c = torch.empty(2 * c_ld + 3, dtype=torch.bfloat16, device="cuda").as_strided((3, 3), (c_ld, 1)) if m == 3 else None
        lay = B.make_blocks(3, 300, ld, b[2].ld_scale)
        b = (far, b[1], lay, b[3])
        if m == 3:
            assert B.rans_block_matmul(*a[:3], *b[:3], B.BF16, c, c_ld, None if not (s := B.rans_matmul_workspace_bytes(a[2], lay)[1]) else B.workspace(s)) == 0
            check(c, a, b, torch.bfloat16)
        else:
            check(product(a, b, torch.float32), a, b, torch.float32)


def test_matmul_binary32_results_keep_binary32():
    """Products that spread over many powers of two: the error stays that of binary32 sums, some 2^-20 of the result."""
    g = torch.Generator().manual_seed(1)
    x, y = (torch.randn(200, 2048, generator=g) * torch.exp(2 * torch.randn(200, 2048, generator=g)) for _ in range(2))
    a, b = B.BlockMatrix(200, 2048).quantize(x.cuda()), B.BlockMatrix(200, 2048).quantize(y.cuda())
    c = a.matmul(b, torch.empty(200, 200, device="cuda")).cpu().double()
    av, bv = (O.decode8(m.code[:, :2048].cpu(), 0) * O.spread(m.scale.cpu().double(), 200, 2048, False) for m in (a, b))
    want = av @ bv.t()
    assert ((c - want).norm() / want.norm()).item() <= 2.0 ** -19


@pytest.mark.parametrize("out", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("tile", (False, True))
def test_matmul_of_more_rows_than_a_launch(out, tile):
    """Two launches along A, two along B."""
    rows = (1 << 17) + 77
    for m, n in ((rows, 3), (3, rows), (40, rows)):
        a, b = coded(m, 160, 0, False, False, 1), coded(n, 160, 0, False, tile, 2)
        check(product(a, b, out), a, b, out, (m, n))


def test_workspace_may_be_absent():
    a, b = B.make_blocks(300, 512), B.make_blocks(200, 512)
    assert B.rans_matmul_workspace_bytes(a, b) == (0, 0)


PARTS = [(64, 64, 4096), (48, 130, 4097), (100, 257, 4400), (40, 33, 16384), (130, 384, 4096), (256, 512, 8000), (33, 1024, 4500)]


@pytest.mark.parametrize("e8m0", (False, True))
@pytest.mark.parametrize("out", tuple(OUT))
def test_matmul_in_parts(out, e8m0):
    """Few tiles and a long K: parts of K, their sums added up in order; the same every time, whatever the workspace held."""
    for i, (m, n, k) in enumerate(PARTS):  # the E5M2 pair at 48 x 130 passes binary16's range in places: infinities there
        a = coded(m, k, 0, e8m0, False, 3 * i, tight=i % 3 == 2)
        b = coded(n, k, 0, e8m0, i % 2 == 0, 3 * i + 1, tight=i % 3 == 2)
        assert B.rans_matmul_workspace_bytes(a[2], b[2])[1] >= 2 * m * n * 4
        c = product(a, b, out, n + (0, 3)[i % 2])
        check(c, a, b, out, (m, n, k))
        assert torch.equal(c, product(a, b, out, n + (0, 3)[i % 2]))
        if i == 1:
            a = coded(m, k, 1, e8m0, False, 5)
            b = coded(n, k, 1, e8m0, False, 6)
            check(product(a, b, out), a, b, out, "e5m2")


def test_matmul_in_parts_workspace_refused():
    a, b = coded(64, 4096, 0, False, False, 1), coded(64, 4096, 0, False, False, 2)
    rc, size = B.rans_matmul_workspace_bytes(a[2], b[2])
    assert rc == 0 and size > 0
    c = torch.full((64, 64), 2.0, device="cuda")
    assert B.rans_block_matmul(*a[:3], *b[:3], B.F32, c, 64, None) == B.ERR_ARG
    assert B.rans_block_matmul(*a[:3], *b[:3], B.F32, c, 64, B.workspace(size)[16:]) == B.ERR_ARG
    assert B.rans_block_matmul(*a[:3], *b[:3], B.F32, c, 64, B.workspace(size)[:size - 256]) == B.ERR_WORKSPACE
    torch.cuda.synchronize()
    assert (c == 2).all()


def test_matmul_in_parts_captured():
    a, b = coded(64, 8192, 0, True, False, 1), coded(200, 8192, 0, True, True, 2)
    ws = B.workspace(B.rans_matmul_workspace_bytes(a[2], b[2])[1])
    c = torch.empty(64, 200, dtype=torch.bfloat16, device="cuda")

    def call():
        assert B.rans_block_matmul(*a[:3], *b[:3], B.BF16, c, 200, ws) == 0

    call()
    torch.cuda.synchronize()
    want = c.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        c.zero_()
        ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c, want)


def test_launched_kernels(launched_kernels):
    """Few rows (a short K has the tiles' fewer steps before it), tiles by whole 16-byte fetches, tiles of operands whose rows start anywhere, and K in parts."""
    for (m, n, k, kw), names in {(1, 384, 4096, ()): {"k_block_matmul_few"}, (1, 384, 512, ()): {"k_block_matmul"}, (300, 384, 512, ()): {"k_block_matmul"},
                                 (300, 384, 510, ("tight",)): {"k_block_matmul_any"}, (64, 96, 8192, ()): {"k_block_matmul", "k_block_matmul_sum"},
                                 (64, 96, 8190, ("tight",)): {"k_block_matmul_any", "k_block_matmul_sum"}}.items():
        a, b = (coded(r, k, 0, False, False, r, tight=bool(kw)) for r in (m, n))
        for out in (torch.bfloat16, torch.float32):
            assert launched_kernels(lambda: product(a, b, out)) == names, (m, n, k)


@pytest.mark.parametrize("long_a", (False, True))
@pytest.mark.parametrize("out", (torch.float32, torch.bfloat16))
def test_matmul_in_parts_behind_a_whole_launch(out, long_a, launched_kernels):
    """More rows than a launch, and so few behind them that their launch alone takes K in parts: 2^17 rows, the same 1024 over and
    over, and 77 others."""
    k, few, again = 4096, 64, 128
    x, y, rest = coded(few, k, 0, False, False, 1), coded(1024, k, 0, False, False, 2), coded(77, k, 0, False, False, 3)
    code, scale = (torch.cat([y[i].repeat(again, 1), rest[i]]) for i in (0, 1))
    long = (code, scale, B.make_blocks(1024 * again + 77, k, k, k // 128))
    a, b = (long, x) if long_a else (x, long)
    m, n = a[2].rows, b[2].rows
    size = B.rans_matmul_workspace_bytes(a[2], b[2])[1]
    assert size >= 2 * few * 77 * 4
    ws, c = B.workspace(size), torch.full((m, n), 99.0, dtype=out, device="cuda")
    assert B.rans_block_matmul(*a[:3], *b[:3], OUT[out], c, n, None) == B.ERR_ARG
    assert B.rans_block_matmul(*a[:3], *b[:3], OUT[out], c, n, ws[:size - 256]) == B.ERR_WORKSPACE
    torch.cuda.synchronize()
    assert (c == 99).all()
    assert "k_block_matmul_sum" in launched_kernels(lambda: B.rans_block_matmul(*a[:3], *b[:3], OUT[out], c, n, ws))
    rows = c if long_a else c.t()
    assert torch.equal(rows[1024:1024 * again].reshape(again - 1, 1024, few), rows[:1024].expand(again - 1, 1024, few))
    for got, part in ((rows[:1024], y), (rows[1024 * again:], rest)):
        check(got if long_a else got.t(), part if long_a else x, x if long_a else part, out, (m, n))
