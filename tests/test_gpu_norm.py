"""The norm with the residual's addition and coded output, and its gradients, on the GPU against 64 bits.

Tolerances, u = 2^-24 the half step of binary32.  rstd: the sum of K squares, added in chains of at most K / 64 + 16 links
(eight a lane and step, six and some between lanes and waves) of positive terms, so its relative error is below
(K / 64 + 18) u, half of that after the root, and 4 u for the mean, eps, the root and the quotient.  y = h rstd w: 3 u more."""
import pytest
import torch

from oracle import blocks as O
from paper_2511_11664_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
CODE = {torch.float32: B.F32, torch.float16: B.F16, torch.bfloat16: B.BF16}
EPS = 1e-5
SHAPES = [(1, 1), (3, 7), (2, 128), (5, 129), (4, 512), (3, 513), (2, 1000), (7, 2048), (2, 4096), (3, 4100), (2, 8192), (2, 8200), (1, 20000), (700, 96)]


def half_step(v, dtype):
    """Half a step of the type at v: eps / 2 of the value, or half the smallest subnormal number."""
    f = torch.finfo(dtype)
    return v.abs() * f.eps / 2 + f.smallest_normal * f.eps / 2


def rstd_tolerance(cols):
    return (cols / 128 + 13) * U


def data(rows, cols, dtype, seed=0):
    g = torch.Generator().manual_seed(rows * 100000 + cols + seed)
    x, r = (torch.randn(rows, cols, generator=g).to(dtype) for _ in range(2))
    x[:, cols // 3] *= 20
    if rows > 2:
        x[1], r[1] = 0, 0
    w = (1 + 0.2 * torch.randn(cols, generator=g))
    return x, r, w


def params(rows, cols, dtype, wdtype, **ld):
    return B.make_norm_params(rows, cols, CODE[dtype], CODE[wdtype], EPS, **ld)


def pitched(t, ld, off=0):
    """A copy of a matrix on the GPU with rows ld apart, its first element off elements into its memory."""
    whole = torch.full((t.shape[0] * ld + off + 16,), 7.0, dtype=t.dtype, device="cuda")
    v = whole.as_strided(t.shape, (ld, 1), off)
    v.copy_(t)
    return v


def check_codes(y, tol, code, scale, fmt, e8m0):
    """code s is y rounded to 8 bits, for y known up to tol: half a step of the format at the code, no code over the largest,
    and the scale that belongs to the largest |y| of its block, up to the same tolerance (a power of two may then be either
    of two neighbours)."""
    rows, cols = y.shape
    s = torch.exp2(scale.cpu().double() - 127) if e8m0 else scale.cpu().double()
    for f in (1 - 1e-4, 1 + 1e-4) if e8m0 else ():
        assert ((s <= O.block_scales((y * 1.0001).float(), fmt, True, False)) & (s >= O.block_scales((y * 0.9999).float(), fmt, True, False))).all()
    b = torch.nn.functional.pad(y.abs(), (0, -cols % 128)).view(rows, -1, 128).amax(2)
    if not e8m0:
        assert (((s - b / O.VMAX[fmt]).abs() <= (tol.max() + 2 * U) * s) | (b == 0)).all()
    each = O.spread(s, rows, cols, False)
    v = O.decode8(code.cpu(), fmt)
    step = 2.0 ** -(3, 2)[fmt] * torch.clamp(v.abs(), min=2.0 ** (-6, -14)[fmt])
    assert ((v * each - y).abs() <= each * step / 2 + (tol + 3 * U) * y.abs()).all()


@pytest.mark.parametrize("wide_weight", (False, True))
@pytest.mark.parametrize("residual", (False, True))
@pytest.mark.parametrize("dtype", tuple(CODE))
def test_norm(dtype, residual, wide_weight):
    for i, (rows, cols) in enumerate(SHAPES):
        x, r, w = data(rows, cols, dtype)
        w = w if wide_weight else w.to(dtype)
        h, rstd, y = O.norm(x, r if residual else None, w, EPS, dtype)
        tol = torch.full((rows, 1), rstd_tolerance(cols) + 3 * U, dtype=torch.float64)
        fmt, e8m0, odd = i % 2, i // 2 % 2 == 1, i % 3 == 2
        ld, off = (cols + 3, 1) if odd else (cols, 0)
        xd, rd = pitched(x, ld, off), pitched(r, ld + 2, off) if residual else None
        total, out = pitched(torch.zeros_like(x), ld, off), pitched(torch.zeros_like(x), ld + 1, off)
        m = B.BlockMatrix(rows, cols, fmt, int(e8m0))
        got_rstd = torch.zeros(rows, device="cuda")
        p = params(rows, cols, dtype, w.dtype, ld_x=ld, ld_res=ld + 2, ld_sum=ld, ld_y=ld + 1)
        assert B.rans_norm_quantize(xd, rd, w.cuda(), p, total, got_rstd, out, m.code, m.scale, m.layout) == 0
        assert torch.equal(total.cpu().double(), h), (rows, cols)
        assert ((got_rstd.cpu().double() - rstd).abs() <= rstd_tolerance(cols) * rstd).all(), (rows, cols)
        assert ((out.cpu().double() - y).abs() <= tol * y.abs() * 1.01 + half_step(y, dtype)).all(), (rows, cols)
        check_codes(y, tol, m.code[:, :cols], m.scale[:, :-(-cols // 128)], fmt, e8m0)


@pytest.mark.parametrize("cols", (96, 4096, 8200, 20000))
def test_norm_in_place_and_parts(cols):
    """Sums in the residual's own memory, each output by itself, no weight."""
    x, r, _ = data(5, cols, torch.bfloat16)
    p = params(5, cols, torch.bfloat16, torch.bfloat16)
    h, rstd, y = O.norm(x, r, None, EPS, torch.bfloat16)
    ref = torch.empty(5, cols, dtype=torch.bfloat16, device="cuda")
    assert B.rans_norm_quantize(x.cuda(), r.cuda(), None, p, None, None, ref, None, None, None) == 0
    assert ((ref.cpu().double() - y).abs() <= (rstd_tolerance(cols) + 3 * U) * 1.01 * y.abs() + half_step(y, torch.bfloat16)).all()
    for which in ("x", "res"):
        xd, rd = x.cuda(), r.cuda()
        total = xd if which == "x" else rd
        out = torch.empty_like(ref)
        assert B.rans_norm_quantize(xd, rd, None, p, total, None, out, None, None, None) == 0
        assert torch.equal(total.cpu().double(), h) and torch.equal(out, ref)
    xd = x.cuda()
    assert B.rans_norm_quantize(xd, r.cuda(), None, p, None, None, xd, None, None, None) == 0  # y over x
    assert torch.equal(xd, ref)
    got = torch.zeros(5, device="cuda")
    assert B.rans_norm_quantize(x.cuda(), r.cuda(), None, p, None, got, None, None, None, None) == 0
    assert ((got.cpu().double() - rstd).abs() <= rstd_tolerance(cols) * rstd).all()
    m = B.BlockMatrix(5, cols)
    assert B.rans_norm_quantize(x.cuda(), r.cuda(), None, p, None, None, None, m.code, m.scale, m.layout) == 0
    check_codes(y, torch.full((5, 1), rstd_tolerance(cols) + 3 * U, dtype=torch.float64), m.code[:, :cols], m.scale[:, :-(-cols // 128)], 0, False)


def test_norm_special_values():
    """A row of zeros, eps = 0 on it, NaN and infinity spoil their own row alone."""
    x, r, w = data(6, 300, torch.float32)
    x[2, 7], x[3, 8] = float("nan"), float("inf")
    p = B.make_norm_params(6, 300, B.F32, B.F32, 0.0)
    out = torch.empty(6, 300, device="cuda")
    assert B.rans_norm_quantize(x.cuda(), r.cuda(), w.cuda(), p, None, None, out, None, None, None) == 0
    want = O.norm(x, r, w, 0.0, torch.float32)[2]
    got = out.cpu().double()
    assert got[1].isnan().all() and got[2].isnan().all()          # 0 * inf; NaN
    assert got[3, 8].isnan() and (got[3, :8] == 0).all()           # inf * 0; finite * 0
    for i in (0, 4, 5):
        assert ((got[i] - want[i]).abs() <= (rstd_tolerance(300) + 4 * U) * want[i].abs()).all()


def bwd_data(rows, cols, dtype, wide_weight, seed=0):
    x, r, w = data(rows, cols, dtype, seed)
    g = torch.Generator().manual_seed(seed + 77)
    dy = torch.randn(rows, cols, generator=g).to(dtype)
    rstd = (1 / torch.sqrt((x.double() ** 2).mean(1) + EPS)).float()
    return dy, r, x, w if wide_weight else w.to(dtype), rstd


def check_backward(rows, cols, dtype, dy, dsum, h, w, rstd, dx, dw):
    """dx: the row's sum of g xh in chains as above, relative to the sum of its magnitudes, then a few operations of one
    rounding; dw: chains of at most rows links."""
    want, want_w = O.norm_backward(dy, dsum, h, w, rstd)
    g, xh = (dy.double() if w is None else dy.double() * w.double()), h.double() * rstd.double()[:, None]
    mean_abs = (g * xh).abs().mean(1, keepdim=True)
    r = rstd.double()[:, None]
    tol = r * (4 * U * g.abs() + xh.abs() * mean_abs * (cols / 64 + 24) * U) + 2 * U * want.abs() + (0 if dsum is None else 2 * U * dsum.double().abs())
    assert ((dx.cpu().double() - want).abs() <= tol * 1.01 + half_step(want, dtype)).all(), (rows, cols)
    if dw is not None:
        assert ((dw.cpu().double() - want_w).abs() <= (rows + 4) * U * (dy.double() * xh).abs().sum(0)).all(), (rows, cols)


@pytest.mark.parametrize("wide_weight", (False, True))
@pytest.mark.parametrize("dtype", tuple(CODE))
def test_norm_backward(dtype, wide_weight):
    for i, (rows, cols) in enumerate(SHAPES + [(1500, 200), (600, 9000), (395, 4500)]):
        dy, ds, h, w, rstd = bwd_data(rows, cols, dtype, wide_weight)
        ds = None if i % 4 == 1 else ds
        ld, off = (cols + 3, 1) if i % 3 == 2 else (cols, 0)
        p = params(rows, cols, dtype, w.dtype, ld_x=ld, ld_res=ld + 2, ld_sum=ld, ld_y=ld + 1)
        dx = pitched(torch.zeros_like(h), ld, off)
        dw = torch.full((cols,), 3.0, device="cuda")
        rc, size = B.rans_norm_workspace_bytes(p)
        assert rc == 0
        args = (pitched(dy, ld + 1, off), None if ds is None else pitched(ds, ld + 2, off), pitched(h, ld, off), w.cuda(), rstd.cuda(), p)
        assert B.rans_norm_backward(*args, dx, dw, B.workspace(size)) == 0
        check_backward(rows, cols, dtype, dy, ds, h, w, rstd, dx, dw)
        dx2, dw2 = torch.zeros_like(dx).as_strided(dx.shape, dx.stride()) if ld == cols else pitched(torch.zeros_like(h), ld, off), torch.empty_like(dw)
        assert B.rans_norm_backward(*args, dx2, dw2, B.workspace(size)) == 0
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2)  # the same order every time
        dx3 = pitched(torch.zeros_like(h), ld, off)
        assert B.rans_norm_backward(*args, dx3, None, None) == 0
        assert torch.equal(dx, dx3)


@pytest.mark.parametrize("cols", (96, 4096, 8200, 20000))
@pytest.mark.parametrize("over", ("dy", "dsum", "h"))
def test_norm_backward_in_place(cols, over):
    dy, ds, h, w, rstd = bwd_data(9, cols, torch.float32, True)
    p = params(9, cols, torch.float32, torch.float32)
    t = dict(dy=dy.cuda(), dsum=ds.cuda(), h=h.cuda())
    assert B.rans_norm_backward(t["dy"], t["dsum"], t["h"], w.cuda(), rstd.cuda(), p, t[over], None, None) == 0
    check_backward(9, cols, torch.float32, dy, ds, h, w, rstd, t[over], None)


def test_norm_backward_of_no_rows_and_no_weight():
    p = params(0, 50, torch.float32, torch.float32)
    dw = torch.ones(50, device="cuda")
    e = torch.empty(0, 50, device="cuda")
    assert B.rans_norm_backward(e, None, e, None, torch.empty(0, device="cuda"), p, e, dw, None) == 0
    assert (dw == 0).all()
    dy, ds, h, _, rstd = bwd_data(4, 333, torch.float16, False)
    dx = torch.empty(4, 333, dtype=torch.float16, device="cuda")
    assert B.rans_norm_backward(dy.cuda(), ds.cuda(), h.cuda(), None, rstd.cuda(), params(4, 333, torch.float16, torch.float16), dx, None, None) == 0
    check_backward(4, 333, torch.float16, dy, ds, h, None, rstd, dx, None)


def test_norm_gradient_against_differences():
    """Central differences of the forward formula in 64 bits, step 1e-4: their error is below 1e-6 of the gradient's size."""
    rows, cols = 2, 40
    g = torch.Generator().manual_seed(5)
    x, dy, ds, w = torch.randn(rows, cols, generator=g), torch.randn(rows, cols, generator=g), torch.randn(rows, cols, generator=g), 1 + 0.3 * torch.randn(cols, generator=g)

    def loss(x_, w_):
        y = x_ / torch.sqrt((x_ * x_).mean(1, keepdim=True) + EPS) * w_
        return (y * dy.double()).sum() + (x_ * ds.double()).sum()

    rstd = torch.empty(rows, device="cuda")
    out = torch.empty(rows, cols, device="cuda")
    p = params(rows, cols, torch.float32, torch.float32)
    assert B.rans_norm_quantize(x.cuda(), None, w.cuda(), p, None, rstd, out, None, None, None) == 0
    dx, dw = torch.empty_like(out), torch.empty(cols, device="cuda")
    assert B.rans_norm_backward(dy.cuda(), ds.cuda(), x.cuda(), w.cuda(), rstd, p, dx, dw, B.workspace(B.rans_norm_workspace_bytes(p)[1])) == 0
    e, scale = 1e-4, 1e-5
    for i in range(rows):
        for j in range(0, cols, 7):
            d = torch.zeros(rows, cols, dtype=torch.float64)
            d[i, j] = e
            diff = (loss(x.double() + d, w.double()) - loss(x.double() - d, w.double())) / (2 * e)
            assert abs(diff.item() - dx[i, j].item()) <= scale * dx.abs().max().item()
    for j in range(0, cols, 7):
        d = torch.zeros(cols, dtype=torch.float64)
        d[j] = e
        diff = (loss(x.double(), w.double() + d) - loss(x.double(), w.double() - d)) / (2 * e)
        assert abs(diff.item() - dw[j].item()) <= scale * dw.abs().max().item()


def test_norm_offsets_beyond_32_bits():
    ld, cols = (1 << 31) + 8, 300
    x, r, w = data(3, cols, torch.bfloat16)
    xd = torch.empty(2 * ld + cols, dtype=torch.bfloat16, device="cuda").as_strided((3, cols), (ld, 1))
    xd.copy_(x)
    p = params(3, cols, torch.bfloat16, torch.bfloat16, ld_x=ld, ld_sum=ld)
    out = torch.empty(3, cols, dtype=torch.bfloat16, device="cuda")
    assert B.rans_norm_quantize(xd, r.cuda(), w.to(torch.bfloat16).cuda(), p, xd, None, out, None, None, None) == 0
    h, _, y = O.norm(x, r, w.to(torch.bfloat16), EPS, torch.bfloat16)
    assert torch.equal(xd.cpu().double(), h)
    assert ((out.cpu().double() - y).abs() <= (rstd_tolerance(cols) + 3 * U) * 1.01 * y.abs() + half_step(y, torch.bfloat16)).all()


@pytest.mark.parametrize("over", ("dy", "dsum", "h", "none"))
def test_norm_backward_weight_gradient_with_dx_in_place(over, launched_kernels):
    """dx in the memory that the weight's gradient is read from: two kernels, one after the other; elsewhere one for both."""
    for rows, cols in ((5, 300), (40, 1000), (395, 4096), (100, 8200)):
        dy, ds, h, w, rstd = bwd_data(rows, cols, torch.bfloat16, False)
        t = dict(dy=dy.cuda(), dsum=ds.cuda(), h=h.cuda(), none=torch.empty_like(h, device="cuda"))
        p = params(rows, cols, torch.bfloat16, w.dtype)
        dw, ws = torch.empty(cols, device="cuda"), B.workspace(B.rans_norm_workspace_bytes(p)[1])
        args = (t["dy"], t["dsum"], t["h"], w.cuda(), rstd.cuda(), p, t[over], dw, ws)

        def call():
            assert B.rans_norm_backward(*args) == 0

        names = launched_kernels(call)
        check_backward(rows, cols, torch.bfloat16, dy, ds, h, w, rstd, t[over], dw)
        assert names == ({"k_norm_bwd", "k_norm_dw"} if over in ("dy", "h") else {"k_norm_bwd_both"})


def test_norm_backward_kernels_by_rows(launched_kernels):
    for (rows, cols), names in {(1, 512): {"k_norm_bwd_both"}, (1000, 512): {"k_norm_bwd", "k_norm_dw"}, (300, 2048): {"k_norm_bwd_both"}, (1100, 4096): {"k_norm_bwd", "k_norm_dw"}}.items():
        dy, ds, h, w, rstd = bwd_data(rows, cols, torch.float16, True)
        p = params(rows, cols, torch.float16, w.dtype)
        dx, dw, ws = torch.empty_like(h, device="cuda"), torch.empty(cols, device="cuda"), B.workspace(B.rans_norm_workspace_bytes(p)[1])
        args = [t.cuda() for t in (dy, ds, h, w, rstd)]
        assert launched_kernels(lambda: B.rans_norm_backward(*args, p, dx, dw, ws)) == names
        check_backward(rows, cols, torch.float16, dy, ds, h, w, rstd, dx, dw)


def test_norm_of_large_and_small_rows_and_infinite_weights():
    """Means far from one; an infinite weight gives infinities of h's sign, NaN where h is zero."""
    x, _, w = data(3, 1000, torch.float32)
    w[5], w[6] = float("inf"), float("-inf")
    x[0, 6] = 0
    for size in (1e17, 1.0, 1e-16):
        h = x * size
        p = B.make_norm_params(3, 1000, B.F32, B.F32, 0.0)
        out = torch.empty(3, 1000, device="cuda")
        assert B.rans_norm_quantize(h.cuda(), None, w.cuda(), p, None, None, out, None, None, None) == 0
        want = O.norm(h, None, w, 0.0, torch.float32)[2]
        got = out.cpu().double()
        assert got[0, 6].isnan() and got[1].isnan().all()  # 0 * inf; the row of zeros without eps
        for row in (0, 2):
            assert got[row, 5] == want[row, 5] and got[row, 5].isinf()
        assert got[2, 6] == want[2, 6] and got[2, 6].isinf()
        rest = torch.ones(1000, dtype=torch.bool)
        rest[5:7] = False
        for row in (0, 2):
            assert ((got - want).abs()[row, rest] <= ((rstd_tolerance(1000) + 4 * U) * want.abs())[row, rest]).all(), size


def test_norm_codes_are_the_definitions():
    """y is half a step of binary32 off and a little, so that of codes under powers of two hardly one is not its definition's."""
    rows, cols = 512, 4096
    x, _, w = data(rows, cols, torch.bfloat16)
    w = w.to(torch.bfloat16)
    m = B.BlockMatrix(rows, cols, B.E4M3, B.SCALE_E8M0)
    assert B.rans_norm_quantize(x.cuda(), None, w.cuda(), params(rows, cols, torch.bfloat16, w.dtype), None, None, None, m.code, m.scale, m.layout) == 0
    y = O.norm(x, None, w, EPS, torch.bfloat16)[2]
    s = O.spread(torch.exp2(m.scale[:, :cols // 128].cpu().double() - 127), rows, cols, False)
    v = y / s
    got = O.decode8(m.code[:, :cols].cpu(), 0)
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(got.abs().clamp(min=2.0 ** -9))), min=-6) - 3)
    off = (got - v).abs() > step / 2 * (1 + 1e-9)
    # a code is wrong where a multiple of half a step lies within y's error, some 2^-23 of y: of 2^21 codes about 2^21 2^-23 2^4 2 = 8
    assert off.sum() <= 40
    assert ((got - v).abs() <= step / 2 + 2.0 ** -22 * v.abs()).all()


def test_norm_backward_of_more_columns_than_a_grid_has_threads():
    """32 threads a column are 2^32 of them for 2^27 columns, more than a launch holds: several launches."""
    cols = (1 << 27) + 300
    g = torch.Generator(device="cuda").manual_seed(1)
    dy, h = (torch.randn(1, cols, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    rstd = torch.full((1,), 0.75, device="cuda")
    p = params(1, cols, torch.bfloat16, torch.bfloat16)
    dx, dw = torch.empty_like(h), torch.full((cols,), 3.0, device="cuda")
    assert B.rans_norm_backward(dy, None, h, None, rstd, p, dx, dw, B.workspace(B.rans_norm_workspace_bytes(p)[1])) == 0
    # one row: a product of three factors of which the first two have few bits, rounded once or twice; then a sum of one
    for at in range(0, cols, 1 << 24):
        part = slice(at, at + (1 << 24))
        want = dy[0, part].double() * h[0, part].double() * 0.75
        assert ((dw[part].double() - want).abs() <= 2 * U * want.abs()).all(), at


@pytest.mark.parametrize("dtype, size", [(torch.float32, s) for s in (1e36, 1e25, 1e18, 1e-18, 1e-25, 1e-36, 1e-40)] + [(torch.bfloat16, 1e30), (torch.bfloat16, 1e-30)])
def test_norm_of_rows_whose_squares_pass_binary32(dtype, size):
    """Squares are binary64: no finite row becomes zeros or infinities.  rstd is one rounding to binary32 off, of half a step of its
    subnormal numbers at least (and an infinity behind the largest); y as everywhere."""
    for rows, cols in ((3, 1000), (2, 8200)):
        x, r, w = data(rows, cols, torch.float32)
        x, r = (x * size).to(dtype), (r * size).to(dtype)
        h, rstd, y = O.norm(x, r, w, 0.0, dtype)
        assert (h == h).all() and torch.isfinite(h).all()
        p = B.make_norm_params(rows, cols, CODE[dtype], B.F32, 0.0)
        got_rstd, out, m = torch.zeros(rows, device="cuda"), torch.empty(rows, cols, dtype=dtype, device="cuda"), B.BlockMatrix(rows, cols)
        assert B.rans_norm_quantize(x.cuda(), r.cuda(), w.cuda(), p, None, got_rstd, out, m.code, m.scale, m.layout) == 0
        for row in range(rows):
            if (h[row] == 0).all():
                continue
            got, want = got_rstd[row].item(), rstd[row].item()
            assert abs(got - want) <= rstd_tolerance(cols) * want + 2.0 ** -150 if want < 3.4e38 else got == float("inf")
            assert ((out[row].cpu().double() - y[row]).abs() <= (rstd_tolerance(cols) + 3 * U) * 1.01 * y[row].abs() + half_step(y[row], dtype)).all()
            check_codes(y[row:row + 1], torch.full((1, 1), rstd_tolerance(cols) + 3 * U, dtype=torch.float64), m.code[row:row + 1, :cols],
                        m.scale[row:row + 1, :-(-cols // 128)], 0, False)


def norm_codes(x, w, fmt, e8m0):
    """Codes, scales (their values) and rstd of a CPU matrix's norm, on the CPU."""
    rows, cols = x.shape
    m, rstd = B.BlockMatrix(rows, cols, fmt, int(e8m0)), torch.empty(rows, device="cuda")
    assert B.rans_norm_quantize(x.cuda(), None, w.cuda(), params(rows, cols, x.dtype, w.dtype), None, rstd, None, m.code, m.scale, m.layout) == 0
    s = m.scale[:, :-(-cols // 128)].cpu()
    return O.decode8(m.code[:, :cols].cpu(), fmt), torch.exp2(s.double() - 127) if e8m0 else s.double(), rstd.cpu().double()


@pytest.mark.parametrize("cols", (300, 4000, 9000))
@pytest.mark.parametrize("fmt", (0, 1))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_norm_codes_on_borders_under_powers_of_two(dtype, fmt, cols):
    """Weights that put y next to a border, less than half a step of binary32 from it: halfway between two codes, normal ones and
    subnormal ones, or at the largest number of a scale.  A code and a scale go by the side on which y lies."""
    g = torch.Generator().manual_seed(cols + fmt)
    mbits, least = ((3, -6), (2, -14))[fmt]
    x = torch.randn(1, cols, generator=g).to(dtype)
    x[x.abs() < 0.01] = 0.01
    odd = 2 * torch.randint(0, 1 << mbits, (cols,), generator=g) + 1
    normal = (1 + odd.double() / (2 << mbits)) * torch.exp2(torch.randint(least, 6, (cols,), generator=g).double())
    z = torch.where(torch.rand(cols, generator=g) < 0.5, normal, odd * 2.0 ** (least - mbits - 1))
    block = torch.arange(cols) // 128
    z[::128] = torch.where(block[::128] % 3 > 0, O.VMAX[fmt], 0.9 * O.VMAX[fmt]).double()
    target = z * torch.exp2((block % 11 - 5).double())
    rstd = O.norm(x, None, None, EPS, dtype)[1]
    w = (target / (x[0].double() * rstd)).float()
    y = O.norm(x, None, w, EPS, dtype)[2]
    assert (y[0].float().double() == target).sum() > cols / 3 and (y[0] != target).all()  # binary32 alone does not see the side
    s = O.block_scales(y, fmt, True, False)
    got, got_s, _ = norm_codes(x, w, fmt, True)
    assert torch.equal(got_s, s)
    assert torch.equal(got, O.round8(y / O.spread(s, 1, cols, False), fmt))


@pytest.mark.parametrize("rows, cols", ((512, 4096), (5000, 1000), (40, 8200), (300, 96)))
@pytest.mark.parametrize("fmt", (0, 1))
@pytest.mark.parametrize("dtype", tuple(CODE))
def test_norm_codes_under_powers_of_two_are_exactly_the_definitions(dtype, fmt, rows, cols):
    """y is known to some 2^-43 (eps is a binary32 number): of 2^21 codes, with 2^5 borders an octave at most, 2^-17 lie within that
    of a border.  rstd is the nearest binary32 number but for as rare ones: half a step, and 2^-30 of it on top."""
    x, _, w = data(rows, cols, dtype)
    w = w.to(dtype)
    _, rstd, y = O.norm(x, None, w, EPS, dtype)
    s = O.block_scales(y, fmt, True, False)
    got, got_s, got_rstd = norm_codes(x, w, fmt, True)
    assert torch.equal(got_s, s)
    assert torch.equal(got, O.round8(y / O.spread(s, rows, cols, False), fmt))
    assert ((got_rstd - rstd).abs() <= U * (1 + 2.0 ** -6) * rstd).all()


@pytest.mark.parametrize("fmt", (0, 1))
def test_norm_codes_under_binary32_scales_are_those_of_y(fmt):
    """The definition of the codes starts from binary32's y: what rans_block_quantize gives for it."""
    for rows, cols in ((200, 4096), (3, 8200), (64, 333)):
        x, r, w = data(rows, cols, torch.float32)
        out, m, q = torch.empty(rows, cols, device="cuda"), B.BlockMatrix(rows, cols, fmt), B.BlockMatrix(rows, cols, fmt)
        assert B.rans_norm_quantize(x.cuda(), r.cuda(), w.cuda(), params(rows, cols, torch.float32, torch.float32), None, None, out, m.code, m.scale, m.layout) == 0
        q.quantize(out)
        nb = -(-cols // 128)
        assert torch.equal(m.code[:, :cols], q.code[:, :cols]) and torch.equal(m.scale[:, :nb], q.scale[:, :nb])
        y = O.norm(x, r, w, EPS, torch.float32)[2]
        assert ((out.cpu().double() - y).abs() <= U * (1 + 2.0 ** -6) * y.abs()).all()  # a rounding, and 2^-30 on top


@pytest.mark.parametrize("fmt", (0, 1))
@pytest.mark.parametrize("dtype", tuple(CODE))
def test_norm_of_many_rows(dtype, fmt):
    """The form for many rows, two vectors a thread and more in flight: whole rows and such that end inside a thread's second one;
    tolerances as above, codes under powers of two exactly."""
    for rows, cols, odd in ((2100, 2500, False), (2048, 4096, False), (2050, 5121, True), (2060, 8190, True)):
        x, r, w = data(rows, cols, dtype)
        w = w.to(dtype)
        h, rstd, y = O.norm(x, r, w, EPS, dtype)
        ld, off = (cols + 3, 1) if odd else (cols, 0)
        total, out, m, got_rstd = pitched(torch.zeros_like(x), ld, off), pitched(torch.zeros_like(x), ld + 1, off), B.BlockMatrix(rows, cols, fmt, 1), torch.zeros(rows, device="cuda")
        p = params(rows, cols, dtype, dtype, ld_x=ld, ld_res=ld + 2, ld_sum=ld, ld_y=ld + 1)
        assert B.rans_norm_quantize(pitched(x, ld, off), pitched(r, ld + 2, off), w.cuda(), p, total, got_rstd, out, m.code, m.scale, m.layout) == 0
        assert torch.equal(total.cpu().double(), h)
        assert ((got_rstd.cpu().double() - rstd).abs() <= U * (1 + 2.0 ** -6) * rstd).all()
        assert ((out.cpu().double() - y).abs() <= U * (1 + 2.0 ** -6) * y.abs() * 1.01 + half_step(y, dtype)).all()
        s = O.block_scales(y, fmt, True, False)
        assert torch.equal(torch.exp2(m.scale[:, :-(-cols // 128)].cpu().double() - 127), s)
        assert torch.equal(O.decode8(m.code[:, :cols].cpu(), fmt), O.round8(y / O.spread(s, rows, cols, False), fmt))
        f = B.BlockMatrix(rows, cols, fmt)
        assert B.rans_norm_quantize(total, None, w.cuda(), params(rows, cols, dtype, dtype, ld_x=ld), None, None, None, f.code, f.scale, f.layout) == 0
        check_codes(y, torch.full((rows, 1), 2 * U, dtype=torch.float64), f.code[:, :cols], f.scale[:, :-(-cols // 128)], fmt, False)


@pytest.mark.parametrize("dtype", tuple(CODE))
def test_norm_backward_of_several_rows_a_work_group(dtype, launched_kernels):
    """Each width's work-groups, with three rows and more one after the other."""
    for rows, cols in ((5000, 300), (2100, 1000), (1100, 4000), (1100, 5000), (1100, 6001), (1100, 8300)):
        dy, ds, h, w, rstd = bwd_data(rows, cols, dtype, False)
        p = params(rows, cols, dtype, w.dtype)
        dx, dw, ws = torch.empty_like(h, device="cuda"), torch.empty(cols, device="cuda"), B.workspace(B.rans_norm_workspace_bytes(p)[1])
        args = [t.cuda() for t in (dy, ds, h, w, rstd)]
        assert launched_kernels(lambda: B.rans_norm_backward(*args, p, dx, dw, ws)) == {"k_norm_bwd", "k_norm_dw"}
        check_backward(rows, cols, dtype, dy, ds, h, w, rstd, dx, dw)
