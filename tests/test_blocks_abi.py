"""Block codes, norm and matrix product: struct layouts, workspace sizes and refusals.  CPU only: every call here is refused
on the host before anything is launched, or has nothing to do."""
import ctypes as C
import os

import pytest
import torch

from oracle import blocks as O
from paper_2511_11664_amd import binding as B

FAKE = 1 << 20  # an aligned address that nothing dereferences


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.SO_PATH):
        B.build_library()
    return B.lib()


def blocks(rows=4, cols=256, **kw):
    base = dict(ld=256, ld_scale=4, format=0, scale_type=0, block=0)
    reserved = kw.pop("reserved", 0)
    base.update(kw)
    b = B.make_blocks(rows, cols, **base)
    b.reserved = reserved
    return b


def test_struct_layouts_match_header():
    assert C.sizeof(B.Blocks) == 48 and C.sizeof(B.NormParams) == 64


def test_default_leading_dimensions():
    b = B.make_blocks(3, 1000)
    assert (b.ld, b.ld_scale) == (1008, 8)
    m = B.BlockMatrix(300, 1000, scale_type=B.SCALE_E8M0, block=B.BLOCK_TILE, device="cpu")
    assert m.code.shape == (300, 1008) and m.scale.shape == (3, 8) and m.scale.dtype == torch.uint8


@pytest.mark.parametrize("change, code", [
    (dict(ld=255), B.ERR_SHAPE), (dict(ld_scale=1), B.ERR_SHAPE), (dict(format=2), B.ERR_ARG), (dict(scale_type=2), B.ERR_ARG),
    (dict(block=2), B.ERR_ARG), (dict(reserved=1), B.ERR_ARG), (dict(rows=(1 << 30) + 1), B.ERR_ARG), (dict(ld=(1 << 32) + 1), B.ERR_ARG)])
def test_layouts_refused(lib, change, code):
    b = blocks(**change)
    assert lib.rans_block_quantize(FAKE, 256, B.F32, 0, FAKE, FAKE, b, None) == code
    assert lib.rans_block_dequantize(FAKE, FAKE, b, B.F32, FAKE, 256, None) == code
    assert lib.rans_block_matmul(FAKE, FAKE, b, FAKE, FAKE, blocks(), B.F32, FAKE, 4, None, 0, None) == code
    size = C.c_size_t()
    assert lib.rans_matmul_workspace_bytes(b, blocks(), C.byref(size)) == code


def test_quantize_arguments_refused(lib):
    b = blocks()
    q = lib.rans_block_quantize
    assert q(None, 256, B.F32, 0, FAKE, FAKE, b, None) == B.ERR_ARG
    assert q(FAKE, 256, B.F32, 0, None, FAKE, b, None) == B.ERR_ARG
    assert q(FAKE, 256, B.F32, 0, FAKE, None, b, None) == B.ERR_ARG
    assert q(FAKE, 256, B.F32, 0, FAKE, FAKE, None, None) == B.ERR_ARG
    assert q(FAKE, 256, 3, 0, FAKE, FAKE, b, None) == B.ERR_ARG
    assert q(FAKE + 2, 256, B.F32, 0, FAKE, FAKE, b, None) == B.ERR_ARG       # misaligned element
    assert q(FAKE, 256, B.F32, 0, FAKE, FAKE + 2, b, None) == B.ERR_ARG       # misaligned scale
    assert q(FAKE, 255, B.F32, 0, FAKE, FAKE, b, None) == B.ERR_SHAPE
    assert q(FAKE, 3, B.F32, 1, FAKE, FAKE, b, None) == B.ERR_SHAPE           # x is 256 x 4 where its transpose is coded
    assert q(FAKE, (1 << 32) + 1, B.F32, 0, FAKE, FAKE, b, None) == B.ERR_ARG
    assert q(None, 256, B.F32, 0, None, None, blocks(rows=0), None) == B.OK   # nothing to do
    assert q(None, 256, B.F32, 0, None, None, blocks(cols=0), None) == B.OK
    d = lib.rans_block_dequantize
    assert d(FAKE, FAKE, b, B.BF16, FAKE + 1, 256, None) == B.ERR_ARG
    assert d(FAKE, FAKE, b, B.BF16, None, 256, None) == B.ERR_ARG
    assert d(FAKE, FAKE, b, 3, FAKE, 256, None) == B.ERR_ARG
    assert d(FAKE, FAKE, b, B.BF16, FAKE, 200, None) == B.ERR_SHAPE
    assert d(None, None, blocks(rows=0), B.BF16, None, 256, None) == B.OK


def norm_params(**kw):
    base = dict(rows=4, cols=256, dtype=B.BF16, weight_dtype=B.BF16, eps=1e-5)
    base.update(kw)
    return B.make_norm_params(**base)


@pytest.mark.parametrize("change, code", [
    (dict(cols=0, ld_x=1, ld_res=1, ld_sum=1, ld_y=1), B.ERR_ARG), (dict(dtype=3), B.ERR_ARG), (dict(weight_dtype=3), B.ERR_ARG),
    (dict(eps=-1.0), B.ERR_ARG), (dict(eps=float("nan")), B.ERR_ARG), (dict(eps=float("inf")), B.ERR_ARG), (dict(ld_x=255), B.ERR_SHAPE),
    (dict(ld_res=255), B.ERR_SHAPE), (dict(ld_sum=255), B.ERR_SHAPE), (dict(ld_y=255), B.ERR_SHAPE), (dict(rows=(1 << 30) + 1), B.ERR_ARG)])
def test_norm_params_refused(lib, change, code):
    p = norm_params(**change)
    size = C.c_size_t()
    assert lib.rans_norm_workspace_bytes(p, C.byref(size)) == code
    assert lib.rans_norm_quantize(FAKE, None, None, p, None, None, FAKE, None, None, None, None) == code
    assert lib.rans_norm_backward(FAKE, None, FAKE, None, FAKE, p, FAKE, None, None, 0, None) == code


def test_norm_arguments_refused(lib):
    p, b = norm_params(), blocks()
    f = lib.rans_norm_quantize
    assert f(None, None, None, p, None, None, FAKE, None, None, None, None) == B.ERR_ARG
    assert f(FAKE, None, None, p, None, None, None, None, None, None, None) == B.ERR_ARG             # no output at all
    assert f(FAKE, None, None, p, None, None, None, FAKE, FAKE, None, None) == B.ERR_ARG             # codes without their layout
    assert f(FAKE, None, None, p, None, None, None, FAKE, FAKE, blocks(block=1), None) == B.ERR_ARG  # a tile spans rows
    assert f(FAKE, None, None, p, None, None, None, FAKE, FAKE, blocks(rows=5), None) == B.ERR_SHAPE
    assert f(FAKE, None, None, p, None, None, None, FAKE, FAKE, blocks(cols=128), None) == B.ERR_SHAPE
    assert f(FAKE + 1, None, None, p, None, None, FAKE, None, None, None, None) == B.ERR_ARG
    assert f(FAKE, None, FAKE + 1, p, None, None, FAKE, None, None, None, None) == B.ERR_ARG
    assert f(FAKE, None, FAKE, norm_params(weight_dtype=B.F16), None, None, FAKE, None, None, None, None) == B.ERR_ARG
    assert f(None, None, None, norm_params(rows=0), None, None, None, None, None, None, None) == B.OK
    g = lib.rans_norm_backward
    assert g(None, None, FAKE, None, FAKE, p, FAKE, None, None, 0, None) == B.ERR_ARG
    assert g(FAKE, None, None, None, FAKE, p, FAKE, None, None, 0, None) == B.ERR_ARG
    assert g(FAKE, None, FAKE, None, None, p, FAKE, None, None, 0, None) == B.ERR_ARG
    assert g(FAKE, None, FAKE, None, FAKE, p, None, None, None, 0, None) == B.ERR_ARG
    assert g(FAKE, None, FAKE, FAKE, FAKE, norm_params(weight_dtype=B.F16), FAKE, None, None, 0, None) == B.ERR_ARG
    size = C.c_size_t()
    assert lib.rans_norm_workspace_bytes(p, C.byref(size)) == B.OK and size.value >= 4 * 256 * 4
    assert lib.rans_norm_workspace_bytes(p, None) == B.ERR_ARG
    assert g(FAKE, None, FAKE, None, FAKE, p, FAKE, FAKE, None, size.value, None) == B.ERR_ARG
    assert g(FAKE, None, FAKE, None, FAKE, p, FAKE, FAKE, FAKE + 16, size.value, None) == B.ERR_ARG
    assert g(FAKE, None, FAKE, None, FAKE, p, FAKE, FAKE, FAKE, size.value - 1, None) == B.ERR_WORKSPACE


def test_matmul_arguments_refused(lib):
    a, b = blocks(), blocks(rows=8)
    f = lib.rans_block_matmul
    assert f(None, FAKE, a, FAKE, FAKE, b, B.BF16, FAKE, 8, None, 0, None) == B.ERR_ARG
    assert f(FAKE, None, a, FAKE, FAKE, b, B.BF16, FAKE, 8, None, 0, None) == B.ERR_ARG
    assert f(FAKE, FAKE, a, None, FAKE, b, B.BF16, FAKE, 8, None, 0, None) == B.ERR_ARG
    assert f(FAKE, FAKE, a, FAKE, FAKE, b, B.BF16, None, 8, None, 0, None) == B.ERR_ARG
    assert f(FAKE, FAKE, a, FAKE, FAKE, b, B.BF16, FAKE + 1, 8, None, 0, None) == B.ERR_ARG
    assert f(FAKE, FAKE, a, FAKE, FAKE, b, 3, FAKE, 8, None, 0, None) == B.ERR_ARG
    assert f(FAKE, FAKE, a, FAKE, FAKE, b, B.BF16, FAKE, 7, None, 0, None) == B.ERR_SHAPE
    assert f(FAKE, FAKE, blocks(block=1), FAKE, FAKE, b, B.BF16, FAKE, 8, None, 0, None) == B.ERR_ARG      # A has row blocks
    assert f(FAKE, FAKE, a, FAKE, FAKE, blocks(scale_type=1), B.BF16, FAKE, 8, None, 0, None) == B.ERR_ARG
    assert f(FAKE, FAKE, a, FAKE, FAKE, blocks(cols=128), B.BF16, FAKE, 8, None, 0, None) == B.ERR_SHAPE
    assert f(None, None, blocks(rows=0), None, None, b, B.BF16, None, 8, None, 0, None) in (B.ERR_ARG, B.OK)
    size = C.c_size_t()
    assert lib.rans_matmul_workspace_bytes(a, b, None) == B.ERR_ARG
    assert lib.rans_matmul_workspace_bytes(a, b, C.byref(size)) == B.OK and size.value == 0
    long = blocks(rows=64, cols=8192, ld=8192, ld_scale=64)
    assert lib.rans_matmul_workspace_bytes(long, long, C.byref(size)) == B.OK and size.value >= 2 * 64 * 64 * 4


def test_binding_refuses_host_tensors_and_short_memory(lib):
    x = torch.zeros(4, 256)
    code, scale = torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(4, 4)
    b = blocks()
    assert B.rans_block_quantize(x, 256, B.F32, False, code, scale, b) == B.ERR_ARG
    assert B.rans_block_dequantize(code, scale, b, B.F32, x, 256) == B.ERR_ARG
    assert B.rans_norm_quantize(x, None, None, norm_params(dtype=B.F32, weight_dtype=B.F32), None, None, x, None, None, None) == B.ERR_ARG
    assert B.rans_norm_backward(x, None, x, None, x[0], norm_params(dtype=B.F32, weight_dtype=B.F32), x, None, None) == B.ERR_ARG
    assert B.rans_block_matmul(code, scale, b, code, scale, b, B.F32, x, 256, None) == B.ERR_ARG
    host = -1

    def holds(t, *want):
        try:
            return B._mem(t, host, *want) == t.data_ptr()
        except B._Refused:
            return False

    assert holds(x, 4, 256, 256, 4) and not holds(x, 4, 256, 257, 4) and not holds(x, 5, 1, 256, 4) and holds(x[:, :7], 4, 7, 256, 4)
    assert not holds(x.half(), 4, 256, 256, 4)                       # elements of half the size
    assert not holds(x[0].expand(8, 256), 8, 256, 256, 4)            # one row of memory, seen eight times
    assert B._mem(None, host, 4, 256, 256, 4) is None
    with pytest.raises(B._Refused):
        B._mem(x, 0, 4, 256, 256, 4)                                 # on another device
    with pytest.raises(B._Refused):
        B._mem_blocks(code, scale, host, blocks(rows=5))
    assert B._mem_blocks(code, scale[:1], host, blocks(block=1)) == (code.data_ptr(), scale.data_ptr())
    with pytest.raises(B.RansError):
        B._ld(x.t())


@pytest.mark.parametrize("fmt, dt", [(0, torch.float8_e4m3fn), (1, torch.float8_e5m2)])
def test_oracle_formats_agree_with_torch(fmt, dt):
    c = torch.arange(256, dtype=torch.uint8)
    assert torch.equal(torch.nan_to_num(O.decode8(c, fmt), nan=-1e9), torch.nan_to_num(c.view(dt).double(), nan=-1e9))
    v = torch.randn(20000, generator=torch.Generator().manual_seed(0)) * torch.exp2(torch.randint(-12, 9, (20000,), generator=torch.Generator().manual_seed(1)))
    v = v.clamp(-O.VMAX[fmt], O.VMAX[fmt])
    assert torch.equal(O.round8(v.double(), fmt), v.to(dt).double())


@pytest.mark.parametrize("fmt", (0, 1))
def test_oracle_scales_are_the_least_power_of_two(fmt):
    """v s >= a > v s / 2, at a = v 2^e and next to it."""
    v = O.VMAX[fmt]
    a = torch.tensor([v, v * 2 ** -30, v * 2 ** 20, 1.0, 1.7499999, 1.75, 1.7500001, 3.0]).float().repeat(2, 1)
    for i in range(a.shape[1]):
        s = O.block_scales(a[:1, i:i + 1], fmt, True, False).item()
        assert v * s >= a[0, i].item() > v * s / 2


def test_calls_go_to_their_tensors_device(monkeypatch):
    """Tensors of a device that is not the current one: the call is made with theirs as the current one, and the current one is put back."""
    current, seen = [0], []

    class Device:
        def __init__(self, dev):
            self.dev = dev

        def __enter__(self):
            self.before, current[0] = current[0], self.dev

        def __exit__(self, *_):
            current[0] = self.before

    monkeypatch.setattr(B, "_current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(B, "_raw_stream", lambda dev: 100 + dev)
    for dev in (0, 1):
        assert B._enqueue(lambda *a: seen.append((current[0], a)) or 7, dev, "x", "y") == 7
    assert seen == [(0, ("x", "y", 100)), (1, ("x", "y", 101))] and current == [0]


def test_memory_of_a_workspace():
    whole = torch.empty(5, 256, dtype=torch.float32)
    at = whole.data_ptr()
    assert B._mem_ws(None, -1) == (None, 0) and B._mem_ws(whole, -1) == (at, 5120) and B._mem_ws(whole[1:], -1) == (at + 1024, 4096)
    assert B._mem_ws(torch.empty(1, dtype=torch.uint8).expand(4096), -1)[1] == 1 and B._mem_ws(whole[:, :128], -1) == (at, (4 * 256 + 128) * 4)
    with pytest.raises(B._Refused):
        B._mem_ws(whole, 0)


@pytest.mark.parametrize("k", (4096, 8192, 16384))
@pytest.mark.parametrize("other", (1, 33, 64, 200, 2048, 4096))
@pytest.mark.parametrize("left", (0, 1, 64, 77, 1024, 4000))
def test_matmul_workspace_holds_every_launch(lib, left, other, k):
    """A product of more than 2^17 rows goes launch by launch: what the whole asks for is enough for the launch of the rows that
    are left, which alone may have few enough tiles to take K in parts."""
    slice_rows = 1 << 17

    def need(m, n):
        size = C.c_size_t()
        assert lib.rans_matmul_workspace_bytes(B.make_blocks(m, k), B.make_blocks(n, k), C.byref(size)) == B.OK
        return size.value

    for whole in (slice_rows + left, 3 * slice_rows + left):
        assert need(whole, other) >= max(need(left, other), need(slice_rows, other))
        assert need(other, whole) >= max(need(other, left), need(other, slice_rows))
        assert need(whole, whole) >= need(left, left)


def refused(code, call):
    with pytest.raises(B.RansError) as e:
        call()
    assert e.value.code == code


def test_block_matrix_refuses_other_shapes_and_types(lib):
    """Larger tensors too, of which only a corner would be coded or written; the right shape passes on to the memory's check, which
    refuses the host's."""
    m, w = B.BlockMatrix(4, 256, device="cpu"), B.BlockMatrix(6, 256, device="cpu")
    for rows, cols in ((8, 512), (8, 256), (4, 512), (3, 256), (4, 255), (256, 4)):
        refused(B.ERR_SHAPE, lambda: m.quantize(torch.zeros(rows, cols)))
        refused(B.ERR_SHAPE, lambda: m.quantize(torch.zeros(cols, rows), transpose=True))
        refused(B.ERR_SHAPE, lambda: m.dequantize(torch.zeros(rows, cols)))
    for rows, cols in ((8, 6), (4, 8), (4, 5), (6, 4), (4, 256)):
        refused(B.ERR_SHAPE, lambda: m.matmul(w, torch.zeros(rows, cols)))
    refused(B.ERR_SHAPE, lambda: m.quantize(torch.zeros(8, 512)[:4, ::2]))
    refused(B.ERR_SHAPE, lambda: m.quantize(torch.zeros(4 * 256)))
    refused(B.ERR_ARG, lambda: m.quantize(torch.zeros(4, 256, dtype=torch.float64)))
    refused(B.ERR_ARG, lambda: m.dequantize(torch.zeros(4, 256, dtype=torch.int16)))
    refused(B.ERR_ARG, lambda: m.matmul(w, torch.zeros(4, 6, dtype=torch.float64)))
    refused(B.ERR_ARG, lambda: m.quantize(torch.zeros(4, 256)))
    refused(B.ERR_ARG, lambda: m.quantize(torch.zeros(256, 9)[:, :4], transpose=True))
    refused(B.ERR_ARG, lambda: m.dequantize(torch.zeros(4, 256)))
    refused(B.ERR_ARG, lambda: m.matmul(w, torch.zeros(4, 6)))


def test_binding_refuses_strided_rows():
    """Elements of a row, of a weight, of rstd follow one another in memory: other strides are not what the entry points read."""
    x = torch.zeros(8, 512)

    def holds(t, *want):
        try:
            return B._mem(t, -1, *want) == t.data_ptr()
        except B._Refused:
            return False

    assert holds(x[:, :256], 8, 256, 512, 4) and holds(x.view(-1)[3:], 1, 256, 256, 4) and holds(x[:, 5:6], 8, 1, 512, 4)
    assert holds(x[0, :256].expand(1, 256), 1, 256, 256, 4) and holds(x[:, 0], 1, 1, 1, 4)
    heads = torch.zeros(8, 6, 64)[:, :4]                # heads next to one another, others behind them in each row
    assert holds(heads, 8, 256, 384, 4) and holds(heads[:, :, None], 8, 256, 384, 4) and not holds(heads, 8, 257, 384, 4)
    assert not holds(x[:, ::2], 8, 256, 512, 4) and not holds(x.t(), 8, 512, 512, 4)
    assert not holds(x.view(-1)[::2], 1, 256, 256, 4)   # every other number
    assert not holds(x[0, :1].expand(256), 1, 256, 256, 4)
    assert not holds(x[:, 0], 1, 8, 8, 4) and not holds(x[:, :1], 1, 8, 8, 4)  # a column as a weight
