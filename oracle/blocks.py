"""Block codes, norm and matrix product in 64 bits, from their definitions in include/rans_if.h (torch on the CPU).

Where the definition names a binary32 operation (a block's scale, its reciprocal, the product that is rounded to 8 bits, the
sum that the norm's stream keeps) that operation is rounded here too; everything else is binary64.
"""
import torch

BLOCK = 128
E4M3, E5M2 = 0, 1
VMAX = (448.0, 57344.0)


def decode8(codes: torch.Tensor, fmt: int) -> torch.Tensor:
    """Values of 8-bit codes, from their fields."""
    c = codes.to(torch.int64)
    mbits, bias = ((3, 7), (2, 15))[fmt]
    e, m = (c & 0x7f) >> mbits, c & ((1 << mbits) - 1)
    v = torch.where(e > 0, (1 + m.double() / (1 << mbits)) * torch.exp2((e - bias).double()), m.double() / (1 << mbits) * 2.0 ** (1 - bias))
    if fmt == E4M3:
        v = torch.where((c & 0x7f) == 0x7f, torch.nan, v)
    else:
        v = torch.where(e == 31, torch.where(m > 0, torch.nan, torch.inf), v)
    return torch.where(c >= 128, -v, v)


def round8(v: torch.Tensor, fmt: int) -> torch.Tensor:
    """Nearest value of the format, ties to the even code; |v| is at most what rounds to the largest."""
    mbits, bias = ((3, 7), (2, 15))[fmt]
    _, e = torch.frexp(v)
    step = torch.exp2((torch.clamp(e - 1, min=1 - bias) - mbits).double())
    return torch.where(torch.isfinite(v), torch.round(v / step) * step, v if fmt == E5M2 else torch.nan)


def _blocks(x, tile):
    """[row blocks, rows of one, column blocks, BLOCK], padded with zeros."""
    h = BLOCK if tile else 1
    rows, cols = x.shape
    nr, nc = -(-rows // h), -(-cols // BLOCK)
    full = x.new_zeros(nr * h, nc * BLOCK)
    full[:rows, :cols] = x
    return full.view(nr, h, nc, BLOCK)


def block_scales(x: torch.Tensor, fmt: int, e8m0: bool, tile: bool) -> torch.Tensor:
    """Scales (binary64 values of binary32 numbers) of the blocks of x."""
    b = _blocks(x.double(), tile).abs()
    a = torch.where(torch.isfinite(b), b, 0.0).amax((1, 3))
    if e8m0:
        m, e = torch.frexp(a / VMAX[fmt])
        s = torch.exp2(torch.clamp(torch.where(m > 0.5, e, e - 1), min=-126).double())
    else:
        s = torch.clamp((a / VMAX[fmt]).float(), min=2.0 ** -126).double()  # a is a binary32 number: one rounding of the quotient
    return torch.where(a > 0, s, 1.0)


def spread(scales: torch.Tensor, rows: int, cols: int, tile: bool) -> torch.Tensor:
    """A scale for each element."""
    r = torch.arange(rows) // (BLOCK if tile else 1)
    return scales[r][:, torch.arange(cols) // BLOCK]


def quantize(x: torch.Tensor, fmt: int, e8m0: bool, tile: bool):
    """(values of the codes, scales) of a binary32 (or narrower) matrix."""
    s = block_scales(x, fmt, e8m0, tile)
    inv = (1 / s).float()  # correctly rounded: one division of binary32 numbers
    y = x.float() * spread(inv, *x.shape, tile)
    return round8(y.double(), fmt), s


def matmul(a: torch.Tensor, b: torch.Tensor):
    """(A B^T, |A| |B|^T) of binary64 values."""
    return a @ b.t(), a.abs() @ b.abs().t()


def norm(x, res, w, eps, dtype):
    """(h, rstd, y): h rounded to the stream's type, the others binary64."""
    h = x.double() if res is None else (x.float() + res.float()).to(dtype).double()
    rstd = 1 / torch.sqrt((h * h).mean(1) + eps)
    y = h * rstd[:, None]
    return h, rstd, y if w is None else y * w.double()


def norm_backward(dy, dsum, h, w, rstd):
    """(dx, dw) in binary64 of what the forward pass left."""
    dy, h, r = dy.double(), h.double(), rstd.double()[:, None]
    g = dy if w is None else dy * w.double()
    xh = h * r
    dx = r * (g - xh * (g * xh).mean(1, keepdim=True))
    return dx if dsum is None else dx + dsum.double(), (dy * xh).sum(0)
