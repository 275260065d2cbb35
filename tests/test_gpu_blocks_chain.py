"""Block codes, norm, matrix product and the codec together, as a split network uses them: a sender's norm and codes through a
container to the receiver's product; a training step's products and gradients; the same captured and on another stream."""
import pytest
import torch

from oracle import blocks as O
from paper_2511_11664_amd import binding as B

pytestmark = pytest.mark.gpu

EPS = 1e-5
TOKENS, HIDDEN, OUT = 150, 384, 260


def inputs(seed=0, tokens=TOKENS, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    x, r = (torch.randn(tokens, HIDDEN, generator=g).to(dtype) for _ in range(2))
    x[:, 7] *= 20
    w = (1 + 0.1 * torch.randn(HIDDEN, generator=g)).to(dtype)
    weight = torch.randn(OUT, HIDDEN, generator=g) * HIDDEN ** -0.5
    return x, r, w, weight


def values(m):
    rows, cols = m.layout.rows, m.layout.cols
    s = m.scale.cpu()
    s = torch.exp2(s.double() - 127) if s.dtype == torch.uint8 else s.double()
    return O.decode8(m.code[:, :cols].cpu(), m.layout.format) * O.spread(s, rows, cols, m.layout.block == B.BLOCK_TILE)


def norm_codes(x, r, w, scale_type=B.SCALE_E8M0):
    rows, cols = x.shape
    m = B.BlockMatrix(rows, cols, scale_type=scale_type)
    h, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
    p = B.make_norm_params(rows, cols, B.BF16, B.BF16, EPS)
    assert B.rans_norm_quantize(x, r, w, p, h, rstd, None, m.code, m.scale, m.layout) == 0
    return m, h, rstd, p


def half_steps(v, total):
    return v.abs() * 2.0 ** -8 + 7 * 2.0 ** -13 * total  # of bf16, and what the 8-bit instruction cuts off


@pytest.mark.parametrize("tokens", (1, 13, TOKENS))
def test_coded_features_through_a_container(tokens):
    """The sender's codes are the symbols of a container; the receiver's product of what it decodes is the product of the
    sender's own codes, bit by bit, and the definition's."""
    x, r, w, weight = inputs(tokens=tokens)
    m, *_ = norm_codes(x.cuda(), r.cuda(), w.cuda())
    n = m.code.numel()
    p = B.make_params(8, 12, tokens, HIDDEN, B.MODE_DENSE, 64, 64 * 32, B.F32)
    codec = B.Codec(p, n)
    codec.qinfo.copy_(torch.tensor([0.0, 255.0, 1.0, 0.0]))
    size = codec.encode(m.code.view(-1))
    got = B.BlockMatrix(tokens, HIDDEN, scale_type=B.SCALE_E8M0)
    codec.decode(size, codec.header(size), got.code.view(-1))
    got.scale.copy_(m.scale)
    assert torch.equal(got.code, m.code)
    wm = B.BlockMatrix(OUT, HIDDEN, scale_type=B.SCALE_E8M0, block=B.BLOCK_TILE).quantize(weight.cuda())
    y = got.matmul(wm, torch.empty(tokens, OUT, dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(y, m.matmul(wm, torch.empty_like(y)))
    want, total = O.matmul(values(m), values(wm))
    assert ((y.cpu().double() - want).abs() <= half_steps(want, total)).all()


def step(x, r, w, weight, dy, dh):
    """Forward and backward of y = codes(norm(x + r)) codes(weight)^T with 8-bit products; -> y, dx, dw of the norm, dweight."""
    m, h, rstd, p = norm_codes(x, r, w, B.SCALE_F32)
    wm = B.BlockMatrix(OUT, HIDDEN, block=B.BLOCK_TILE).quantize(weight)
    y = m.matmul(wm, torch.empty(TOKENS, OUT, dtype=torch.bfloat16, device="cuda"))
    g = B.BlockMatrix(TOKENS, OUT, B.E5M2).quantize(dy)
    wt = B.BlockMatrix(HIDDEN, OUT, block=B.BLOCK_TILE).quantize(weight, transpose=True)
    dn = g.matmul(wt, torch.empty(TOKENS, HIDDEN, dtype=torch.bfloat16, device="cuda"))
    dx, dw = torch.empty_like(x), torch.empty(HIDDEN, device="cuda")
    rc, size = B.rans_norm_workspace_bytes(p)
    assert rc == 0
    assert B.rans_norm_backward(dn, dh, h, w, rstd, p, dx, dw, B.workspace(size)) == 0
    n = m.dequantize(torch.empty(TOKENS, HIDDEN, dtype=torch.bfloat16, device="cuda"))
    gt = B.BlockMatrix(OUT, TOKENS, B.E5M2).quantize(dy, transpose=True)
    nt = B.BlockMatrix(HIDDEN, TOKENS).quantize(n, transpose=True)
    dweight = gt.matmul(nt, torch.empty(OUT, HIDDEN, device="cuda"))
    return dict(m=m, wm=wm, y=y, g=g, wt=wt, dn=dn, dx=dx, dw=dw, h=h, rstd=rstd, n=n, gt=gt, nt=nt, dweight=dweight)


def test_training_step():
    """Each result against the definition in 64 bits of what it was made from."""
    x, r, w, weight = inputs(1)
    g = torch.Generator().manual_seed(9)
    dy, dh = (torch.randn(TOKENS, c, generator=g).to(torch.bfloat16) for c in (OUT, HIDDEN))
    s = step(*(t.cuda() for t in (x, r, w, weight, dy, dh)))
    want, total = O.matmul(values(s["m"]), values(s["wm"]))
    assert ((s["y"].cpu().double() - want).abs() <= half_steps(want, total)).all()
    want, total = O.matmul(values(s["g"]), values(s["wt"]))
    assert ((s["dn"].cpu().double() - want).abs() <= half_steps(want, total)).all()
    assert torch.equal(values(s["wt"]), values(s["wm"]).t())
    want, total = O.matmul(values(s["gt"]), values(s["nt"]))
    assert ((s["dweight"].cpu().double() - want).abs() <= (128 + 2 + 4) * 2.0 ** -23 * total).all()
    assert torch.equal(O.quantize(dy.t(), B.E5M2, False, False)[0], O.decode8(s["gt"].code[:, :TOKENS].cpu(), B.E5M2))
    dx, dw = O.norm_backward(s["dn"].cpu(), dh, s["h"].cpu(), w, s["rstd"].cpu())
    assert ((s["dx"].cpu().double() - dx).abs() <= 2.0 ** -8 * dx.abs() + 1e-5).all()
    assert ((s["dw"].cpu().double() - dw).abs() <= 1e-5 * (1 + dw.abs())).all()
    # and the coded step as a whole next to the uncoded one: 8-bit operands, 3 and 2 mantissa bits, a few percent
    h = (x.float() + r.float()).to(torch.bfloat16).double()
    n = h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * w.double()
    for got, ref in ((s["y"], n @ weight.double().t()), (s["dweight"], dy.double().t() @ n), (s["dn"], dy.double() @ weight.double())):
        assert ((got.cpu().double() - ref).norm() / ref.norm()).item() < 0.1


def test_captured_chain_replays_like_eager_calls():
    """One graph of the whole step; other inputs at every replay, eager work of the same kind between them."""
    t = [v.cuda() for v in inputs(2)]
    dy, dh = torch.empty(TOKENS, OUT, dtype=torch.bfloat16, device="cuda").normal_(), torch.empty(TOKENS, HIDDEN, dtype=torch.bfloat16, device="cuda").normal_()
    step(*t, dy, dh)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*t, dy, dh)
    for seed in range(3, 7):
        new = [v.cuda() for v in inputs(seed)]
        for a, b in zip(t, new):
            a.copy_(b)
        dy.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = {k: out[k].clone() for k in ("y", "dn", "dx", "dw", "dweight")}
        eager = step(*new, dy, dh)
        for k in got:
            assert torch.equal(got[k], eager[k]), (seed, k)


def test_two_graphs_with_a_workspace_each_in_turn_and_on_two_streams():
    p = B.make_norm_params(700, 512, B.F32, B.F32, EPS)
    rc, size = B.rans_norm_workspace_bytes(p)
    assert rc == 0
    sets, graphs = [], []
    for _ in range(2):
        dy, h = torch.randn(700, 512, device="cuda"), torch.randn(700, 512, device="cuda")
        rstd = torch.rsqrt(h.square().mean(1) + EPS)
        sets.append((dy, h, rstd, torch.empty_like(h), torch.empty(512, device="cuda"), B.workspace(size)))

    def call(s):
        assert B.rans_norm_backward(s[0], None, s[1], None, s[2], p, s[3], s[4], s[5]) == 0

    want = []
    for s in sets:
        call(s)
        torch.cuda.synchronize()
        want.append((s[3].clone(), s[4].clone()))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(s)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(4):
        for s in sets:
            s[3].zero_(), s[4].zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for s, (dx, dw) in zip(sets, want):
            assert torch.equal(s[3], dx) and torch.equal(s[4], dw)


def test_another_stream():
    """A call goes to the current stream, behind what that stream still has to do."""
    x, r, w, weight = (t.cuda() for t in inputs(3))
    ref, *_ = norm_codes(x, r, w)
    st = torch.cuda.Stream()
    late = torch.empty_like(x)
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        torch.cuda._sleep(20_000_000)
        late.copy_(x)
        m, *_ = norm_codes(late, r, w)
    st.synchronize()
    nb = HIDDEN // 128  # scales behind a row are never written
    assert torch.equal(m.code, ref.code) and torch.equal(m.scale[:, :nb], ref.scale[:, :nb])


def test_launched_kernels(launched_kernels):
    x, r, w, weight = (t.cuda() for t in inputs(4))
    assert launched_kernels(lambda: norm_codes(x, r, w)) == {"k_norm_quant"}
    m = B.BlockMatrix(TOKENS, HIDDEN)
    assert launched_kernels(lambda: m.quantize(x)) == {"k_block_quant"}
    assert launched_kernels(lambda: B.BlockMatrix(HIDDEN, TOKENS).quantize(x, transpose=True)) == {"k_block_quant_tile"}
    assert launched_kernels(lambda: m.dequantize(torch.empty_like(x))) == {"k_block_dequant"}
