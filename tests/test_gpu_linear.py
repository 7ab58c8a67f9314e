"""Linear layers and their gradients against their definitions in 64 bits, at the sizes, strides, alignments and
epilogues where they can go wrong (marked gpu).

Tolerances, element by element, from the arithmetic.  A product's sum over K terms carries at most
(K + 8) 2^-23 of sum |a| |b| from its fp32 additions (truncated ones included), and in 32 bits 2^-19 of it from
the split products (each within a few 2^-21).  Epilogues multiply that by the activation's largest slope (below
1.2) and add a few 2^-22 of their own value; a bf16 result is within half a unit in the last place, 2^-8, of it.
"""
import pytest
import torch

import _operators as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = [(1, 1, 1), (1, 5, 3), (2, 64, 64), (3, 2048, 256), (17, 33, 65), (64, 64, 64), (65, 130, 33), (128, 128, 128),
         (129, 257, 100), (200, 333, 777), (256, 512, 64), (300, 264, 1032), (31, 1000, 2040), (520, 136, 72),
         (1000, 24, 3000), (384, 768, 520)]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


def _mat(rows, cols, dt, gen, pad=0, shift=0, scale=1.0):
    buf = torch.zeros(rows * (cols + pad) + shift, device="cuda", dtype=dt)
    x = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    x.copy_(scale * torch.randn(rows, cols, generator=gen))
    return x


def _out(rows, cols, dt, pad=0, shift=0):
    """An output in a buffer of a marker value, whose rest must stay as it is."""
    buf = torch.full((rows * (cols + pad) + shift + 64,), 7.0, device="cuda", dtype=dt)
    return buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols], buf


def _untouched(buf, x):
    keep = buf.clone()
    off = (x.data_ptr() - buf.data_ptr()) // buf.element_size()
    keep.as_strided(x.shape, x.stride(), off).fill_(7.0)
    return bool((keep == 7.0).all())


def _sum_tol(a, b, k, dt):
    """The bound on a product's error: a (M x K) and b (N x K) in 64 bits."""
    return (a.abs() @ b.abs().T) * ((k + 8) * 2.0 ** -23 + (2.0 ** -19 if dt == torch.float32 else 0)) + 1e-30


def _check(got, want, tol, dt):
    got = got.double().cpu()
    tol = tol + want.abs() * (2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -21) + 1e-7 * (dt == torch.float32)
    assert torch.isfinite(got).all()
    bad = (got - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()), float(tol.max()))


@pytest.mark.parametrize("rows,n,k", SIZES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (1, 3)])
def test_forward(rows, n, k, dt, pad, shift):
    import paper_2507_08784_gb300 as glr
    dt = DT[dt]
    gen = torch.Generator().manual_seed(rows + 7 * n + 13 * k)
    for act, bias, residual, preact in (("none", False, False, False), ("gelu", True, False, True), ("silu", False, True, True),
                                        ("gelu_tanh", True, True, False), ("relu", True, True, True)):
        X, W = _mat(rows, k, dt, gen, pad, shift), _mat(n, k, dt, gen, pad, shift, k ** -0.5)
        b = torch.randn(n, generator=gen).to(dt).cuda() if bias else None
        R = _mat(rows, n, dt, gen, pad, shift) if residual else None
        Y, ybuf = _out(rows, n, dt, pad, shift)
        P, pbuf = _out(rows, n, dt, 2 * pad, shift) if preact else (None, None)
        glr.glr_linear(X, W, Y, bias=b, act=act, residual=R, preact=P)
        torch.cuda.synchronize()
        Xc, Wc = X.cpu(), W.cpu()
        Z, want = ref.linear(Xc, Wc, None if b is None else b.cpu(), act, None if R is None else R.cpu())
        tol = 1.2 * _sum_tol(Xc.double(), Wc.double(), k, dt) + 2.0 ** -21 * (Z.abs() + 1)
        _check(Y, want, tol + (0 if R is None else 2.0 ** -22 * R.cpu().double().abs()), dt)
        assert _untouched(ybuf, Y)
        if preact:
            _check(P, Z, tol, dt)
            assert _untouched(pbuf, P)
    glr.glr_operator_status()


@pytest.mark.parametrize("rows,n,k", SIZES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (1, 3)])
def test_grad_input(rows, n, k, dt, pad, shift):
    import paper_2507_08784_gb300 as glr
    dt = DT[dt]
    gen = torch.Generator().manual_seed(rows + 5 * n + 11 * k)
    for act, residual, grad_out in (("none", False, False), ("none", True, True), ("gelu", True, False), ("silu", False, True),
                                    ("gelu_tanh", True, True), ("relu", False, False)):
        dZ, W = _mat(rows, n, dt, gen, pad, shift), _mat(n, k, dt, gen, pad, shift, n ** -0.5)
        D = _mat(rows, k, dt, gen, pad, shift) if residual else None
        P = _mat(rows, k, dt, gen, pad, shift, 2.0) if act != "none" else None
        dX, xbuf = _out(rows, k, dt, pad, shift)
        G, gbuf = _out(rows, k, dt, 0, shift) if grad_out else (None, None)
        glr.glr_linear_grad_input(dZ, W, dX, residual=D, preact=P, act=act, grad_out=G)
        torch.cuda.synchronize()
        a, b = dZ.cpu().double(), W.cpu().double()
        g = a @ b + (0 if D is None else D.cpu().double())
        slope = torch.ones_like(g) if P is None else ref.act_slope(P.cpu().double(), act)
        tol = _sum_tol(a, b.T.contiguous(), n, dt) + 2.0 ** -22 * g.abs()
        # the slopes' own error: a few 2^-22 of terms of the size of 1 + |z|^3
        extra = 0 if P is None else 2.0 ** -20 * g.abs() * (1 + P.cpu().double().abs())
        _check(dX, g * slope, tol * 1.2 + extra, dt)
        assert _untouched(xbuf, dX)
        if grad_out:
            _check(G, g, tol, dt)
            assert _untouched(gbuf, G)
    glr.glr_operator_status()


@pytest.mark.parametrize("nodes,rows,n,k", [(1, 1, 1, 1), (2, 3, 5, 7), (4, 32, 256, 128), (3, 65, 100, 33), (1, 1000, 64, 64),
                                            (8, 128, 128, 256), (2, 777, 72, 136), (5, 64, 520, 24), (64, 5, 40, 48),
                                            (1, 4100, 136, 200), (4, 40, 333, 777), (2, 300, 768, 384)])
@pytest.mark.parametrize("dt,gd", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (1, 1)])
def test_grad_weight(nodes, rows, n, k, dt, gd, pad, shift):
    import paper_2507_08784_gb300 as glr
    dt, gd = DT[dt], DT[gd]
    gen = torch.Generator().manual_seed(nodes + 3 * rows + 5 * n + 11 * k)
    dZ, X = _mat(nodes * rows, n, dt, gen, pad, shift), _mat(nodes * rows, k, dt, gen, pad, shift)
    for bias in (False, True):
        outs = [_out(n, k, gd) for _ in range(nodes)]
        sums = [_out(1, n, gd) for _ in range(nodes)] if bias else None
        glr.glr_linear_grad_weight(dZ, X, [o[0] for o in outs], db=[s[0].view(n) for s in sums] if bias else None)
        torch.cuda.synchronize()
        for i in range(nodes):
            a, b = (t[i * rows:(i + 1) * rows].cpu().double().T.contiguous() for t in (dZ, X))
            _check(outs[i][0], a @ b.T, _sum_tol(a, b, rows, dt), gd)
            assert _untouched(outs[i][1], outs[i][0])
            if bias:
                _check(sums[i][0].view(n), a.sum(1), (rows + 8) * 2.0 ** -23 * a.abs().sum(1), gd)
                assert _untouched(sums[i][1], sums[i][0])
    glr.glr_operator_status()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_nothing_to_do(dt):
    """No rows, no inputs: the sums are empty, the epilogues still run."""
    import paper_2507_08784_gb300 as glr
    dt = DT[dt]
    e = lambda *s: torch.empty(*s, device="cuda", dtype=dt)  # noqa: E731
    glr.glr_linear(e(0, 8), e(16, 8), e(0, 16))
    b, Y = torch.randn(16, device="cuda").to(dt), e(3, 16)
    glr.glr_linear(e(3, 0), e(16, 0), Y, bias=b, act="relu")
    assert torch.equal(Y, b.clamp(min=0).expand(3, 16))
    dX = e(3, 8)
    glr.glr_linear_grad_input(e(3, 0), e(0, 8), dX)
    assert not dX.any()
    dW, db = [torch.full((16, 8), 3.0, device="cuda") for _ in range(2)], [torch.full((16,), 3.0, device="cuda") for _ in range(2)]
    glr.glr_linear_grad_weight(e(0, 16), e(0, 8), dW, db=db)
    assert not any(x.any() for x in dW + db)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,k", [(70, 90, 50), (256, 256, 192)])
def test_in_place_residual_stream_and_graph(rows, n, k, dt):
    """The residual in the output's own memory, on another stream, and replayed from a graph: the same bits."""
    import paper_2507_08784_gb300 as glr
    dt = DT[dt]
    gen = torch.Generator().manual_seed(1)
    X, W, R = _mat(rows, k, dt, gen), _mat(n, k, dt, gen), _mat(rows, n, dt, gen)
    want = torch.empty_like(R)
    glr.glr_linear(X, W, want, residual=R, act="silu")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    Y = R.clone()
    s.wait_stream(torch.cuda.current_stream())
    glr.glr_linear(X, W, Y, residual=Y, act="silu", stream=s)
    s.synchronize()
    assert torch.equal(Y, want)
    graph, Y = torch.cuda.CUDAGraph(), torch.zeros_like(R)
    with torch.cuda.graph(graph):
        glr.glr_linear(X, W, Y, residual=R, act="silu")
    for _ in range(2):
        Y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, want)


def test_not_a_number_and_infinity_stay_in_their_rows():
    """A row of X with NaN, one with infinity: the other rows' results are as without them."""
    import paper_2507_08784_gb300 as glr
    for dt in DT.values():
        for rows, n, k in ((130, 70, 90), (256, 256, 256)):
            gen = torch.Generator().manual_seed(2)
            X, W = _mat(rows, k, dt, gen), _mat(n, k, dt, gen)
            Y, Z = torch.empty(rows, n, device="cuda", dtype=dt), torch.empty(rows, n, device="cuda", dtype=dt)
            glr.glr_linear(X, W, Y)
            X[3, 5] = float("nan")
            X[64, 7] = float("inf")
            glr.glr_linear(X, W, Z)
            assert torch.isnan(Z[3]).all() and not torch.isfinite(Z[64]).any()
            keep = [i for i in range(rows) if i not in (3, 64)]
            assert torch.equal(Z[keep], Y[keep])


def test_gradients_against_differences():
    """Two layers, L = <C, Y>: the chain of the three gradients against central differences of the forward pass
    along random directions.  |L''| along a unit direction is below 4 here and L is within 1e-5, so a step of
    1e-2 is good to 1e-3 + 1e-2^2."""
    import paper_2507_08784_gb300 as glr
    gen = torch.Generator().manual_seed(5)
    rows, d, h, o = 24, 20, 31, 12
    X, W1, b1, W2 = (torch.randn(*s, generator=gen).cuda() for s in ((rows, d), (h, d), (h,), (o, h)))
    X.mul_(0.5), W1.mul_(0.3), W2.mul_(0.2)
    R, C = torch.randn(rows, o, generator=gen).cuda(), torch.randn(rows, o, generator=gen).cuda() / 10

    def forward(X, W1, b1, W2):
        Z1, H, Y = torch.empty(rows, h, device="cuda"), torch.empty(rows, h, device="cuda"), torch.empty(rows, o, device="cuda")
        glr.glr_linear(X, W1, H, bias=b1, act=act, preact=Z1)
        glr.glr_linear(H, W2, Y, residual=R)
        return Z1, H, float((C * Y).double().sum())

    for act in ("gelu", "gelu_tanh", "silu"):
        Z1, H, _ = forward(X, W1, b1, W2)
        dZ1, dX, dW1, dW2, db = (torch.empty_like(t) for t in (Z1, X, W1, W2, b1))
        glr.glr_linear_grad_input(C, W2, dZ1, preact=Z1, act=act)
        glr.glr_linear_grad_weight(C, H, dW2)
        glr.glr_linear_grad_weight(dZ1, X, dW1, db=db)
        glr.glr_linear_grad_input(dZ1, W1, dX)
        for which, grad in enumerate((dX, dW1, db, dW2)):
            v = torch.randn(grad.shape, generator=gen).cuda()
            v /= v.norm()
            vals = []
            for e in (1e-2, -1e-2):
                args = [X, W1, b1, W2]
                args[which] = args[which] + e * v
                vals.append(forward(*args)[2])
            assert abs((vals[0] - vals[1]) / 2e-2 - float((grad * v).sum())) < 1.1e-3, (act, which)


def test_results_are_reproducible():
    import paper_2507_08784_gb300 as glr
    for dt in DT.values():
        gen = torch.Generator().manual_seed(4)
        dZ, X = _mat(4 * 300, 264, dt, gen), _mat(4 * 300, 136, dt, gen)
        a, b = ([torch.empty(264, 136, device="cuda") for _ in range(4)] for _ in range(2))
        da, db = ([torch.empty(264, device="cuda") for _ in range(4)] for _ in range(2))
        glr.glr_linear_grad_weight(dZ, X, a, db=da)
        glr.glr_linear_grad_weight(dZ, X, b, db=db)
        assert all(torch.equal(x, y) for x, y in zip(a + da, b + db))


@pytest.mark.parametrize("nodes,rows,n,k", [(2, 64, 1, 64), (3, 40, 64, 1), (4, 7, 1, 1), (2, 1, 128, 192), (8, 1, 8, 8)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_grad_weight_of_single_columns_and_rows(nodes, rows, n, k, dt):
    import paper_2507_08784_gb300 as glr
    dt = DT[dt]
    gen = torch.Generator().manual_seed(12)
    dZ, X = _mat(nodes * rows, n, dt, gen), _mat(nodes * rows, k, dt, gen)
    dW, db = [torch.empty(n, k, device="cuda") for _ in range(nodes)], [torch.empty(n, device="cuda") for _ in range(nodes)]
    glr.glr_linear_grad_weight(dZ, X, dW, db=db)
    for i in range(nodes):
        a, b = (t[i * rows:(i + 1) * rows].cpu().double().T.contiguous() for t in (dZ, X))
        _check(dW[i], a @ b.T, _sum_tol(a, b, rows, dt), torch.float32)
        _check(db[i], a.sum(1), (rows + 8) * 2.0 ** -23 * a.abs().sum(1), torch.float32)


LARGE = [(700, 640, 1111), (257, 2048, 1024), (2048, 300, 901), (4100, 256, 513), (130, 1000, 4096)]


@pytest.mark.parametrize("rows,n,k", LARGE)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 3)])
def test_large_products(rows, n, k, dt, pad, shift):
    """Products large enough to be laid out for the tensor cores first (fp32, and rows off 16 bytes), with positive
    inputs too, where a truncated sum would drift: every sum within 2^-20 of sum |a| |b|, which rounded additions
    of up to 4100 products meet (their errors add up like their square root) and truncated ones do not."""
    import paper_2507_08784_gb300 as glr
    dt = DT[dt]
    gen = torch.Generator().manual_seed(rows)
    for positive in (False, True):
        X, W, Z = _mat(rows, k, dt, gen, pad, shift), _mat(n, k, dt, gen, pad, shift), _mat(rows, n, dt, gen, pad, shift)
        if positive:
            X.abs_(), W.abs_(), Z.abs_()
        Y, ybuf = _out(rows, n, dt, pad, shift)
        dX, xbuf = _out(rows, k, dt, pad, shift)
        dW = [torch.empty(n, k, device="cuda")]
        glr.glr_linear(X, W, Y, act="relu")
        glr.glr_linear_grad_input(Z, W, dX)
        glr.glr_linear_grad_weight(Z, X, dW)
        torch.cuda.synchronize()
        x, w, z = X.double(), W.double(), Z.double()
        for got, a, b in ((Y, x, w), (dX, z, w.T), (dW[0], z.T, x.T)):
            want, size = a @ b.T, a.abs() @ b.abs().T
            want = want.clamp(min=0) if got is Y else want
            tol = 2.0 ** -20 * size + (2.0 ** -8 * want.abs() if got.dtype == torch.bfloat16 else 2.0 ** -22 * want.abs())
            if got.dtype == torch.bfloat16:
                tol += (a.shape[1] + 8) * 2.0 ** -23 * size       # bf16 results may be summed by truncation
            assert ((got.double() - want).abs() <= tol).all(), (positive, float(((got.double() - want).abs() / size).max()))
        assert _untouched(ybuf, Y) and _untouched(xbuf, dX)
    glr.glr_operator_status()


def test_large_products_without_workspace():
    """The C entry point with no workspace takes another way to the same product."""
    import ctypes
    import paper_2507_08784_gb300 as glr
    from paper_2507_08784_gb300 import _lib
    gen = torch.Generator().manual_seed(3)
    X, W, Y, Z = (_mat(*s, torch.float32, gen) for s in ((600, 900), (700, 900), (600, 700), (600, 700)))
    args = _lib.GlrLinearArgs(600, 700, 900, X.data_ptr(), 900, W.data_ptr(), 900, Y.data_ptr(), 700, None, None, 0, None, 0, None, 0, 0, 0)
    need = ctypes.c_int64(-1)
    assert glr.load().glr_linear_workspace(ctypes.byref(args), ctypes.byref(need)) == 0 and need.value >= 3 * 2 * 1300 * 900
    assert glr.load().glr_linear(ctypes.byref(args), torch.cuda.current_stream().cuda_stream) == 0
    glr.glr_linear(X, W, Z)
    torch.cuda.synchronize()
    size, want = X.double().abs() @ W.double().abs().T, X.double() @ W.double().T
    for got in (Y, Z):
        assert ((got.double() - want).abs() <= 2.0 ** -19 * size).all()


def test_infinities_survive_the_layout():
    """fp32 matrices cut into planes: an infinity or a NaN stays in its row, and the type's extremes are finite."""
    import paper_2507_08784_gb300 as glr
    gen = torch.Generator().manual_seed(4)
    X, W = _mat(300, 1500, torch.float32, gen), _mat(1200, 1500, torch.float32, gen)
    Y, Z = torch.empty(300, 1200, device="cuda"), torch.empty(300, 1200, device="cuda")
    glr.glr_linear(X, W, Y)
    X[5, 7], X[90, 1400], X[200] = float("nan"), float("inf"), 0.0
    X[200, 3] = 1.5e38
    glr.glr_linear(X, W, Z)
    assert torch.isnan(Z[5]).all() and not torch.isfinite(Z[90]).any()
    keep = [i for i in range(300) if i not in (5, 90, 200)]
    assert torch.equal(Z[keep], Y[keep])
    small = W[:, 3].abs() < 2
    want = 1.5e38 * W[:, 3].double()
    assert ((Z[200].double() - want).abs()[small] <= 2.0 ** -19 * want.abs()[small]).all()


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 7, 8, 9])
@pytest.mark.parametrize("n,k", [(1, 8), (2, 3), (5, 1032), (63, 515), (64, 2048), (1001, 4100), (6000, 8193)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_few_rows(rows, n, k, dt):
    """Rows on 16 bytes of any length, whose last vector is whole or not."""
    import paper_2507_08784_gb300 as glr
    dt = DT[dt]
    gen = torch.Generator().manual_seed(rows + 7 * n + 13 * k)
    pad = -k % 8 + 8
    X, W = _mat(rows, k, dt, gen, pad), _mat(n, k, dt, gen, pad, scale=k ** -0.5)
    b = torch.randn(n, generator=gen).to(dt).cuda()
    R = _mat(rows, n, dt, gen, 1, 1)
    Y, ybuf = _out(rows, n, dt, 3, 1)
    P, pbuf = _out(rows, n, dt, 5, 2)
    glr.glr_linear(X, W, Y, bias=b, act="silu", residual=R, preact=P)
    Xc, Wc, Rc = X.cpu(), W.cpu(), R.cpu()
    Z, want = ref.linear(Xc, Wc, b.cpu(), "silu", Rc)
    tol = 1.2 * _sum_tol(Xc.double(), Wc.double(), k, dt) + 2.0 ** -21 * (Z.abs() + 1)
    _check(Y, want, tol + 2.0 ** -22 * Rc.double().abs(), dt)
    _check(P, Z, tol, dt)
    assert _untouched(ybuf, Y) and _untouched(pbuf, P)
    glr.glr_operator_status()


@pytest.mark.parametrize("rows,n,k", [(1000, 2048, 8200), (1000, 8200, 2048), (8200, 1000, 2048), (20, 4100, 4097), (400, 1100, 2100)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_long_contractions_of_few_tiles(rows, n, k, dt, pad, shift):
    """Contractions that pairs of SMs or single ones share, of the product and of each gradient in turn."""
    test_large_products(rows, n, k, dt, pad, shift)


@pytest.mark.parametrize("nodes,rows,n,k", [(2, 600, 700, 900), (1, 3000, 1000, 1032), (8, 64, 512, 1001)])
def test_bf16_gradients_of_fp32_matrices(nodes, rows, n, k):
    """Products of fp32 matrices large enough to be laid out in planes, rounded to bf16 once at the end."""
    import paper_2507_08784_gb300 as glr
    gen = torch.Generator().manual_seed(rows)
    dZ, X = _mat(nodes * rows, n, torch.float32, gen), _mat(nodes * rows, k, torch.float32, gen)
    dW = [torch.empty(n, k, device="cuda", dtype=torch.bfloat16) for _ in range(nodes)]
    db = [torch.empty(n, device="cuda", dtype=torch.bfloat16) for _ in range(nodes)]
    glr.glr_linear_grad_weight(dZ, X, dW, db=db)
    for i in range(nodes):
        a, b = (t[i * rows:(i + 1) * rows].double().T.contiguous().cpu() for t in (dZ, X))
        _check(dW[i], a @ b.T, _sum_tol(a, b, rows, torch.float32), torch.bfloat16)
        _check(db[i], a.sum(1), (rows + 8) * 2.0 ** -23 * a.abs().sum(1), torch.bfloat16)
    glr.glr_operator_status()


@pytest.mark.parametrize("rows,n,k", [(1, 5, 3), (20, 64, 64), (65, 130, 33), (129, 257, 200), (300, 264, 1032), (40, 1000, 2040), (384, 768, 520)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 1])
def test_c_entries_without_workspace(rows, n, k, dt, pad):
    """All three products through the C entry points with no workspace, whatever one they would ask for."""
    import ctypes
    import paper_2507_08784_gb300 as glr
    from paper_2507_08784_gb300 import _lib
    code, dt = (0, torch.float32) if dt == "f32" else (1, torch.bfloat16)
    assert (_lib.GLR_F32, _lib.GLR_BF16) == (0, 1)
    gen = torch.Generator().manual_seed(rows + n)
    X, W, Z = _mat(rows, k, dt, gen, pad), _mat(n, k, dt, gen, pad, scale=k ** -0.5), _mat(rows, n, dt, gen, pad)
    (Y, ybuf), (D, dbuf) = _out(rows, n, dt, pad), _out(rows, k, dt, pad)
    G = torch.empty(n, k, device="cuda", dtype=dt)
    at = (ctypes.c_void_p * 1)(G.data_ptr())
    lib, st = glr.load(), torch.cuda.current_stream().cuda_stream
    p = lambda t: t.data_ptr()  # noqa: E731
    calls = [(lib.glr_linear, _lib.GlrLinearArgs(rows, n, k, p(X), k + pad, p(W), k + pad, p(Y), n + pad, None, None, 0, None, 0, None, 0, code, 0)),
             (lib.glr_linear_grad_input, _lib.GlrLinearGradInputArgs(rows, n, k, p(Z), n + pad, p(W), k + pad, p(D), k + pad, None, 0,
                                                                     None, 0, None, 0, None, 0, code, 0)),
             (lib.glr_linear_grad_weight, _lib.GlrLinearGradWeightArgs(1, rows, n, k, p(Z), n + pad, p(X), k + pad, ctypes.addressof(at),
                                                                       None, None, 0, code, code))]
    for fn, args in calls:
        assert fn(ctypes.byref(args), st) == 0
    torch.cuda.synchronize()
    x, w, z = (t.cpu().double() for t in (X, W, Z))
    for got, a, b in ((Y, x, w), (D, z, w.T.contiguous()), (G, z.T.contiguous(), x.T.contiguous())):
        _check(got, a @ b.T, _sum_tol(a, b, a.shape[1], dt), dt)
    assert _untouched(ybuf, Y) and _untouched(dbuf, D)
    glr.glr_operator_status()


@pytest.mark.parametrize("pad", [0, 1])
def test_matrices_past_32_bits_of_elements(pad):
    """70000 x 32768: as the input, as the input's gradient, as the weights of one row and as the weights' gradient."""
    import paper_2507_08784_gb300 as glr
    rows, k, n, dt = 70000, 32768, 24, torch.bfloat16
    big = torch.empty(rows, k + pad, device="cuda", dtype=dt).normal_()[:, :k]
    W, Z = torch.randn(n, k, device="cuda").to(dt), torch.randn(rows, n, device="cuda").to(dt)
    at = torch.tensor([0, 1, 32767, 32768, 65535, 65536, 69999], device="cuda")

    def close(got, a, b, k):
        want, size = a @ b.T, a.abs() @ b.abs().T
        assert ((got.double() - want).abs() <= (k + 8) * 2.0 ** -23 * size + 2.0 ** -8 * want.abs()).all()

    Y = torch.empty(rows, n, device="cuda", dtype=dt)
    glr.glr_linear(big, W, Y)
    close(Y[at], big[at].double(), W.double(), k)
    y = torch.empty(1, rows, device="cuda", dtype=dt)
    glr.glr_linear(W[:1], big, y)
    close(y[:, at], W[:1].double(), big[at].double(), k)
    dW = torch.empty(n, k, device="cuda", dtype=dt)
    glr.glr_linear_grad_weight(Z, big, dW)
    close(dW[:, at % k], Z.double().T, big[:, at % k].double().T, rows)
    out = torch.full((rows, k + pad), 7.0, device="cuda", dtype=dt)
    glr.glr_linear_grad_input(Z, W, out[:, :k])
    close(out[at, :k], Z[at].double(), W.double().T, n)
    assert pad == 0 or bool((out[:, k:] == 7).all())
    del out
    G = torch.empty(rows, k, device="cuda", dtype=dt)
    glr.glr_linear_grad_weight(Z.T[:8].contiguous(), W[:8].contiguous(), G)
    close(G[at], Z.T[:8, at].double().T, W[:8].double().T, 8)
    glr.glr_operator_status()
