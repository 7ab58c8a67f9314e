"""The row operators (embeddings, norms, activations in 8 bits, tokens' log-probabilities) against their definitions in
64 bits, at the sizes, masks, strides and alignments where they can go wrong (marked gpu).

Tolerances, from the arithmetic, with u = 2^-24 (half a step of fp32) and h = 2^-8 (half a step of bf16; 0 for fp32
results).  A sum of n terms in any order is within n u of the sum of their absolute values; the kernels' longest
chain of additions is stated at each test.  Codes and scales of given values are exact.
"""
import math

import pytest
import torch

import _operators as ops
import _rows as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


@pytest.fixture(scope="module")
def glr(_lib):
    import paper_2507_08784_gb300
    return paper_2507_08784_gb300


class Guarded:
    """rows x cols on the GPU inside a buffer of a known filling, which has to be there around it afterwards."""

    def __init__(self, rows, cols, dt, pad=0, shift=0, fill=None, value=None):
        self.fill = fill if fill is not None else (77 if dt in (torch.int8, torch.uint8, torch.int32, torch.int64) else 77.0)
        self.rows, self.cols, self.shift, self.ld = rows, cols, shift, cols + pad
        self.buf = torch.full((rows * self.ld + shift + 64,), self.fill, device="cuda", dtype=dt)
        self.t = self.buf[shift:shift + rows * self.ld].view(rows, self.ld)[:, :cols]
        if value is not None:
            self.t.copy_(value)

    def check(self):
        outside = torch.ones_like(self.buf, dtype=torch.bool)
        outside[self.shift:self.shift + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols] = False
        assert (self.buf[outside] == self.fill).all(), "written outside"
        return self.t


def _near(got, want, tol):
    """|got - want| <= tol, element by element (tol a tensor or a number)."""
    got, want = got.double().cpu(), torch.as_tensor(want, dtype=torch.float64)
    assert got.shape == want.shape
    assert torch.isfinite(got).all()
    over = (got - want).abs() - tol
    assert (over <= 0).all(), (float(over.max()), float((got - want).abs().max()), float(want.abs().max()))


# ---------------------------------------------------------------------------------------------------- embeddings

@pytest.mark.parametrize("rows,vocab,d,pad,shift,wide", [
    (1, 1, 1, 0, 0, False), (3, 5, 7, 1, 1, True), (17, 100, 64, 0, 0, False), (33, 50, 255, 1, 3, True), (64, 31, 256, 0, 0, True),
    (5, 1000, 2048, 8, 8, False), (9, 20, 2056, 0, 0, False), (300, 40, 33, 3, 0, True), (2, 3, 20001, 0, 1, False),
])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1.0, 22.627416610717773])
def test_lookup(glr, rows, vocab, d, pad, shift, wide, dt, scale):
    dt, gen = DT[dt], torch.Generator().manual_seed(rows + d)
    tokens = torch.randint(0, vocab, (rows,), generator=gen)
    tokens[::5] = -1
    tokens[1::7] = vocab
    if wide:
        tokens[2::7] = 2 ** 40
    E = Guarded(vocab, d, dt, pad, shift, value=torch.randn(vocab, d, generator=gen))
    Y = Guarded(rows, d, dt, pad, shift)
    glr.glr_embedding(E.t, tokens.to(torch.int64 if wide else torch.int32).cuda(), Y.t, scale=scale)
    want = ref.lookup(E.t.cpu(), tokens, scale)
    # the scale is an fp32 number, so the product is rounded once, or once more to bf16
    tol = 0 if scale == 1.0 else (U + HALF[dt]) * want.abs()
    _near(Y.check(), want, tol)


def test_lookup_keeps_infinities_and_nan(glr):
    E = torch.tensor([[math.inf, -math.inf, math.nan, -0.0, 1.0], [0, 0, 0, 0, 0]], device="cuda")
    Y = torch.empty(2, 5, device="cuda")
    glr.glr_embedding(E, torch.tensor([0, -1], device="cuda"), Y, scale=2.0)
    assert Y[0, 0] == math.inf and Y[0, 1] == -math.inf and Y[0, 2].isnan() and Y[0, 4] == 2 and (Y[1] == 0).all()


def _embedding_grad(glr, nodes, rows, vocab, d, dt, gd, tokens, pad=0, shift=0, scale=1.0, accumulate=False, wide=True, stream=None, seed=0):
    gen = torch.Generator().manual_seed(seed + rows + d)
    dY = Guarded(nodes * rows, d, dt, pad, shift, value=torch.randn(nodes * rows, d, generator=gen))
    dE = [Guarded(vocab, d, gd, value=torch.randn(vocab, d, generator=gen) if accumulate else None) for _ in range(nodes)]
    before = torch.stack([g.t.double().cpu() for g in dE]) if accumulate else 0
    tok = tokens.to(torch.int64 if wide else torch.int32).cuda()
    glr.glr_embedding_grad(dY.t, tok, [g.t for g in dE], scale=scale, accumulate=accumulate, stream=stream)
    got = torch.stack([g.check() for g in dE])
    want, terms, n = ref.embedding_grad(dY.t.cpu(), tokens, nodes, vocab, scale)
    # a chain of at most n additions, the scaling, the addition to what was there, the rounding
    tol = (n + 2) * U * terms + (U + HALF[gd]) * (want + before).abs()
    _near(got, want + before, tol)
    return got


@pytest.mark.parametrize("nodes,rows,vocab,d,pad,shift", [
    (1, 1, 1, 1, 0, 0), (1, 1, 1000, 64, 0, 0), (2, 3, 63, 7, 1, 1), (3, 50, 64, 256, 0, 0), (1, 100, 65, 257, 3, 1), (4, 32, 1000, 128, 0, 0),
    (2, 1000, 300, 264, 8, 8), (1, 4095, 129, 40, 0, 0), (1, 4096, 5000, 16, 0, 0), (1, 4097, 128, 24, 0, 0), (2, 9000, 20, 8, 0, 3),
])
@pytest.mark.parametrize("dt,gd", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
def test_embedding_grad(glr, nodes, rows, vocab, d, pad, shift, dt, gd):
    gen = torch.Generator().manual_seed(vocab)
    tokens = torch.randint(0, vocab, (nodes * rows,), generator=gen)
    tokens[::6] = -1
    tokens[3::11] = vocab
    _embedding_grad(glr, nodes, rows, vocab, d, DT[dt], DT[gd], tokens, pad, shift, scale=1.5, wide=rows % 2 == 0)


@pytest.mark.parametrize("kind", ["one", "few", "none", "skewed", "ends"])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("d", [48, 51, 600])
def test_embedding_grad_distributions(glr, kind, accumulate, d):
    """One token for all rows, a handful of them (all warps share a row), none, the usual skew, the vocabulary's ends."""
    nodes, rows, vocab, gen = 2, 5000, 700, torch.Generator().manual_seed(3)
    n = nodes * rows
    tokens = {"one": torch.full((n,), 333), "few": torch.randint(0, 3, (n,), generator=gen) * 320, "none": torch.full((n,), -5),
              "skewed": (torch.rand(n, generator=gen) ** 6 * vocab).long(),
              "ends": torch.where(torch.rand(n, generator=gen) < 0.5, 0, vocab - 1)}[kind]
    got = _embedding_grad(glr, nodes, rows, vocab, d, torch.bfloat16, torch.float32, tokens, accumulate=accumulate)
    again = _embedding_grad(glr, nodes, rows, vocab, d, torch.bfloat16, torch.float32, tokens, accumulate=accumulate)
    assert torch.equal(got, again)


@pytest.mark.parametrize("rows,vocab,d", [(135000, 300, 8), (40000, 70000, 16)])
def test_embedding_grad_of_many_chunks(glr, rows, vocab, d):
    """More sorted chunks than a tile's table holds, and tiles of many rows with a table of several chunks."""
    gen = torch.Generator().manual_seed(5)
    tokens = (torch.rand(rows, generator=gen) ** 3 * vocab).long()
    tokens[::1000] = -1
    _embedding_grad(glr, 1, rows, vocab, d, torch.float32, torch.float32, tokens, scale=0.25)


@pytest.mark.parametrize("nodes,rows,vocab,d,pad,shift", [
    (2, 900, 130, 264, 3, 0), (1, 5000, 700, 600, 1, 0), (2, 3000, 400, 40, 0, 1), (3, 300, 40000, 520, 5, 2), (1, 2000, 70000, 256, 1, 1),
])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dt,gd", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_embedding_grad_of_rows_off_16_bytes(glr, nodes, rows, vocab, d, pad, shift, accumulate, dt, gd):
    """Whole vectors of dE from rows of dY at any alignment; a token of hundreds of rows, and single ones."""
    gen = torch.Generator().manual_seed(d)
    tokens = (torch.rand(nodes * rows, generator=gen) ** 5 * vocab).long()
    tokens[::17] = -1
    _embedding_grad(glr, nodes, rows, vocab, d, DT[dt], DT[gd], tokens, pad, shift, scale=0.5, accumulate=accumulate)


def test_embedding_grad_of_no_rows(glr):
    dE = [torch.full((9, 16), 5.0, device="cuda") for _ in range(2)]
    args = (torch.empty(0, 16, device="cuda"), torch.empty(0, device="cuda", dtype=torch.int32), dE)
    glr.glr_embedding_grad(*args, accumulate=True)
    assert all((g == 5).all() for g in dE)
    glr.glr_embedding_grad(*args)
    assert all((g == 0).all() for g in dE)
    glr.glr_embedding(dE[0], torch.empty(0, device="cuda", dtype=torch.int64), torch.empty(0, 16, device="cuda"))


def test_embedding_gradient_is_the_lookups(glr):
    """The derivative of sum(C * lookup(E)) along a direction, by differences (the lookup is linear: exact but for rounding)."""
    gen = torch.Generator().manual_seed(1)
    vocab, d, rows = 37, 24, 90
    E, D = (torch.randn(vocab, d, generator=gen).cuda() for _ in range(2))
    C, tokens = torch.randn(rows, d, generator=gen).cuda(), torch.randint(-2, vocab + 2, (rows,), generator=gen).cuda()
    out = []
    for sign in (1, -1):
        Y = torch.empty(rows, d, device="cuda")
        glr.glr_embedding(E + sign * D, tokens, Y, scale=0.5)
        out.append(float((C.double() * Y.double()).sum()))
    dE = torch.empty(vocab, d, device="cuda")
    glr.glr_embedding_grad(C, tokens, dE, scale=0.5)
    slope = float((dE.double() * D.double()).sum())
    assert abs((out[0] - out[1]) / 2 - slope) <= 64 * U * float((C.abs().sum() * 4))


# --------------------------------------------------------------------------------------------------- 8 bits

def _edge_values(dt):
    """Blocks at the edges of the scales: largest elements of 127 2^p and its neighbours, zeros, the smallest and largest
    numbers, ties, signs."""
    f = torch.finfo(dt)
    rows = []
    for p in (-6, 0, 5):
        for m in (127, 127.5, 126.5, 64, 63.5, 127.9, 128):
            rows.append([m * 2.0 ** p, -m * 2.0 ** p / 3, 0.5 * 2.0 ** p, 1.5 * 2.0 ** p, 2.5 * 2.0 ** p, -0.5 * 2.0 ** p] + [0.3 * 2.0 ** p] * 26)
    rows.append([0.0] * 32)
    rows.append([-0.0] * 31 + [f.tiny])
    rows.append([f.smallest_normal * (q + 1) for q in range(32)])
    rows.append([f.smallest_normal / 64 * q for q in range(32)])
    rows.append([f.max, f.min] + [f.max / 2, f.max / 300] * 15)
    rows.append([2.0 ** -120 * q for q in range(32)])
    return torch.tensor(rows, dtype=torch.float64).to(dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_codes_at_the_edges(glr, dt):
    X = _edge_values(DT[dt])
    codes, scales, values = ref.pack(X)
    got, s = torch.empty(X.shape, device="cuda", dtype=torch.int8), torch.empty(X.shape[0], 1, device="cuda", dtype=torch.uint8)
    glr.glr_checkpoint_pack(X.cuda(), got, s)
    assert torch.equal(s.cpu(), scales) and torch.equal(got.cpu(), codes)
    for to in (torch.float32, torch.bfloat16):
        Y = torch.empty(X.shape, device="cuda", dtype=to)
        glr.glr_checkpoint_unpack(got, s, Y)
        assert torch.equal(Y.double().cpu(), values)
    step = 2.0 ** (scales.double() - 127)
    assert ((values - X.double()).abs() <= torch.where(X.double().abs() > 127 * 2.0 ** 121, step, step / 2)).all()


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_codes_of_what_is_not_finite(glr, bad):
    X = torch.randn(2, 70, generator=torch.Generator().manual_seed(2))
    X[0, 40] = bad
    codes, scales, values = ref.pack(X)
    got, s = torch.empty(2, 70, device="cuda", dtype=torch.int8), torch.empty(2, 3, device="cuda", dtype=torch.uint8)
    glr.glr_checkpoint_pack(X.cuda(), got, s)
    assert torch.equal(s.cpu(), scales) and torch.equal(got.cpu(), codes) and s[0, 1] == 255
    for act in ("none", "relu", "gelu", "gelu_tanh", "silu"):
        Y = torch.empty(2, 70, device="cuda")
        glr.glr_checkpoint_unpack(got, s, Y, act=act)
        assert torch.equal(Y.isnan().cpu(), values.isnan())


@pytest.mark.parametrize("rows,cols,pad,shift", [
    (1, 1, 0, 0), (2, 31, 1, 1), (3, 32, 0, 0), (5, 33, 0, 3), (7, 64, 8, 8), (4, 255, 1, 0), (3, 2048, 0, 0), (2, 2049, 0, 1), (600, 40, 0, 0),
    (2, 5000, 3, 5), (5000, 8, 0, 0), (1500, 520, 0, 0), (3, 40000, 0, 0),
])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_pack_and_unpack(glr, rows, cols, pad, shift, dt):
    dt, gen = DT[dt], torch.Generator().manual_seed(cols)
    X = Guarded(rows, cols, dt, pad, shift, value=torch.randn(rows, cols, generator=gen) * torch.exp(3 * torch.randn(rows, 1, generator=gen)))
    codes, scales = Guarded(rows, cols, torch.int8, pad, shift), Guarded(rows, (cols + 31) // 32, torch.uint8, pad, shift)
    glr.glr_checkpoint_pack(X.t, codes.t, scales.t)
    want_codes, want_scales, values = ref.pack(X.t.cpu())
    assert torch.equal(codes.check().cpu(), want_codes) and torch.equal(scales.check().cpu(), want_scales)
    Y = Guarded(rows, cols, dt, pad, shift)
    glr.glr_checkpoint_unpack(codes.t, scales.t, Y.t)
    assert torch.equal(Y.check().double().cpu(), values)
    for act in ("relu", "gelu", "gelu_tanh", "silu"):
        glr.glr_checkpoint_unpack(codes.t, scales.t, Y.t, act=act)
        # an activation within 2^-19 of max(|z|, 1): the functions' few ulps, gelu's cancellation at 1 + erf
        _near(Y.check(), ops.act(values, act), 2.0 ** -19 * values.abs().clamp(max=1) + HALF[dt] * ops.act(values, act).abs() + 1e-38)


def _checkpoint_case(nodes, rows, n, k, dt, act, pad, seed):
    gen = torch.Generator().manual_seed(seed)
    dZ = Guarded(nodes * rows, n, dt, pad, value=torch.randn(nodes * rows, n, generator=gen))
    W = Guarded(n, k, dt, pad, value=torch.randn(n, k, generator=gen) * max(1, n) ** -0.5)
    R = Guarded(nodes * rows, k, dt, pad, value=torch.randn(nodes * rows, k, generator=gen))
    codes, scales, Z = ref.pack(1.5 * torch.randn(nodes * rows, k, generator=gen))
    return dZ, W, R, codes.cuda(), scales.cuda(), Z


@pytest.mark.parametrize("nodes,rows,n,k,pad", [
    (1, 1, 1, 1, 0), (2, 3, 5, 33, 1), (1, 17, 64, 32, 0), (3, 40, 31, 100, 3), (2, 128, 96, 257, 0), (4, 64, 128, 256, 0), (1, 300, 200, 520, 8),
    (2, 1000, 264, 136, 0),
])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dt,gd", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_linear_grad_checkpoint(glr, nodes, rows, n, k, pad, act, dt, gd):
    dt, gd = DT[dt], DT[gd]
    dZ, W, R, codes, scales, Z = _checkpoint_case(nodes, rows, n, k, dt, act, pad, n + k)
    dX = Guarded(nodes * rows, k, dt, pad)
    dW, db = [Guarded(n, k, gd) for _ in range(nodes)], [Guarded(1, n, gd) for _ in range(nodes)]
    glr.glr_linear_grad_checkpoint(dZ.t, codes, scales, W=W.t, dX=dX.t, dW=[g.t for g in dW], db=[g.t[0] for g in db], act=act, residual=R.t)
    z = dZ.t.double().cpu()
    X = ops.act(Z, act)
    # X is rounded to the layer's type, which it may have been to either side; products within 2^-20 of their absolute sum in fp32
    # and, for bf16 results, 2^-12 (truncated sums); the activation's own error as in test_pack_and_unpack
    x_off = 2.0 ** -19 * (1 + Z.abs()) + HALF[dt] * X.abs()
    per = lambda t: t.view(nodes, rows, -1)  # noqa: E731
    want = per(z).transpose(1, 2) @ per(X)
    mass = per(z.abs()).transpose(1, 2) @ per(X.abs())
    chain = 2.0 ** -20 if gd == torch.float32 else 2.0 ** -12
    tol = chain * mass + per(z.abs()).transpose(1, 2) @ per(x_off) + HALF[gd] * want.abs()
    _near(torch.stack([g.check() for g in dW]), want, tol + 1e-30)
    _near(torch.stack([g.check()[0] for g in db]), per(z).sum(1), rows * U * per(z.abs()).sum(1) + HALF[gd] * per(z).sum(1).abs())
    G = z @ W.t.double().cpu() + R.t.double().cpu()
    mass = z.abs() @ W.t.double().cpu().abs() + R.t.double().cpu().abs()
    slope = ref.act_slope(Z, act)
    chain = 2.0 ** -20 if dt == torch.float32 else 2.0 ** -12
    want = G * slope
    _near(dX.check(), want, (chain * mass) * slope.abs() + 2.0 ** -18 * (1 + Z.abs()) * G.abs() + HALF[dt] * want.abs() + 1e-30)


def test_linear_grad_checkpoint_parts(glr):
    """dX alone, dW alone, dX in the residual's place: the same bits as together."""
    nodes, rows, n, k = 2, 70, 40, 96
    dZ, W, R, codes, scales, _ = _checkpoint_case(nodes, rows, n, k, torch.bfloat16, "silu", 0, 5)
    out = lambda *s: torch.empty(*s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    dX, dW, db = out(nodes * rows, k), [out(n, k) for _ in range(nodes)], [out(n) for _ in range(nodes)]
    glr.glr_linear_grad_checkpoint(dZ.t, codes, scales, W=W.t, dX=dX, dW=dW, db=db, act="silu", residual=R.t)
    dX2, dW2 = out(nodes * rows, k), [out(n, k) for _ in range(nodes)]
    glr.glr_linear_grad_checkpoint(dZ.t, codes, scales, W=W.t, dX=dX2, act="silu", residual=R.t)
    glr.glr_linear_grad_checkpoint(dZ.t, codes, scales, dW=dW2, act="silu")
    assert torch.equal(dX, dX2) and all(torch.equal(a, b) for a, b in zip(dW, dW2))
    glr.glr_linear_grad_checkpoint(dZ.t, codes, scales, W=W.t, dX=R.t, act="silu", residual=R.t)
    assert torch.equal(dX, R.check())


def test_linear_grad_checkpoint_of_no_rows(glr):
    dW, db = torch.full((5, 40), 3.0, device="cuda"), torch.full((5,), 3.0, device="cuda")
    none = lambda n, dt: torch.empty(0, n, device="cuda", dtype=dt)  # noqa: E731
    glr.glr_linear_grad_checkpoint(none(5, torch.float32), none(40, torch.int8), none(2, torch.uint8), W=torch.ones(5, 40, device="cuda"),
                                   dX=none(40, torch.float32), dW=dW, db=db, act="relu")
    assert (dW == 0).all() and (db == 0).all()


# ----------------------------------------------------------------------------------------------------- norms

NORM_SIZES = [(1, 1, 0, 0), (3, 5, 1, 1), (9, 32, 0, 0), (5, 33, 3, 5), (70, 64, 8, 8), (17, 1000, 0, 0), (8, 1024, 0, 0), (6, 1025, 1, 0),
              (4, 2048, 0, 0), (3, 2049, 7, 3), (5, 4096, 0, 0), (2, 8200, 8, 0), (3, 16384, 0, 0), (2, 16385, 0, 1), (2, 32768, 0, 0)]


@pytest.mark.parametrize("rows,n,pad,shift", NORM_SIZES + [(5000, 136, 0, 0), (1400, 4096, 0, 0), (700, 4100, 0, 0), (2000, 515, 0, 0)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("full", [True, False])
def test_norm(glr, rows, n, pad, shift, dt, full):
    dt, gen = DT[dt], torch.Generator().manual_seed(n)
    new = lambda: Guarded(rows, n, dt, pad, shift, value=torch.randn(rows, n, generator=gen) * 3)  # noqa: E731
    X, R = new(), new() if full else None
    w = (1 + 0.2 * torch.randn(n, generator=gen)).to(dt).cuda() if full else None
    H, Y = Guarded(rows, n, dt, pad, shift) if full else None, Guarded(rows, n, dt, pad, shift)
    rstd = torch.full((rows,), math.nan, device="cuda")
    codes, scales = Guarded(rows, n, torch.int8, pad, shift), Guarded(rows, (n + 31) // 32, torch.uint8, pad, shift)
    glr.glr_norm(X.t, Y.t, weight=w, residual=R.t if full else None, H=H.t if full else None, rstd=rstd, codes=codes.t, scales=scales.t, eps=1e-5)
    S, want_r, want = ref.norm(X.t.cpu(), R.t.cpu() if full else None, w.cpu() if full else None, 1e-5)
    # S: one addition, to within u (|X| + |R|) by which squares and their sum move; 40 chained additions and 10 across lanes and
    # warps for the squares, at half their effect through the root; root, quotient and two products
    mass = X.t.double().cpu().abs() + (R.t.double().cpu().abs() if full else 0)
    rel_s = U * (mass * S.abs()).sum(1) / (S * S).sum(1).clamp(min=1e-300)
    rel_r = 30 * U + rel_s
    _near(rstd, want_r, rel_r * want_r)
    off = want_r[:, None] * U * mass * (w.double().cpu().abs() if full else 1)
    near = off + (rel_r[:, None] + 4 * U) * want.abs()
    _near(Y.check(), want, near + HALF[dt] * want.abs())
    if full:
        _near(H.check(), S, U * mass + HALF[dt] * S.abs())
    # the codes stand for Y to within half a step, and a step is that of the largest element, by which it may be twice as large
    # where that element lies at 127 steps
    got = torch.empty(rows, n, device="cuda")
    glr.glr_checkpoint_unpack(codes.check(), scales.check(), got)
    step = (2.0 ** (scales.t.double().cpu() - 127)).repeat_interleave(32, 1)[:, :n]
    _near(got, want, step / 2 + near)
    _, want_scales, _ = ref.pack(want)
    differ = scales.t.cpu() != want_scales
    top = torch.nn.functional.pad(want.abs(), (0, -n % 32)).view(rows, -1, 32).amax(2)
    border = 127 * 2.0 ** (torch.minimum(scales.t.cpu(), want_scales).double() - 127)
    assert ((top - border).abs()[differ] <= 1e-5 * border[differ]).all()


def test_norm_in_place_and_without(glr):
    """H over X, Y over the residual, no Y, nothing but rstd: the same bits as into matrices of their own."""
    gen = torch.Generator().manual_seed(4)
    X, R, w = (torch.randn(*s, generator=gen).bfloat16().cuda() for s in ((37, 776), (37, 776), (776,)))
    new = lambda: torch.empty_like(X)  # noqa: E731
    H, Y, r, r2 = new(), new(), torch.empty(37, device="cuda"), torch.empty(37, device="cuda")
    c, s = torch.empty(37, 776, device="cuda", dtype=torch.int8), torch.empty(37, 25, device="cuda", dtype=torch.uint8)
    c2, s2 = torch.empty_like(c), torch.empty_like(s)
    glr.glr_norm(X, Y, weight=w, residual=R, H=H, rstd=r, codes=c, scales=s)
    glr.glr_norm(X, None, weight=w, residual=R, codes=c2, scales=s2)
    glr.glr_norm(X, None, residual=R, rstd=r2)
    assert torch.equal(c, c2) and torch.equal(s, s2) and torch.equal(r, r2)
    X2, R2 = X.clone(), R.clone()
    glr.glr_norm(X2, R2, weight=w, residual=R2, H=X2)
    assert torch.equal(X2, H) and torch.equal(R2, Y)


@pytest.mark.parametrize("big", [1e18, 3e19, 1e30, 3e38])
@pytest.mark.parametrize("n", [40, 3000])
def test_norm_beyond_the_squares_range(glr, big, n):
    X = torch.randn(3, n, generator=torch.Generator().manual_seed(1)).clamp(-3, 3) / 3 * big
    X[1] = 0
    Y, r = torch.empty(3, n, device="cuda"), torch.empty(3, device="cuda")
    glr.glr_norm(X.cuda(), Y, rstd=r, eps=1e-6)
    _, want_r, want = ref.norm(X, None, None, 1e-6)
    _near(r, want_r, 34 * U * want_r)
    _near(Y, want, 38 * U * want.abs())


def test_norm_of_what_is_not_finite(glr):
    X = torch.ones(4, 300, device="cuda")
    X[0, 7], X[1, 9] = math.nan, math.inf
    Y, r = torch.empty_like(X), torch.empty(4, device="cuda")
    c, s = torch.empty(4, 300, device="cuda", dtype=torch.int8), torch.empty(4, 10, device="cuda", dtype=torch.uint8)
    glr.glr_norm(X, Y, rstd=r, codes=c, scales=s)
    assert Y[0].isnan().all() and r[1] == 0 and Y[1, 9].isnan() and torch.isfinite(Y[2:]).all()
    assert (s[0] == 255).all() and s[1, 0] == 255 and (s[2:] != 255).all()


@pytest.mark.parametrize("rows,n,pad,shift", NORM_SIZES + [(700, 200, 0, 0), (900, 1030, 0, 0)])
@pytest.mark.parametrize("dt,gd", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("full", [True, False])
def test_norm_grad(glr, rows, n, pad, shift, dt, gd, full):
    dt, gd, nodes, gen = DT[dt], DT[gd], 2, torch.Generator().manual_seed(n + 1)
    new = lambda: Guarded(nodes * rows, n, dt, pad, shift, value=torch.randn(nodes * rows, n, generator=gen))  # noqa: E731
    dY, H, R = new(), new(), new() if full else None
    w = (1 + 0.2 * torch.randn(n, generator=gen)).to(dt).cuda() if full else None
    rstd = (1 / torch.sqrt((H.t.double() ** 2).mean(1) + 1e-5)).float()
    dX, dw = Guarded(nodes * rows, n, dt, pad, shift), [Guarded(1, n, gd) for _ in range(nodes)]
    glr.glr_norm_grad(dY.t, H.t, rstd, dX.t, weight=w, residual=R.t if full else None, dweight=[g.t[0] for g in dw])
    cpu = lambda x: None if x is None else x.cpu()  # noqa: E731
    want, want_w = ref.norm_grad(dY.t.cpu(), H.t.cpu(), rstd.cpu(), cpu(w), cpu(R.t) if full else None, nodes)
    x = H.t.double().cpu() * rstd.double().cpu()[:, None]
    g = dY.t.double().cpu() * (w.double().cpu() if full else 1)
    # the row's sum: 40 chained additions, ten across lanes and warps, three roundings a term; then five operations
    r = rstd.double().cpu()[:, None]
    tol = r * (8 * U * g.abs() + 60 * U * x.abs() * (g * x).abs().mean(1, keepdim=True)) + (U + HALF[dt]) * want.abs()
    tol = tol + (U * R.t.double().cpu().abs() if full else 0)
    _near(dX.check(), want, tol)
    mass = (dY.t.double().cpu() * x).abs().view(nodes, rows, n).sum(1)
    _near(torch.stack([v.check()[0] for v in dw]), want_w, (rows + 4) * U * mass + HALF[gd] * want_w.abs())


def test_norm_grad_in_place_and_without(glr):
    gen = torch.Generator().manual_seed(6)
    dY, H, R, w = (torch.randn(*s, generator=gen).bfloat16().cuda() for s in ((64, 520), (64, 520), (64, 520), (520,)))
    rstd = torch.rand(64, generator=gen).cuda() + 0.5
    dX, dw = torch.empty_like(dY), torch.empty(520, device="cuda")
    glr.glr_norm_grad(dY, H, rstd, dX, weight=w, residual=R, dweight=dw)
    dX2, dw2 = torch.empty_like(dY), torch.empty(520, device="cuda")
    glr.glr_norm_grad(dY, H, rstd, dX2, weight=w, residual=R)
    glr.glr_norm_grad(dY, H, rstd, None, weight=w, residual=R, dweight=dw2)
    assert torch.equal(dX, dX2) and torch.equal(dw, dw2)
    R2, dY2 = R.clone(), dY.clone()
    glr.glr_norm_grad(dY, H, rstd, R2, weight=w, residual=R2)
    glr.glr_norm_grad(dY2, H, rstd, dY2, weight=w, residual=R)
    assert torch.equal(dX, R2) and torch.equal(dX, dY2)
    none = torch.empty(0, 520, device="cuda", dtype=torch.bfloat16)
    glr.glr_norm_grad(none, none, torch.empty(0, device="cuda"), none, dweight=[dw, dw2])
    assert (dw == 0).all() and (dw2 == 0).all()


def test_norm_gradient_by_differences(glr):
    """dX and dweight against differences of sum(C * norm) in 64 bits, at H = X + residual."""
    gen = torch.Generator().manual_seed(8)
    X, R, C, D = (torch.randn(5, 77, generator=gen) for _ in range(4))
    w, dv = 1 + 0.3 * torch.randn(77, generator=gen), torch.randn(77, generator=gen)
    H, Y, r = torch.empty(5, 77, device="cuda"), torch.empty(5, 77, device="cuda"), torch.empty(5, device="cuda")
    glr.glr_norm(X.cuda(), Y, weight=w.cuda(), residual=R.cuda(), H=H, rstd=r, eps=1e-4)
    dX, dw = torch.empty(5, 77, device="cuda"), torch.empty(77, device="cuda")
    glr.glr_norm_grad(C.cuda(), H, r, dX, weight=w.cuda(), dweight=dw)

    def f(e):
        S, _, y = ref.norm(X.double() + e * D.double(), R, w.double() + e * dv.double(), 1e-4)
        return float((C.double() * y).sum())
    slope = float((dX.double().cpu() * D).sum() + (dw.double().cpu() * dv).sum())
    assert abs((f(1e-5) - f(-1e-5)) / 2e-5 - slope) < 1e-4 * abs(C).sum()


# ------------------------------------------------------------------------------------------- log-probabilities

def _run_logp(glr, z, tokens=None, tau=1.0, topk=0, ids=torch.int32, stream=None):
    rows = z.shape[0]
    new = lambda: torch.full((rows,), 55.0, device="cuda")  # noqa: E731
    logp, lse, ent = new() if tokens is not None else None, new(), new()
    top = Guarded(rows, topk, torch.float32, 3) if topk else None
    top_ids = Guarded(rows, topk, ids, 1) if topk else None
    glr.glr_token_logp(z, tokens=tokens, logp=logp, lse=lse, entropy=ent, top_logp=top.t if topk else None,
                       top_ids=top_ids.t if topk else None, temperature=tau, stream=stream)
    torch.cuda.synchronize()
    return logp, lse, ent, top.check() if topk else None, top_ids.check() if topk else None


def _logits(rows, vocab, dt, pad, shift, gen, scale=3.0):
    return Guarded(rows, vocab, dt, pad, shift, value=torch.randn(rows, vocab, generator=gen) * scale)


def _logp_tol(z, tau):
    """Absolute error of a log-probability: (z - m) / tau is rounded twice, exp2's argument once more (2^-23 |z - m| / tau and
    2^-22 of the exponential's own in every term of the sum), the sum is a chain of vocab / 256 additions and 13 joins."""
    f = z[torch.isfinite(z)].double()
    span = float((f.max() - f.min()).clamp(max=1e4)) / tau if f.numel() else 0.0
    return 2.0 ** -22 * (min(span, 104) + 4) + (z.shape[1] / 256 + 40) * U


def _check_logp(glr, z, tokens, tau, topk, ids, got=None):
    logp, lse, ent, top, top_ids = got or _run_logp(glr, z, tokens.cuda() if tokens is not None else None, tau, topk, ids)
    w_logp, w_lse, w_ent, w_top, w_ids = ref.token_logp(z.cpu(), tokens, tau, topk)
    tol = _logp_tol(z.cpu(), tau)
    some = w_lse != -math.inf
    assert torch.equal(lse.cpu() == -math.inf, ~some)
    far = z.float().cpu()
    far = torch.where(torch.isfinite(far), far, 0.0).abs().amax(1).double() / tau          # the rounding of lse, and of z - m
    def near(a, b, t):
        a, b = a.double().cpu(), b
        same = a == b
        assert torch.equal(torch.isfinite(a), torch.isfinite(b))
        assert (same | ((a - b).abs() <= t)).all(), (float((a - b)[~same].abs().max()), t)
    if logp is not None:
        near(logp, w_logp, tol + 4 * U * far + 4 * U * torch.where(torch.isfinite(w_logp), w_logp, 0.0).abs())
    near(lse, w_lse, tol + 4 * U * far)
    # the entropy's second sum has terms p (log p) of one sign: the relative error of a term times the sum of them
    near(ent, w_ent, (2 * tol + 2.0 ** -18) * (1 + w_ent))
    if topk:
        assert torch.equal(top_ids.cpu().long(), w_ids)
        near(top, w_top, tol + 4 * U * far[:, None] + 4 * U * torch.where(torch.isfinite(w_top), w_top, 0.0).abs())


LOGP_SIZES = [(1, 1, 1, 0, 0), (3, 2, 2, 1, 1), (5, 7, 3, 0, 3), (9, 8, 8, 0, 0), (6, 31, 40, 2, 0), (17, 255, 16, 0, 0), (12, 1000, 33, 3, 5),
              (7, 4099, 64, 8, 0), (5, 16384, 256, 0, 0), (4, 20000, 257, 1, 0), (3, 32771, 1024, 0, 1), (2, 65536, 128, 0, 0), (2, 131071, 100, 1, 0),
              (1, 262144, 5, 0, 0)]


@pytest.mark.parametrize("rows,vocab,topk,pad,shift", LOGP_SIZES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("tau", [1.0, 0.6])
def test_token_logp(glr, rows, vocab, topk, pad, shift, dt, tau):
    gen = torch.Generator().manual_seed(vocab)
    z = _logits(rows, vocab, DT[dt], pad, shift, gen)
    tokens = torch.randint(0, vocab, (rows,), generator=gen)
    tokens[::4], tokens[2::5] = -1, vocab
    wide = rows % 2 == 1
    _check_logp(glr, z.t, tokens.to(torch.int64 if wide else torch.int32), tau, topk, torch.int64 if wide else torch.int32)
    z.check()


@pytest.mark.parametrize("rows,vocab,topk", [(330, 20000, 48), (900, 9001, 200), (2000, 1500, 90), (400, 40000, 300), (500, 3000, 128)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_token_logp_of_many_rows(glr, rows, vocab, topk, dt):
    """A CTA a row: alternatives as a stable sort orders them, log-probabilities as log_softmax in 64 bits."""
    gen = torch.Generator().manual_seed(rows)
    z = _logits(rows, vocab, DT[dt], 0, 0, gen, 2.0).t
    z[:, ::97] = -math.inf
    tokens = torch.randint(0, vocab, (rows,), generator=gen)
    tokens[tokens % 97 == 0] += 1
    logp, lse, ent, top, ids = _run_logp(glr, z, tokens.cuda(), 0.9, topk)
    lp = torch.log_softmax(z.double() / 0.9, 1).cpu()
    tol = _logp_tol(z.cpu(), 0.9) + 4 * U * 40
    order = torch.sort(z.cpu(), dim=1, descending=True, stable=True).indices[:, :topk]
    assert torch.equal(ids.cpu().long(), order)
    _near(top, lp.gather(1, order), tol)
    _near(logp, lp.gather(1, tokens.clamp(max=vocab - 1)[:, None])[:, 0], tol)
    _near(lse, torch.logsumexp(z.double().cpu() / 0.9, 1), tol)
    w_ent = -torch.where(lp > -math.inf, lp.exp() * torch.where(lp > -math.inf, lp, 0.0), 0.0).sum(1)
    _near(ent, w_ent, (2 * tol + 2.0 ** -18) * (1 + w_ent))
    again = _run_logp(glr, z, tokens.cuda(), 0.9, topk)
    assert all(torch.equal(a, b) for a, b in zip((logp, lse, ent, top, ids), again))


@pytest.mark.parametrize("vocab", [50, 5000, 70000])
@pytest.mark.parametrize("kind", ["equal", "two", "ascending", "descending", "strided", "steps", "zeros"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_alternatives_in_awkward_orders(glr, vocab, kind, dt):
    """Equal logits go by their index; orders in which every element is larger than all before it; large ones far apart."""
    v = torch.arange(vocab, dtype=torch.float64)
    z = {"equal": torch.zeros(vocab) + 2.5, "two": (v % 3 == 1) * 1.0, "ascending": v / vocab * 20 - 10, "descending": 10 - v / vocab * 20,
         "strided": torch.where(v % 2048 < 8, 5 + v / vocab, -v / vocab), "steps": torch.floor(v / 700) % 5,
         "zeros": torch.where(v % 2 == 0, 0.0, -0.0)}[kind].to(DT[dt]).cuda()
    rows = torch.stack([z, z.flip(0)])
    for topk in (1, 3, 64, 300):
        _check_logp(glr, rows, torch.tensor([0, vocab - 1]), 1.0, topk, torch.int32)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [37, 3001, 40000])
def test_ruled_out_entries(glr, dt, vocab):
    """Rows with -infinity in places, everywhere, everywhere but one or few entries; the type's lowest value as a mask."""
    dt, gen = DT[dt], torch.Generator().manual_seed(9)
    z = torch.randn(7, vocab, generator=gen).to(dt)
    z[0, :vocab // 2] = -math.inf
    z[1] = -math.inf
    z[2] = -math.inf
    z[2, vocab - 2] = -1.0
    z[3, :-5] = -math.inf
    z[4] = torch.finfo(dt).min
    z[5, ::2] = torch.finfo(dt).min
    z[6, 5:] = torch.finfo(dt).min
    tokens = torch.tensor([0, 3, vocab - 2, vocab - 1, 5, 1, 7])
    got = _run_logp(glr, z.cuda(), tokens.cuda(), 1.0, 20)
    w_logp, w_lse, w_ent, w_top, w_ids = ref.token_logp(z, tokens, 1.0, 20)
    assert torch.equal(got[4].cpu().long(), w_ids)
    for a, b in zip(got[:4], (w_logp, w_lse, w_ent, w_top)):
        a = a.double().cpu()
        assert torch.equal(a == -math.inf, b == -math.inf)
        ok = b != -math.inf
        assert ((a - b).abs()[ok] <= 2.0 ** -16 * (1 + b[ok].abs())).all()
    assert got[0][0] == -math.inf and got[0][1] == 0 and got[1][1] == -math.inf and got[2][1] == 0 and (got[4][1] == -1).all()
    assert abs(float(got[2][2])) < 1e-6 and abs(float(got[0][2])) < 1e-6


def test_logits_that_are_not_finite(glr):
    z = torch.randn(3, 500, device="cuda")
    z[0, 17], z[1, 30] = math.nan, math.inf
    logp, lse, ent, top, ids = _run_logp(glr, z, torch.tensor([1, 2, 3], device="cuda"), 1.0, 4)
    for x in (logp, lse, ent):
        assert x[0].isnan() and x[1].isnan() and torch.isfinite(x[2])
    assert ids[0, 0] == 17 and ids[1, 0] == 30 and top[:2].isnan().all()


@pytest.mark.parametrize("shift", [0.0, 1e4, -1e6, 1e30])
@pytest.mark.parametrize("tau", [1.0, 1e-3, 1e3])
def test_logits_far_from_zero(glr, shift, tau):
    """Log-probabilities come from differences to the maximum."""
    z = (torch.randn(4, 3000, generator=torch.Generator().manual_seed(1)) * 2 + shift).float()
    _check_logp(glr, z.cuda(), torch.tensor([1, 2, 3, 4]), tau, 9, torch.int64)


def test_outputs_may_be_left_out(glr):
    z, t = torch.randn(6, 777, device="cuda").bfloat16(), torch.arange(6, device="cuda")
    logp, lse, ent, top, ids = _run_logp(glr, z, t, 1.3, 11)
    one, two, three = torch.empty(6, device="cuda"), torch.empty(6, 11, device="cuda"), torch.empty(6, 11, device="cuda", dtype=torch.int32)
    glr.glr_token_logp(z, tokens=t, logp=one, temperature=1.3)
    assert torch.equal(one, logp)
    glr.glr_token_logp(z, entropy=one, temperature=1.3)
    assert torch.equal(one, ent)
    glr.glr_token_logp(z, top_logp=two, temperature=1.3)
    glr.glr_token_logp(z, top_ids=three, temperature=1.3)
    assert torch.equal(two, top) and torch.equal(three, ids)


@pytest.mark.parametrize("rows,vocab,pad,shift", [s[:2] + s[3:] for s in LOGP_SIZES])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("which", ["both", "logp", "entropy"])
def test_token_logp_grad(glr, rows, vocab, pad, shift, dt, which):
    dt, tau, gen = DT[dt], 0.8, torch.Generator().manual_seed(vocab + 1)
    z = _logits(rows, vocab, dt, pad, shift, gen, 2.0)
    if vocab > 10:
        z.t[:, 3:7] = -math.inf
    tokens = torch.randint(0, vocab, (rows,), generator=gen)
    tokens[1::4] = -7
    a = torch.randn(rows, generator=gen) if which != "entropy" else None
    b = torch.randn(rows, generator=gen) if which != "logp" else None
    _, lse, ent, _, _ = _run_logp(glr, z.t, tau=tau)
    d = Guarded(rows, vocab, dt, pad, (shift + 1) % 4 if rows % 2 else shift)
    gpu = lambda x: None if x is None else x.cuda()  # noqa: E731
    glr.glr_token_logp_grad(z.t, lse, d.t, tokens=gpu(tokens) if a is not None else None, dlogp=gpu(a), entropy=ent if b is not None else None,
                            dentropy=gpu(b), temperature=tau)
    leaf = z.t.double().cpu().requires_grad_(True)
    lp = torch.log_softmax(leaf / tau, 1)
    ok = (tokens >= 0) & (tokens < vocab)
    loss = 0
    if a is not None:
        loss = loss + (a.double() * torch.where(ok, lp.gather(1, tokens.clamp(0, vocab - 1)[:, None])[:, 0], 0.0)).sum()
    if b is not None:
        fin = torch.isfinite(z.t.cpu())
        lps = torch.where(fin, lp, 0.0)
        loss = loss - (b.double()[:, None] * torch.where(fin, lps.exp() * lps, 0.0)).sum()
    (want,) = torch.autograd.grad(loss, leaf)
    want = torch.nan_to_num(want, nan=0.0)
    p = torch.softmax(z.t.double().cpu() / tau, 1)
    lpa = torch.where(p > 0, lp.detach(), 0.0).abs()
    # log p is off by tol and the rounding of lse (|lse| u) and of z / tau, p by as much of its value; exp2 by 2^-22
    tol_lp = _logp_tol(z.t.cpu(), tau) + 4 * U * (lse.double().cpu().abs()[:, None] + lpa)
    A = 0 if a is None else a.double().abs()[:, None]
    B = 0 if b is None else b.double().abs()[:, None]
    H = ent.double().cpu()[:, None]
    tol = (A * p * (tol_lp + 2.0 ** -21) + B * p * ((tol_lp + 2.0 ** -21) * (lpa + H + 1) + 2.0 ** -17 * (1 + H)) + 2 * U * A) / tau + HALF[dt] * want.abs()
    _near(d.check(), want, tol + 1e-37)
    # in place of the logits: the same bits
    glr.glr_token_logp_grad(z.t, lse, z.t, tokens=gpu(tokens) if a is not None else None, dlogp=gpu(a), entropy=ent if b is not None else None,
                            dentropy=gpu(b), temperature=tau)
    assert torch.equal(z.check(), d.t)


def test_rows_without_a_gradient(glr):
    """A row without a distribution, and one with neither term, is zero whatever its logits hold."""
    z = torch.randn(4, 300, device="cuda")
    z[0] = -math.inf
    z[1] = math.nan
    _, lse, ent, _, _ = _run_logp(glr, z)
    d = torch.full_like(z, 9.0)
    glr.glr_token_logp_grad(z, lse, d, tokens=torch.tensor([5, 400, 6, -1], device="cuda"), dlogp=torch.ones(4, device="cuda"), entropy=ent,
                            dentropy=torch.tensor([1.0, 0.0, 1.0, 0.0], device="cuda"))
    assert (d[0] == 0).all() and (d[1] == 0).all() and (d[3] == 0).all() and torch.isfinite(d[2]).all() and (d[2] != 0).any()


def test_alternatives_are_a_teachers(glr):
    """top_logp and top_ids as glr_distill_loss takes a teacher: its own distribution restricted to them is the nearest there is."""
    gen = torch.Generator().manual_seed(3)
    z = torch.randn(20, 900, generator=gen)
    z[3, 5:] = -math.inf                              # five entries left of 32
    z = z.cuda()
    top, ids = torch.empty(20, 32, device="cuda"), torch.empty(20, 32, device="cuda", dtype=torch.int32)
    glr.glr_token_logp(z, top_logp=top, top_ids=ids)
    loss, row, d = torch.empty(1, device="cuda"), torch.empty(20, device="cuda"), torch.empty_like(z)
    glr.glr_distill_loss(z, top, ids, loss=loss, row_loss=row, dlogits=d)
    # KL(q || p) with q = p / P on the alternatives is -log P
    want = -torch.log(top.double().exp().sum(1)).cpu()
    assert ((row.double().cpu() - want).abs() < 1e-5).all() and abs(float(row[3])) < 1e-5


# ------------------------------------------------------------------------------------------- streams and graphs

def _everything(glr, dt):
    """Inputs, outputs and a function that calls every row operator once."""
    gen = torch.Generator().manual_seed(12)
    nodes, rows, d, vocab = 2, 40, 136, 500
    r = lambda *s: torch.randn(*s, generator=gen).to(dt).cuda()  # noqa: E731
    new = lambda *s, dtype=dt: torch.zeros(*s, device="cuda", dtype=dtype)  # noqa: E731
    f32 = lambda *s: new(*s, dtype=torch.float32)  # noqa: E731
    t = nodes * rows
    i = dict(E=r(vocab, d), tokens=torch.randint(-1, vocab, (t,), generator=gen).cuda(), R=r(t, d), w=r(d), W=r(64, d), dZ=r(t, 64), z=r(t, vocab),
             a=r(t).float(), b=r(t).float())
    o = dict(Y=new(t, d), H=new(t, d), N=new(t, d), rstd=f32(t), codes=new(t, d, dtype=torch.int8), scales=new(t, 5, dtype=torch.uint8),
             V=new(t, d), dX=new(t, d), dW=[new(64, d) for _ in range(nodes)], db=[new(64) for _ in range(nodes)], dH=new(t, d),
             dw=[f32(d) for _ in range(nodes)], dE=[new(vocab, d) for _ in range(nodes)], logp=f32(t), lse=f32(t), ent=f32(t), top=f32(t, 7),
             ids=new(t, 7, dtype=torch.int32), dz=new(t, vocab))

    def run(stream=None):
        glr.glr_embedding(i["E"], i["tokens"], o["Y"], scale=2.0, stream=stream)
        glr.glr_norm(o["Y"], o["N"], weight=i["w"], residual=i["R"], H=o["H"], rstd=o["rstd"], codes=o["codes"], scales=o["scales"], stream=stream)
        glr.glr_checkpoint_unpack(o["codes"], o["scales"], o["V"], act="silu", stream=stream)
        glr.glr_linear_grad_checkpoint(i["dZ"], o["codes"], o["scales"], W=i["W"], dX=o["dX"], dW=o["dW"], db=o["db"], act="silu", stream=stream)
        glr.glr_norm_grad(o["dX"], o["H"], o["rstd"], o["dH"], weight=i["w"], dweight=o["dw"], stream=stream)
        glr.glr_embedding_grad(o["dH"], i["tokens"], o["dE"], scale=2.0, stream=stream)
        glr.glr_token_logp(i["z"], tokens=i["tokens"], logp=o["logp"], lse=o["lse"], entropy=o["ent"], top_logp=o["top"], top_ids=o["ids"], stream=stream)
        glr.glr_token_logp_grad(i["z"], o["lse"], o["dz"], tokens=i["tokens"], dlogp=i["a"], entropy=o["ent"], dentropy=i["b"], stream=stream)

    flat = lambda: [x for v in o.values() for x in (v if isinstance(v, list) else [v])]  # noqa: E731
    return i, flat, run


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_other_streams_and_graphs(glr, dt):
    """Another stream, and a graph that is captured and replayed on new inputs, give the bits of the plain calls."""
    i, flat, run = _everything(glr, DT[dt])
    run()
    want = [x.clone() for x in flat()]

    def clear():
        for x in flat():
            x.zero_()
        torch.cuda.synchronize()

    clear()
    side = torch.cuda.Stream()
    run(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, flat()))
    clear()
    with torch.cuda.stream(side):
        run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, flat()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    # another graph of the same calls: each has workspaces of its own
    other = torch.cuda.CUDAGraph()
    with torch.cuda.graph(other):
        run()
    for k in range(3):
        clear()
        (graph if k != 1 else other).replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, flat()))
    i["tokens"].add_(1)
    i["z"].mul_(0.5)
    run()
    torch.cuda.synchronize()
    want = [x.clone() for x in flat()]
    clear()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, flat()))


def test_two_calls_at_once(glr):
    """Calls on two streams that overlap share nothing."""
    sets = [_everything(glr, torch.bfloat16) for _ in range(2)]
    for _, _, run in sets:
        run()
    torch.cuda.synchronize()
    want = [[x.clone() for x in flat()] for _, flat, _ in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(10):
        for (_, _, run), s in zip(sets, streams):
            run(s)
    torch.cuda.synchronize()
    for (_, flat, _), w in zip(sets, want):
        assert all(torch.equal(a, b) for a, b in zip(w, flat()))


@pytest.mark.parametrize("name", ["lookup", "grad", "pack", "norm", "logp"])
def test_matrices_past_32_bits_of_elements(glr, name):
    """Rows far beyond 2^31 elements into their buffers."""
    cols, rows = 1 << 20, 2100
    if torch.cuda.mem_get_info()[0] < 3 * 2 * rows * cols:
        pytest.skip("not enough memory")
    big = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16)
    far = torch.tensor([0, 2047, 2049, 2099], device="cuda")
    fill = torch.randn(4, cols, device="cuda").bfloat16()
    big[far] = fill
    if name == "lookup":
        out = torch.empty(4, cols, device="cuda", dtype=torch.bfloat16)
        glr.glr_embedding(big, far, out)
        assert torch.equal(out, fill)
    elif name == "grad":
        tokens = torch.full((rows,), -1, device="cuda")
        tokens[far] = torch.tensor([0, 1, 2, 1], device="cuda")
        out = torch.empty(3, cols, device="cuda", dtype=torch.float32)
        glr.glr_embedding_grad(big, tokens, out)
        assert torch.equal(out, torch.stack([fill[0].float(), fill[1].float() + fill[3].float(), fill[2].float()]))
    elif name == "pack":
        codes, scales = torch.empty(rows, cols, device="cuda", dtype=torch.int8), torch.empty(rows, cols // 32, device="cuda", dtype=torch.uint8)
        big[:] = 0
        big[far] = fill
        glr.glr_checkpoint_pack(big, codes, scales)
        c4, s4 = torch.empty(4, cols, device="cuda", dtype=torch.int8), torch.empty(4, cols // 32, device="cuda", dtype=torch.uint8)
        glr.glr_checkpoint_pack(fill, c4, s4)
        assert torch.equal(codes[far], c4) and torch.equal(scales[far], s4)
        glr.glr_checkpoint_unpack(codes, scales, big)
        out = torch.empty_like(fill)
        glr.glr_checkpoint_unpack(c4, s4, out)
        assert torch.equal(big[far], out)
    elif name == "norm":
        wide = big.view(rows * 64, cols // 64)
        small = wide[far * 64 + 1].clone()
        wide[torch.isnan(wide.float()).any(1)] = 0
        wide[far * 64 + 1] = small
        y, y4 = torch.empty_like(wide), torch.empty_like(small)
        glr.glr_norm(wide, y)
        glr.glr_norm(small, y4)
        assert torch.equal(y[far * 64 + 1], y4)
    else:
        wide = big.view(rows * 2, cols // 2)
        wide[:] = 0
        wide[far * 2 + 1] = fill[:, :cols // 2]
        got, small = torch.empty(rows * 2, 9, device="cuda", dtype=torch.int32), torch.empty(4, 9, device="cuda", dtype=torch.int32)
        glr.glr_token_logp(wide, top_ids=got)
        glr.glr_token_logp(fill[:, :cols // 2].contiguous(), top_ids=small)
        assert torch.equal(got[far * 2 + 1], small)
        assert (got[0].cpu() == torch.arange(9)).all()
