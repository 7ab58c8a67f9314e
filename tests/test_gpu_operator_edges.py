"""The operators around the step at the edges of what they promise: kernels that read what the one before them wrote,
the ends of the floating-point range, terms without a coefficient (marked gpu)."""
import math

import pytest
import torch

import _operators as ref
from test_gpu_losses import _check_grad, _close, _dprob, _run_distill, _run_policy, _run_preference

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 4, 8, 24, 2048])
def test_kernels_read_what_the_one_before_wrote(rows, dt):
    """Two layers and the second one's gradients back to back, each reading the buffers that the call before has just
    written, which change from repetition to repetition: the same bits as with a pause after every call."""
    import paper_2507_08784_gb300 as glr
    dt, d, h, o = DT[dt], 512, 1024, 264
    gen = torch.Generator().manual_seed(rows)
    W1, W2 = (torch.randn(*s, generator=gen).to(dt).cuda() for s in ((h, d), (o, h)))
    xs = [torch.randn(rows, d, generator=gen).to(dt).cuda() for _ in range(12)]
    hid, out = torch.empty(rows, h, device="cuda", dtype=dt), torch.empty(rows, o, device="cuda", dtype=dt)

    def run(pause):
        hid.zero_(), out.zero_()
        torch.cuda.synchronize()
        results = []
        for x in xs:
            dW, db = torch.empty(o, h, device="cuda", dtype=dt), torch.empty(o, device="cuda", dtype=dt)
            for call in (lambda: glr.glr_linear(x, W1, hid, act="silu"), lambda: glr.glr_linear(hid, W2, out),
                         lambda: glr.glr_linear_grad_weight(out, hid, dW, db=db)):
                call()
                if pause:
                    torch.cuda.synchronize()
            results.append((out.clone(), dW, db) if pause else (dW, db))
        torch.cuda.synchronize()
        return results

    for (want_out, want_dw, want_db), (dw, db) in zip(run(True), run(False)):
        assert torch.equal(dw, want_dw) and torch.equal(db, want_db) and want_out.any()


# ---------------------------------------------------------------------------------------- preference, far from zero

@pytest.mark.parametrize("vocab", [777, 32769])
@pytest.mark.parametrize("offset", [0.0, 1e4, 1e6])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_preference_gradient_of_logits_far_from_zero(vocab, offset, dt):
    """Logits with a common offset, and rows that hold the type's lowest value throughout or but for one entry:
    everything is a function of z - max z, so the tolerances are those of the logits' span, as for the other losses."""
    dt = DT[dt]
    gen = torch.Generator().manual_seed(41)
    lengths = [4, 7, 1, 5]
    rows = sum(lengths)
    z = (3 * torch.randn(rows, vocab, generator=gen) + offset).to(dt)
    span = max(float(x.max() - x.min()) for x in z.float())
    z[2] = z[13] = torch.finfo(dt).min
    z[6] = torch.finfo(dt).min
    z[6, 5] = offset
    tokens = torch.randint(0, vocab, (rows,), generator=gen)
    tokens[6] = 5
    offsets = torch.tensor([0] + lengths).cumsum(0)
    want = ref.preference(z, tokens, offsets, None, None, "sigmoid", 0.1, 0.1, False)
    loss, pair, seq, row, d = _run_preference(z.cuda(), tokens.cuda(), offsets.cuda(), None, None, "sigmoid", 0.1, 0.1)
    rel = 2.0 ** -19 + 2.0 ** -22 * span
    _close(row, want[3], 4 * rel)
    _close(seq, want[2], 4 * rel)
    grad_rel = rel + 0.1 * 4 * rel * (2 + 2 * float(want[2].abs().max()))
    biggest = want[4].abs().max(1, keepdim=True).values
    _check_grad(d, want[4], grad_rel, dt, biggest * (_dprob(z) + (want[4].abs() == biggest)))


# ------------------------------------------------------------------------------- terms without a coefficient: preference

@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_preference_of_a_ruled_out_answer(dt):
    """A rejected answer with a token of logit -infinity is infinitely far behind: -log sigmoid(infinity) = 0 without
    smoothing, and its mirror image with the smoothing at 1.  With both terms the loss is infinite."""
    dt = DT[dt]
    gen = torch.Generator().manual_seed(42)
    tokens, offsets = torch.randint(0, 300, (16,), generator=gen), torch.tensor([0, 4, 8, 12, 16])
    for smoothing, answer in ((0.0, 1), (1.0, 0), (0.1, 1)):
        z = torch.randn(16, 300, generator=gen).to(dt)
        banned = 4 * answer + 2
        z[banned, tokens[banned]] = -math.inf
        other = ref.preference(z[8:], tokens[8:], torch.tensor([0, 4, 8]), None, None, "sigmoid", 0.1, smoothing, False)
        loss, pair, _, _, d = _run_preference(z.cuda(), tokens.cuda(), offsets.cuda(), None, None, "sigmoid", 0.1, smoothing)
        if smoothing == 0.1:
            assert float(pair[0]) == math.inf and float(loss) == math.inf
            continue
        assert float(pair[0]) == 0.0 and not d[:8].any()
        _close(pair[1:], other[1], 2.0 ** -15)
        _close(loss, other[0] / 2, 2.0 ** -15)
        _check_grad(d[8:], other[4] / 2, 2.0 ** -16, dt, other[4].abs() + 1e-2)


# ----------------------------------------------------------------------------- terms without a coefficient: distillation

@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("topk", [3, 100])
def test_distillation_without_the_soft_term(dt, topk):
    """soft = 0 and a teacher's entry that the student rules out (their divergence is infinite): the hard term alone."""
    dt = DT[dt]
    gen = torch.Generator().manual_seed(43)
    z = torch.randn(5, 500, generator=gen).to(dt)
    ids, teacher = torch.randint(0, 250, (5, topk), generator=gen), torch.randn(5, topk, generator=gen)
    labels = torch.randint(250, 500, (5,), generator=gen)
    z[torch.arange(5), ids[:, 1]] = -math.inf
    for tau in (1.0, 2.0, 3.0):
        lp = torch.log_softmax(z.double(), 1)
        want = -0.5 * lp.gather(1, labels[:, None])[:, 0]
        grad = 0.1 * lp.exp()
        grad[torch.arange(5), labels] -= 0.1
        loss, row, d = _run_distill(z.cuda(), teacher.cuda(), ids.cuda(), labels.cuda(), None, tau, 0.0, 0.5)
        _close(row, want, 2.0 ** -16)
        _close(loss, want.mean(), 2.0 ** -16)
        _check_grad(d, grad, 2.0 ** -16, dt, grad.abs())
        assert float(_run_distill(z.cuda(), teacher.cuda(), ids.cuda(), labels.cuda(), None, tau, 1.0, 0.5)[1].min()) == math.inf


# ----------------------------------------------------------------------------------- terms without a coefficient: policy

@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_policy_terms_without_a_coefficient(dt):
    """kl = 0 where exp(ref - logp) leaves the range, and an advantage of 0 where the ratio does: nothing of either."""
    dt = DT[dt]
    gen = torch.Generator().manual_seed(44)
    z = torch.randn(6, 400, generator=gen).to(dt)
    tokens, adv = torch.randint(0, 400, (6,), generator=gen).cuda(), torch.randn(6, generator=gen)
    z[1, tokens[1]] = -160.0
    z[2, tokens[2]] = -math.inf
    old, refl = torch.full((6,), -5.0), torch.full((6,), -1.0)
    a = _run_policy(z.cuda(), tokens, old.cuda(), adv.cuda(), None, None)
    b = _run_policy(z.cuda(), tokens, old.cuda(), adv.cuda(), refl.cuda(), None, kl=0.0)
    assert all(torch.isfinite(x).all() for x in (a[0], a[1], a[3]))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    adv[3], adv[4], old[3:5] = 0.0, 1.5, -120.0
    loss, row, _, d = _run_policy(z.cuda(), tokens, old.cuda(), adv.cuda(), None, None, high=0.28)
    assert float(row[3]) == 0.0 and not d[3:5].any()
    assert abs(float(row[4]) + 1.28 * 1.5) < 1e-6 and torch.isfinite(loss).all()


# --------------------------------------------------------------------------------------------- confident predictions

@pytest.mark.parametrize("kind", ["policy", "distill"])
def test_losses_of_confident_tokens(kind):
    """Two fp32 logits d apart, -log p = log1p(exp(-d)): the sum 1 + exp(-d) is rounded once (2^-24) and its logarithm
    correct to a unit in its last place or two."""
    gap = torch.linspace(8.0, 16.0, 4096)
    z = torch.stack([gap, torch.zeros_like(gap)], 1).contiguous()
    want = torch.log1p(torch.exp(-gap.double()))
    first, rows = torch.zeros(4096, dtype=torch.int64, device="cuda"), 4096
    if kind == "policy":
        zero = torch.zeros(rows, device="cuda")
        got = -_run_policy(z.cuda(), first, zero, zero + 1, grad=False)[2]
    else:
        got = _run_distill(z.cuda(), torch.empty(rows, 0, device="cuda"), torch.empty(rows, 0, device="cuda", dtype=torch.int32), first, None,
                           1.0, 0.0, 1.0, grad=False)[1]
    assert ((got.double().cpu() - want).abs() <= 1.05 * 2.0 ** -24 + 2.0 ** -22 * want).all(), float((got.double().cpu() - want).abs().max())


# ------------------------------------------------------------------------------------ ends of the range: activations

# few rows; a shared contraction (bf16) or the small products (fp32); whole tiles one after the other; the same laid out first
PATHS = [(3, 64, 64, 0), (70, 72, 64, 0), (70, 72, 64, 1), (4096, 2048, 256, 0), (4096, 2048, 256, 1)]


def _ends(n, dt):
    m = torch.finfo(dt).max
    v = torch.tensor([0.0, 100.0, 1e4, 3e18, 3e19, 1e30, 1e36, m], dtype=torch.float64)
    return torch.cat([v, -v]).to(dt).repeat(-(-n // 16))[:n]


def _check_ends(rows, n, k, pad, act, dt):
    import paper_2507_08784_gb300 as glr
    dt = DT[dt]
    z = _ends(n, dt)
    X, W = torch.zeros(rows, k + pad, device="cuda", dtype=dt)[:, :k], torch.randn(n, k + pad, device="cuda").to(dt)[:, :k]
    Y, P = torch.empty(rows, n + pad, device="cuda", dtype=dt)[:, :n], torch.empty(rows, n, device="cuda", dtype=dt)
    glr.glr_linear(X, W, Y, bias=z.cuda(), act=act, preact=P)
    zd = z.double()
    want = zd if act == "none" else zd.clamp(min=0)
    assert torch.equal(P.cpu(), z.expand(rows, n))
    tol = want.abs() * 2.0 ** -20 + 1e-30
    assert ((Y.double().cpu() - want).abs() <= tol).all(), (Y[0], want)

    z = _ends(k, dt)
    D, G = torch.zeros(rows, n + pad, device="cuda", dtype=dt)[:, :n], torch.ones(rows, k, device="cuda", dtype=dt)
    dX = torch.empty(rows, k + pad, device="cuda", dtype=dt)[:, :k]
    glr.glr_linear_grad_input(D, W, dX, residual=G, preact=z.cuda().expand(rows, k).contiguous(), act=act)
    slope = (z.double() > 0).double() if act != "none" else torch.ones(k, dtype=torch.float64)
    if act in ("gelu", "gelu_tanh", "silu"):
        slope[z == 0] = 0.5
    assert ((dX.double().cpu() - slope).abs() <= 2.0 ** -20).all(), (dX[0], slope)
    glr.glr_operator_status()


@pytest.mark.parametrize("rows,n,k,pad", PATHS)
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_activations_at_the_ends_of_the_range(rows, n, k, pad, act, dt):
    """Pre-activations from 100 to the type's largest, of either sign: an activation is there 0 or the value itself, its
    slope 0 or 1."""
    _check_ends(rows, n, k, pad, act, dt)


# --------------------------------------------------------------------------------------------- ends of the range: gelu_tanh

@pytest.mark.parametrize("rows,n,k,pad", PATHS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_gelu_tanh_at_the_ends_of_the_range(rows, n, k, pad, dt):
    _check_ends(rows, n, k, pad, "gelu_tanh", dt)


# ----------------------------------------------------------------------------------------- ends of the range: fp32 products

# rows, outputs and inputs of the three ways of an fp32 product: few rows, small, laid out (a shared contraction, whole tiles)
FP32_PATHS = [(8, 200, 100), (130, 70, 90), (300, 1200, 1500), (2048, 2048, 512)]


def _same_or_close(got, want, tol):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], want[inf])
    fin = torch.isfinite(want)
    assert ((got - want).abs()[fin] <= tol[fin]).all(), float(((got - want).abs() / tol)[fin].max())


@pytest.mark.parametrize("rows,n,k", FP32_PATHS)
def test_extremes_in_fp32_products(rows, n, k):
    """The type's largest values, of either sign, in single places of X and of W, against factors below 0.4."""
    import paper_2507_08784_gb300 as glr
    gen = torch.Generator().manual_seed(rows)
    X, W = 0.4 * torch.rand(rows, k, generator=gen), 0.4 * torch.rand(n, k, generator=gen)
    big = torch.finfo(torch.float32).max
    X[1], W[7] = 0.0, 0.0
    X[1, 3], X[2, 5], W[6, 11], W[7, 20] = big, -big, -big, big
    want = X.double() @ W.double().T
    tol = 2.0 ** -19 * (X.double().abs() @ W.double().abs().T) + 1e-30
    Y, dX, dW = (torch.empty(rows, n, device="cuda") for _ in range(3))
    glr.glr_linear(X.cuda(), W.cuda(), Y)
    glr.glr_linear_grad_input(X.cuda(), W.T.contiguous().cuda(), dX)
    glr.glr_linear_grad_weight(X.T.contiguous().cuda(), W.T.contiguous().cuda(), dW)
    for got in (Y, dX, dW):
        _same_or_close(got, want, tol)
    glr.glr_operator_status()


# ----------------------------------------------------------------------------------------- infinities in fp32 products

@pytest.mark.parametrize("rows,n,k", FP32_PATHS)
def test_infinities_in_fp32_products(rows, n, k):
    """The type's largest values, infinities of either sign in X and in W, one against a zero and two against each other:
    every result is what the definition gives, and its finite ones as close as always."""
    import paper_2507_08784_gb300 as glr
    gen = torch.Generator().manual_seed(rows)
    X, W = torch.randn(rows, k, generator=gen), 3000 * torch.randn(n, k, generator=gen)
    big = torch.finfo(torch.float32).max
    X[1], X[2] = 0.0, 0.0
    X[1, 3], X[2, 5], X[3, 7], X[4, k - 1], X[5, 11], X[6, 2] = big, -big, math.inf, -math.inf, math.inf, math.nan
    W[:, 3], W[:, 5] = 0.4 * torch.rand(n, generator=gen), -0.4 * torch.rand(n, generator=gen)
    X[3, 9] = math.inf                                      # with W's column 9 of either sign: infinite or not a number
    W[4, 11] = 0.0
    W[5, 13], W[6, 11] = math.inf, -math.inf
    W[7] = 0.0
    W[7, 20] = big
    X[:, 20] = 0.3 * torch.rand(rows, generator=gen)
    a, b = X.double(), W.double()
    want = a @ b.T
    size = torch.where(torch.isfinite(a), a, 0).abs() @ torch.where(torch.isfinite(b), b, 0).abs().T
    want = torch.where(want.abs() > big, want.sign() * math.inf, want)
    tol = 2.0 ** -19 * size + 1e-30
    Y, R = (torch.empty(rows, n, device="cuda") for _ in range(2))
    glr.glr_linear(X.cuda(), W.cuda(), Y)
    glr.glr_linear(X.cuda(), W.cuda(), R, act="relu")
    _same_or_close(Y, want, tol)
    _same_or_close(R, torch.where(want <= 0, 0.0, want), tol)
    # the same products as gradients: dZ W with dZ = X and W's transpose, and dZ^T X
    dX, dW = torch.empty(rows, n, device="cuda"), torch.empty(rows, n, device="cuda")
    glr.glr_linear_grad_input(X.cuda(), W.T.contiguous().cuda(), dX)
    _same_or_close(dX, want, tol)
    glr.glr_linear_grad_weight(X.T.contiguous().cuda(), W.T.contiguous().cuda(), dW)
    _same_or_close(dW, want, tol)
    glr.glr_operator_status()


# --------------------------------------------------------------------------------------------- very long contractions

@pytest.mark.parametrize("dt,rows", [("bf16", 1 << 20), ("f32", 1 << 17)])
def test_long_sums_rounded_to_bf16_do_not_drift(dt, rows):
    """bf16 gradients of positive matrices of many rows.  A truncated sum is short by 2^-25 of itself or more for
    every 16 of its terms, always the same way; roundings to bf16 (2^-8) cancel in the mean over n k / 32 results of
    different size, to 2^-8 / sqrt(n k / 32) < 2^-16.  So the mean relative error tells them apart: below 2^-12, a sixteenth of
    the final rounding."""
    import paper_2507_08784_gb300 as glr
    dt, n, k = DT[dt], 2048, 2048
    gen = torch.Generator("cuda").manual_seed(6)

    def positive(cols):
        scale = 1 + torch.rand(cols, device="cuda", generator=gen)
        return torch.rand(rows, cols, device="cuda", generator=gen).mul_(scale).to(dt)

    dZ, X = positive(n), positive(k)
    dW = torch.empty(n, k, device="cuda", dtype=torch.bfloat16)
    glr.glr_linear_grad_weight(dZ, X, dW)
    at = slice(0, n, 32)
    want = torch.zeros(n // 32, k, device="cuda", dtype=torch.float64)
    for i in range(0, rows, 1 << 14):
        part = slice(i, i + (1 << 14))
        want += dZ[part, at].double().T @ X[part].double()
    error = (dW[at].double() - want) / want
    assert float(error.abs().max()) <= 2.0 ** -8 + 2.0 ** -12
    assert abs(float(error.mean())) <= 2.0 ** -12, float(error.mean())
    glr.glr_operator_status()


# --------------------------------------------------------------------------------------------------- waits that gave up

def test_waits_that_gave_up_are_reported_once(tmp_path):
    """tests/operator_status_check.cu, run with the built library: a call after the report says what came since."""
    import os
    import shutil
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    pkg, exe = os.path.join(root, "paper_2507_08784_gb300"), str(tmp_path / "check")
    subprocess.run([shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc", "-std=c++17", "-O1", "--expt-relaxed-constexpr",
                    "-gencode", "arch=compute_103a,code=sm_103a", "-I", os.path.join(root, "include"), "-I",
                    os.path.join(pkg, "csrc"), os.path.join(root, "tests", "operator_status_check.cu"), "-o", exe, "-L",
                    os.path.join(pkg, "lib"), "-lglr", "-Xlinker", "-rpath", "-Xlinker", os.path.join(pkg, "lib")], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout


# ------------------------------------------------------------------------------------ epilogues of very long contractions

@pytest.mark.parametrize("rows,n,k", [(2000, 2300, 33001), (2048, 2304, 40960), (300, 40, 70000)])
@pytest.mark.parametrize("pad", [0, 3])
def test_epilogues_of_very_long_contractions(rows, n, k, pad):
    """bf16 layers and input gradients with everything in their epilogues, results on 16 bytes and off: sums within
    (k + 8) 2^-23 of those of the absolute values, as in the tests of shorter ones, results within 2^-8 of their value."""
    import paper_2507_08784_gb300 as glr
    gen = torch.Generator("cuda").manual_seed(rows)

    def mat(r, c, scale=1.0, extra=0):
        x = torch.empty(r, -(-c // 8) * 8 + extra, device="cuda", dtype=torch.bfloat16)
        return x.normal_(0.0, scale, generator=gen)[:, :c]

    X, W, R, P = mat(rows, k), mat(n, k, k ** -0.5), mat(rows, n, extra=pad), torch.empty(rows, n, device="cuda", dtype=torch.bfloat16)
    bias, Y = mat(1, n)[0].contiguous(), torch.empty(rows, n + pad, device="cuda", dtype=torch.bfloat16)[:, :n]
    glr.glr_linear(X, W, Y, bias=bias, act="silu", residual=R, preact=P)
    x, w = X.double(), W.double()
    z, size = x @ w.T + bias.double(), x.abs() @ w.abs().T
    tol = 1.2 * (k + 8) * 2.0 ** -23 * size + 2.0 ** -20 * (1 + z.abs())
    for got, want in ((P, z), (Y, z * torch.sigmoid(z) + R.double())):
        assert ((got.double() - want).abs() <= tol + 2.0 ** -8 * want.abs()).all()
    # the same contraction as an input gradient: dZ = X, and W's transpose
    D, G, S = torch.empty_like(Y), torch.empty(rows, n + pad, device="cuda", dtype=torch.bfloat16)[:, :n], mat(rows, n, extra=pad)
    Wt = mat(k, n)
    Wt.copy_(W.T)
    glr.glr_linear_grad_input(X, Wt, D, residual=R, preact=S, act="silu", grad_out=G)
    g, p = x @ w.T + R.double(), torch.sigmoid(S.double())
    for got, want in ((G, g), (D, g * p * (1 + S.double() * (1 - p)))):
        assert ((got.double() - want).abs() <= tol + 2.0 ** -20 * g.abs() * (1 + S.double().abs()) + 2.0 ** -8 * want.abs()).all()
    glr.glr_operator_status()
