"""The row operators at the edges of what they promise: the order of an embedding gradient's sums, alternatives of rows that
hold NaNs, gradients of log-probabilities of logits far from zero (marked gpu)."""
import math

import pytest
import torch

from test_gpu_rows import HALF, U, Guarded, _logp_tol

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


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


# ---------------------------------------------------------------------------------------------------- embeddings

# narrow and wide slices, looked through and sorted
@pytest.mark.parametrize("nodes,rows,vocab,d", [(2, 700, 90, 48), (4, 1000, 40000, 512), (1, 6000, 300, 264), (8, 2000, 32000, 256)])
@pytest.mark.parametrize("gd", ["f32", "bf16"])
def test_order_of_the_sums(glr, nodes, rows, vocab, d, gd):
    """It is fixed by the sizes and the tokens: strides, alignment, the tokens' type, the type of equal values and a run
    beside other work change no bit."""
    gen = torch.Generator().manual_seed(d)
    n = nodes * rows
    tokens = ((torch.rand(n, generator=gen) ** 5 * (vocab + 40)).long() - 20).cuda()
    value = torch.randn(n, d, generator=gen).bfloat16()

    def run(dt, pad, shift, index, stream=None):
        dY = Guarded(n, d, dt, pad, shift, value=value)
        dE = [torch.empty(vocab, d, device="cuda", dtype=DT[gd]) for _ in range(nodes)]
        torch.cuda.synchronize()
        glr.glr_embedding_grad(dY.t, tokens.to(index), dE, scale=1.25, stream=stream)
        torch.cuda.synchronize()
        return torch.stack(dE)

    want = run(torch.bfloat16, 0, 0, torch.int64)
    side = torch.cuda.Stream()
    for dt, pad, shift, index, stream in ((torch.bfloat16, 1, 0, torch.int32, None), (torch.bfloat16, 8, 3, torch.int64, side),
                                          (torch.float32, 0, 0, torch.int32, None), (torch.float32, 3, 1, torch.int64, side)):
        assert torch.equal(run(dt, pad, shift, index, stream), want)


# ------------------------------------------------------------------------------------------- log-probabilities

def _alternatives(glr, z, topk, tau=0.7):
    """top_logp, top_ids, logp, lse and entropy on the CPU."""
    rows = z.shape[0]
    top, ids = Guarded(rows, topk, torch.float32, 1), Guarded(rows, topk, torch.int32, 3)
    out = [torch.full((rows,), 55.0, device="cuda") for _ in range(3)]
    glr.glr_token_logp(z, tokens=torch.zeros(rows, dtype=torch.int32, device="cuda"), logp=out[0], lse=out[1], entropy=out[2], top_logp=top.t,
                       top_ids=ids.t, temperature=tau)
    torch.cuda.synchronize()
    return top.check().cpu(), ids.check().cpu().long(), [x.cpu() for x in out]


def _ordered(z, topk):
    """Ids in descending order of the logits, a NaN above all, equal ones by index, -1 where only ruled-out entries are left."""
    rows, vocab = z.shape
    order = torch.sort(torch.where(z.isnan(), math.inf, z.double()), dim=1, descending=True, stable=True).indices
    ids = torch.where(z.gather(1, order) == -math.inf, -1, order)[:, :topk]
    return torch.nn.functional.pad(ids, (0, max(0, topk - vocab)), value=-1)


# a CTA a row of 64, 128 and 256 threads, and clusters of two, four and eight
@pytest.mark.parametrize("rows,vocab", [(3, 8), (400, 64), (200, 1000), (200, 5000), (160, 24576), (2, 16384), (2, 40000), (1, 131072)])
@pytest.mark.parametrize("topk", [1, 12, 64, 300, 1024])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_alternatives_of_whole_vectors_of_nan(glr, rows, vocab, topk, dt):
    """NaNs that fill whole groups of eight on 16 bytes count as the largest logits like any others, and their rows' results are NaN."""
    gen = torch.Generator().manual_seed(vocab + topk)
    z = torch.randn(rows, vocab, generator=gen).to(DT[dt])
    z[:, 5::11] = -math.inf
    z[0] = math.nan                                                   # a whole row
    if rows > 1:
        z[1, vocab // 16 * 8:vocab // 16 * 8 + 8] = math.nan          # one group among finite and ruled-out entries
    if rows > 2:
        z[2, :vocab // 2] = math.nan                                  # half a row
        z[2, vocab - 1] = math.nan
    top, ids, rest = _alternatives(glr, z.cuda(), topk)
    assert torch.equal(ids, _ordered(z, topk))
    nan = z.isnan().any(1)
    assert torch.equal(top[nan].isnan(), ids[nan] >= 0) and (top[nan][ids[nan] < 0] == -math.inf).all()
    assert torch.equal(top[~nan] == -math.inf, ids[~nan] < 0) and not top[~nan].isnan().any()
    for x in rest:
        assert torch.equal(x.isnan(), nan)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 5])
def test_alternatives_of_a_broken_teacher(glr, dt, shift):
    """A row of NaNs, at any place in memory, is a teacher whose loss is NaN, not one that costs nothing."""
    rows, vocab, topk = 4, 800, 16
    z = Guarded(rows, vocab, DT[dt], 0, shift, value=torch.randn(rows, vocab, generator=torch.Generator().manual_seed(2)))
    z.t[2] = math.nan
    top, ids = torch.empty(rows, topk, device="cuda"), torch.empty(rows, topk, device="cuda", dtype=torch.int32)
    glr.glr_token_logp(z.t, top_logp=top, top_ids=ids)
    assert ids[2].tolist() == list(range(topk)) and top[2].isnan().all()
    student = torch.randn(rows, vocab, device="cuda")
    loss, row, d = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(student)
    glr.glr_distill_loss(student, top, ids, loss=loss, row_loss=row, dlogits=d)
    assert loss.isnan().all() and row.isnan().tolist() == [False, False, True, False]


def _logp_grad(z, tokens, a, b, tau):
    """The gradient, p, log p (0 where p is) and the entropy in 64 bits, from differences to the rows' maxima."""
    x = z.double().cpu()
    some = (x.amax(1, keepdim=True) > -math.inf)
    lp = torch.log_softmax((x - torch.where(some, x.amax(1, keepdim=True), 0.0)) / tau, 1)
    p = torch.where(some, lp.exp(), 0.0)
    lp = torch.where(p > 0, lp, 0.0)
    H = -(p * lp).sum(1, keepdim=True)
    ok = some & (tokens >= 0)[:, None]
    e = torch.zeros_like(p).scatter_(1, tokens.clamp(min=0)[:, None], 1.0)
    return (torch.where(ok, a.double()[:, None] * (e - p), 0.0) - b.double()[:, None] * p * (lp + H)) / tau, p, lp, H


def _far(kind, rows, vocab, dt, gen):
    """Logits whose lse is far from zero, or not finite where m / tau leaves the range."""
    low, z = torch.finfo(dt).min, torch.randn(rows, vocab, generator=gen) * 2
    if kind == "least":                                               # the type's lowest value as a mask
        z = z.to(dt)
        z[0] = low
        z[1::3] = low
        z[1::3, vocab // 3] = torch.tensor(low).to(dt) / 2            # ... and one that is not quite
        z[2::3, ::2] = low
        return z
    if kind == "most":
        z = z.to(dt)
        z[::2] = -low
        z[1::2, 4:] = -math.inf
        z[1::2, :4] = -low
        return z
    return (z + kind).to(dt)


@pytest.mark.parametrize("rows,vocab,pad", [(9, 300, 0), (200, 1003, 1), (4, 20000, 0), (3, 40000, 0), (2, 70001, 3), (1, 140000, 0)])
@pytest.mark.parametrize("kind", [56.0, 70.0, 1e4, -1e6, 1e30, "least", "most"])
@pytest.mark.parametrize("tau", [1.0, 2.0 ** -10, 0.5, 1024.0])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_gradients_far_from_zero(glr, rows, vocab, pad, kind, tau, dt):
    """They come from differences to the maximum, as the log-probabilities do: p within its own error, whatever lse's rounding
    is, and every row of them adds up to 0."""
    dt, gen = DT[dt], torch.Generator().manual_seed(rows)
    z = Guarded(rows, vocab, dt, pad, value=_far(kind, rows, vocab, dt, gen))
    tokens = torch.randint(0, vocab, (rows,), generator=gen)
    tokens[5::6] = -1
    a, b = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen)
    lse, ent = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    glr.glr_token_logp(z.t, lse=lse, entropy=ent, temperature=tau)
    d = Guarded(rows, vocab, dt, pad)
    args = dict(tokens=tokens.cuda(), dlogp=a.cuda(), entropy=ent, dentropy=b.cuda(), temperature=tau)
    glr.glr_token_logp_grad(z.t, lse, d.t, **args)
    want, p, lp, H = _logp_grad(z.t, tokens, a, b, tau)
    # log p is off by the forward pass's tolerance, and up to |lse| = 64 by the roundings of lse and of z / tau (at most 104 beyond
    # it where p is not 0), twice each; p by as much of its value and by exp2's 2^-22, and it is 0 below 2^-126; the entropy by
    # what its own test allows; products of dlogp, dentropy and 1 / tau by 2 u
    near = torch.where(lse.double().cpu().abs() <= 64, 2 * U * (64 + 64 + 104), 0.0)[:, None]
    spread = z.t.double().cpu()
    spread = torch.where(p > 0, spread, spread.amax(1, keepdim=True))                     # of what has a probability
    tol_lp = _logp_tol(spread, tau) + 4 * U * lp.abs() + near + 2.0 ** -21
    tol_H = (2 * _logp_tol(z.t.cpu(), tau) + 2.0 ** -18) * (1 + H)
    A, B = a.double().abs()[:, None], b.double().abs()[:, None]
    tol = (A * p * tol_lp + B * p * (tol_lp * (lp.abs() + H + 1) + tol_H) + 2 * U * A + 2.0 ** -126 * (A + B * (lp.abs() + H + 1))) / tau
    tol = tol * (1 + HALF[dt]) + HALF[dt] * want.abs() + 1e-37
    got = d.check().double().cpu()
    assert torch.isfinite(got).all()
    over = (got - want).abs() - tol
    assert (over <= 0).all(), (float(over.max()), float((got - want).abs().max()), float(want.abs().max()))
    assert ((got - want).sum(1).abs() <= tol.sum(1)).all() and (want.sum(1).abs() <= 1e-9 / tau * vocab).all()
    # in place of the logits: the same bits
    glr.glr_token_logp_grad(z.t, lse, z.t, **args)
    assert torch.equal(z.check(), d.t)


def test_rows_that_are_read_again_beside_others(glr):
    """Near, far, ruled-out and untouched rows in one call, captured and replayed: each as it is alone."""
    gen = torch.Generator().manual_seed(4)
    z = torch.randn(40, 9000, generator=gen)
    z[1::4] += 3000.0
    z[2::4] = -math.inf
    z[3::4] = torch.finfo(torch.float32).min
    z = z.cuda()
    tokens, a, b = torch.randint(0, 9000, (40,), generator=gen).cuda(), torch.randn(40, generator=gen).cuda(), torch.randn(40, generator=gen).cuda()
    a[8:12], b[8:12] = 0.0, 0.0
    lse, ent, d = torch.empty(40, device="cuda"), torch.empty(40, device="cuda"), torch.empty_like(z)
    glr.glr_token_logp(z, lse=lse, entropy=ent, temperature=0.5)
    run = lambda: glr.glr_token_logp_grad(z, lse, d, tokens=tokens, dlogp=a, entropy=ent, dentropy=b, temperature=0.5)  # noqa: E731
    run()
    for i in range(40):
        one = torch.empty(1, 9000, device="cuda")
        glr.glr_token_logp_grad(z[i:i + 1], lse[i:i + 1], one, tokens=tokens[i:i + 1], dlogp=a[i:i + 1], entropy=ent[i:i + 1],
                                dentropy=b[i:i + 1], temperature=0.5)
        assert torch.equal(one[0], d[i])
    want = d.clone()
    assert (want[2::4] == 0).all() and (want[8:12] == 0).all() and (want[5] != 0).any() and (want[7] != 0).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    d.fill_(5.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(d, want)
