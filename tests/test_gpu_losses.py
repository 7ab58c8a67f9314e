"""The losses on logits (distillation, policy, preference) against their definitions in 64 bits, at the sizes,
masks, strides and alignments where they can go wrong (marked gpu).

Tolerances, from the arithmetic: an exponential exp2((z - m) log2(e) / tau) in fp32 is off by the rounding of
its argument (2^-23 of |z - m| / tau) and a few 2^-23 of its own, a sum over the vocabulary by at most
2^-24 times the terms one thread adds (vocab / 512, at most 2^9 here) and the merges; so a probability is
within REL = 2^-19 + 2^-22 max|z - m| / tau of its value, a log-probability within the same absolute error, and
products of them with the coefficients within a few times that.  bf16 results add half a unit in the last place, 2^-8.
"""
import math

import pytest
import torch

import _operators as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


def _logits(rows, vocab, dt, gen, pad=0, shift=0, scale=3.0):
    """rows x vocab on the GPU in rows of vocab + pad elements, the first one `shift` elements into its buffer."""
    buf = torch.zeros(rows * (vocab + pad) + shift, device="cuda", dtype=dt)
    z = buf[shift:shift + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    z.copy_(torch.randn(rows, vocab, generator=gen) * scale)
    return z


def _rel(z, tau=1.0):
    f = z[torch.isfinite(z)]
    span = float((f.max() - f.min()).clamp(max=400)) if f.numel() else 0.0
    return 2.0 ** -19 + 2.0 ** -22 * span / tau


def _check_grad(got, want, rel, dt, coef):
    """|got - want| <= rel (|want| + coef) + the rounding of the result; coef bounds p's and q's factors times
    the probabilities themselves (a difference of two of them keeps their absolute errors)."""
    got, want = got.double().cpu(), want
    tol = 4 * rel * (want.abs() + coef) + (2.0 ** -8 * want.abs() if dt == torch.bfloat16 else 0) + 1e-38
    bad = (got - want).abs() > tol
    assert torch.isfinite(got).all()
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()), float(want.abs().max()))


def _close(got, want, tol):
    got, want = got.double().cpu().flatten(), torch.as_tensor(want, dtype=torch.float64).flatten()
    assert torch.isfinite(got).all()
    assert ((got - want).abs() <= tol * (1 + want.abs())).all(), (got, want)


def _dprob(logits, tau=1.0):
    """softmax of every row in 64 bits, zero for rows with none."""
    p = torch.softmax(logits.double().cpu() / tau, 1)
    return torch.nan_to_num(p, nan=0.0)


# ------------------------------------------------------------------------------------------------ distillation

def _run_distill(z, teacher, ids, labels=None, weight=None, tau=1.0, soft=1.0, hard=0.0, inplace=False, stream=None,
                 grad=True, pad=0):
    import paper_2507_08784_gb300 as glr
    rows, vocab = z.shape
    loss, row = torch.full((1,), math.nan, device="cuda"), torch.full((rows,), math.nan, device="cuda")
    d = None
    if grad:
        d = z if inplace else torch.full((rows, vocab + pad), math.nan, device="cuda", dtype=z.dtype)[:, :vocab]
    glr.glr_distill_loss(z, teacher, ids, loss=loss, row_loss=row, dlogits=d, labels=labels, weight=weight,
                         temperature=tau, soft=soft, hard=hard, stream=stream)
    torch.cuda.synchronize()
    glr.glr_operator_status()
    return loss, row, d


def _distill_case(rows, vocab, topk, dt, tau, hard, pad, shift, seed, wide):
    gen = torch.Generator().manual_seed(seed)
    z = _logits(rows, vocab, dt, gen, pad, shift)
    ids = torch.randint(0, vocab, (rows, topk), generator=gen)
    ids[::3, : topk // 4] = -1
    if topk > 2:
        ids[::4, -1] = ids[::4, 0]                        # given twice
    teacher = (2 * torch.randn(rows, topk, generator=gen)).to(dt)
    labels = torch.randint(0, vocab, (rows,), generator=gen)
    labels[::5] = -100
    weight = torch.rand(rows, generator=gen)
    weight[1::4] = 0
    it = torch.int64 if wide else torch.int32
    zc = z.cpu()
    dev = (teacher.cuda(), ids.to(it).cuda(), labels.to(it).cuda() if hard else None, weight.cuda())
    want = ref.distill(zc, teacher, ids, labels if hard else None, weight, tau, 1.5, hard)
    return z, zc, dev, want


@pytest.mark.parametrize("rows,vocab,topk,tau,hard,pad,shift,wide", [
    (1, 1, 1, 1.0, 0.0, 0, 0, False),
    (3, 2, 2, 2.0, 0.5, 1, 1, True),
    (5, 7, 4, 1.0, 0.5, 0, 3, False),
    (9, 8, 8, 2.0, 0.0, 0, 0, True),
    (6, 31, 0, 1.0, 1.0, 2, 0, True),
    (17, 255, 16, 4.0, 0.5, 0, 0, False),
    (12, 1000, 33, 2.0, 0.3, 3, 5, True),
    (7, 4099, 64, 1.0, 0.0, 8, 0, False),
    (5, 16384, 513, 2.0, 0.5, 0, 0, True),
    (3, 32771, 1024, 1.5, 0.5, 0, 1, False),
    (4, 65536, 128, 1.0, 0.0, 0, 0, False),
    (2, 131071, 100, 2.0, 0.5, 1, 0, True),
    (2, 262144, 256, 1.0, 0.5, 0, 0, False),
])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_distill(rows, vocab, topk, tau, hard, pad, shift, wide, dt):
    dt = DT[dt]
    z, zc, (teacher, ids, labels, weight), want = _distill_case(rows, vocab, topk, dt, tau, hard, pad, shift, 11, wide)
    loss, row, d = _run_distill(z, teacher, ids, labels, weight, tau, 1.5, hard, pad=pad)
    rel = _rel(zc.float(), tau)
    _close(loss, want[0], 8 * rel)
    _close(row, want[1], 8 * rel)
    coef = weight.cpu().double()[:, None] * (1.5 / tau + hard)
    p = coef * torch.maximum(_dprob(zc, tau), _dprob(zc))
    q = (want[2] - 0).abs()
    _check_grad(d, want[2], rel, dt, p + q)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,pad", [(1003, 0), (40000, 0), (131072, 0), (70001, 5)])
def test_distill_in_place_and_on_another_stream(vocab, pad, dt):
    dt = DT[dt]
    z, zc, (teacher, ids, labels, weight), _ = _distill_case(19, vocab, 20, dt, 2.0, 0.5, pad, 0, 5, False)
    a = _run_distill(z, teacher, ids, labels, weight, 2.0, 1.0, 0.5)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = _run_distill(z, teacher, ids, labels, weight, 2.0, 1.0, 0.5, stream=s)
    c = _run_distill(z, teacher, ids, labels, weight, 2.0, 1.0, 0.5, inplace=True)
    for x, y in ((b, a), (c, a)):
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1]) and torch.equal(x[2], y[2])
    z.copy_(zc)                                           # the same memory: sums go by how rows lie on 16 bytes
    f = _run_distill(z, teacher, ids, labels, weight, 2.0, 1.0, 0.5, grad=False)
    assert torch.equal(f[1], a[1])


def test_distill_masks_that_leave_nothing():
    """Rows of weight 0 hold NaN, a row is ruled out entirely, one holds the type's lowest value throughout,
    one has a single allowed entry, one no teacher entry, one only teacher entries of -infinity."""
    for dt in DT.values():
        gen = torch.Generator().manual_seed(3)
        z = _logits(8, 3001, dt, gen)
        low = torch.finfo(dt).min
        z[0] = math.nan
        z[1] = -math.inf
        z[2] = low
        z[3] = -math.inf
        z[3, 17] = 2.0
        z[6, :2000] = low
        z[7, ::2] = -math.inf
        ids = torch.randint(0, 3001, (8, 9), generator=gen)
        ids[4] = torch.tensor([-1, 3001, 1 << 30, -5, -1, -1, -1, -1, -1])
        ids[3] = 17
        ids[6], ids[7] = 2000 + torch.arange(9), 1 + 2 * torch.arange(9)
        teacher = torch.randn(8, 9, generator=gen)
        teacher[5] = -math.inf
        teacher[7, 3:] = -math.inf
        weight = torch.ones(8)
        weight[0] = 0
        labels = torch.tensor([0, 5, 5, 17, -1, 4, 2500, 1])
        want = ref.distill(z.cpu(), teacher, ids, labels, weight, 2.0, 1.0, 0.5)
        loss, row, d = _run_distill(z, teacher.cuda(), ids.cuda(), labels.cuda(), weight.cuda(), 2.0, 1.0, 0.5)
        rel = 2.0 ** -16
        assert not d[0].any() and not d[1].any() and row[0] == 0 and row[1] == 0
        _close(row, want[1], 8 * rel)
        _close(loss, want[0], 8 * rel)
        _check_grad(d, want[2], rel, dt, want[2].abs() + 1e-2)


def test_distill_without_rows():
    import paper_2507_08784_gb300 as glr
    loss = torch.full((1,), math.nan, device="cuda")
    e = torch.empty(0, 77, device="cuda")
    glr.glr_distill_loss(e, torch.empty(0, 4, device="cuda"), torch.empty(0, 4, device="cuda", dtype=torch.int32),
                         loss=loss, row_loss=torch.empty(0, device="cuda"), dlogits=e)
    assert float(loss) == 0.0


def test_distill_gradient_against_differences():
    """Central differences of the loss itself along random directions; the loss is within 1e-6 of its value,
    so a step of 0.05 leaves 1e-6 / 0.05 = 2e-5 of noise, and the third derivative (below 1) 0.05^2 / 6."""
    gen = torch.Generator().manual_seed(8)
    rows, vocab, topk = 6, 500, 12
    z = _logits(rows, vocab, torch.float32, gen, scale=1.0)
    ids = torch.stack([torch.randperm(vocab, generator=gen)[:topk] for _ in range(rows)]).cuda()
    teacher, labels = torch.randn(rows, topk, generator=gen).cuda(), torch.randint(0, vocab, (rows,), generator=gen).cuda()
    _, _, d = _run_distill(z, teacher, ids, labels, None, 2.0, 4.0, 0.5)
    for s in range(4):
        v = torch.randn(rows, vocab, generator=gen).cuda()
        up, down = (float(_run_distill(z + e * v, teacher, ids, labels, None, 2.0, 4.0, 0.5, grad=False)[0])
                    for e in (0.05, -0.05))
        assert abs((up - down) / 0.1 - float((d * v).sum())) < 1e-3


# ------------------------------------------------------------------------------------------------------ policy

def _run_policy(z, tokens, old, adv, refl=None, weight=None, tau=1.0, low=0.2, high=0.2, kl=0.0, grad=True,
                inplace=False):
    import paper_2507_08784_gb300 as glr
    rows, vocab = z.shape
    loss, row, logp = torch.full((1,), math.nan, device="cuda"), *(torch.full((rows,), math.nan, device="cuda") for _ in range(2))
    d = (z if inplace else torch.full_like(z, math.nan)) if grad else None
    glr.glr_policy_loss(z, tokens, old, adv, loss=loss, row_loss=row, logp=logp, dlogits=d, ref_logp=refl, weight=weight,
                        temperature=tau, clip_low=low, clip_high=high, kl=kl)
    torch.cuda.synchronize()
    glr.glr_operator_status()
    return loss, row, logp, d


def _policy_case(rows, vocab, dt, tau, pad, shift, seed):
    gen = torch.Generator().manual_seed(seed)
    z = _logits(rows, vocab, dt, gen, pad, shift)
    tokens = torch.randint(0, vocab, (rows,), generator=gen)
    zc = z.cpu()
    lp = torch.log_softmax(zc.double() / tau, 1).gather(1, tokens[:, None])[:, 0]
    old = (lp + 0.4 * torch.randn(rows, generator=gen)).float()
    refl = (lp + 0.3 * torch.randn(rows, generator=gen)).float()
    adv = torch.randn(rows, generator=gen)
    adv[::6] = 0
    tokens[2::7] = -1
    weight = torch.rand(rows, generator=gen)
    weight[1::4] = 0
    return z, zc, tokens, old, adv, refl, weight


@pytest.mark.parametrize("rows,vocab,tau,kl,pad,shift,wide", [
    (1, 1, 1.0, 0.0, 0, 0, True), (2, 3, 0.7, 0.1, 1, 1, False), (11, 64, 1.0, 0.05, 0, 0, True),
    (40, 1001, 1.3, 0.1, 0, 3, False), (9, 32768, 0.7, 0.0, 0, 0, True), (5, 100003, 1.0, 0.2, 5, 0, False),
    (3, 300000, 1.0, 0.1, 0, 0, True),
])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_policy(rows, vocab, tau, kl, pad, shift, wide, dt):
    dt = DT[dt]
    z, zc, tokens, old, adv, refl, weight = _policy_case(rows, vocab, dt, tau, pad, shift, 21)
    want = ref.policy(zc, tokens, old, adv, refl if kl else None, weight, tau, 0.2, 0.28, kl)
    cu = lambda x: x.cuda()  # noqa: E731
    loss, row, logp, d = _run_policy(z, cu(tokens if wide else tokens.int()), cu(old), cu(adv), cu(refl) if kl else None,
                                     cu(weight), tau, 0.2, 0.28, kl)
    rel = _rel(zc.float(), tau) * 4                       # ratio and exp(e) are exponentials of log-probabilities
    _close(loss, want[0], 8 * rel)
    _close(row, want[1], 8 * rel)
    _close(logp, want[2], 4 * rel)
    _check_grad(d, want[3], rel, dt, (want[3].abs().sum(1, keepdim=True) * (_dprob(zc, tau) + (want[3].abs() > 0.3 * want[3].abs().sum(1, keepdim=True)))))
    # no gradient wanted, the gradient in the logits' place, equal weights
    assert torch.equal(_run_policy(z, cu(tokens), cu(old), cu(adv), cu(refl) if kl else None, cu(weight), tau, 0.2, 0.28, kl, grad=False)[1], row)
    even = _run_policy(z, cu(tokens), cu(old), cu(adv), None, None, tau)
    same = _run_policy(z, cu(tokens), cu(old), cu(adv), None, torch.full((rows,), 1.0 / rows, device="cuda"), tau, inplace=True)
    assert torch.equal(even[3], same[3]) and torch.equal(even[0], same[0])


def test_policy_masks_that_leave_nothing():
    for dt in DT.values():
        gen = torch.Generator().manual_seed(4)
        z = _logits(6, 2049, dt, gen)
        z[0] = math.nan                                     # weight 0
        z[1] = -math.inf                                    # nothing allowed
        z[2] = math.inf                                     # token outside: not read
        z[3] = -math.inf
        z[3, 5] = -7.0                                      # one allowed entry, the token
        z[4, 1:] = torch.finfo(dt).min                      # masked by the lowest value
        z[5, :] = torch.finfo(dt).min                       # ... throughout: uniform
        tokens = torch.tensor([1, 1, 2049, 5, 0, 9])
        weight = torch.tensor([0.0, 1, 1, 1, 1, 1])
        old, adv, refl = -torch.rand(6, generator=gen), torch.randn(6, generator=gen), -torch.rand(6, generator=gen)
        want = ref.policy(z.cpu(), tokens, old, adv, refl, weight, 1.0, 0.2, 0.2, 0.1)
        loss, row, logp, d = _run_policy(z, tokens.cuda(), old.cuda(), adv.cuda(), refl.cuda(), weight.cuda(), kl=0.1)
        assert not d[:3].any() and not row[:3].any() and not logp[:3].any()
        _close(loss, want[0], 2.0 ** -14)
        _close(logp, want[2], 2.0 ** -16)
        _check_grad(d, want[3], 2.0 ** -16, dt, want[3].abs() + 1e-2)


def test_policy_gradient_against_differences():
    gen = torch.Generator().manual_seed(9)
    rows, vocab = 8, 300
    z = _logits(rows, vocab, torch.float32, gen, scale=1.0)
    tokens = torch.randint(0, vocab, (rows,), generator=gen)
    lp = torch.log_softmax(z.double().cpu(), 1).gather(1, tokens[:, None])[:, 0]
    # ratios well inside or well outside the clip range, so that a small step stays on one side
    old = (lp + torch.tensor([0.0, 0.6, -0.6, 0.05, 0.0, 0.6, -0.6, -0.05])).float().cuda()
    adv = torch.tensor([1.0, 1, 1, 1, -1, -1, -1, -1]).cuda()
    refl, tokens = (lp + 0.2).float().cuda(), tokens.cuda()
    _, _, _, d = _run_policy(z, tokens, old, adv, refl, None, kl=0.3)
    for s in range(4):
        v = torch.randn(rows, vocab, generator=gen).cuda()
        v /= v.abs().max()
        up, down = (float(_run_policy(z + e * v, tokens, old, adv, refl, None, kl=0.3, grad=False)[0]) for e in (0.02, -0.02))
        assert abs((up - down) / 0.04 - float((d * v).sum())) < 1e-3


# -------------------------------------------------------------------------------------------------- preference

def _run_preference(z, tokens, offsets, refl=None, weight=None, kind="sigmoid", beta=0.1, smoothing=0.0, average=False,
                    grad=True, inplace=False, stream=None):
    import paper_2507_08784_gb300 as glr
    rows, vocab = z.shape
    pairs = (offsets.numel() - 1) // 2
    nan = lambda n: torch.full((n,), math.nan, device="cuda")  # noqa: E731
    loss, pair, seq, row = nan(1), nan(pairs), nan(2 * pairs), nan(rows)
    d = (z if inplace else torch.full_like(z, math.nan)) if grad else None
    glr.glr_preference_loss(z, tokens, offsets, loss=loss, pair_loss=pair, seq_logp=seq, row_logp=row, dlogits=d,
                            ref_logp=refl, weight=weight, kind=kind, beta=beta, smoothing=smoothing, average=average,
                            stream=stream)
    torch.cuda.synchronize()
    glr.glr_operator_status()
    return loss, pair, seq, row, d


def _preference_case(lengths, vocab, dt, pad, shift, seed, extra=0):
    gen = torch.Generator().manual_seed(seed)
    rows = sum(lengths) + extra
    z = _logits(rows, vocab, dt, gen, pad, shift)
    tokens = torch.randint(0, vocab, (rows,), generator=gen)
    tokens[torch.rand(rows, generator=gen) < 0.25] = -100
    offsets = torch.tensor([0] + lengths).cumsum(0)
    return z, z.cpu(), tokens, offsets, gen


@pytest.mark.parametrize("lengths,vocab,kind,average,smoothing,pad,shift,wide,extra", [
    ([1, 1], 1, "sigmoid", False, 0.0, 0, 0, True, 0),
    ([3, 0], 17, "ipo", True, 0.0, 1, 1, False, 2),
    ([0, 0, 1, 5], 200, "sigmoid", False, 0.1, 0, 0, True, 0),
    ([9, 14, 30, 2, 1, 1], 1001, "sigmoid", True, 0.2, 0, 3, False, 3),
    ([20, 33], 32768, "ipo", False, 0.0, 0, 0, True, 0),
    ([5, 7, 6, 4], 100001, "sigmoid", False, 0.0, 3, 0, False, 1),
    ([300, 411, 2, 700], 130, "sigmoid", False, 0.1, 0, 0, True, 0),
])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_preference(lengths, vocab, kind, average, smoothing, pad, shift, wide, extra, dt):
    dt = DT[dt]
    z, zc, tokens, offsets, gen = _preference_case(lengths, vocab, dt, pad, shift, 31, extra)
    seqs = len(lengths)
    base = ref.preference(zc, tokens, offsets, None, None, kind, 0.1, smoothing, average)[2]
    refl = (base + 2 * torch.randn(seqs, generator=gen)).float()
    want = ref.preference(zc, tokens, offsets, refl, None, kind, 0.1, smoothing, average)
    it = torch.int64 if wide else torch.int32
    loss, pair, seq, row, d = _run_preference(z, tokens.to(it).cuda(), offsets.to(it).cuda(), refl.cuda(), None, kind, 0.1,
                                              smoothing, average)
    rel = _rel(zc.float())
    _close(row, want[3], 4 * rel)
    _close(seq, want[2], 4 * rel)
    # h is a difference of sequence sums: its error is theirs, and the pair loss moves by at most 2 |h - 5| + 1 of it
    habs = 4 * rel * (2 + 2 * float(want[2].abs().max() if seqs else 0))
    slope = 1 + 2 * float(want[1].abs().max()) ** 0.5 if kind == "ipo" else 0.1
    assert float((pair.double().cpu() - want[1]).abs().max()) <= slope * habs + 8 * rel * float(1 + want[1].abs().max())
    grad_rel = rel + (2 if kind == "ipo" else 0.1) * habs
    biggest = want[4].abs().max(1, keepdim=True).values
    _check_grad(d, want[4], grad_rel, dt, biggest * (_dprob(zc) + (want[4].abs() == biggest)))
    f = _run_preference(z, tokens.cuda(), offsets.cuda(), refl.cuda(), None, kind, 0.1, smoothing, average, grad=False)
    assert torch.equal(f[0], loss) and torch.equal(f[1], pair)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = _run_preference(z, tokens.cuda(), offsets.cuda(), refl.cuda(), None, kind, 0.1, smoothing, average, inplace=True, stream=s)
    assert torch.equal(g[4], d)


def test_preference_masks_that_leave_nothing():
    """Prompt rows that hold NaN, a row ruled out entirely, a sequence without counted tokens, a pair of weight
    0, offsets beyond the rows."""
    for dt in DT.values():
        gen = torch.Generator().manual_seed(6)
        z = _logits(20, 777, dt, gen)
        tokens = torch.randint(0, 777, (20,), generator=gen)
        tokens[0], z[0] = -1, math.nan
        z[2] = -math.inf
        z[3, :700] = torch.finfo(dt).min
        tokens[3] = 705
        tokens[5:8] = 777
        z[5:8] = math.inf
        offsets = torch.tensor([-3, 5, 8, 12, 15, 17, 400])
        weight = torch.tensor([1.0, 0.0, 2.0])
        for average in (False, True):
            want = ref.preference(z.cpu(), tokens, offsets, None, weight, "sigmoid", 0.3, 0.1, average)
            loss, pair, seq, row, d = _run_preference(z, tokens.cuda(), offsets.cuda(), None, weight.cuda(), "sigmoid", 0.3,
                                                      0.1, average)
            assert not d[0].any() and not d[2].any() and not d[5:8].any() and not d[8:15].any() and row[2] == 0
            _close(seq, want[2], 2.0 ** -15)
            _close(pair, want[1], 2.0 ** -13)
            _close(loss, want[0], 2.0 ** -13)
            _check_grad(d, want[4], 2.0 ** -14, dt, want[4].abs() + 1e-2)


def test_preference_without_pairs():
    z, _, tokens, _, _ = _preference_case([4], 50, torch.float32, 0, 0, 1)
    loss, pair, seq, row, d = _run_preference(z, tokens.cuda(), torch.zeros(1, dtype=torch.int64, device="cuda"))
    assert float(loss) == 0 and not d.any()


def test_preference_gradient_against_differences():
    z, _, tokens, offsets, gen = _preference_case([5, 8, 3, 6], 120, torch.float32, 0, 0, 2)
    z.mul_(1 / 3)
    tokens, offsets = tokens.cuda(), offsets.cuda()
    for kw in (dict(kind="sigmoid", smoothing=0.1), dict(kind="ipo", average=True, beta=0.5)):
        d = _run_preference(z, tokens, offsets, **kw)[4]
        for s in range(3):
            v = torch.randn(z.shape, generator=gen).cuda()
            v /= v.abs().max()
            up, down = (float(_run_preference(z + e * v, tokens, offsets, grad=False, **kw)[0]) for e in (0.02, -0.02))
            assert abs((up - down) / 0.04 - float((d * v).sum())) < 2e-3


# ------------------------------------------------------------------------------------------- large and repeated

def test_rows_past_32_bits_of_elements():
    """2.3e9 logits: the rows at the end are right."""
    rows, vocab = 17600, 131072
    free, _ = torch.cuda.mem_get_info()
    if free < 14 << 30:
        pytest.skip("needs 14 GB")
    z = torch.zeros(rows, vocab, device="cuda", dtype=torch.bfloat16)
    gen = torch.Generator().manual_seed(2)
    z[-2:] = (2 * torch.randn(2, vocab, generator=gen)).cuda()
    tokens = torch.zeros(rows, dtype=torch.int64)
    tokens[-2:] = torch.tensor([vocab - 1, 77])
    weight = torch.zeros(rows)
    weight[0] = weight[-2:] = 1
    old = torch.full((rows,), -11.0)
    adv = torch.ones(rows)
    loss, row, logp, d = _run_policy(z, tokens.cuda(), old.cuda(), adv.cuda(), None, weight.cuda(), low=100.0, high=100.0, inplace=False)
    want = ref.policy(z[-2:].cpu(), tokens[-2:], old[-2:], adv[-2:], None, weight[-2:], 1.0, 100.0, 100.0, 0.0)
    _close(logp[-2:], want[2], 2.0 ** -17)
    _check_grad(d[-2:], want[3], 2.0 ** -16, torch.bfloat16, want[3].abs())
    assert abs(float(logp[0]) + math.log(vocab)) < 1e-5 and not d[1:-2].any()


def test_results_do_not_depend_on_the_launch():
    """The same call twice gives the same bits."""
    for vocab in (999, 50000):
        z, zc, (teacher, ids, labels, weight), _ = _distill_case(700, vocab, 8, torch.bfloat16, 2.0, 0.5, 0, 0, 13, False)
        a = _run_distill(z, teacher, ids, labels, weight, 2.0, 1.0, 0.5)
        b = _run_distill(z, teacher, ids, labels, weight, 2.0, 1.0, 0.5)
        assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])


@pytest.mark.parametrize("vocab,rows", [(37, 9000), (2048, 5003), (8191, 3001), (32768, 1500), (65536, 700), (131071, 400)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_many_rows_a_group(vocab, rows, dt):
    """Many more rows than the GPU takes at once: every row against 64-bit sums over all of them, with a gradient
    and without one."""
    dt = DT[dt]
    gen = torch.Generator().manual_seed(17)
    z = _logits(rows, vocab, dt, gen)
    ids = torch.randint(0, vocab, (rows, 5), generator=gen).cuda()
    teacher, labels = torch.randn(rows, 5, generator=gen).cuda(), torch.randint(0, vocab, (rows,), generator=gen).cuda()
    weight = torch.ones(rows)
    weight[::3] = 0
    zc = z.clone()
    loss, row, d = _run_distill(z, teacher, ids, labels, weight.cuda(), 2.0, 1.0, 0.5)
    f_loss, f_row, _ = _run_distill(zc, teacher, ids, labels, weight.cuda(), 2.0, 1.0, 0.5, grad=False)
    _, p_row, p_logp, _ = _run_policy(zc, labels, torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda"), None,
                                      weight.cuda(), grad=False)
    assert torch.equal(row, f_row) and torch.equal(loss, f_loss)
    rel, q = _rel(zc[:50].float().cpu()) * 2, torch.softmax(teacher.double() / 2.0, 1)
    for at in range(0, rows, 256):
        part = slice(at, min(rows, at + 256))
        x = zc[part].double()
        lp, lp1 = torch.log_softmax(x / 2.0, 1), torch.log_softmax(x, 1).gather(1, labels[part, None])[:, 0]
        want = (q[part] * (q[part].log() - lp.gather(1, ids[part]))).sum(1) - 0.5 * lp1
        live = (weight[part] != 0).cuda()
        assert ((row[part].double() - torch.where(live, want, 0)).abs() <= 8 * rel * (1 + want.abs())).all(), at
        assert ((p_logp[part].double() - torch.where(live, lp1, 0)).abs() <= 8 * rel * (1 + lp1.abs())).all(), at
        g = (0.5 * lp.exp() + 0.5 * torch.softmax(x, 1)).scatter_add_(1, ids[part], -0.5 * q[part])
        g.scatter_add_(1, labels[part, None], torch.full((g.shape[0], 1), -0.5, device="cuda", dtype=torch.float64))
        g = torch.where(live[:, None], g, 0)
        tol = 16 * rel * (g.abs() + lp.exp() + torch.softmax(x, 1) + 1e-6) + (2.0 ** -8 * g.abs() if dt == torch.bfloat16 else 0)
        tol.scatter_add_(1, ids[part], 16 * rel * q[part]).scatter_add_(1, labels[part, None], torch.full((g.shape[0], 1), 16 * rel, device="cuda").double())
        assert ((d[part].double() - g).abs() <= tol).all(), at


@pytest.mark.parametrize("vocab,rows,topk,tau", [(70, 5000, 65, 2.0), (2048, 3001, 100, 1.0), (8191, 1500, 128, 3.0), (32768, 700, 129, 2.0),
                                                 (131071, 200, 257, 1.0), (131072, 300, 128, 2.0), (390001, 60, 1024, 1.5)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("inplace", [False, True])
def test_many_entries_a_row(vocab, rows, topk, tau, dt, inplace):
    """More of the teacher's entries than a warp's first loads, ids given twice among them, over many rows a group; the
    last size leaves room for two rows' entries beside the row itself."""
    dt = DT[dt]
    gen = torch.Generator().manual_seed(23)
    z = _logits(rows, vocab, dt, gen)
    ids = torch.randint(0, vocab, (rows, topk), generator=gen)
    ids[::2, 1] = ids[::2, topk - 1]
    ids, labels = ids.int().cuda(), torch.randint(0, vocab, (rows,), generator=gen).cuda()
    teacher, weight = torch.randn(rows, topk, generator=gen).cuda(), torch.ones(rows)
    weight[::5] = 0
    zc = z.clone()
    loss, row, d = _run_distill(z, teacher, ids, labels, weight.cuda(), tau, 1.0, 0.5, inplace=inplace)
    rel, q = _rel(zc[:50].float().cpu()) * 2, torch.softmax(teacher.double() / tau, 1)
    wants = torch.zeros((), device="cuda", dtype=torch.float64)
    for at in range(0, rows, 64):
        part = slice(at, min(rows, at + 64))
        x, k = zc[part].double(), ids[part].long()
        lp, lp1 = torch.log_softmax(x / tau, 1), torch.log_softmax(x, 1).gather(1, labels[part, None])[:, 0]
        live = (weight[part] != 0).cuda()
        want = torch.where(live, (q[part] * (q[part].log() - lp.gather(1, k))).sum(1) - 0.5 * lp1, 0)
        wants += want.sum()
        assert ((row[part].double() - want).abs() <= 8 * rel * (1 + want.abs())).all(), at
        g = (lp.exp() / tau + 0.5 * torch.softmax(x, 1)).scatter_add_(1, k, -q[part] / tau)
        g.scatter_add_(1, labels[part, None], torch.full((g.shape[0], 1), -0.5, device="cuda", dtype=torch.float64))
        g = torch.where(live[:, None], g, 0)
        tol = 16 * rel * (g.abs() + lp.exp() + torch.softmax(x, 1) + 1e-6) + (2.0 ** -8 * g.abs() if dt == torch.bfloat16 else 0)
        tol.scatter_add_(1, k, 16 * rel * q[part]).scatter_add_(1, labels[part, None], torch.full((g.shape[0], 1), 16 * rel, device="cuda").double())
        assert ((d[part].double() - g).abs() <= tol).all(), at
    assert abs(float(loss) - float(wants)) <= 8 * rel * (rows + abs(float(wants)))
