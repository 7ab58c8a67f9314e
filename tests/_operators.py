"""Definitions of the operators around the step in 64 bits, for the tests: plain loops over rows, written from
the formulas in include/glr.h, on CPU tensors."""
import math

import torch


def act(z, name):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z.clone()


def act_slope(z, name):
    z = z.clone().requires_grad_(True)
    act(z, name).sum().backward()
    return z.grad


def linear(X, W, bias, name, residual):
    Z = X.double() @ W.double().T
    if bias is not None:
        Z = Z + bias.double()
    Y = act(Z, name)
    return Z, Y if residual is None else Y + residual.double()


def log_softmax(z):
    """log softmax of a 64-bit row; None for a row ruled out entirely."""
    m = z.max()
    if m == -math.inf:
        return None
    return (z - m) - torch.log(torch.exp(z - m).sum())


def distill(logits, teacher, ids, labels, weight, tau, soft, hard):
    rows, vocab = logits.shape
    d = torch.zeros(rows, vocab, dtype=torch.float64)
    row_loss = torch.zeros(rows, dtype=torch.float64)
    total = 0.0
    for t in range(rows):
        w = float(weight[t]) if weight is not None else 1.0 / rows
        z = logits[t].double()
        if w == 0:
            continue
        lp, lp1 = log_softmax(z / tau), log_softmax(z)
        if lp is None:
            continue
        have = [(int(i), float(a)) for i, a in zip(ids[t], teacher[t]) if 0 <= int(i) < vocab and float(a) != -math.inf]
        loss = 0.0
        if have:
            top = max(a for _, a in have)
            e = [math.exp((a - top) / tau) for _, a in have]
            for (i, a), x in zip(have, e):
                q = x / sum(e)
                if q > 0:
                    loss += soft * q * (math.log(q) - float(lp[i]))
                d[t, i] -= w * soft / tau * q
            d[t] += w * soft / tau * lp.exp()
        if labels is not None and 0 <= int(labels[t]) < vocab:
            y = int(labels[t])
            loss -= hard * float(lp1[y])
            d[t] += w * hard * lp1.exp()
            d[t, y] -= w * hard
        row_loss[t] = loss
        total += w * loss
    return total, row_loss, d


def policy(logits, tokens, old, adv, ref, weight, tau, low, high, kl):
    rows, vocab = logits.shape
    d = torch.zeros(rows, vocab, dtype=torch.float64)
    row_loss, logp = torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    total = 0.0
    for t in range(rows):
        w = float(weight[t]) if weight is not None else 1.0 / rows
        y = int(tokens[t])
        if w == 0 or not 0 <= y < vocab:
            continue
        row = log_softmax(logits[t].double() / tau)
        if row is None:
            continue
        lp = float(row[y])
        A, r = float(adv[t]), math.exp(lp - float(old[t]))
        loss = -min(r * A, min(max(r, 1 - low), 1 + high) * A)
        slope = 0.0 if (r > 1 + high if A > 0 else r < 1 - low) else -A * r
        if ref is not None:
            e = float(ref[t]) - lp
            loss += kl * (math.expm1(e) - e)
            slope -= kl * math.expm1(e)
        row_loss[t], logp[t] = loss, lp
        total += w * loss
        d[t] = -w * slope / tau * row.exp()
        d[t, y] += w * slope / tau
    return total, row_loss, logp, d


def preference(logits, tokens, offsets, ref, weight, kind, beta, smoothing, average):
    rows, vocab = logits.shape
    pairs = (len(offsets) - 1) // 2
    row_logp = torch.zeros(rows, dtype=torch.float64)
    probs, counts = {}, [False] * rows
    for t in range(rows):
        y = int(tokens[t])
        if 0 <= y < vocab:
            lp = log_softmax(logits[t].double())
            if lp is not None:
                row_logp[t], probs[t], counts[t] = lp[y], lp.exp(), True
    spans = []
    for s in range(2 * pairs):
        b = min(max(int(offsets[s]), 0), rows)
        spans.append((b, min(max(int(offsets[s + 1]), b), rows)))
    n = [sum(counts[b:e]) for b, e in spans]
    share = [1.0 / max(1, c) if average else 1.0 for c in n]
    seq = torch.tensor([float(row_logp[b:e].sum()) * s for (b, e), s in zip(spans, share)], dtype=torch.float64)
    d = torch.zeros(rows, vocab, dtype=torch.float64)
    pair_loss, total = torch.zeros(pairs, dtype=torch.float64), 0.0
    for q in range(pairs):
        w = float(weight[q]) if weight is not None else 1.0 / pairs
        r = [float(seq[2 * q + i]) - (float(ref[2 * q + i]) if ref is not None else 0.0) for i in (0, 1)]
        h = r[0] - r[1]
        if kind == "ipo":
            e = h - 0.5 / beta
            loss, slope = e * e, 2 * e
        else:
            soft = lambda x: max(x, 0) + math.log1p(math.exp(-abs(x)))  # noqa: E731
            sig = lambda x: 1 / (1 + math.exp(-x)) if x > -700 else 0.0  # noqa: E731
            loss = (1 - smoothing) * soft(-beta * h) + smoothing * soft(beta * h)
            slope = beta * (smoothing * sig(beta * h) - (1 - smoothing) * sig(-beta * h))
        pair_loss[q] = loss
        if w == 0:
            continue
        total += w * loss
        for i, sign in ((0, 1.0), (1, -1.0)):
            b, e = spans[2 * q + i]
            coef = sign * slope * w * share[2 * q + i]
            for t in range(b, e):
                if counts[t]:
                    d[t] = -coef * probs[t]
                    d[t, int(tokens[t])] += coef
    return total, pair_loss, seq, row_logp, d
