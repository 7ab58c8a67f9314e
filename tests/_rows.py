"""Definitions of the row operators (embeddings, norms, 8-bit checkpoints, token log-probabilities) in 64 bits, for the
tests: plain loops, written from the formulas in include/glr.h, on CPU tensors."""
import math

import torch

import _operators


def act_slope(z, name):
    """The activations' slopes; relu's at 0, which a code of 0 stands for, is 0."""
    return (z > 0).double() if name == "relu" else _operators.act_slope(z, name)


def lookup(E, tokens, scale):
    Y = torch.zeros(len(tokens), E.shape[1], dtype=torch.float64)
    for t, v in enumerate(tokens.tolist()):
        if 0 <= v < E.shape[0]:
            Y[t] = scale * E[v].double()
    return Y


def embedding_grad(dY, tokens, nodes, vocab, scale):
    """The gradients, and for each element the sum of absolute terms and the number of terms."""
    rows = dY.shape[0] // nodes
    ok = (tokens >= 0) & (tokens < vocab)
    at = (tokens.long() + vocab * (torch.arange(len(tokens)) // max(1, rows)))[ok]
    add = lambda x: torch.zeros(nodes * vocab, x.shape[1], dtype=torch.float64).index_add_(0, at, x[ok]).view(nodes, vocab, -1)  # noqa: E731
    d = dY.double()
    return add(scale * d), add(abs(scale) * d.abs()), add(torch.ones(len(tokens), 1, dtype=torch.float64))


def pack(X):
    """Codes, scale bytes and values of a matrix (float32 or bfloat16; exact in 64 bits)."""
    rows, cols = X.shape
    blocks = (cols + 31) // 32
    x = torch.nn.functional.pad(X.double(), (0, 32 * blocks - cols)).view(rows, blocks, 32)
    finite = torch.isfinite(x).all(2, keepdim=True)
    x = torch.where(finite, x, 0.0)
    # the smallest p with 2^p >= most / 127, a quotient that no rounding takes to a power of two from above
    part, p = torch.frexp(x.abs().amax(2, keepdim=True) / 127)
    p = torch.where(part == 0.5, p - 1, p)
    p = torch.where(part == 0, -127, p).clamp(-127, 121)
    codes = torch.round(x * 2.0 ** -p.double()).clamp(-127, 127)                    # ties to even
    values = torch.where(finite, codes * 2.0 ** p.double(), math.nan)
    flat = lambda t: t.reshape(rows, -1)[:, :cols]  # noqa: E731
    return flat(codes).to(torch.int8), torch.where(finite, p + 127, 255)[:, :, 0].to(torch.uint8), flat(values)


def norm(X, residual, weight, eps):
    S = X.double() + (0 if residual is None else residual.double())
    rstd = 1 / torch.sqrt((S * S).mean(1) + eps)
    Y = S * rstd[:, None] * (1 if weight is None else weight.double())
    return S, rstd, Y


def norm_grad(dY, H, rstd, weight, residual, nodes):
    x = H.double() * rstd.double()[:, None]
    g = dY.double() * (1 if weight is None else weight.double())
    dX = rstd.double()[:, None] * (g - x * (g * x).mean(1, keepdim=True))
    if residual is not None:
        dX = dX + residual.double()
    dw = (dY.double() * x).view(nodes, -1, H.shape[1]).sum(1)
    return dX, dw


def token_logp(logits, tokens, tau, topk):
    """logp, lse, entropy, and the alternatives, of finite or ruled-out logits."""
    rows, vocab = logits.shape
    logp, lse, ent = (torch.zeros(rows, dtype=torch.float64) for _ in range(3))
    top = torch.full((rows, topk), -math.inf, dtype=torch.float64)
    ids = torch.full((rows, topk), -1, dtype=torch.int64)
    for t in range(rows):
        z = logits[t].double()
        if float(z.max()) == -math.inf:
            lse[t] = -math.inf
            continue
        x = z / tau
        m = x.max()
        e = torch.exp(x - m)
        lse[t] = m + torch.log(e.sum())
        lp = (x - m) - torch.log(e.sum())
        p = lp.exp()
        ent[t] = -torch.where(p > 0, p * lp, 0.0).sum()
        y = int(tokens[t]) if tokens is not None else -1
        if 0 <= y < vocab:
            logp[t] = lp[y]
        order = sorted((v for v in range(vocab) if float(z[v]) != -math.inf), key=lambda v: (-float(z[v]), v))[:topk]
        for q, v in enumerate(order):
            top[t, q], ids[t, q] = lp[v], v
    return logp, lse, ent, top, ids
