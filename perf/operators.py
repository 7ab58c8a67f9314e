"""The operators around a compressed training step, as timed cases.

GreedyLore takes the nodes' gradients of a layer matrix.  The operators here make them: the layers' products
with their epilogues and gradients, and the losses on the logits that the last layer gives, each with the
gradient that the backward pass starts from.

* ``linear``      Y = act(X W^T + b) + R, and the pre-activation that the backward pass reads;
* ``grad``        a layer's backward pass: the gradient of its input with the activation below it,
                  (dZ W + D) act'(Z), and every node's gradient of the weights and the bias, dZ_i^T X_i and
                  the column sums of dZ_i, as ``GreedyLore.step`` takes them;
* ``distill``     distillation from a teacher's top logits: KL(q || softmax(z / tau)) with q the softmax of
                  the teacher's logits at its top ids, and the cross entropy of a label, with d loss / d z;
* ``preference``  a loss on the log ratios of pairs of answers (sigmoid with label smoothing, or squared),
                  from the packed tokens' logits to their gradient;
* ``policy``      the clipped policy loss with a KL term to a reference, per token, with its gradient.

``run`` gives each operator's outputs whole, from elementary torch operations in 32 bits, or with ``own`` from
the package's entry points.  ``exact`` is the same from the definitions in 64 bits.
"""
import math

import torch

own = False            # set from outside: run() uses the package's operators
_glr = None


def _package():
    global _glr
    if _glr is None:
        import paper_2507_08784_gb300 as glr
        _glr = glr
    return _glr


def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


# ---------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one row through a d = 2048 layer's square matrix: latency, and the weights' bytes
        dict(name="linear-one-row", op="linear", dtype="bf16", rows=1, k=2048, n=2048, act="silu", bias=True,
             residual=False, preact=False, pad=0),
        # a classifier head or small embedding whose sizes fit no tile, in 32 bits
        dict(name="linear-ragged", op="linear", dtype="f32", rows=555, k=777, n=333, act="gelu", bias=True,
             residual=True, preact=True, pad=1),
        # the widening product of a d = 4096 feed-forward block over eight sequences of 1024 tokens
        dict(name="linear-ffn", op="linear", dtype="bf16", rows=8192, k=4096, n=11008, act="silu", bias=False,
             residual=False, preact=True, pad=0),
        # the smallest backward pass: the 256 x 128 matrix of four nodes with 32 rows each
        dict(name="grad-small", op="grad", dtype="f32", gdtype="f32", nodes=4, rows=32, k=128, n=256, act="gelu_tanh",
             residual=False, bias=True, pad=0),
        # a d = 2048 block's 5632 x 2048 matrix for eight nodes with 1024 tokens each
        dict(name="grad-ffn", op="grad", dtype="bf16", gdtype="bf16", nodes=8, rows=1024, k=2048, n=5632, act="silu",
             residual=True, bias=True, pad=0),
        # a small student with few classes: launches and latency
        dict(name="distill-small", op="distill", dtype="f32", rows=64, vocab=1000, topk=8, tau=1.0, soft=1.0, hard=0.0,
             weights=False, banned=0, pad=0),
        # language-model distillation: four sequences of 1024 tokens, 64 teacher logits a token, half hard labels
        dict(name="distill", op="distill", dtype="bf16", rows=4096, vocab=32768, topk=64, tau=2.0, soft=2.0, hard=0.5,
             weights=True, banned=0, pad=0),
        # the same with a large vocabulary of odd size: rows that begin at every alignment
        dict(name="distill-large", op="distill", dtype="bf16", rows=8192, vocab=131071, topk=128, tau=1.0, soft=1.0,
             hard=0.0, weights=True, banned=0, pad=0),
        # three pairs of short answers, odd vocabulary, 32 bits
        dict(name="preference-small", op="preference", dtype="f32", pairs=3, longest=40, vocab=5003, kind="ipo", beta=0.1,
             smoothing=0.0, average=True, ref=True, pad=0),
        # a node's batch of preference training: eight pairs of answers of up to 1024 tokens
        dict(name="preference", op="preference", dtype="bf16", pairs=8, longest=1024, vocab=32768, kind="sigmoid", beta=0.1,
             smoothing=0.1, average=False, ref=True, pad=0),
        # one short sampled answer
        dict(name="policy-small", op="policy", dtype="bf16", rows=33, vocab=32768, tau=1.0, low=0.2, high=0.2, kl=0.0,
             weights=True, banned=0, pad=0),
        # a node's sampled answers, with the reference policy's KL term and a part of the vocabulary ruled out
        dict(name="policy", op="policy", dtype="bf16", rows=6000, vocab=65536, tau=0.7, low=0.2, high=0.28, kl=0.05,
             weights=True, banned=500, pad=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    v = _log(rng, lo, hi)
    how = rng.random()
    v = max(8, v - v % 8) if how < 0.4 else v | 1 if how < 0.7 else v
    return 3080 if v == 3072 else v


def draw(rng):
    op = rng.choice(["linear", "grad", "distill", "preference", "policy"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([0, 0, 0, 8, 3])
    if op in ("linear", "grad"):
        most = 2e11 if dtype == "bf16" else 5e10
        act = rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])
        while True:
            nodes = rng.choice([1, 2, 4, 8]) if op == "grad" else 1
            rows, k, n = _log(rng, 1, 8192 // nodes), _size(rng, 64, 11008), _size(rng, 64, 11008)
            if 2.0 * nodes * rows * k * n <= most:
                break
        if op == "linear":
            return dict(op=op, dtype=dtype, rows=rows, k=k, n=n, act=act, bias=rng.random() < 0.5,
                        residual=rng.random() < 0.5, preact=act != "none" and rng.random() < 0.7, pad=pad)
        return dict(op=op, dtype=dtype, gdtype=rng.choice([dtype, "f32"]), nodes=nodes, rows=rows, k=k, n=n, act=act,
                    residual=rng.random() < 0.5, bias=rng.random() < 0.5, pad=pad)
    most = 4e8 if dtype == "bf16" else 2e8
    vocab = _size(rng, 500, 131072)
    if op == "preference":
        longest = _log(rng, 1, 1024)
        while True:
            pairs = _log(rng, 1, 16)
            if 1.5 * pairs * longest * vocab <= most:
                break
            longest = max(1, longest * 2 // 3)
        kind = rng.choice(["sigmoid", "ipo"])
        return dict(op=op, dtype=dtype, pairs=pairs, longest=longest, vocab=vocab, kind=kind,
                    beta=rng.choice([0.05, 0.1, 0.5]), smoothing=rng.choice([0.0, 0.1]) if kind == "sigmoid" else 0.0,
                    average=kind == "ipo", ref=rng.random() < 0.8, pad=pad)
    rows = _log(rng, 1, max(1, min(8192, int(most / vocab))))
    if op == "policy":
        return dict(op=op, dtype=dtype, rows=rows, vocab=vocab, tau=rng.choice([1.0, 0.7, 1.3]), low=0.2,
                    high=rng.choice([0.2, 0.28]), kl=rng.choice([0.0, 0.02, 0.1]), weights=rng.random() < 0.7,
                    banned=rng.choice([0, 0, 100]), pad=pad)
    hard = rng.choice([0.0, 0.5])
    return dict(op=op, dtype=dtype, rows=rows, vocab=vocab, topk=_log(rng, 1, 256), tau=rng.choice([1.0, 2.0, 4.0]),
                soft=rng.choice([1.0, 4.0]), hard=hard, weights=rng.random() < 0.7, banned=rng.choice([0, 0, 100]), pad=pad)


def work(case):
    b = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op == "linear":
        m, k, n = case["rows"], case["k"], case["n"]
        out = 1 + bool(case["preact"]) + bool(case["residual"])
        return {"bytes": b * (m * k + n * k + out * m * n + (n if case["bias"] else 0)), "flops": 2.0 * m * n * k}
    if op == "grad":
        g = 2 if case["gdtype"] == "bf16" else 4
        m, k, n = case["nodes"] * case["rows"], case["k"], case["n"]
        extra = (case["act"] != "none") + bool(case["residual"])
        small = case["nodes"] * n * g if case["bias"] else 0
        return {"bytes": b * (m * n + n * k + m * k * (2 + extra)) + g * case["nodes"] * n * k + small,
                "flops": 4.0 * m * n * k}
    # logits of rows that do not count need not be read; their gradient, zero, is written
    if op == "preference":
        t, read, p = sum(_lengths(case)), sum(n - n // 4 for n in _lengths(case)), case["pairs"]
        return {"bytes": b * (t + read) * case["vocab"] + 8 * t + 16 * t + 8 * 5 * p, "flops": 8.0 * read * case["vocab"]}
    t, v = case["rows"], case["vocab"]
    read = 0.875 * t if case["weights"] else t
    side = t * case["topk"] * (4 + b) + 12 * t if op == "distill" else 32 * t
    return {"bytes": b * (t + read) * v + side, "flops": (8.0 if op == "policy" else 12.0) * read * v}


# --------------------------------------------------------------------------------------------------- inputs

def _lengths(case):
    """Lengths of the 2 P answers: the longest, a single token, and others between, fixed by the case."""
    most, state, out = case["longest"], 12345, []
    for i in range(2 * case["pairs"]):
        state = (1103515245 * state + 12345) % (1 << 31)
        out.append(most if i == 0 else 1 if i == 1 else 1 + state % most)
    return out


def _matrix(g, rows, cols, dt, scale, pad):
    """rows x cols in rows of cols + pad elements."""
    x = torch.empty(rows, cols + pad, device="cuda", dtype=dt)
    x.normal_(0.0, 1.0, generator=g).mul_(scale)
    return x[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, op, pad = _dt(case["dtype"]), case["op"], case["pad"]
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    s = dict(case=case)
    if op == "linear":
        m, k, n = case["rows"], case["k"], case["n"]
        s["X"] = _matrix(g, m, k, dt, 1.0, pad)
        s["W"] = _matrix(g, n, k, dt, k ** -0.5, pad)
        s["bias"] = (0.5 * rand(n)).to(dt) if case["bias"] else None
        s["residual"] = _matrix(g, m, n, dt, 1.0, pad) if case["residual"] else None
        s["Y"] = torch.empty(m, n + pad, device="cuda", dtype=dt)[:, :n]
        s["preact"] = torch.empty(m, n, device="cuda", dtype=dt) if case["preact"] else None
        return s
    if op == "grad":
        m, k, n, nodes, gd = case["nodes"] * case["rows"], case["k"], case["n"], case["nodes"], _dt(case["gdtype"])
        s["dZ"] = _matrix(g, m, n, dt, 0.02, pad)
        s["W"] = _matrix(g, n, k, dt, n ** -0.5, pad)
        s["X"] = _matrix(g, m, k, dt, 1.0, pad)
        s["preact"] = _matrix(g, m, k, dt, 1.0, pad) if case["act"] != "none" else None
        s["residual"] = _matrix(g, m, k, dt, 0.02, pad) if case["residual"] else None
        s["dX"] = torch.empty(m, k, device="cuda", dtype=dt)
        s["dW"] = [torch.empty(n, k, device="cuda", dtype=gd) for _ in range(nodes)]
        s["db"] = [torch.empty(n, device="cuda", dtype=gd) for _ in range(nodes)] if case["bias"] else None
        return s
    v = case["vocab"]
    rows = sum(_lengths(case)) if op == "preference" else case["rows"]
    z = _matrix(g, rows, v, dt, 1.5, pad)
    s["logits"] = z
    s["dlogits"] = torch.empty(rows, v + pad, device="cuda", dtype=dt)[:, :v]
    s["loss"] = torch.empty(1, device="cuda")
    draw_ids = lambda n: torch.randint(0, v, (n,), device="cuda", generator=g)  # noqa: E731
    at = torch.arange(rows, device="cuda")
    if op == "distill":
        k = min(case["topk"], v)
        step = torch.randint(1, max(2, v // k), (rows, 1), device="cuda", generator=g)
        ids = (draw_ids(rows)[:, None] + step * torch.arange(k, device="cuda")) % v       # distinct in a row
        teacher = (2.0 * rand(rows, k)).sort(dim=1, descending=True).values
        z.scatter_(1, ids, (2.0 + teacher + 0.5 * rand(rows, k)).to(dt))
        ids = ids.to(torch.int32)
        if k > 1:
            ids[::7, -1] = -1                                                                # a shorter list
        s.update(teacher=teacher.to(dt), ids=ids, row_loss=torch.empty(rows, device="cuda"))
        s["labels"] = draw_ids(rows) if case["hard"] else None
        if case["banned"]:
            z[:, :case["banned"]] = -math.inf
            s["ids"] = torch.where((ids >= 0) & (ids < case["banned"]), -1, ids).to(torch.int32)
            s["labels"] = None if s["labels"] is None else s["labels"].clamp(min=case["banned"])
        s["weight"] = _weights(g, rows) if case["weights"] else None
        return s
    tokens = draw_ids(rows).clamp(min=case.get("banned", 0))
    z[at, tokens] += math.log(v) + 0.5                                                       # about 0.4 of the mass
    if case.get("banned"):
        z[:, :case["banned"]] = -math.inf
    if op == "policy":
        zt = z.float() / case["tau"]
        logp = zt[at, tokens] - torch.logsumexp(zt, 1)
        del zt
        s.update(tokens=tokens, old_logp=logp + 0.2 * rand(rows), advantage=0.5 + rand(rows),
                 ref_logp=logp + 0.3 * rand(rows) if case["kl"] else None, logp=torch.empty(rows, device="cuda"),
                 row_loss=torch.empty(rows, device="cuda"), weight=_weights(g, rows) if case["weights"] else None)
        return s
    lengths = _lengths(case)
    s["sequence"] = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"),
                                            torch.tensor(lengths, device="cuda"))
    s["offsets"] = torch.tensor([0] + lengths, device="cuda").cumsum(0)
    start = s["offsets"][s["sequence"]]
    prompt = (at - start) < (s["offsets"][s["sequence"] + 1] - start) // 4                     # a quarter is prompt
    s["tokens"] = torch.where(prompt, -1, tokens)
    counted = s["tokens"] >= 0
    zf = z.float()
    logp = torch.where(counted, zf[at, tokens] - torch.logsumexp(zf, 1), 0.0)
    del zf
    per = lambda x: torch.stack([y.sum() for y in x.double().split(lengths)])  # noqa: E731
    seq = per(logp) / (per(counted).clamp(min=1) if case["average"] else 1)
    s["ref_logp"] = (seq + (1.0 if case["average"] else 3.0) * rand(len(lengths))).float() if case["ref"] else None
    s.update(pair_loss=torch.empty(case["pairs"], device="cuda"), seq_logp=torch.empty(len(lengths), device="cuda"),
             row_logp=torch.empty(rows, device="cuda"),
             workspace=torch.empty(4 * rows + 16 * case["pairs"] + 1024, device="cuda"))
    return s


def _weights(g, rows):
    """Weights of a masked mean: an eighth of the rows does not count."""
    w = (torch.rand(rows, device="cuda", generator=g) > 0.125).float()
    return w / w.sum().clamp(min=1)


# ------------------------------------------------------------------------------------------------------ run

def run(s):
    return (_own if own else _plain)[s["case"]["op"]](s)


def _own_linear(s):
    c = s["case"]
    _package().glr_linear(s["X"], s["W"], s["Y"], bias=s["bias"], act=c["act"], residual=s["residual"], preact=s["preact"])
    return {"y": s["Y"], "preact": s["preact"]}


def _own_grad(s):
    c, glr = s["case"], _package()
    glr.glr_linear_grad_input(s["dZ"], s["W"], s["dX"], residual=s["residual"], preact=s["preact"], act=c["act"])
    glr.glr_linear_grad_weight(s["dZ"], s["X"], s["dW"], db=s["db"])
    return {"dx": s["dX"], "dw": s["dW"], "db": s["db"]}


def _own_distill(s):
    c = s["case"]
    _package().glr_distill_loss(s["logits"], s["teacher"], s["ids"], loss=s["loss"], row_loss=s["row_loss"],
                                dlogits=s["dlogits"], labels=s["labels"], weight=s["weight"], temperature=c["tau"],
                                soft=c["soft"], hard=c["hard"])
    return {"loss": s["loss"], "row_loss": s["row_loss"], "dlogits": s["dlogits"]}


def _own_preference(s):
    c = s["case"]
    _package().glr_preference_loss(s["logits"], s["tokens"], s["offsets"], loss=s["loss"], pair_loss=s["pair_loss"],
                                   seq_logp=s["seq_logp"], row_logp=s["row_logp"], workspace=s["workspace"],
                                   dlogits=s["dlogits"], ref_logp=s["ref_logp"], kind=c["kind"], beta=c["beta"],
                                   smoothing=c["smoothing"], average=c["average"])
    return {"loss": s["loss"], "pair_loss": s["pair_loss"], "seq_logp": s["seq_logp"], "row_logp": s["row_logp"],
            "dlogits": s["dlogits"]}


def _own_policy(s):
    c = s["case"]
    _package().glr_policy_loss(s["logits"], s["tokens"], s["old_logp"], s["advantage"], loss=s["loss"],
                               row_loss=s["row_loss"], logp=s["logp"], dlogits=s["dlogits"], ref_logp=s["ref_logp"],
                               weight=s["weight"], temperature=c["tau"], clip_low=c["low"], clip_high=c["high"],
                               kl=c["kl"])
    return {"loss": s["loss"], "row_loss": s["row_loss"], "logp": s["logp"], "dlogits": s["dlogits"]}


def _act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, 0.0)
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _plain_linear(s):
    dt = s["X"].dtype
    z = s["X"].float() @ s["W"].float().T
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, s["case"]["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(dt), "preact": None if s["preact"] is None else z.to(dt)}


def _plain_grad(s):
    c, dt = s["case"], s["dZ"].dtype
    dz, x = s["dZ"].float(), s["X"].float()
    dx = dz @ s["W"].float()
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    if s["preact"] is not None:
        dx = dx * _act_slope(s["preact"].float(), c["act"])
    dzn, xn, gd = dz.view(c["nodes"], c["rows"], -1), x.view(c["nodes"], c["rows"], -1), _dt(c["gdtype"])
    dw = torch.matmul(dzn.transpose(1, 2), xn).to(gd)
    db = None if s["db"] is None else list(dzn.sum(1).to(gd))
    return {"dx": dx.to(dt), "dw": list(dw), "db": db}


def _softmax(z):
    m = z.max(dim=1, keepdim=True).values
    lse = m + torch.log(torch.exp(z - m).sum(dim=1, keepdim=True))
    return torch.exp(z - lse), lse[:, 0]


def _plain_distill(s):
    c, z = s["case"], s["logits"].float()
    rows, v = z.shape
    w = s["weight"] if s["weight"] is not None else torch.full((rows,), 1.0 / rows, device="cuda")
    p, lse = _softmax(z / c["tau"])
    valid = (s["ids"] >= 0) & (s["ids"] < v)
    ids = torch.where(valid, s["ids"], 0).long()
    a = torch.where(valid, s["teacher"].float() / c["tau"], -math.inf)
    some = valid.any(dim=1, keepdim=True)
    q = torch.where(valid & some, torch.exp(a - torch.where(some, a.max(dim=1, keepdim=True).values, 0.0)), 0.0)
    q = q / torch.where(some, q.sum(dim=1, keepdim=True), 1.0)
    zq = z.gather(1, ids) / c["tau"]
    row = c["soft"] * torch.where(q > 0, q * (torch.log(torch.where(q > 0, q, 1.0)) - zq + lse[:, None]), 0.0).sum(1)
    d = (c["soft"] / c["tau"]) * p * some
    d.scatter_add_(1, ids, (-c["soft"] / c["tau"]) * q)
    if s["labels"] is not None:
        p1, lse1 = _softmax(z)
        row = row + c["hard"] * (lse1 - z.gather(1, s["labels"][:, None])[:, 0])
        d += c["hard"] * p1
        d.scatter_add_(1, s["labels"][:, None], torch.full((rows, 1), -c["hard"], device="cuda"))
    row = torch.where(w != 0, row, 0.0)
    d = torch.where((w != 0)[:, None], d * w[:, None], 0.0)
    return {"loss": (w * row).sum().view(1), "row_loss": row, "dlogits": d.to(s["logits"].dtype)}


def _plain_preference(s):
    c, z, tokens = s["case"], s["logits"].float(), s["tokens"]
    counted = tokens >= 0
    at = torch.where(counted, tokens, 0)[:, None]
    p, lse = _softmax(z)
    row = torch.where(counted, z.gather(1, at)[:, 0] - lse, 0.0)
    seqs = 2 * c["pairs"]
    member = (s["sequence"][:, None] == torch.arange(seqs, device="cuda")).float()
    seq = (member * row[:, None]).sum(0)
    length = (member * counted.float()[:, None]).sum(0).clamp(min=1)
    share = 1 / length if c["average"] else torch.ones_like(length)
    seq = seq * share
    ratio = seq if s["ref_logp"] is None else seq - s["ref_logp"]
    h = ratio[0::2] - ratio[1::2]
    if c["kind"] == "ipo":
        e = h - 1 / (2 * c["beta"])
        pair, slope = e * e, 2 * e
    else:
        up, down = 1 / (1 + torch.exp(-c["beta"] * h)), 1 / (1 + torch.exp(c["beta"] * h))
        pair = -(1 - c["smoothing"]) * torch.log(up) - c["smoothing"] * torch.log(down)
        slope = c["beta"] * (-(1 - c["smoothing"]) * down + c["smoothing"] * up)
    coef = torch.stack([slope, -slope], 1).view(-1) * share / c["pairs"]
    coef = torch.where(counted, coef[s["sequence"]], 0.0)[:, None]
    d = -coef * p
    d.scatter_add_(1, at, coef)
    return {"loss": pair.sum().view(1) / c["pairs"], "pair_loss": pair, "seq_logp": seq, "row_logp": row,
            "dlogits": d.to(s["logits"].dtype)}


def _plain_policy(s):
    c, z = s["case"], s["logits"].float() / s["case"]["tau"]
    rows = z.shape[0]
    w = s["weight"] if s["weight"] is not None else torch.full((rows,), 1.0 / rows, device="cuda")
    at, adv = s["tokens"][:, None], s["advantage"]
    p, lse = _softmax(z)
    logp = z.gather(1, at)[:, 0] - lse
    ratio = torch.exp(logp - s["old_logp"])
    row = -torch.minimum(ratio * adv, ratio.clamp(1 - c["low"], 1 + c["high"]) * adv)
    open_ = torch.where(adv > 0, ratio <= 1 + c["high"], ratio >= 1 - c["low"])
    slope = torch.where(open_, -adv * ratio, 0.0)
    if s["ref_logp"] is not None:
        e = s["ref_logp"] - logp
        row = row + c["kl"] * (torch.exp(e) - e - 1)
        slope = slope + c["kl"] * (1 - torch.exp(e))
    coef = (slope * w / c["tau"])[:, None]
    d = -coef * p
    d.scatter_add_(1, at, coef)
    row, logp = torch.where(w != 0, row, 0.0), torch.where(w != 0, logp, 0.0)
    d = torch.where((w != 0)[:, None], d, 0.0)
    return {"loss": (w * row).sum().view(1), "row_loss": row, "logp": logp, "dlogits": d.to(s["logits"].dtype)}


_own = dict(linear=_own_linear, grad=_own_grad, distill=_own_distill, preference=_own_preference, policy=_own_policy)
_plain = dict(linear=_plain_linear, grad=_plain_grad, distill=_plain_distill, preference=_plain_preference,
              policy=_plain_policy)


# ------------------------------------------------------------------------------------- definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return dict(linear=_exact_linear, grad=_exact_grad, distill=_exact_rows, preference=_exact_preference,
                policy=_exact_rows)[case["op"]](s)


def _exact_act(z, name):
    """The activation and its derivative, the latter by differentiating the former."""
    z = z.detach().requires_grad_(True)
    with torch.enable_grad():
        if name == "relu":
            y = torch.nn.functional.relu(z)
        elif name == "silu":
            y = z * torch.sigmoid(z)
        elif name == "gelu":
            y = z * torch.special.ndtr(z)
        elif name == "gelu_tanh":
            y = z * torch.sigmoid(2 * (2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3))
        else:
            y = z * 1.0
        (slope,) = torch.autograd.grad(y.sum(), z)
    return y.detach(), slope


def _exact_linear(s):
    z = torch.nn.functional.linear(s["X"].double(), s["W"].double(), None if s["bias"] is None else s["bias"].double())
    y = _exact_act(z, s["case"]["act"])[0] + (0 if s["residual"] is None else s["residual"].double())
    return {"y": y, "preact": None if s["preact"] is None else z}


def _exact_grad(s):
    c = s["case"]
    dz, x = s["dZ"].double(), s["X"].double()
    g = torch.einsum("mn,nk->mk", dz, s["W"].double()) + (0 if s["residual"] is None else s["residual"].double())
    if s["preact"] is not None:
        g = g * _exact_act(s["preact"].double(), c["act"])[1]
    parts = [slice(i * c["rows"], (i + 1) * c["rows"]) for i in range(c["nodes"])]
    return {"dx": g, "dw": [torch.einsum("mn,mk->nk", dz[p], x[p]) for p in parts],
            "db": None if s["db"] is None else [dz[p].sum(0) for p in parts]}


def _chunks(rows, vocab):
    size = max(1, (1 << 27) // vocab)
    return [slice(i, min(rows, i + size)) for i in range(0, rows, size)]


def _exact_rows(s):
    """Distillation and policy loss: the rows' losses as functions of the logits, differentiated."""
    c = s["case"]
    rows, v = s["logits"].shape
    grad = torch.empty(rows, v, device="cuda", dtype=torch.float64)
    row, logp = (torch.zeros(rows, device="cuda", dtype=torch.float64) for _ in range(2))
    w = s["weight"].double() if s["weight"] is not None else torch.full((rows,), 1.0 / rows, device="cuda").double()
    for part in _chunks(rows, v):
        z = s["logits"][part].double().requires_grad_(True)
        with torch.enable_grad():
            if c["op"] == "distill":
                zero = torch.zeros((), device="cuda", dtype=torch.float64)
                lp = torch.log_softmax(z / c["tau"], 1)
                ids = s["ids"][part].long()
                a = (s["teacher"][part].double() / c["tau"]).masked_fill(ids < 0, -math.inf)
                has = (ids >= 0).any(1)
                lq = torch.log_softmax(torch.where(has[:, None], a, zero), 1)
                term = lq.exp() * (lq - lp.gather(1, ids.clamp(min=0)))
                loss = c["soft"] * torch.where((ids >= 0) & has[:, None], term, zero).sum(1)
                if s["labels"] is not None:
                    loss = loss - c["hard"] * torch.log_softmax(z, 1).gather(1, s["labels"][part][:, None])[:, 0]
            else:
                lp = torch.log_softmax(z / c["tau"], 1).gather(1, s["tokens"][part][:, None])[:, 0]
                adv = s["advantage"][part].double()
                ratio = torch.exp(lp - s["old_logp"][part].double())
                stop = torch.where(adv > 0, torch.clamp(ratio, max=1 + c["high"]), torch.clamp(ratio, min=1 - c["low"]))
                loss = -stop * adv
                if s["ref_logp"] is not None:
                    e = s["ref_logp"][part].double() - lp
                    loss = loss + c["kl"] * (torch.expm1(e) - e)
                logp[part] = lp.detach()
            grad[part] = torch.autograd.grad((loss * w[part]).sum(), z)[0]
        row[part] = loss.detach()
    dead = w == 0
    row[dead], logp[dead], grad[dead] = 0, 0, 0
    out = {"loss": (w * row).sum().view(1), "row_loss": row, "dlogits": grad}
    return out if c["op"] == "distill" else {**out, "logp": logp}


def _exact_preference(s):
    c, off = s["case"], s["offsets"].tolist()
    rows, v = s["logits"].shape
    counted = s["tokens"] >= 0
    at = s["tokens"].clamp(min=0)
    row = torch.zeros(rows, device="cuda", dtype=torch.float64)
    for part in _chunks(rows, v):
        row[part] = torch.log_softmax(s["logits"][part].double(), 1).gather(1, at[part][:, None])[:, 0]
    row[~counted] = 0
    spans = [slice(off[i], off[i + 1]) for i in range(len(off) - 1)]
    seq = torch.stack([row[q].sum() / (counted[q].sum().clamp(min=1) if c["average"] else 1) for q in spans])
    leaf = seq.clone().requires_grad_(True)
    with torch.enable_grad():
        ratio = leaf if s["ref_logp"] is None else leaf - s["ref_logp"].double()
        h = ratio[::2] - ratio[1::2]
        if c["kind"] == "ipo":
            pair = (h - 0.5 / c["beta"]) ** 2
        else:
            soft = torch.nn.functional.softplus
            pair = (1 - c["smoothing"]) * soft(-c["beta"] * h) + c["smoothing"] * soft(c["beta"] * h)
        (slope,) = torch.autograd.grad(pair.mean(), leaf)
    coef = torch.zeros(rows, device="cuda", dtype=torch.float64)
    for i, q in enumerate(spans):
        coef[q] = slope[i] / (counted[q].sum().clamp(min=1) if c["average"] else 1)
    coef[~counted] = 0
    grad = torch.empty(rows, v, device="cuda", dtype=torch.float64)
    for part in _chunks(rows, v):
        grad[part] = -coef[part, None] * torch.softmax(s["logits"][part].double(), 1)
        grad[part] = grad[part].scatter_add(1, at[part][:, None], coef[part, None])
    return {"loss": pair.detach().mean().view(1), "pair_loss": pair.detach(), "seq_logp": seq, "row_logp": row, "dlogits": grad}
