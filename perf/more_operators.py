"""More operators around a compressed training step, as timed cases.

What stands around the layers' products and the losses: the embedding, whose matrix's gradient GreedyLore takes like
any other layer's, the norm between layers, what is kept of activations for the backward pass, and the
log-probabilities that the losses read.

* ``embedding``   ``lookup``: Y_t = scale E[token_t]; ``grad``: every node's gradient of E, scale times the sum of the
                  rows of dY of each token, zero for tokens that do not occur; a token outside the vocabulary is padding;
* ``norm``        ``forward``: H = X + R, Y = H rstd w with rstd = (mean H^2 + eps)^(-1/2), and Y in 8 bits with scales;
                  ``grad``: dX = rstd (w dY - x mean(w dY x)) + D with x = H rstd, and every node's sum of dY x;
* ``checkpoint``  ``save``: activations in 8 bits, for every 32 columns of a row a scale s, the smallest power of two with
                  |x| <= 127 s, and the codes round(x / s); ``grad``: a layer's backward pass from the saved
                  pre-activation Z of its input X = act(Z): dZ_i^T X and the column sums of dZ_i for every node, and
                  (dZ W + D) act'(Z);
* ``logp``        ``forward``: log softmax(z / tau) of every row's token, the logarithm of the sum, the entropy, and the
                  most probable alternatives (equal ones by index); ``grad``: the logits' gradient from those
                  of the log-probability and of the entropy.

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
        # a small student's vocabulary, four nodes with 32 tokens each, 32 bits: launches and latency
        dict(name="embedding-grad-small", op="embedding", way="grad", dtype="f32", gdtype="f32", nodes=4, rows=32, vocab=1000,
             d=128, scale=1.0, pad=0),
        # eight nodes with 1024 tokens each into a d = 2048 model's embedding
        dict(name="embedding-grad", op="embedding", way="grad", dtype="bf16", gdtype="bf16", nodes=8, rows=1024, vocab=32768,
             d=2048, scale=1.0, pad=0),
        # sixteen sequences of 1024 tokens from a d = 4096 model's large vocabulary, scaled by sqrt(d)
        dict(name="embedding-lookup", op="embedding", way="lookup", dtype="bf16", nodes=1, rows=16384, vocab=131071, d=4096,
             scale=64.0, pad=0),
        # one token through a d = 2048 model's norm
        dict(name="norm-one-row", op="norm", way="forward", dtype="bf16", nodes=1, rows=1, n=2048, residual=True, weight=True,
             packed=True, pad=0),
        # eight sequences of 1024 tokens between the blocks of a d = 4096 model, the output saved for the backward pass
        dict(name="norm", op="norm", way="forward", dtype="bf16", nodes=1, rows=8192, n=4096, residual=True, weight=True,
             packed=True, pad=0),
        # its backward pass for eight nodes
        dict(name="norm-grad", op="norm", way="grad", dtype="bf16", gdtype="f32", nodes=8, rows=1024, n=4096, residual=True,
             weight=True, pad=0),
        # a layer whose sizes fit no tile and no block of columns, in 32 bits
        dict(name="checkpoint-grad-small", op="checkpoint", way="grad", dtype="f32", gdtype="f32", nodes=2, rows=111, k=333, n=157,
             act="gelu", residual=True, bias=True, pad=1),
        # the widened activations of a d = 2048 feed-forward block, eight sequences of 1024 tokens
        dict(name="checkpoint-save", op="checkpoint", way="save", dtype="bf16", nodes=1, rows=8192, k=5632, pad=0),
        # the backward pass of the block's narrowing product for eight nodes, its input from the saved pre-activation
        dict(name="checkpoint-grad", op="checkpoint", way="grad", dtype="bf16", gdtype="bf16", nodes=8, rows=1024, k=5632, n=2048,
             act="silu", residual=False, bias=True, pad=0),
        # one sampled token with its alternatives
        dict(name="logp-one-row", op="logp", way="forward", dtype="bf16", rows=1, vocab=32768, topk=16, tau=1.0, entropy=True,
             banned=0, pad=0),
        # a teacher's top logits for distillation, four sequences of 1024 tokens, a large vocabulary of odd size
        dict(name="logp", op="logp", way="forward", dtype="bf16", rows=4096, vocab=131071, topk=64, tau=0.7, entropy=True,
             banned=500, pad=0),
        # the gradient of a policy's log-probabilities with a bonus for its entropy
        dict(name="logp-grad", op="logp", way="grad", dtype="bf16", rows=6000, vocab=65536, topk=0, tau=1.0, entropy=True,
             banned=0, pad=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    v = _log(rng, lo, hi)
    how = rng.random()
    return max(8, v - v % 8) if how < 0.4 else v | 1 if how < 0.7 else v


def draw(rng):
    op = rng.choice(["embedding", "norm", "checkpoint", "logp"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    small = 1 if dtype == "bf16" else 2
    pad = rng.choice([0, 0, 0, 8, 3])
    nodes = rng.choice([1, 2, 4, 8])
    if op == "embedding":
        way = rng.choice(["lookup", "grad", "grad"])
        if way == "lookup":
            while True:
                vocab, d, rows = _size(rng, 500, 131072), _size(rng, 64, 8192), _log(rng, 1, 16384)
                if small * rows * d <= 6.7e7 and small * vocab * d <= 5.4e8:
                    break
            return dict(op=op, way=way, dtype=dtype, nodes=1, rows=rows, vocab=vocab, d=d, scale=rng.choice([1.0, 16.0, d ** 0.5]),
                        pad=pad)
        gdtype = rng.choice([dtype, "f32"])
        while True:
            vocab, d, rows = _size(rng, 500, 131072), _size(rng, 64, 8192), _log(rng, 1, 32768 // nodes)
            if (1 if gdtype == "bf16" else 2) * nodes * vocab * d <= 5e8 and small * nodes * rows * d <= 3e7:
                break
        return dict(op=op, way=way, dtype=dtype, gdtype=gdtype, nodes=nodes, rows=rows, vocab=vocab, d=d,
                    scale=rng.choice([1.0, 16.0, d ** 0.5]), pad=pad)
    if op == "norm":
        way = rng.choice(["forward", "grad"])
        nodes = nodes if way == "grad" else 1
        while True:
            rows, n = _log(rng, 1, 16384 // nodes), _size(rng, 64, 16384)
            if small * nodes * rows * n <= 3.3e7:
                break
        if way == "grad":
            return dict(op=op, way=way, dtype=dtype, gdtype=rng.choice([dtype, "f32"]), nodes=nodes, rows=rows, n=n,
                        residual=rng.random() < 0.5, weight=rng.random() < 0.8, pad=pad)
        return dict(op=op, way=way, dtype=dtype, nodes=1, rows=rows, n=n, residual=rng.random() < 0.7,
                    weight=rng.random() < 0.8, packed=rng.random() < 0.6, pad=pad)
    if op == "checkpoint":
        if rng.random() < 0.4:
            while True:
                rows, k = _log(rng, 1, 16384), _size(rng, 64, 16384)
                if small * rows * k <= 4.6e7:
                    break
            return dict(op=op, way="save", dtype=dtype, nodes=1, rows=rows, k=k, pad=pad)
        most = 1.8e11 if dtype == "bf16" else 4e10
        while True:
            rows, k, n = _log(rng, 1, 8192 // nodes), _size(rng, 64, 11008), _size(rng, 64, 11008)
            if 2.0 * nodes * rows * k * n <= most and nodes * n * k <= 1.2e8:
                break
        return dict(op=op, way="grad", dtype=dtype, gdtype=dtype, nodes=nodes, rows=rows, k=k, n=n,
                    act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), residual=rng.random() < 0.5,
                    bias=rng.random() < 0.5, pad=pad)
    way = rng.choice(["forward", "forward", "grad"])
    vocab = _size(rng, 500, 131072)
    rows = _log(rng, 1, max(1, min(8192, int((4e8 if dtype == "bf16" else 2e8) / vocab))))
    return dict(op=op, way=way, dtype=dtype, rows=rows, vocab=vocab, topk=rng.choice([0, _log(rng, 1, 256)]) if way == "forward" else 0,
                tau=rng.choice([1.0, 0.7, 1.3]), entropy=rng.random() < 0.7, banned=rng.choice([0, 0, 100]), pad=pad)


def work(case):
    b = 2 if case["dtype"] == "bf16" else 4
    op, way = case["op"], case["way"]
    g = 2 if case.get("gdtype") == "bf16" else 4
    if op == "embedding":
        t, d = case["nodes"] * case["rows"], case["d"]
        if way == "lookup":
            return {"bytes": 4 * t + 2.0 * b * t * d, "flops": 1.0 * t * d}
        return {"bytes": 4 * t + 0.9375 * b * t * d + 1.0 * g * case["nodes"] * case["vocab"] * d, "flops": 1.0 * t * d}
    if op == "norm":
        t, n = case["nodes"] * case["rows"], case["n"]
        if way == "forward":
            # the codes are written, and read once more for the values that they stand for
            packed = 2 * (t * n + t * ((n + 31) // 32)) + 2 * t * n if case["packed"] else 0
            return {"bytes": (4 if case["residual"] else 2) * b * t * n + 4 * t + b * n + packed, "flops": 8.0 * t * n}
        return {"bytes": (4 if case["residual"] else 3) * b * t * n + 4 * t + b * n + g * case["nodes"] * n, "flops": 12.0 * t * n}
    if op == "checkpoint":
        t, k = case["nodes"] * case["rows"], case["k"]
        codes = t * k + t * ((k + 31) // 32)
        if way == "save":
            return {"bytes": b * t * k + 2 * codes + 2 * t * k, "flops": 3.0 * t * k}
        n = case["n"]
        small = case["nodes"] * n * g if case["bias"] else 0
        return {"bytes": codes + b * (t * n + n * k + t * k * (2 if case["residual"] else 1)) + g * case["nodes"] * n * k + small,
                "flops": 4.0 * t * n * k}
    t, v = case["rows"], case["vocab"]
    if way == "forward":
        return {"bytes": b * t * v + (16 + 8 * case["topk"]) * t, "flops": 8.0 * t * v}
    return {"bytes": 2 * b * t * v + 20 * t, "flops": 8.0 * t * v}


# --------------------------------------------------------------------------------------------------- inputs

def _matrix(g, rows, cols, dt, scale, pad):
    """rows x cols in rows of cols + pad elements."""
    x = torch.empty(rows, cols + pad, device="cuda", dtype=dt)
    x.normal_(0.0, 1.0, generator=g).mul_(scale)
    return x[:, :cols]


def _out(rows, cols, dt, pad=0):
    return torch.empty(rows, cols + pad, device="cuda", dtype=dt)[:, :cols]


def _saved(x):
    """The codes (int8) and scales (their exponents, biased by 127) of a 32-bit matrix."""
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    y = torch.zeros(rows, 32 * blocks, device="cuda")
    y[:, :cols] = x
    y = y.view(rows, blocks, 32)
    part, power = torch.frexp(y.abs().amax(2))                     # part 2^power, 0.5 <= part < 1
    power = (power - 7 + (part > 127 / 128).int()).clamp(min=-127)
    codes = torch.round(torch.ldexp(y, -power[:, :, None])).to(torch.int8)
    return codes.view(rows, -1)[:, :cols].contiguous(), (power + 127).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, gd, op, way, pad = _dt(case["dtype"]), _dt(case.get("gdtype")), case["op"], case["way"], case["pad"]
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    s = dict(case=case)
    rows = case.get("nodes", 1) * case["rows"]
    if op == "embedding":
        v, d = case["vocab"], case["d"]
        # words by rank as 1 / rank, in an order of their own; a sixteenth of the rows is padding
        rank = torch.exp(torch.rand(rows, device="cuda", generator=g) * math.log(v)).long() - 1
        tokens = (rank * 7919 + 12345) % v
        pads = torch.rand(rows, device="cuda", generator=g) < 0.0625
        s["tokens"] = torch.where(pads, -1, tokens)
        if way == "lookup":
            s["E"] = _matrix(g, v, d, dt, 0.02, pad)
            s["Y"] = _out(rows, d, dt, pad)
        else:
            s["dY"] = _matrix(g, rows, d, dt, 0.02, pad)
            s["dE"] = [torch.empty(v, d, device="cuda", dtype=gd) for _ in range(case["nodes"])]
        return s
    if op == "norm":
        n = case["n"]
        s["weight"] = (1 + 0.1 * rand(n)).to(dt) if case["weight"] else None
        if way == "forward":
            s["X"] = _matrix(g, rows, n, dt, 0.3, pad)
            s["residual"] = _matrix(g, rows, n, dt, 2.0, pad) if case["residual"] else None
            s["H"] = _out(rows, n, dt, pad) if case["residual"] else None
            s["Y"], s["rstd"] = _out(rows, n, dt, pad), torch.empty(rows, device="cuda")
            if case["packed"]:
                s["codes"] = torch.empty(rows, n, device="cuda", dtype=torch.int8)
                s["scales"] = torch.empty(rows, (n + 31) // 32, device="cuda", dtype=torch.uint8)
                s["values"] = torch.empty(rows, n, device="cuda", dtype=torch.bfloat16)
            return s
        s["H"] = _matrix(g, rows, n, dt, 2.0, pad)
        s["rstd"] = torch.rsqrt(s["H"].float().square().mean(1) + 1e-6)
        s["dY"] = _matrix(g, rows, n, dt, 0.02, pad)
        s["residual"] = _matrix(g, rows, n, dt, 0.02, pad) if case["residual"] else None
        s["dX"] = _out(rows, n, dt, pad)
        s["dw"] = [torch.empty(n, device="cuda", dtype=gd) for _ in range(case["nodes"])] if case["weight"] else None
        return s
    if op == "checkpoint":
        k = case["k"]
        z = _matrix(g, rows, k, dt, 1.0, pad)
        z.mul_(torch.exp(0.7 * rand(k)).to(dt))                       # columns of unlike size
        if way == "save":
            s["X"] = z
            s["codes"] = torch.empty(rows, k, device="cuda", dtype=torch.int8)
            s["scales"] = torch.empty(rows, (k + 31) // 32, device="cuda", dtype=torch.uint8)
            s["values"] = torch.empty(rows, k, device="cuda", dtype=torch.bfloat16)
            return s
        n = case["n"]
        s["codes"], s["scales"] = _saved(z.float())
        s["dZ"] = _matrix(g, rows, n, dt, 0.02, pad)
        s["W"] = _matrix(g, n, k, dt, n ** -0.5, pad)
        s["residual"] = _matrix(g, rows, k, dt, 0.02, pad) if case["residual"] else None
        s["dX"] = _out(rows, k, dt, pad)
        s["dW"] = [torch.empty(n, k, device="cuda", dtype=gd) for _ in range(case["nodes"])]
        s["db"] = [torch.empty(n, device="cuda", dtype=gd) for _ in range(case["nodes"])] if case["bias"] else None
        return s
    v = case["vocab"]
    z = _matrix(g, rows, v, dt, 1.5, pad)
    at = torch.arange(rows, device="cuda")
    tokens = torch.randint(case["banned"], v, (rows,), device="cuda", generator=g)
    z[at, tokens] += math.log(v)
    if case["banned"]:
        z[:, :case["banned"]] = -math.inf
    s["logits"] = z
    s["tokens"] = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.125, -1, tokens)
    if way == "forward":
        s["logp"], s["lse"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        s["entropy"] = torch.empty(rows, device="cuda") if case["entropy"] else None
        k = case["topk"]
        s["top_logp"] = torch.empty(rows, k, device="cuda") if k else None
        s["top_ids"] = torch.empty(rows, k, device="cuda", dtype=torch.int32) if k else None
        return s
    zt = z.float() / case["tau"]
    s["lse"] = torch.logsumexp(zt, 1)
    s["entropy"] = s["dentropy"] = None
    if case["entropy"]:
        p = torch.exp(zt - s["lse"][:, None])
        s["entropy"] = -torch.where(p > 0, p * (zt - s["lse"][:, None]), 0.0).sum(1)
        s["dentropy"] = -0.01 / rows * torch.ones(rows, device="cuda")
        del p
    del zt
    s["dlogp"] = rand(rows) / rows
    s["dlogits"] = _out(rows, v, dt, pad)
    return s


# ------------------------------------------------------------------------------------------------------ run

def run(s):
    name = s["case"]["op"] + "-" + s["case"]["way"]
    return (_own if own else _plain)[name](s)


def _own_lookup(s):
    _package().glr_embedding(s["E"], s["tokens"], s["Y"], scale=s["case"]["scale"])
    return {"y": s["Y"]}


def _own_embedding_grad(s):
    _package().glr_embedding_grad(s["dY"], s["tokens"], s["dE"], scale=s["case"]["scale"])
    return {"de": s["dE"]}


def _own_norm(s):
    glr, packed = _package(), s["case"]["packed"]
    glr.glr_norm(s["X"], s["Y"], weight=s["weight"], residual=s["residual"], H=s["H"], rstd=s["rstd"], eps=1e-6,
                 codes=s["codes"] if packed else None, scales=s["scales"] if packed else None)
    if packed:
        glr.glr_checkpoint_unpack(s["codes"], s["scales"], s["values"])
    return {"y": s["Y"], "h": s["H"], "rstd": s["rstd"], "values": s["values"] if packed else None}


def _own_norm_grad(s):
    _package().glr_norm_grad(s["dY"], s["H"], s["rstd"], s["dX"], weight=s["weight"], residual=s["residual"], dweight=s["dw"])
    return {"dx": s["dX"], "dw": s["dw"]}


def _own_save(s):
    glr = _package()
    glr.glr_checkpoint_pack(s["X"], s["codes"], s["scales"])
    glr.glr_checkpoint_unpack(s["codes"], s["scales"], s["values"])
    return {"values": s["values"]}


def _own_checkpoint_grad(s):
    _package().glr_linear_grad_checkpoint(s["dZ"], s["codes"], s["scales"], W=s["W"], dX=s["dX"], dW=s["dW"], db=s["db"],
                                          act=s["case"]["act"], residual=s["residual"])
    return {"dx": s["dX"], "dw": s["dW"], "db": s["db"]}


def _own_logp(s):
    _package().glr_token_logp(s["logits"], tokens=s["tokens"], logp=s["logp"], lse=s["lse"], entropy=s["entropy"],
                              top_logp=s["top_logp"], top_ids=s["top_ids"], temperature=s["case"]["tau"])
    return {"logp": s["logp"], "lse": s["lse"], "entropy": s["entropy"], "top_logp": s["top_logp"], "top_ids": s["top_ids"]}


def _own_logp_grad(s):
    _package().glr_token_logp_grad(s["logits"], s["lse"], s["dlogits"], tokens=s["tokens"], dlogp=s["dlogp"],
                                   entropy=s["entropy"], dentropy=s["dentropy"], temperature=s["case"]["tau"])
    return {"dlogits": s["dlogits"]}


def _plain_lookup(s):
    e, t = s["E"], s["tokens"]
    rows = e[t.clamp(min=0)].float() * s["case"]["scale"]
    return {"y": torch.where((t >= 0)[:, None], rows, 0.0).to(e.dtype)}


def _plain_embedding_grad(s):
    c, t = s["case"], s["tokens"]
    nodes, v = c["nodes"], c["vocab"]
    at = torch.where(t >= 0, t + v * (torch.arange(t.numel(), device="cuda") // c["rows"]), nodes * v)
    de = torch.zeros(nodes * v + 1, c["d"], device="cuda")
    de.index_add_(0, at, s["dY"].float())
    return {"de": list((de[:-1] * c["scale"]).to(_dt(c["gdtype"])).view(nodes, v, -1))}


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


def _values(codes, scales):
    """What codes and scales stand for, in 32 bits."""
    power = (scales.int() - 127).repeat_interleave(32, dim=1)[:, :codes.shape[1]]
    return torch.ldexp(codes.float(), power)


def _plain_norm(s):
    c, dt = s["case"], s["X"].dtype
    h = s["X"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    rstd = torch.rsqrt((h * h).mean(1) + 1e-6)
    y = h * rstd[:, None]
    if s["weight"] is not None:
        y = y * s["weight"].float()
    values = _values(*_saved(y)).to(torch.bfloat16) if c["packed"] else None
    return {"y": y.to(dt), "h": None if s["residual"] is None else h.to(dt), "rstd": rstd, "values": values}


def _plain_norm_grad(s):
    c, dt = s["case"], s["dY"].dtype
    dy, x = s["dY"].float(), s["H"].float() * s["rstd"][:, None]
    dw = None if s["dw"] is None else list((dy * x).view(c["nodes"], c["rows"], -1).sum(1).to(_dt(c["gdtype"])))
    if s["weight"] is not None:
        dy = dy * s["weight"].float()
    dx = (dy - x * (dy * x).mean(1, keepdim=True)) * s["rstd"][:, None]
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return {"dx": dx.to(dt), "dw": dw}


def _plain_save(s):
    return {"values": _values(*_saved(s["X"].float())).to(torch.bfloat16)}


def _plain_checkpoint_grad(s):
    c, dt, gd = s["case"], s["dZ"].dtype, _dt(s["case"]["gdtype"])
    z, dz = _values(s["codes"], s["scales"]), s["dZ"].float()
    x = _act(z, c["act"]).to(dt).float()                    # the layer's input, as the forward pass had it
    dzn, xn = dz.view(c["nodes"], c["rows"], -1), x.view(c["nodes"], c["rows"], -1)
    dw = torch.matmul(dzn.transpose(1, 2), xn).to(gd)
    db = None if s["db"] is None else list(dzn.sum(1).to(gd))
    dx = dz @ s["W"].float()
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return {"dx": (dx * _act_slope(z, c["act"])).to(dt), "dw": list(dw), "db": db}


def _plain_logp(s):
    c, z, t = s["case"], s["logits"].float(), s["tokens"]
    x = z / c["tau"]
    m = x.max(dim=1, keepdim=True).values
    e = torch.exp(x - m)
    total = e.sum(dim=1, keepdim=True)
    lse = m + torch.log(total)
    logp = torch.where(t >= 0, x.gather(1, t.clamp(min=0)[:, None])[:, 0] - lse[:, 0], 0.0)
    entropy = None
    if s["entropy"] is not None:
        entropy = torch.log(total)[:, 0] - torch.where(e > 0, e * (x - m), 0.0).sum(1) / total[:, 0]
    top = ids = None
    if c["topk"]:
        top, ids = torch.sort(s["logits"], dim=1, descending=True, stable=True)
        top, ids = top[:, :c["topk"]].float() / c["tau"] - lse, ids[:, :c["topk"]].to(torch.int32)
    return {"logp": logp, "lse": lse[:, 0], "entropy": entropy, "top_logp": top, "top_ids": ids}


def _plain_logp_grad(s):
    c, t = s["case"], s["tokens"]
    lp = s["logits"].float() / c["tau"] - s["lse"][:, None]
    p = torch.exp(lp)
    coef = torch.where(t >= 0, s["dlogp"], 0.0)[:, None]
    d = -coef * p
    d.scatter_add_(1, t.clamp(min=0)[:, None], coef)
    if s["dentropy"] is not None:
        d = d - s["dentropy"][:, None] * torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0)
    return {"dlogits": (d / c["tau"]).to(s["logits"].dtype)}


_own = {"embedding-lookup": _own_lookup, "embedding-grad": _own_embedding_grad, "norm-forward": _own_norm,
        "norm-grad": _own_norm_grad, "checkpoint-save": _own_save, "checkpoint-grad": _own_checkpoint_grad,
        "logp-forward": _own_logp, "logp-grad": _own_logp_grad}
_plain = {"embedding-lookup": _plain_lookup, "embedding-grad": _plain_embedding_grad, "norm-forward": _plain_norm,
          "norm-grad": _plain_norm_grad, "checkpoint-save": _plain_save, "checkpoint-grad": _plain_checkpoint_grad,
          "logp-forward": _plain_logp, "logp-grad": _plain_logp_grad}


# ------------------------------------------------------------------------------------- definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"embedding": _exact_embedding, "norm": _exact_norm, "checkpoint": _exact_checkpoint, "logp": _exact_logp}[case["op"]](s)


def _exact_embedding(s):
    c, t = s["case"], s["tokens"]
    if c["way"] == "lookup":
        y = torch.zeros(c["rows"], c["d"], device="cuda", dtype=torch.float64)
        at = torch.nonzero(t >= 0)[:, 0]
        y[at] = c["scale"] * s["E"][t[at]].double()
        return {"y": y}
    # a node's rows in the order of their tokens; a token's sum is the difference of two running sums
    out = []
    for i in range(c["nodes"]):
        part = slice(i * c["rows"], (i + 1) * c["rows"])
        tok, order = torch.sort(t[part], stable=True)
        run_ = torch.zeros(c["rows"] + 1, c["d"], device="cuda", dtype=torch.float64)
        run_[1:] = s["dY"][part][order].double().cumsum(0)
        some = torch.unique(tok[tok >= 0])
        lo, hi = torch.searchsorted(tok, some), torch.searchsorted(tok, some, right=True)
        de = torch.zeros(c["vocab"], c["d"], device="cuda", dtype=torch.float64)
        de[some] = c["scale"] * (run_[hi] - run_[lo])
        out.append(de)
    return {"de": out}


def _exact_save(x):
    """The values nearest to a 64-bit matrix among those that 8 bits and the blocks' scales can hold."""
    out = torch.empty_like(x)
    full = x.shape[1] // 32 * 32
    for lo, hi, width in ((0, full, 32), (full, x.shape[1], x.shape[1] - full)):
        if hi > lo:
            block = x[:, lo:hi].unflatten(1, (-1, width))
            most = block.abs().amax(-1, keepdim=True)
            step = torch.exp2(torch.ceil(torch.log2(most.clamp(min=1e-30) / 127)))
            step = torch.where(most > 127 * step, 2 * step, torch.where(2 * most <= 127 * step, step / 2, step))
            out[:, lo:hi] = (torch.round(block / step) * step).flatten(1)
    return out


def _exact_norm(s):
    c = s["case"]
    w = torch.ones(c["n"], device="cuda", dtype=torch.float64) if s["weight"] is None else s["weight"].double()
    if c["way"] == "forward":
        h = s["X"].double() if s["residual"] is None else torch.add(s["X"].double(), s["residual"].double())
        rstd = 1 / torch.sqrt(torch.linalg.vector_norm(h, dim=1) ** 2 / c["n"] + 1e-6)
        y = torch.einsum("tn,t,n->tn", h, rstd, w)
        return {"y": y, "h": None if s["residual"] is None else h, "rstd": rstd, "values": _exact_save(y) if c["packed"] else None}
    # with the statistic given, Y = S rstd(S) w at S = H: the derivative of rstd is -rstd^3 S / n
    rstd, h, dy = s["rstd"].double(), s["H"].double(), s["dY"].double()
    dx = torch.empty_like(h)
    for part in torch.arange(h.shape[0], device="cuda").split(1024):
        g = dy[part] * w
        inner = torch.einsum("tn,tn->t", g, h[part])
        dx[part] = g * rstd[part, None] - h[part] * (rstd[part] ** 3 * inner / c["n"])[:, None]
        if s["residual"] is not None:
            dx[part] += s["residual"][part].double()
    rows = c["rows"]
    dw = None if s["dw"] is None else [torch.einsum("tn,tn,t->n", dy[i:i + rows], h[i:i + rows], rstd[i:i + rows])
                                       for i in range(0, h.shape[0], rows)]
    return {"dx": dx, "dw": dw}


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


def _exact_checkpoint(s):
    c = s["case"]
    if c["way"] == "save":
        return {"values": _exact_save(s["X"].double())}
    step = torch.exp2(s["scales"].double() - 127)
    z = s["codes"].double() * step[:, torch.arange(c["k"], device="cuda") // 32]
    x, slope = _exact_act(z, c["act"])
    x, dz = x.to(s["dZ"].dtype).double(), s["dZ"].double()
    g = torch.einsum("mn,nk->mk", dz, s["W"].double()) + (0 if s["residual"] is None else s["residual"].double())
    parts = [slice(i * c["rows"], (i + 1) * c["rows"]) for i in range(c["nodes"])]
    return {"dx": g * slope, "dw": [torch.einsum("mn,mk->nk", dz[p], x[p]) for p in parts],
            "db": None if s["db"] is None else [dz[p].sum(0) for p in parts]}


def _exact_logp(s):
    c, t = s["case"], s["tokens"]
    rows, v = s["logits"].shape
    chunks = torch.arange(rows, device="cuda").split(max(1, (1 << 26) // v))
    grad = torch.empty(rows, v, device="cuda", dtype=torch.float64) if c["way"] == "grad" else None
    logp, lse, entropy = (torch.zeros(rows, device="cuda", dtype=torch.float64) for _ in range(3))
    k = c["topk"]
    top = torch.empty(rows, k, device="cuda", dtype=torch.float64)
    for at in chunks:
        z = s["logits"][at].double() / c["tau"]
        if grad is not None:
            # with the statistics given: p = exp(z - lse)
            lp = z - s["lse"][at].double()[:, None]
            p = lp.exp()
            coef = s["dlogp"][at].double() * (t[at] >= 0)
            d = torch.zeros_like(p).scatter_(1, t[at].clamp(min=0)[:, None], coef[:, None]) - coef[:, None] * p
            if s["dentropy"] is not None:
                d += s["dentropy"][at].double()[:, None] * (torch.special.entr(p) - p * s["entropy"][at].double()[:, None])
            grad[at] = d / c["tau"]
            continue
        lse[at] = torch.logsumexp(z, 1)
        lp = z - lse[at, None]
        entropy[at] = torch.special.entr(lp.exp()).sum(1)
        logp[at] = torch.where(t[at] >= 0, lp.gather(1, t[at].clamp(min=0)[:, None])[:, 0], 0.0)
        if k:
            top[at] = lp.topk(k, dim=1).values
    if grad is not None:
        return {"dlogits": grad}
    return {"logp": logp, "lse": lse, "entropy": entropy if c["entropy"] else None, "top_logp": top if k else None, "top_ids": None}
