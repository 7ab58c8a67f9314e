"""The operators around the step, as declared in ``include/glr.h``: a linear layer with its epilogue, the
gradients of its input, weights and bias (the weights' per node, as ``GreedyLore.step`` takes them), embeddings,
norms, activations kept in 8 bits, and the losses on logits and tokens' log-probabilities with their gradients.

Every function marshals its tensors to the C entry point of its name and returns nothing: the outputs are the
caller's tensors.  The library cannot see the tensors' shapes, so they are checked here; what it can check
itself (ranges, alignment, strides) it refuses with ``GlrError``.  All tensors lie on the current device.  Work is
enqueued on ``stream`` (the current one by default) without synchronising; tensors last used on another stream are
the caller's to order.
Matrices are 2-D CUDA tensors, float32 or bfloat16, with unit column stride and any row stride.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Union

import torch

from . import GLR_BF16, GLR_F32, GLR_OK, _check, _lib, _raw_stream, _stream_ptr, load

_DTYPES = {torch.float32: GLR_F32, torch.bfloat16: GLR_BF16}
_INDEX = {torch.int32: 0, torch.int64: 1}
ACTIVATIONS = {"none": _lib.GLR_ACT_NONE, "relu": _lib.GLR_ACT_RELU, "gelu": _lib.GLR_ACT_GELU,
               "gelu_tanh": _lib.GLR_ACT_GELU_TANH, "silu": _lib.GLR_ACT_SILU}
PREFERENCES = {"sigmoid": _lib.GLR_PREF_SIGMOID, "ipo": _lib.GLR_PREF_IPO}


def _dtype(x: torch.Tensor, name: str) -> int:
    code = _DTYPES.get(x.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32 or bfloat16")
    return code


def _elsewhere(x: torch.Tensor, name: str):
    if x.get_device() < 0:
        raise ValueError(f"{name} must be a CUDA tensor")
    raise ValueError(f"{name} must be on the device of the call's first tensor")


def _mat(x: Optional[torch.Tensor], name: str, dev: int, rows: int, cols: int, dtype=None):
    """Address and row stride of a rows x cols matrix argument (None: absent)."""
    if x is None:
        return None, 0
    if x.shape != (rows, cols):
        raise ValueError(f"{name} must be {rows} x {cols}, got {tuple(x.shape)}")
    if x.get_device() != dev:
        _elsewhere(x, name)
    if dtype is not None and x.dtype != dtype:
        raise ValueError(f"{name} must be a CUDA tensor of {dtype}")
    ld, step = x.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name} must have unit column stride")
    return x.data_ptr(), ld if rows > 1 else cols


def _vec(x: Optional[torch.Tensor], name: str, dev: int, n: int, dtype=torch.float32):
    """Address of a contiguous vector argument of n elements (None: absent)."""
    if x is None:
        return None
    if x.numel() != n or x.dtype != dtype or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor of {n} {dtype} elements")
    if x.get_device() != dev:
        _elsewhere(x, name)
    return x.data_ptr()


def _index(x: Optional[torch.Tensor], name: str, dev: int, n: int):
    if x is None:
        return None, 0
    wide = _INDEX.get(x.dtype)
    if wide is None or x.numel() != n or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor of {n} int32 or int64 elements")
    if x.get_device() != dev:
        _elsewhere(x, name)
    return x.data_ptr(), wide


def _here(dev: int, stream) -> int:
    """The stream's address, for tensors on the current device: the library launches there, and knows them by address alone."""
    if dev < 0:
        raise ValueError("the tensors must be CUDA tensors")
    if dev != torch.cuda.current_device():
        raise ValueError(f"the tensors are on cuda:{dev}, which is not the current device")
    return _raw_stream(dev) if stream is None and _raw_stream is not None else _stream_ptr(stream)


def _call(fn, args, on: int) -> None:
    rc = fn(ctypes.byref(args), on)
    if rc != GLR_OK:
        _check(rc)


def _space(args, query, x: torch.Tensor, work: float, ragged: int, stream):
    """The workspace that a product asks for (float32 or rows off 16 bytes, where it is large), from PyTorch's
    allocator in the stream's own pool: its memory is reused in the order of the work that runs there."""
    if (x.dtype == torch.bfloat16 and not ragged) or work < 1e7:
        return None
    need = ctypes.c_int64(0)
    _check(query(ctypes.byref(args), ctypes.byref(need)))
    if need.value == 0:
        return None
    space = _alloc(need.value, torch.uint8, x.device, stream)
    args.workspace, args.workspace_bytes = space.data_ptr(), need.value
    return space


def _alloc(n: int, dtype, device, stream) -> torch.Tensor:
    if stream is None:
        return torch.empty(n, dtype=dtype, device=device)
    own = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(_stream_ptr(stream))
    with torch.cuda.stream(own):
        return torch.empty(n, dtype=dtype, device=device)


def _activation(act: str) -> int:
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}")
    return ACTIVATIONS[act]


def glr_linear(X: torch.Tensor, W: torch.Tensor, Y: torch.Tensor, *, bias: Optional[torch.Tensor] = None,
               act: str = "none", residual: Optional[torch.Tensor] = None, preact: Optional[torch.Tensor] = None,
               stream=None) -> None:
    """Y = act(X W^T + bias) + residual; preact receives X W^T + bias.  X rows x k, W n x k, Y rows x n."""
    dtype, dev = _dtype(X, "X"), X.get_device()
    rows, k = X.shape
    n = W.shape[0]
    dt = X.dtype
    x, ldx = _mat(X, "X", dev, rows, k)
    w, ldw = _mat(W, "W", dev, n, k, dt)
    y, ldy = _mat(Y, "Y", dev, rows, n, dt)
    r, ldr = _mat(residual, "residual", dev, rows, n, dt)
    p, ldp = _mat(preact, "preact", dev, rows, n, dt)
    lib, on = load(), _here(dev, stream)
    args = _lib.GlrLinearArgs(rows, n, k, x, ldx, w, ldw, y, ldy, _vec(bias, "bias", dev, n, dt), r, ldr, p, ldp, None, 0, dtype,
                              _activation(act))
    space = _space(args, lib.glr_linear_workspace, X, 2.0 * rows * n * k, ((x | w) & 15) | ((ldx | ldw) & 7), stream)
    _call(lib.glr_linear, args, on)
    del space


def glr_linear_grad_input(dZ: torch.Tensor, W: torch.Tensor, dX: torch.Tensor, *,
                          residual: Optional[torch.Tensor] = None, preact: Optional[torch.Tensor] = None,
                          act: str = "none", grad_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """G = dZ W + residual; dX = G act'(preact); grad_out receives G.  dZ rows x n, W n x k, dX rows x k."""
    dtype, dev = _dtype(dZ, "dZ"), dZ.get_device()
    rows, n = dZ.shape
    k = W.shape[1]
    dt = dZ.dtype
    z, lddz = _mat(dZ, "dZ", dev, rows, n)
    w, ldw = _mat(W, "W", dev, n, k, dt)
    x, lddx = _mat(dX, "dX", dev, rows, k, dt)
    r, ldr = _mat(residual, "residual", dev, rows, k, dt)
    p, ldp = _mat(preact, "preact", dev, rows, k, dt)
    g, ldg = _mat(grad_out, "grad_out", dev, rows, k, dt)
    lib, on = load(), _here(dev, stream)
    args = _lib.GlrLinearGradInputArgs(rows, n, k, z, lddz, w, ldw, x, lddx, r, ldr, p, ldp, g, ldg, None, 0, dtype,
                                       _activation(act))
    space = _space(args, lib.glr_linear_grad_input_workspace, dZ, 2.0 * rows * n * k, ((z | w) & 15) | ((lddz | ldw) & 7), stream)
    _call(lib.glr_linear_grad_input, args, on)
    del space


def glr_linear_grad_weight(dZ: torch.Tensor, X: torch.Tensor, dW: Union[torch.Tensor, Sequence[torch.Tensor]], *,
                           db: Union[None, torch.Tensor, Sequence[torch.Tensor]] = None, stream=None) -> None:
    """dW[i] = dZ_i^T X_i and db[i] = the column sums of dZ_i for the nodes' equal shares of the rows.

    dZ is (nodes rows) x n, X (nodes rows) x k; dW holds the nodes' n x k gradients (contiguous, float32 or
    bfloat16: the G of ``GreedyLore.step``), db their n-vectors of the same dtype.  A tensor is one node's."""
    dtype, dev = _dtype(dZ, "dZ"), dZ.get_device()
    dW = [dW] if isinstance(dW, torch.Tensor) else list(dW)
    db = [db] if isinstance(db, torch.Tensor) else db if db is None else list(db)
    nodes, (rows, n), k = len(dW), dZ.shape, X.shape[1]
    if nodes < 1 or rows % nodes:
        raise ValueError("dZ must hold the same number of rows for each of the dW")
    if db is not None and len(db) != nodes:
        raise ValueError("db must hold as many tensors as dW")
    gd = dW[0].dtype
    grad_dtype = _dtype(dW[0], "dW")
    z, lddz = _mat(dZ, "dZ", dev, rows, n)
    x, ldx = _mat(X, "X", dev, rows, k, dZ.dtype)
    wp, bp = (ctypes.c_void_p * nodes)(), (ctypes.c_void_p * nodes)()
    for i, g in enumerate(dW):
        if g.dim() != 2 or g.shape[0] != n or g.shape[1] != k:
            raise ValueError(f"dW[{i}] must be {n} x {k}")
        wp[i] = _vec(g, f"dW[{i}]", dev, n * k, gd)
    for i, g in enumerate(db or ()):
        bp[i] = _vec(g, f"db[{i}]", dev, n, gd)
    lib, on = load(), _here(dev, stream)
    args = _lib.GlrLinearGradWeightArgs(nodes, rows // nodes, n, k, z, lddz, x, ldx, ctypes.addressof(wp),
                                        None if db is None else ctypes.addressof(bp), None, 0, dtype, grad_dtype)
    space = _space(args, lib.glr_linear_grad_weight_workspace, dZ, 2.0 * rows * n * k, ((z | x) & 15) | ((lddz | ldx) & 7), stream)
    _call(lib.glr_linear_grad_weight, args, on)
    del space


def glr_distill_loss(logits: torch.Tensor, teacher: torch.Tensor, ids: torch.Tensor, *, loss: torch.Tensor,
                     row_loss: torch.Tensor, dlogits: Optional[torch.Tensor] = None,
                     labels: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                     temperature: float = 1.0, soft: float = 1.0, hard: float = 0.0, stream=None) -> None:
    """soft KL(q || softmax(z / tau)) + hard CE(label), q the softmax of the teacher's logits (rows x topk) at ids.

    loss (1) = sum of weight (rows; None: 1 / rows each) times row_loss (rows); dlogits (None: no gradient) may
    be logits itself.  The usual tau^2 factor of the soft term is the caller's, in ``soft``."""
    dtype, dev = _dtype(logits, "logits"), logits.get_device()
    rows, vocab = logits.shape
    topk = teacher.shape[1] if teacher.dim() == 2 else -1
    z, ldz = _mat(logits, "logits", dev, rows, vocab)
    t, ldt = _mat(teacher, "teacher", dev, rows, topk)
    d, ldd = _mat(dlogits, "dlogits", dev, rows, vocab, logits.dtype)
    i, ldi = _mat(ids, "ids", dev, rows, topk)
    if ids.dtype not in _INDEX:
        raise ValueError("ids must be int32 or int64")
    y, ywide = _index(labels, "labels", dev, rows)
    on = _here(dev, stream)
    _call(load().glr_distill_loss,
          _lib.GlrDistillArgs(rows, vocab, topk, z, ldz, t, ldt, i, ldi, y, _vec(weight, "weight", dev, rows),
                              _vec(loss, "loss", dev, 1), _vec(row_loss, "row_loss", dev, rows), d, ldd, dtype,
                              _dtype(teacher, "teacher"), _INDEX[ids.dtype], ywide, temperature, soft, hard, 0), on)


def glr_policy_loss(logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor, advantage: torch.Tensor, *,
                    loss: torch.Tensor, row_loss: torch.Tensor, logp: torch.Tensor,
                    dlogits: Optional[torch.Tensor] = None, ref_logp: Optional[torch.Tensor] = None,
                    weight: Optional[torch.Tensor] = None, temperature: float = 1.0, clip_low: float = 0.2,
                    clip_high: float = 0.2, kl: float = 0.0, stream=None) -> None:
    """The clipped policy loss -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl (exp(e) - e - 1) of every
    row's token, r = exp(logp - old_logp), e = ref_logp - logp, with its gradient (see glr.h)."""
    dtype, dev = _dtype(logits, "logits"), logits.get_device()
    rows, vocab = logits.shape
    z, ldz = _mat(logits, "logits", dev, rows, vocab)
    d, ldd = _mat(dlogits, "dlogits", dev, rows, vocab, logits.dtype)
    y, wide = _index(tokens, "tokens", dev, rows)
    on = _here(dev, stream)
    _call(load().glr_policy_loss,
          _lib.GlrPolicyArgs(rows, vocab, z, ldz, y, _vec(old_logp, "old_logp", dev, rows), _vec(advantage, "advantage", dev, rows),
                             _vec(ref_logp, "ref_logp", dev, rows), _vec(weight, "weight", dev, rows), _vec(loss, "loss", dev, 1),
                             _vec(row_loss, "row_loss", dev, rows), _vec(logp, "logp", dev, rows), d, ldd, dtype, wide,
                             temperature, clip_low, clip_high, kl), on)


def glr_preference_loss(logits: torch.Tensor, tokens: torch.Tensor, offsets: torch.Tensor, *, loss: torch.Tensor,
                        pair_loss: torch.Tensor, seq_logp: torch.Tensor, row_logp: torch.Tensor,
                        dlogits: Optional[torch.Tensor] = None, ref_logp: Optional[torch.Tensor] = None,
                        weight: Optional[torch.Tensor] = None, kind: str = "sigmoid", beta: float = 0.1,
                        smoothing: float = 0.0, average: bool = False, workspace: Optional[torch.Tensor] = None,
                        stream=None) -> None:
    """A loss on the log ratios of pairs of packed answers, from the logits to their gradient (see glr.h).

    offsets (2 pairs + 1) bounds the sequences' rows, chosen and rejected in turn; pair_loss (pairs), seq_logp
    (2 pairs), row_logp (rows).  workspace: float32, 4 rows + 16 pairs + 1024 elements (None: taken from
    PyTorch's allocator for this call)."""
    dtype, dev = _dtype(logits, "logits"), logits.get_device()
    rows, vocab = logits.shape
    pairs = (offsets.numel() - 1) // 2
    if offsets.numel() < 1 or offsets.numel() % 2 == 0:
        raise ValueError("offsets must have 2 pairs + 1 elements")
    if kind not in PREFERENCES:
        raise ValueError(f"kind must be one of {sorted(PREFERENCES)}")
    z, ldz = _mat(logits, "logits", dev, rows, vocab)
    d, ldd = _mat(dlogits, "dlogits", dev, rows, vocab, logits.dtype)
    y, ywide = _index(tokens, "tokens", dev, rows)
    o, owide = _index(offsets, "offsets", dev, 2 * pairs + 1)
    on, need = _here(dev, stream), 4 * rows + 16 * pairs + 1024
    if workspace is None:
        workspace = _alloc(need, torch.float32, logits.device, stream)
    elif workspace.dtype != torch.float32 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous float32 CUDA tensor")
    elif workspace.get_device() != dev:
        _elsewhere(workspace, "workspace")
    _call(load().glr_preference_loss,
          _lib.GlrPreferenceArgs(rows, vocab, pairs, z, ldz, y, o, _vec(ref_logp, "ref_logp", dev, 2 * pairs),
                                 _vec(weight, "weight", dev, pairs), _vec(loss, "loss", dev, 1), _vec(pair_loss, "pair_loss", dev, pairs),
                                 _vec(seq_logp, "seq_logp", dev, 2 * pairs), _vec(row_logp, "row_logp", dev, rows), d, ldd,
                                 workspace.data_ptr(), 4 * workspace.numel(), dtype, ywide, owide, PREFERENCES[kind],
                                 beta, smoothing, 1 if average else 0, 0), on)


def _codes(codes: Optional[torch.Tensor], scales: Optional[torch.Tensor], dev: int, rows: int, cols: int):
    """Addresses and row strides of an 8-bit matrix and its scales."""
    if (codes is None) != (scales is None):
        raise ValueError("codes and scales go together")
    c, ldc = _mat(codes, "codes", dev, rows, cols, torch.int8)
    s, lds = _mat(scales, "scales", dev, rows, (cols + 31) // 32, torch.uint8)
    return c, ldc, s, lds


def _nodes(grads, name: str, rows: int):
    """The nodes' gradient tensors as a list, and the rows of each."""
    grads = [grads] if isinstance(grads, torch.Tensor) else list(grads)
    if len(grads) < 1 or rows % len(grads):
        raise ValueError(f"the rows must be the same number for each of the {name}")
    return grads, rows // len(grads)


def _pointers(grads, name: str, dev: int, shape, dtype):
    arr = (ctypes.c_void_p * len(grads))()
    for i, g in enumerate(grads):
        if tuple(g.shape) != shape:
            raise ValueError(f"{name}[{i}] must be {' x '.join(map(str, shape))}")
        arr[i] = _vec(g, f"{name}[{i}]", dev, g.numel(), dtype)
    return arr


def _scratch(args, query, device, stream):
    """The workspace that a call needs, from PyTorch's allocator in the stream's own pool."""
    need = ctypes.c_int64(0)
    _check(query(ctypes.byref(args), ctypes.byref(need)))
    if need.value == 0:
        return None
    space = _alloc(need.value, torch.uint8, device, stream)
    args.workspace, args.workspace_bytes = space.data_ptr(), need.value
    return space


def glr_embedding(E: torch.Tensor, tokens: torch.Tensor, Y: torch.Tensor, *, scale: float = 1.0, stream=None) -> None:
    """Y[t] = scale E[tokens[t]], zero for a token outside the vocabulary.  E vocab x d, Y rows x d."""
    dtype, dev = _dtype(E, "E"), E.get_device()
    (vocab, d), rows = E.shape, tokens.numel()
    e, lde = _mat(E, "E", dev, vocab, d)
    y, ldy = _mat(Y, "Y", dev, rows, d, E.dtype)
    t, wide = _index(tokens, "tokens", dev, rows)
    on = _here(dev, stream)
    _call(load().glr_embedding, _lib.GlrEmbeddingArgs(rows, vocab, d, e, lde, t, y, ldy, dtype, wide, scale, 0), on)


def glr_embedding_grad(dY: torch.Tensor, tokens: torch.Tensor, dE: Union[torch.Tensor, Sequence[torch.Tensor]], *,
                       scale: float = 1.0, accumulate: bool = False, stream=None) -> None:
    """dE[i][v] = scale times the sum of the rows of dY of token v among node i's equal share of the rows.

    dE holds the nodes' vocab x d gradients (contiguous, float32 or bfloat16: the G of ``GreedyLore.step``); with
    accumulate the sums are added to what they hold.  A tensor is one node's."""
    dtype, dev = _dtype(dY, "dY"), dY.get_device()
    all_rows, d = dY.shape
    dE, rows = _nodes(dE, "dE", all_rows)
    vocab, gd = dE[0].shape[0], dE[0].dtype
    grad_dtype = _dtype(dE[0], "dE")
    y, lddy = _mat(dY, "dY", dev, all_rows, d)
    t, wide = _index(tokens, "tokens", dev, all_rows)
    ep = _pointers(dE, "dE", dev, (vocab, d), gd)
    lib, on = load(), _here(dev, stream)
    args = _lib.GlrEmbeddingGradArgs(len(dE), rows, vocab, d, y, lddy, t, ctypes.addressof(ep), None, 0, dtype, grad_dtype, wide,
                                     1 if accumulate else 0, scale, 0)
    space = _scratch(args, lib.glr_embedding_grad_workspace, dY.device, stream)
    _call(lib.glr_embedding_grad, args, on)
    del space


def glr_checkpoint_pack(X: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, *, stream=None) -> None:
    """X (rows x cols) in 8 bits: codes (int8) and, for every 32 columns of a row, scales (uint8, rows x ceil(cols / 32))."""
    dtype, dev = _dtype(X, "X"), X.get_device()
    rows, cols = X.shape
    x, ldx = _mat(X, "X", dev, rows, cols)
    c, ldc, s, lds = _codes(codes, scales, dev, rows, cols)
    on = _here(dev, stream)
    _call(load().glr_checkpoint_pack, _lib.GlrCheckpointPackArgs(rows, cols, x, ldx, c, ldc, s, lds, dtype, 0), on)


def glr_checkpoint_unpack(codes: torch.Tensor, scales: torch.Tensor, Y: torch.Tensor, *, act: str = "none", stream=None) -> None:
    """Y = act of the values that codes and scales stand for."""
    dtype, dev = _dtype(Y, "Y"), Y.get_device()
    rows, cols = Y.shape
    y, ldy = _mat(Y, "Y", dev, rows, cols)
    c, ldc, s, lds = _codes(codes, scales, dev, rows, cols)
    on = _here(dev, stream)
    _call(load().glr_checkpoint_unpack, _lib.GlrCheckpointUnpackArgs(rows, cols, c, ldc, s, lds, y, ldy, dtype, _activation(act)), on)


def glr_linear_grad_checkpoint(dZ: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, *, W: Optional[torch.Tensor] = None,
                               dX: Optional[torch.Tensor] = None, dW: Union[None, torch.Tensor, Sequence[torch.Tensor]] = None,
                               db: Union[None, torch.Tensor, Sequence[torch.Tensor]] = None, act: str = "none",
                               residual: Optional[torch.Tensor] = None, nodes: int = 1, stream=None) -> None:
    """A layer's backward pass from its input's checkpoint: X = act(value), dW[i] = dZ_i^T X_i, db[i] the column sums
    of dZ_i, and dX = (dZ W + residual) act'(value); dW or dX may be left out.  The nodes are those of dW (nodes: without dW)."""
    dtype, dev = _dtype(dZ, "dZ"), dZ.get_device()
    all_rows, n = dZ.shape
    k = codes.shape[1]
    dt, grad_dtype, wp, bp = dZ.dtype, dtype, None, None
    z, lddz = _mat(dZ, "dZ", dev, all_rows, n)
    c, ldc, s, lds = _codes(codes, scales, dev, all_rows, k)
    if dX is not None and W is None:
        raise ValueError("dX needs W")
    w, ldw = _mat(W, "W", dev, n, k, dt)
    r, ldr = _mat(residual, "residual", dev, all_rows, k, dt)
    x, lddx = _mat(dX, "dX", dev, all_rows, k, dt)
    if dW is not None:
        dW, rows = _nodes(dW, "dW", all_rows)
        nodes, gd, grad_dtype = len(dW), dW[0].dtype, _dtype(dW[0], "dW")
        wp = _pointers(dW, "dW", dev, (n, k), gd)
        if db is not None:
            db = [db] if isinstance(db, torch.Tensor) else list(db)
            if len(db) != nodes:
                raise ValueError("db must hold as many tensors as dW")
            bp = _pointers(db, "db", dev, (n,), gd)
    elif db is not None:
        raise ValueError("db needs dW")
    elif nodes < 1 or all_rows % nodes:
        raise ValueError("the rows must be the same number for each of the nodes")
    lib, on = load(), _here(dev, stream)
    args = _lib.GlrLinearGradCheckpointArgs(nodes, all_rows // nodes, n, k, z, lddz, w, ldw, c, ldc, s, lds, r, ldr, x, lddx,
                                            None if wp is None else ctypes.addressof(wp), None if bp is None else ctypes.addressof(bp),
                                            None, 0, dtype, grad_dtype, _activation(act), 0)
    space = _scratch(args, lib.glr_linear_grad_checkpoint_workspace, dZ.device, stream)
    _call(lib.glr_linear_grad_checkpoint, args, on)
    del space


def glr_norm(X: torch.Tensor, Y: Optional[torch.Tensor], *, weight: Optional[torch.Tensor] = None,
             residual: Optional[torch.Tensor] = None, H: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None,
             codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None, eps: float = 1e-6, stream=None) -> None:
    """S = X + residual, H = S, rstd = (mean S^2 + eps)^(-1/2) of each row, Y = S rstd weight, codes and scales Y in 8 bits."""
    dtype, dev = _dtype(X, "X"), X.get_device()
    rows, n = X.shape
    dt = X.dtype
    x, ldx = _mat(X, "X", dev, rows, n)
    r, ldr = _mat(residual, "residual", dev, rows, n, dt)
    h, ldh = _mat(H, "H", dev, rows, n, dt)
    y, ldy = _mat(Y, "Y", dev, rows, n, dt)
    c, ldc, s, lds = _codes(codes, scales, dev, rows, n)
    on = _here(dev, stream)
    _call(load().glr_norm,
          _lib.GlrNormArgs(rows, n, x, ldx, r, ldr, _vec(weight, "weight", dev, n, dt), h, ldh, y, ldy, _vec(rstd, "rstd", dev, rows),
                           c, ldc, s, lds, dtype, eps), on)


def glr_norm_grad(dY: torch.Tensor, H: torch.Tensor, rstd: torch.Tensor, dX: Optional[torch.Tensor], *,
                  weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                  dweight: Union[None, torch.Tensor, Sequence[torch.Tensor]] = None, stream=None) -> None:
    """dX = rstd (weight dY - x mean(weight dY x)) + residual with x = H rstd, and dweight[i] = the column sums of dY x
    over node i's equal share of the rows (vectors of n, float32 or bfloat16; a tensor is one node's)."""
    dtype, dev = _dtype(dY, "dY"), dY.get_device()
    all_rows, n = dY.shape
    dt, nodes, grad_dtype, wp = dY.dtype, 1, dtype, None
    y, lddy = _mat(dY, "dY", dev, all_rows, n)
    h, ldh = _mat(H, "H", dev, all_rows, n, dt)
    r, ldr = _mat(residual, "residual", dev, all_rows, n, dt)
    x, lddx = _mat(dX, "dX", dev, all_rows, n, dt)
    if dweight is not None:
        dweight, _ = _nodes(dweight, "dweight", all_rows)
        nodes, grad_dtype = len(dweight), _dtype(dweight[0], "dweight")
        wp = _pointers(dweight, "dweight", dev, (n,), dweight[0].dtype)
    lib, on = load(), _here(dev, stream)
    args = _lib.GlrNormGradArgs(nodes, all_rows // nodes, n, y, lddy, h, ldh, _vec(rstd, "rstd", dev, all_rows),
                                _vec(weight, "weight", dev, n, dt), r, ldr, x, lddx, None if wp is None else ctypes.addressof(wp),
                                None, 0, dtype, grad_dtype)
    space = None if wp is None else _scratch(args, lib.glr_norm_grad_workspace, dY.device, stream)
    _call(lib.glr_norm_grad, args, on)
    del space


def glr_token_logp(logits: torch.Tensor, *, tokens: Optional[torch.Tensor] = None, logp: Optional[torch.Tensor] = None,
                   lse: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                   top_logp: Optional[torch.Tensor] = None, top_ids: Optional[torch.Tensor] = None, temperature: float = 1.0,
                   stream=None) -> None:
    """log softmax(logits / temperature) of every row's token, the logarithm of the sum, the entropy, and the most probable
    alternatives (rows x topk: float32 log-probabilities, int32 or int64 ids; equal ones by ascending id; see glr.h)."""
    dtype, dev = _dtype(logits, "logits"), logits.get_device()
    rows, vocab = logits.shape
    z, ldz = _mat(logits, "logits", dev, rows, vocab)
    top = top_logp if top_logp is not None else top_ids
    topk = 0 if top is None else top.shape[1] if top.dim() == 2 else -1
    p, ldp = _mat(top_logp, "top_logp", dev, rows, topk, torch.float32)
    i, ldi = _mat(top_ids, "top_ids", dev, rows, topk)
    if top_ids is not None and top_ids.dtype not in _INDEX:
        raise ValueError("top_ids must be int32 or int64")
    t, wide = _index(tokens, "tokens", dev, rows)
    on = _here(dev, stream)
    _call(load().glr_token_logp,
          _lib.GlrTokenLogpArgs(rows, vocab, topk, z, ldz, t, _vec(logp, "logp", dev, rows), _vec(lse, "lse", dev, rows),
                                _vec(entropy, "entropy", dev, rows), p, ldp, i, ldi, dtype, wide,
                                0 if top_ids is None else _INDEX[top_ids.dtype], temperature), on)


def glr_token_logp_grad(logits: torch.Tensor, lse: torch.Tensor, dlogits: torch.Tensor, *, tokens: Optional[torch.Tensor] = None,
                        dlogp: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                        dentropy: Optional[torch.Tensor] = None, temperature: float = 1.0, stream=None) -> None:
    """The logits' gradient from those of the tokens' log-probabilities and of the rows' entropies, with lse and entropy as
    glr_token_logp left them; dlogits may be logits itself."""
    dtype, dev = _dtype(logits, "logits"), logits.get_device()
    rows, vocab = logits.shape
    z, ldz = _mat(logits, "logits", dev, rows, vocab)
    d, ldd = _mat(dlogits, "dlogits", dev, rows, vocab, logits.dtype)
    t, wide = _index(tokens, "tokens", dev, rows)
    on = _here(dev, stream)
    _call(load().glr_token_logp_grad,
          _lib.GlrTokenLogpGradArgs(rows, vocab, z, ldz, t, _vec(lse, "lse", dev, rows), _vec(entropy, "entropy", dev, rows),
                                    _vec(dlogp, "dlogp", dev, rows), _vec(dentropy, "dentropy", dev, rows), d, ldd, dtype, wide,
                                    temperature, 0), on)


def glr_operator_status() -> int:
    """Raises GlrError (GLR_ETIMEOUT) when a bounded wait in an operator's kernel has given up since the last call; else 0."""
    n = ctypes.c_int32(0)
    _check(load().glr_operator_status(ctypes.byref(n)))
    return int(n.value)
