"""What the row operators' entry points and their binding answer without a GPU: struct layouts, workspace queries and
refusals, which come before any device work."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import __graft_entry__
from paper_2507_08784_gb300 import _lib
from test_operator_checks import _Elsewhere

STRUCTS = {"glr_embedding_args": _lib.GlrEmbeddingArgs, "glr_embedding_grad_args": _lib.GlrEmbeddingGradArgs,
           "glr_checkpoint_pack_args": _lib.GlrCheckpointPackArgs, "glr_checkpoint_unpack_args": _lib.GlrCheckpointUnpackArgs,
           "glr_linear_grad_checkpoint_args": _lib.GlrLinearGradCheckpointArgs, "glr_norm_args": _lib.GlrNormArgs,
           "glr_norm_grad_args": _lib.GlrNormGradArgs, "glr_token_logp_args": _lib.GlrTokenLogpArgs,
           "glr_token_logp_grad_args": _lib.GlrTokenLogpGradArgs}
P = 1 << 20      # an address that nothing reads: every call here is refused before device work


@pytest.fixture(scope="module")
def lib():
    __graft_entry__.build()
    return _lib.load()


def test_struct_layouts(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "glr.h"', 'int main(void) {']
    for cname, cls in STRUCTS.items():
        lines.append(f'printf("{cname} %zu\\n", sizeof({cname}));')
        lines += [f'printf("{cname}.{f} %zu\\n", offsetof({cname}, {f}));' for f, _ in cls._fields_]
    lines.append('printf("GLR_MAX_NORM %d\\n", (int)GLR_MAX_NORM);')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ['return 0;', '}']) + "\n")
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run([cc, "-std=c99", "-I", inc, str(src), "-o", str(tmp_path / "layout")], check=True)
    out = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout
    got = dict(line.split() for line in out.splitlines())
    for cname, cls in STRUCTS.items():
        assert int(got[cname]) == ctypes.sizeof(cls), cname
        for f, _ in cls._fields_:
            assert int(got[f"{cname}.{f}"]) == getattr(cls, f).offset, f"{cname}.{f}"
    assert int(got["GLR_MAX_NORM"]) == _lib.GLR_MAX_NORM


def _array(*addresses):
    arr = (ctypes.c_void_p * 64)(*addresses)
    return arr


NODES = _array(*[P + 4096 * i for i in range(64)])
HOLE, TWICE = _array(P, None), _array(P, P)
A = ctypes.addressof
GOOD = {
    "glr_embedding": (_lib.GlrEmbeddingArgs, dict(rows=4, vocab=10, d=8, E=P, lde=8, tokens=P, Y=P, ldy=8, scale=1.0)),
    "glr_embedding_grad": (_lib.GlrEmbeddingGradArgs, dict(nodes=2, rows=4, vocab=10, d=8, dY=P, lddy=8, tokens=P, dE=A(NODES),
                                                           workspace=P, workspace_bytes=1 << 20, scale=1.0)),
    "glr_checkpoint_pack": (_lib.GlrCheckpointPackArgs, dict(rows=4, cols=33, X=P, ldx=33, codes=P, ld_codes=33, scales=P, ld_scales=2)),
    "glr_checkpoint_unpack": (_lib.GlrCheckpointUnpackArgs, dict(rows=4, cols=33, codes=P, ld_codes=33, scales=P, ld_scales=2, Y=P, ldy=33)),
    "glr_linear_grad_checkpoint": (_lib.GlrLinearGradCheckpointArgs,
                                   dict(nodes=2, rows=4, n=8, k=33, dZ=P, lddz=8, W=P, ldw=33, codes=P, ld_codes=33, scales=P, ld_scales=2,
                                        dX=P, lddx=33, dW=A(NODES), db=A(NODES), workspace=P, workspace_bytes=1 << 20, act=1)),
    "glr_norm": (_lib.GlrNormArgs, dict(rows=4, n=33, X=P, ldx=33, H=P + 4096, ldh=33, Y=P + 8192, ldy=33, rstd=P, codes=P, ld_codes=33,
                                        scales=P, ld_scales=2, eps=1e-6)),
    "glr_norm_grad": (_lib.GlrNormGradArgs, dict(nodes=2, rows=4, n=33, dY=P, lddy=33, H=P + 4096, ldh=33, rstd=P, dX=P + 8192, lddx=33,
                                                 dweight=A(NODES), workspace=P, workspace_bytes=1 << 20)),
    "glr_token_logp": (_lib.GlrTokenLogpArgs, dict(rows=4, vocab=100, topk=3, logits=P, ld_logits=100, tokens=P, logp=P, lse=P, entropy=P,
                                                   top_logp=P, ld_top_logp=3, top_ids=P, ld_top_ids=3, temperature=1.0)),
    "glr_token_logp_grad": (_lib.GlrTokenLogpGradArgs, dict(rows=4, vocab=100, logits=P, ld_logits=100, tokens=P, lse=P, entropy=P, dlogp=P,
                                                            dentropy=P, dlogits=P, ld_dlogits=100, temperature=1.0)),
}


@pytest.mark.parametrize("name,change,says", [
    ("glr_embedding", dict(dtype=2), "unknown dtype"), ("glr_embedding", dict(index64=2), "index64"),
    ("glr_embedding", dict(rows=-1), "rows"), ("glr_embedding", dict(vocab=1 << 24), "2^24"), ("glr_embedding", dict(d=1 << 21), "2^20"),
    ("glr_embedding", dict(scale=float("inf")), "scale"), ("glr_embedding", dict(E=None), "E null"), ("glr_embedding", dict(lde=7), "E null"),
    ("glr_embedding", dict(Y=P + 2), "Y null"), ("glr_embedding", dict(tokens=None), "tokens"),
    ("glr_embedding", dict(tokens=P + 4, index64=1), "tokens"),
    ("glr_embedding_grad", dict(grad_dtype=2), "grad_dtype"), ("glr_embedding_grad", dict(nodes=0), "nodes"),
    ("glr_embedding_grad", dict(nodes=65), "nodes"), ("glr_embedding_grad", dict(rows=1 << 30), "nodes * rows"),
    ("glr_embedding_grad", dict(accumulate=2), "accumulate"), ("glr_embedding_grad", dict(dE=None), "dE is null"),
    ("glr_embedding_grad", dict(dE=A(HOLE)), "dE[1]"), ("glr_embedding_grad", dict(dE=A(TWICE)), "twice"),
    ("glr_embedding_grad", dict(lddy=7), "dY null"), ("glr_embedding_grad", dict(scale=float("nan")), "scale"),
    ("glr_embedding_grad", dict(rows=5000, workspace=None), "workspace"), ("glr_embedding_grad", dict(rows=5000, workspace_bytes=100), "workspace"),
    ("glr_embedding_grad", dict(rows=5000, workspace=P + 8), "workspace"), ("glr_embedding_grad", dict(vocab=-1), "vocab"),
    ("glr_checkpoint_pack", dict(dtype=-1), "unknown dtype"), ("glr_checkpoint_pack", dict(cols=1 << 25), "cols"),
    ("glr_checkpoint_pack", dict(X=None), "X null"), ("glr_checkpoint_pack", dict(codes=None), "codes"),
    ("glr_checkpoint_pack", dict(scales=None), "scales"), ("glr_checkpoint_pack", dict(ld_codes=32), "ld <"),
    ("glr_checkpoint_pack", dict(ld_scales=1), "ld <"),
    ("glr_checkpoint_unpack", dict(act=5), "activation"), ("glr_checkpoint_unpack", dict(Y=None), "Y null"),
    ("glr_checkpoint_unpack", dict(codes=None), "codes"),
    ("glr_linear_grad_checkpoint", dict(act=-1), "activation"), ("glr_linear_grad_checkpoint", dict(dW=None, db=None, dX=None), "neither"),
    ("glr_linear_grad_checkpoint", dict(dW=None), "db needs dW"), ("glr_linear_grad_checkpoint", dict(dZ=None), "dZ null"),
    ("glr_linear_grad_checkpoint", dict(codes=None), "codes"), ("glr_linear_grad_checkpoint", dict(W=None), "W null"),
    ("glr_linear_grad_checkpoint", dict(lddx=32), "dX"), ("glr_linear_grad_checkpoint", dict(residual=P, ldr=34), "same ld"),
    ("glr_linear_grad_checkpoint", dict(residual=P + 64, ldr=3), "residual"), ("glr_linear_grad_checkpoint", dict(dW=A(HOLE)), "dW[1]"),
    ("glr_linear_grad_checkpoint", dict(db=A(HOLE)), "db[1]"), ("glr_linear_grad_checkpoint", dict(dW=A(TWICE)), "twice"),
    ("glr_linear_grad_checkpoint", dict(workspace=None), "workspace"), ("glr_linear_grad_checkpoint", dict(workspace_bytes=64), "workspace"),
    ("glr_linear_grad_checkpoint", dict(nodes=0), "nodes"), ("glr_linear_grad_checkpoint", dict(grad_dtype=9), "grad_dtype"),
    ("glr_norm", dict(n=0), "need 1 <= n"), ("glr_norm", dict(n=32769), "need 1 <= n"), ("glr_norm", dict(eps=0.0), "eps"),
    ("glr_norm", dict(eps=float("nan")), "eps"), ("glr_norm", dict(X=None), "X null"), ("glr_norm", dict(ldh=32), "ld < n"),
    ("glr_norm", dict(codes=None), "go together"), ("glr_norm", dict(ld_scales=1), "ld <"), ("glr_norm", dict(H=P, ldh=34), "same ld"),
    ("glr_norm", dict(H=P + 8192), "one matrix"), ("glr_norm", dict(weight=P + 1), "weight"), ("glr_norm", dict(rows=-1), "rows"),
    ("glr_norm_grad", dict(dY=None), "dY null"), ("glr_norm_grad", dict(H=None), "H null"), ("glr_norm_grad", dict(rstd=None), "rstd"),
    ("glr_norm_grad", dict(dX=P, lddx=40), "same ld"), ("glr_norm_grad", dict(dX=P + 4096), "must not be H"),
    ("glr_norm_grad", dict(dweight=A(HOLE)), "dweight[1]"), ("glr_norm_grad", dict(dweight=A(TWICE)), "twice"),
    ("glr_norm_grad", dict(workspace=None), "workspace"), ("glr_norm_grad", dict(residual=P + 64, ldr=1), "residual"),
    ("glr_norm_grad", dict(n=40000), "need 1 <= n"), ("glr_norm_grad", dict(nodes=70), "nodes"),
    ("glr_token_logp", dict(topk=1025), "topk"), ("glr_token_logp", dict(topk=-1), "topk"), ("glr_token_logp", dict(vocab=0), "vocab"),
    ("glr_token_logp", dict(vocab=400000, ld_logits=400000), "bytes"), ("glr_token_logp", dict(tokens=None), "tokens"),
    ("glr_token_logp", dict(ld_top_ids=2), "top_ids"), ("glr_token_logp", dict(top_ids=P + 4, ids_index64=1), "top_ids"),
    ("glr_token_logp", dict(ld_top_logp=2), "top_logp"), ("glr_token_logp", dict(temperature=0.0), "temperature"),
    ("glr_token_logp", dict(temperature=1e-39), "temperature"), ("glr_token_logp", dict(ids_index64=3), "index64"),
    ("glr_token_logp", dict(rows=1 << 25), "rows"), ("glr_token_logp", dict(lse=P + 2), "lse"),
    ("glr_token_logp_grad", dict(lse=None), "lse"), ("glr_token_logp_grad", dict(tokens=None), "tokens"),
    ("glr_token_logp_grad", dict(entropy=None), "entropy"), ("glr_token_logp_grad", dict(ld_dlogits=101), "same ld"),
    ("glr_token_logp_grad", dict(dlogits=None), "dlogits"), ("glr_token_logp_grad", dict(temperature=float("nan")), "temperature"),
])
def test_refusals(lib, name, change, says):
    cls, good = GOOD[name]
    args = cls(**{**good, **change})
    assert getattr(lib, name)(ctypes.byref(args), None) == _lib.GLR_EINVAL
    msg = lib.glr_last_error(None).decode()
    assert msg.startswith(name) and says in msg, msg


def test_null_arguments(lib):
    need = ctypes.c_int64(0)
    for name in GOOD:
        assert getattr(lib, name)(None, None) == _lib.GLR_EINVAL
    for name in ("glr_embedding_grad", "glr_linear_grad_checkpoint", "glr_norm_grad"):
        cls, good = GOOD[name]
        assert getattr(lib, name + "_workspace")(None, ctypes.byref(need)) == _lib.GLR_EINVAL
        assert getattr(lib, name + "_workspace")(ctypes.byref(cls(**good)), None) == _lib.GLR_EINVAL


def test_workspace_queries(lib):
    def need(name, **change):
        cls, good = GOOD[name]
        n = ctypes.c_int64(-1)
        assert getattr(lib, name + "_workspace")(ctypes.byref(cls(**{**good, **change})), ctypes.byref(n)) == 0
        return n.value

    assert need("glr_embedding_grad", rows=5000) > 0 and need("glr_embedding_grad", rows=0) == 0 and need("glr_embedding_grad", rows=5000, d=0) == 0
    assert need("glr_norm_grad") > 0 and need("glr_norm_grad", dweight=None) == 0
    both = need("glr_linear_grad_checkpoint")
    assert both >= 8 * 33 * 4
    assert need("glr_linear_grad_checkpoint", dX=None) <= both and need("glr_linear_grad_checkpoint", dW=None, db=None) < both


def _calls():
    t, i, c, u = _Elsewhere, lambda *s: _Elsewhere(*s, dtype=torch.int64), lambda *s: _Elsewhere(*s, dtype=torch.int8), lambda *s: _Elsewhere(*s, dtype=torch.uint8)
    return {
        "glr_embedding": ((t(10, 8), i(4), t(4, 8)), {}),
        "glr_embedding_grad": ((t(4, 8), i(4), [t(10, 8), t(10, 8)]), {}),
        "glr_norm": ((t(4, 33), t(4, 33)), dict(weight=t(33), residual=t(4, 33), H=t(4, 33), rstd=t(4), codes=c(4, 33), scales=u(4, 2))),
        "glr_norm_grad": ((t(4, 33), t(4, 33), t(4), t(4, 33)), dict(weight=t(33), residual=t(4, 33), dweight=[t(33), t(33)])),
        "glr_checkpoint_pack": ((t(4, 33), c(4, 33), u(4, 2)), {}),
        "glr_checkpoint_unpack": ((c(4, 33), u(4, 2), t(4, 33)), {}),
        "glr_linear_grad_checkpoint": ((t(4, 6), c(4, 33), u(4, 2)), dict(W=t(6, 33), dX=t(4, 33), dW=[t(6, 33), t(6, 33)], db=[t(6), t(6)],
                                                                          act="silu", residual=t(4, 33))),
        "glr_token_logp": ((t(4, 9),), dict(tokens=i(4), logp=t(4), lse=t(4), entropy=t(4), top_logp=t(4, 3), top_ids=i(4, 3))),
        "glr_token_logp_grad": ((t(4, 9), t(4), t(4, 9)), dict(tokens=i(4), dlogp=t(4), entropy=t(4), dentropy=t(4))),
    }


@pytest.mark.parametrize("name", sorted(_calls()))
def test_tensors_of_a_call_lie_on_the_current_device(name, monkeypatch):
    """An argument on another device, or all of them there, never reaches the library, which takes plain addresses."""
    from paper_2507_08784_gb300 import operators
    reached = []

    class Library:
        def __getattr__(self, entry):
            return lambda *a: entry.endswith("_workspace") or reached.append(entry) or 0

    monkeypatch.setattr(operators, "load", Library)
    monkeypatch.setattr(operators, "_check", lambda rc: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    fn = getattr(operators, name)
    args, named = _calls()[name]
    fn(*args, **named, stream=0)
    assert reached == [name]
    tensors = [x for a in (*args, *named.values()) for x in (a if isinstance(a, list) else [a]) if isinstance(x, _Elsewhere)]
    for x in tensors:
        x.at = 1
        with pytest.raises(ValueError, match="device"):
            fn(*args, **named, stream=0)
        x.at = 0
    for x in tensors:
        x.at = 1
    with pytest.raises(ValueError, match="device"):
        fn(*args, **named, stream=0)
    assert reached == [name]


def test_binding_refuses_what_the_library_cannot_see():
    import paper_2507_08784_gb300 as glr
    x, i = torch.zeros(4, 6), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        glr.glr_embedding(x.double(), i, x)
    with pytest.raises(ValueError, match="int32 or int64"):
        glr.glr_embedding(x, i.float(), x)
    with pytest.raises(ValueError, match="same number"):
        glr.glr_embedding_grad(torch.zeros(5, 2), torch.zeros(5, dtype=torch.int64), [x, x])
    with pytest.raises(ValueError, match="go together"):
        glr.glr_norm(x, x, codes=torch.zeros(4, 6, dtype=torch.int8))
    with pytest.raises(ValueError, match="int8"):
        glr.glr_checkpoint_pack(x, torch.zeros(4, 6, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8))
    with pytest.raises(ValueError, match="scales must be 4 x 1"):
        glr.glr_checkpoint_pack(x, torch.zeros(4, 6, dtype=torch.int8), torch.zeros(4, 6, dtype=torch.uint8))
    with pytest.raises(ValueError, match="dX needs W"):
        glr.glr_linear_grad_checkpoint(x, torch.zeros(4, 6, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8), dX=x)
    with pytest.raises(ValueError, match="top_ids"):
        glr.glr_token_logp(x, top_logp=torch.zeros(4, 2), top_ids=torch.zeros(4, 3, dtype=torch.int64))
