"""Host-side checks of the operators' C entry points and their binding that need no GPU: struct layouts, and
the refusals, which come before any device work."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import __graft_entry__
from paper_2507_08784_gb300 import _lib

STRUCTS = {"glr_linear_args": _lib.GlrLinearArgs, "glr_linear_grad_input_args": _lib.GlrLinearGradInputArgs,
           "glr_linear_grad_weight_args": _lib.GlrLinearGradWeightArgs, "glr_distill_args": _lib.GlrDistillArgs,
           "glr_policy_args": _lib.GlrPolicyArgs, "glr_preference_args": _lib.GlrPreferenceArgs}


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
    for c in ("GLR_MAX_TOPK", "GLR_MAX_LOGIT_BYTES", "GLR_ACT_SILU", "GLR_ACT_GELU_TANH", "GLR_PREF_IPO"):
        lines.append(f'printf("{c} %d\\n", (int){c});')
    lines.append('printf("workspace %d\\n", (int)GLR_PREFERENCE_WORKSPACE(10, 3));')
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
    for c in ("GLR_MAX_TOPK", "GLR_MAX_LOGIT_BYTES", "GLR_ACT_SILU", "GLR_ACT_GELU_TANH", "GLR_PREF_IPO"):
        assert int(got[c]) == getattr(_lib, c)
    assert int(got["workspace"]) == 4 * (4 * 10 + 16 * 3 + 1024)


P = 1 << 20      # an address that nothing reads: every call here is refused before device work

LINEAR = dict(rows=4, n=8, k=16, X=P, ldx=16, W=P, ldw=16, Y=P, ldy=8, dtype=0, act=0)
GRAD_INPUT = dict(rows=4, n=8, k=16, dZ=P, lddz=8, W=P, ldw=16, dX=P, lddx=16, dtype=0, act=0)
DISTILL = dict(rows=4, vocab=100, topk=3, logits=P, ld_logits=100, teacher=P, ld_teacher=3, ids=P, ld_ids=3, loss=P,
               row_loss=P, dtype=0, teacher_dtype=0, temperature=1.0, soft=1.0)
POLICY = dict(rows=4, vocab=100, logits=P, ld_logits=100, tokens=P, old_logp=P, advantage=P, loss=P, row_loss=P, logp=P,
              dtype=1, temperature=1.0, clip_low=0.2, clip_high=0.2)
PREFERENCE = dict(rows=4, vocab=100, pairs=1, logits=P, ld_logits=100, tokens=P, offsets=P, loss=P, pair_loss=P, seq_logp=P,
                  row_logp=P, workspace=P, workspace_bytes=1 << 20, dtype=0, beta=0.1)


@pytest.mark.parametrize("name,cls,good,change,says", [
    ("glr_linear", _lib.GlrLinearArgs, LINEAR, dict(dtype=2), "unknown dtype"),
    ("glr_linear", _lib.GlrLinearArgs, LINEAR, dict(act=5), "unknown activation"),
    ("glr_linear", _lib.GlrLinearArgs, LINEAR, dict(rows=-1), "rows"),
    ("glr_linear", _lib.GlrLinearArgs, LINEAR, dict(n=1 << 25), "2^24"),
    ("glr_linear", _lib.GlrLinearArgs, LINEAR, dict(X=None), "X or W"),
    ("glr_linear", _lib.GlrLinearArgs, LINEAR, dict(ldw=15), "ld < k"),
    ("glr_linear", _lib.GlrLinearArgs, LINEAR, dict(X=P + 2), "misaligned"),
    ("glr_linear", _lib.GlrLinearArgs, LINEAR, dict(Y=None), "Y null"),
    ("glr_linear", _lib.GlrLinearArgs, LINEAR, dict(bias=P + 1), "bias"),
    ("glr_linear", _lib.GlrLinearArgs, LINEAR, dict(residual=P + 64, ldr=7), "residual"),
    ("glr_linear", _lib.GlrLinearArgs, LINEAR, dict(residual=P, ldr=9), "same ld"),
    ("glr_linear", _lib.GlrLinearArgs, LINEAR, dict(preact=P, ldp=1), "preact"),
    ("glr_linear_grad_input", _lib.GlrLinearGradInputArgs, GRAD_INPUT, dict(act=1), "needs preact"),
    ("glr_linear_grad_input", _lib.GlrLinearGradInputArgs, GRAD_INPUT, dict(dZ=None), "dZ null"),
    ("glr_linear_grad_input", _lib.GlrLinearGradInputArgs, GRAD_INPUT, dict(W=None), "W null"),
    ("glr_linear_grad_input", _lib.GlrLinearGradInputArgs, GRAD_INPUT, dict(lddx=15), "dX null"),
    ("glr_linear_grad_input", _lib.GlrLinearGradInputArgs, GRAD_INPUT, dict(grad_out=P, ldg=3), "grad_out"),
    ("glr_linear_grad_input", _lib.GlrLinearGradInputArgs, GRAD_INPUT, dict(residual=P, ldr=20), "same ld"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(topk=1025), "topk"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(vocab=0), "vocab"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(vocab=400000, ld_logits=400000), "bytes"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(ids=None), "ids"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(ids=P + 4, ids_index64=1), "ids"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(ids_index64=2), "index64"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(teacher=None), "teacher"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(teacher_dtype=7), "teacher_dtype"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(temperature=0.0), "temperature"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(temperature=float("nan")), "temperature"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(soft=float("inf")), "soft"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(row_loss=None), "row_loss"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(loss=None), "loss is null"),
    ("glr_distill_loss", _lib.GlrDistillArgs, DISTILL, dict(dlogits=P, ld_dlogits=101), "same ld"),
    ("glr_policy_loss", _lib.GlrPolicyArgs, POLICY, dict(tokens=None), "tokens"),
    ("glr_policy_loss", _lib.GlrPolicyArgs, POLICY, dict(old_logp=None), "old_logp"),
    ("glr_policy_loss", _lib.GlrPolicyArgs, POLICY, dict(clip_low=-0.1), "clip_low"),
    ("glr_policy_loss", _lib.GlrPolicyArgs, POLICY, dict(clip_high=float("nan")), "clip_low"),
    ("glr_policy_loss", _lib.GlrPolicyArgs, POLICY, dict(logp=None), "logp"),
    ("glr_policy_loss", _lib.GlrPolicyArgs, POLICY, dict(ref_logp=P + 2), "ref_logp"),
    ("glr_policy_loss", _lib.GlrPolicyArgs, POLICY, dict(ld_logits=99), "logits"),
    ("glr_preference_loss", _lib.GlrPreferenceArgs, PREFERENCE, dict(workspace_bytes=100), "workspace"),
    ("glr_preference_loss", _lib.GlrPreferenceArgs, PREFERENCE, dict(workspace=P + 4), "workspace"),
    ("glr_preference_loss", _lib.GlrPreferenceArgs, PREFERENCE, dict(offsets=None), "offsets"),
    ("glr_preference_loss", _lib.GlrPreferenceArgs, PREFERENCE, dict(beta=0.0), "beta"),
    ("glr_preference_loss", _lib.GlrPreferenceArgs, PREFERENCE, dict(smoothing=1.5), "smoothing"),
    ("glr_preference_loss", _lib.GlrPreferenceArgs, PREFERENCE, dict(kind=2), "kind"),
    ("glr_preference_loss", _lib.GlrPreferenceArgs, PREFERENCE, dict(average=2), "average"),
    ("glr_preference_loss", _lib.GlrPreferenceArgs, PREFERENCE, dict(pairs=-1), "pairs"),
])
def test_refusals(lib, name, cls, good, change, says):
    args = cls(**{**good, **change})
    assert getattr(lib, name)(ctypes.byref(args), None) == _lib.GLR_EINVAL
    msg = lib.glr_last_error(None).decode()
    assert msg.startswith(name) and says in msg


@pytest.mark.parametrize("change,says", [
    (dict(nodes=0), "nodes"), (dict(nodes=65), "nodes"), (dict(dW=None), "dW is null"), (dict(grad_dtype=3), "grad_dtype"),
    (dict(lddz=7), "dZ null"), (dict(X=None), "X null"), (dict(hole=1), "dW[1]"), (dict(db_hole=1), "db[1]"),
])
def test_grad_weight_refusals(lib, change, says):
    dw, db = (ctypes.c_void_p * 64)(*[P] * 64), (ctypes.c_void_p * 64)(*[P] * 64)
    if "hole" in change:
        dw[1] = None
    if "db_hole" in change:
        db[1] = P + 2
    good = dict(nodes=2, rows=4, n=8, k=16, dZ=P, lddz=8, X=P, ldx=16, dW=ctypes.addressof(dw), db=ctypes.addressof(db))
    good.update({k: v for k, v in change.items() if "hole" not in k})
    args = _lib.GlrLinearGradWeightArgs(**good)
    assert lib.glr_linear_grad_weight(ctypes.byref(args), None) == _lib.GLR_EINVAL
    assert says in lib.glr_last_error(None).decode()


def test_null_arguments(lib):
    for name in ("glr_linear", "glr_linear_grad_input", "glr_linear_grad_weight", "glr_distill_loss", "glr_policy_loss",
                 "glr_preference_loss"):
        assert getattr(lib, name)(None, None) == _lib.GLR_EINVAL


def test_binding_refuses_what_the_library_cannot_see():
    """Shapes, types and devices are the binding's to check (CPU tensors never reach the library)."""
    import paper_2507_08784_gb300 as glr
    x = torch.zeros(4, 6)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        glr.glr_linear(x.double(), x, x)
    with pytest.raises(ValueError, match="CUDA"):
        glr.glr_linear(x, torch.zeros(3, 6), torch.zeros(4, 3))
    with pytest.raises(ValueError, match="one of"):
        glr.glr_preference_loss(x, torch.zeros(4), torch.zeros(3), loss=x, pair_loss=x, seq_logp=x, row_logp=x, kind="no")
    with pytest.raises(ValueError, match="same number of rows"):
        glr.glr_linear_grad_weight(torch.zeros(5, 2), torch.zeros(5, 3), [x, x])
