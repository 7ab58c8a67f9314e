"""What the operators' entry points and their binding answer without a GPU: workspace queries and refusals."""
import ctypes

import pytest
import torch

import __graft_entry__
from paper_2507_08784_gb300 import _lib

P = 1 << 20      # an address that nothing reads


@pytest.fixture(scope="module")
def lib():
    __graft_entry__.build()
    return _lib.load()


@pytest.mark.parametrize("n,k", [(4096, 4096), (11008, 4096), (4096, 11008)])
@pytest.mark.parametrize("rows,some", [(1, False), (8, False), (16, False), (24, False), (25, True), (300, True)])
def test_workspace_is_asked_for_where_it_is_used(lib, rows, n, k, some):
    """Up to 24 rows of fp32 on 16 bytes go through the kernel that reads the weights as they are."""
    args = _lib.GlrLinearArgs(rows=rows, n=n, k=k, X=P, ldx=k, W=P, ldw=k, Y=P, ldy=n, dtype=_lib.GLR_F32, act=0)
    need = ctypes.c_int64(-1)
    assert lib.glr_linear_workspace(ctypes.byref(args), ctypes.byref(need)) == 0
    assert (need.value > 0) == some, need.value
    args.dtype = _lib.GLR_BF16
    assert lib.glr_linear_workspace(ctypes.byref(args), ctypes.byref(need)) == 0 and need.value == 0


class _Elsewhere:
    """What the binding asks of a tensor on a GPU that this machine need not have."""
    is_cuda = True

    def __init__(self, *shape, dtype=torch.float32, at=0):
        self.shape, self.dtype, self.at, self.device = torch.Size(shape), dtype, at, torch.device("cuda", at)

    def stride(self):
        return tuple(torch.empty(self.shape, device="meta").stride())

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def get_device(self):
        return self.at

    def data_ptr(self):
        return P

    def is_contiguous(self):
        return True


def _calls():
    t, i = _Elsewhere, lambda *s: _Elsewhere(*s, dtype=torch.int64)
    return {
        "glr_linear": ((t(4, 8), t(6, 8), t(4, 6)), dict(bias=t(6), residual=t(4, 6), preact=t(4, 6))),
        "glr_linear_grad_input": ((t(4, 6), t(6, 8), t(4, 8)), dict(residual=t(4, 8), preact=t(4, 8), act="silu", grad_out=t(4, 8))),
        "glr_linear_grad_weight": ((t(4, 6), t(4, 8), [t(6, 8), t(6, 8)]), dict(db=[t(6), t(6)])),
        "glr_distill_loss": ((t(4, 9), t(4, 2), i(4, 2)), dict(loss=t(1), row_loss=t(4), dlogits=t(4, 9), labels=i(4), weight=t(4))),
        "glr_policy_loss": ((t(4, 9), i(4), t(4), t(4)), dict(loss=t(1), row_loss=t(4), logp=t(4), dlogits=t(4, 9), ref_logp=t(4), weight=t(4))),
        "glr_preference_loss": ((t(4, 9), i(4), i(3)), dict(loss=t(1), pair_loss=t(1), seq_logp=t(2), row_logp=t(4), dlogits=t(4, 9),
                                                             ref_logp=t(2), weight=t(1), workspace=t(2000))),
    }


@pytest.mark.parametrize("name", sorted(_calls()))
def test_tensors_of_a_call_lie_on_the_current_device(name, monkeypatch):
    """An argument on another device, or all of them there, never reaches the library, which takes plain addresses."""
    from paper_2507_08784_gb300 import operators
    reached = []

    class Library:
        def __getattr__(self, entry):
            return lambda *a: reached.append(entry) or 0

    monkeypatch.setattr(operators, "load", Library)
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


@pytest.mark.parametrize("value", [1e-39, 1e-45, 3.1e38])
def test_reciprocals_out_of_range_are_refused(lib, value):
    """A temperature or beta whose reciprocal is not finite would make NaN of every probability."""
    distill = _lib.GlrDistillArgs(rows=4, vocab=100, topk=3, logits=P, ld_logits=100, teacher=P, ld_teacher=3, ids=P, ld_ids=3, loss=P,
                                  row_loss=P, temperature=value, soft=1.0)
    policy = _lib.GlrPolicyArgs(rows=4, vocab=100, logits=P, ld_logits=100, tokens=P, old_logp=P, advantage=P, loss=P, row_loss=P, logp=P,
                                temperature=value, clip_low=0.2, clip_high=0.2)
    preference = _lib.GlrPreferenceArgs(rows=4, vocab=100, pairs=1, logits=P, ld_logits=100, tokens=P, offsets=P, loss=P, pair_loss=P,
                                        seq_logp=P, row_logp=P, workspace=P, workspace_bytes=1 << 20, beta=value)
    for name, args, says in (("glr_distill_loss", distill, "temperature"), ("glr_policy_loss", policy, "temperature"),
                             ("glr_preference_loss", preference, "beta")):
        assert getattr(lib, name)(ctypes.byref(args), None) == _lib.GLR_EINVAL
        assert says in lib.glr_last_error(None).decode()
