"""What the operators' entry points and their binding answer without a GPU: workspace queries and refusals."""
import ctypes

import pytest

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
