"""The row operators at the edges of what they promise: alternatives of rows that hold NaNs (marked gpu)."""
import math

import pytest
import torch

from test_gpu_rows import Guarded

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


@pytest.fixture(scope="module")
def glr(_lib):
    import paper_2507_08784_gb300
    return paper_2507_08784_gb300


# ------------------------------------------------------------------------------------------- log-probabilities

def _alternatives(glr, z, topk, tau=0.7):
    """top_logp, top_ids, logp, lse and entropy on the CPU."""
    rows = z.shape[0]
    top, ids = Guarded(rows, topk, torch.float32, 1), Guarded(rows, topk, torch.int32, 3)
    out = [torch.full((rows,), 55.0, device="cuda") for _ in range(3)]
    glr.glr_token_logp(z, tokens=torch.zeros(rows, dtype=torch.int32, device="cuda"), logp=out[0], lse=out[1], entropy=out[2], top_logp=top.t,
                       top_ids=ids.t, temperature=tau)
    torch.cuda.synchronize()
    return top.check().cpu(), ids.check().cpu().long(), [x.cpu() for x in out]


def _ordered(z, topk):
    """Ids in descending order of the logits, a NaN above all, equal ones by index, -1 where only ruled-out entries are left."""
    rows, vocab = z.shape
    order = torch.sort(torch.where(z.isnan(), math.inf, z.double()), dim=1, descending=True, stable=True).indices
    ids = torch.where(z.gather(1, order) == -math.inf, -1, order)[:, :topk]
    return torch.nn.functional.pad(ids, (0, max(0, topk - vocab)), value=-1)


# a CTA a row of 64, 128 and 256 threads, and clusters of two, four and eight
@pytest.mark.parametrize("rows,vocab", [(3, 8), (400, 64), (200, 1000), (200, 5000), (160, 24576), (2, 16384), (2, 40000), (1, 131072)])
@pytest.mark.parametrize("topk", [1, 12, 64, 300, 1024])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_alternatives_of_whole_vectors_of_nan(glr, rows, vocab, topk, dt):
    """NaNs that fill whole groups of eight on 16 bytes count as the largest logits like any others, and their rows' results are NaN."""
    gen = torch.Generator().manual_seed(vocab + topk)
    z = torch.randn(rows, vocab, generator=gen).to(DT[dt])
    z[:, 5::11] = -math.inf
    z[0] = math.nan                                                   # a whole row
    if rows > 1:
        z[1, vocab // 16 * 8:vocab // 16 * 8 + 8] = math.nan          # one group among finite and ruled-out entries
    if rows > 2:
        z[2, :vocab // 2] = math.nan                                  # half a row
        z[2, vocab - 1] = math.nan
    top, ids, rest = _alternatives(glr, z.cuda(), topk)
    assert torch.equal(ids, _ordered(z, topk))
    nan = z.isnan().any(1)
    assert torch.equal(top[nan].isnan(), ids[nan] >= 0) and (top[nan][ids[nan] < 0] == -math.inf).all()
    assert torch.equal(top[~nan] == -math.inf, ids[~nan] < 0) and not top[~nan].isnan().any()
    for x in rest:
        assert torch.equal(x.isnan(), nan)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 5])
def test_alternatives_of_a_broken_teacher(glr, dt, shift):
    """A row of NaNs, at any place in memory, is a teacher whose loss is NaN, not one that costs nothing."""
    rows, vocab, topk = 4, 800, 16
    z = Guarded(rows, vocab, DT[dt], 0, shift, value=torch.randn(rows, vocab, generator=torch.Generator().manual_seed(2)))
    z.t[2] = math.nan
    top, ids = torch.empty(rows, topk, device="cuda"), torch.empty(rows, topk, device="cuda", dtype=torch.int32)
    glr.glr_token_logp(z.t, top_logp=top, top_ids=ids)
    assert ids[2].tolist() == list(range(topk)) and top[2].isnan().all()
    student = torch.randn(rows, vocab, device="cuda")
    loss, row, d = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(student)
    glr.glr_distill_loss(student, top, ids, loss=loss, row_loss=row, dlogits=d)
    assert loss.isnan().all() and row.isnan().tolist() == [False, False, True, False]
