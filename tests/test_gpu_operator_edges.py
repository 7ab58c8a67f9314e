"""The operators around the step at the edges of what they promise: kernels that read what the one before them wrote,
the ends of the floating-point range, terms without a coefficient (marked gpu)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 4, 8, 24, 2048])
def test_kernels_read_what_the_one_before_wrote(rows, dt):
    """Two layers and the second one's gradients back to back, each reading the buffers that the call before has just
    written, which change from repetition to repetition: the same bits as with a pause after every call."""
    import paper_2507_08784_gb300 as glr
    dt, d, h, o = DT[dt], 512, 1024, 264
    gen = torch.Generator().manual_seed(rows)
    W1, W2 = (torch.randn(*s, generator=gen).to(dt).cuda() for s in ((h, d), (o, h)))
    xs = [torch.randn(rows, d, generator=gen).to(dt).cuda() for _ in range(12)]
    hid, out = torch.empty(rows, h, device="cuda", dtype=dt), torch.empty(rows, o, device="cuda", dtype=dt)

    def run(pause):
        hid.zero_(), out.zero_()
        torch.cuda.synchronize()
        results = []
        for x in xs:
            dW, db = torch.empty(o, h, device="cuda", dtype=dt), torch.empty(o, device="cuda", dtype=dt)
            for call in (lambda: glr.glr_linear(x, W1, hid, act="silu"), lambda: glr.glr_linear(hid, W2, out),
                         lambda: glr.glr_linear_grad_weight(out, hid, dW, db=db)):
                call()
                if pause:
                    torch.cuda.synchronize()
            results.append((out.clone(), dW, db) if pause else (dW, db))
        torch.cuda.synchronize()
        return results

    for (want_out, want_dw, want_db), (dw, db) in zip(run(True), run(False)):
        assert torch.equal(dw, want_dw) and torch.equal(db, want_db) and want_out.any()
