"""The student example: its gradients against automatic differentiation of the definitions in 64 bits, and its
losses over steps of the compressed optimizer (marked gpu).

Tolerance of a node's fp32 gradient, against its largest entry: each of the six products on the way carries a few
2^-19 of its terms' absolute sum, which cancellation leaves some tens of times larger than the result: 2^-12.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


def _loss(kind, task, logits, rows):
    """Each node's share of the nodes' mean loss, from 64-bit logits."""
    per = logits.shape[0] // task.nodes
    if kind == "distill":
        q = torch.softmax(task.teacher.double().cpu() / 2.0, 1)
        ids = task.ids.long().cpu()
        lp = torch.log_softmax(logits / 2.0, 1).gather(1, ids)
        hard = -torch.log_softmax(logits, 1).gather(1, task.labels.cpu()[:, None])[:, 0]
        each = 4.0 * (q * (q.log() - lp)).sum(1) + 0.5 * hard
        return each.view(task.nodes, per).mean(1)
    logp = torch.log_softmax(logits, 1).gather(1, task.tokens.cpu()[:, None])[:, 0]
    if kind == "preference":
        seq = logp.view(-1, task.length).sum(1) - task.ref.double().cpu()
        each = -torch.nn.functional.logsigmoid(0.1 * (seq[0::2] - seq[1::2]))
        return each.view(task.nodes, -1).mean(1)
    old, adv = task.old.double().cpu(), task.advantage.double().cpu()
    ratio = torch.exp(logp - old)
    each = -torch.minimum(ratio * adv, ratio.clamp(0.8, 1.2) * adv) + 0.02 * (torch.exp(old - logp) - (old - logp) - 1)
    return each.view(task.nodes, per).mean(1)


@pytest.mark.parametrize("kind", ["distill", "preference", "policy"])
@pytest.mark.parametrize("nodes,d,hidden,vocab", [(2, 33, 50, 101), (3, 64, 96, 200)])
def test_gradients(kind, nodes, d, hidden, vocab):
    from examples import student as ex
    rows = 48 * nodes
    net = ex.Student(d, hidden, vocab, nodes, 4, dtype=torch.float32)
    gen = torch.Generator("cuda").manual_seed(5)
    x = torch.randn(rows, d, device="cuda", generator=gen)
    task = ex.LOSSES[kind](net, x, torch.randn(vocab, d, device="cuda", generator=gen) * d ** -0.5)
    for w in net.W:                                   # away from where the reference probabilities were taken
        w += 0.02 * torch.randn(w.shape, device="cuda", generator=gen) * w.shape[1] ** -0.5
    logits = net.forward(x)
    loss = task(logits)
    net.backward(logits)
    W = [w.double().cpu().requires_grad_() for w in net.W]
    b = [v.double().cpu().requires_grad_() for v in net.b]
    X = x.double().cpu()
    Y = X + torch.nn.functional.silu(X @ W[0].T + b[0]) @ W[1].T + b[1]
    shares = _loss(kind, task, Y @ W[2].T, rows)
    mean = float(shares.detach().mean())
    assert abs(float(loss) - mean) <= 1e-4 * (1 + abs(mean))
    for i in range(nodes):
        grads = torch.autograd.grad(shares[i], W + b, retain_graph=True)
        for got, want in zip([g[i] for g in net.dW] + [g[i] for g in net.db], grads):
            assert float((got.double().cpu() - want).abs().max()) <= 2.0 ** -12 * float(want.abs().max()), (kind, i, want.shape)
    net.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["distill", "preference", "policy"])
def test_losses_fall(kind, dtype):
    from examples import student as ex
    losses = ex.train(kind, steps=40, dtype=dtype).tolist()
    assert all(v == v for v in losses)
    assert losses[-1] < losses[0] - 0.05 * abs(losses[0]), losses


def test_the_same_run_gives_the_same_losses():
    from examples import student as ex
    a, b = (ex.train("distill", steps=12) for _ in range(2))
    assert torch.equal(a, b)
