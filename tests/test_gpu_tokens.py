"""The tokens example: embeddings, norms, layers from 8-bit checkpoints, log-probabilities and the compressed step
together, its gradients against the formulas in 64 bits and against differences (marked gpu).

Tolerance of a node's fp32 gradient, against its largest entry: each of the products and sums on the way carries a few
2^-19 of its terms' absolute sum, which cancellation leaves some tens of times larger than the result: 2^-12.
"""
import pytest
import torch

import _rows as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


def _case(nodes, vocab, d, hidden, per):
    from examples import tokens as ex
    net = ex.Model(vocab, d, hidden, nodes, 4, dtype=torch.float32)
    gen = torch.Generator("cuda").manual_seed(3)
    rows = nodes * per
    for g in net.g:
        g += 0.1 * torch.randn(d, device="cuda", generator=gen)
    tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=gen)
    tokens[::9] = -1                                       # padding
    answers = torch.randint(-1, vocab, (rows,), device="cuda", generator=gen)
    return net, tokens, answers, torch.randn(rows, device="cuda", generator=gen)


def _loss64(net, E, W1, W2, W3, g1, g2, tokens, answers, advantage, bonus):
    """Each node's loss, in 64 bits, from the weights."""
    keep = (tokens >= 0).double()[:, None]
    h0 = keep * net.scale * E[tokens.clamp(min=0)]
    norm = lambda h, g: h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * g  # noqa: E731
    h1 = h0 + torch.nn.functional.silu(norm(h0, g1) @ W1.T) @ W2.T
    lp = torch.log_softmax(norm(h1, g2) @ W3.T, 1)
    logp = torch.where(answers >= 0, lp.gather(1, answers.clamp(min=0)[:, None])[:, 0], 0.0)
    each = -(advantage * logp - bonus * (lp.exp() * lp).sum(1))
    return each.view(net.nodes, -1).mean(1)


@pytest.mark.parametrize("nodes,vocab,d,hidden,per", [(2, 101, 33, 50, 24), (3, 200, 64, 96, 40), (2, 300, 40, 72, 1100)])
def test_gradients(nodes, vocab, d, hidden, per):
    import paper_2507_08784_gb300 as glr
    net, tokens, answers, advantage = _case(nodes, vocab, d, hidden, per)
    logits = net.forward(tokens)
    before = logits.double().cpu()
    net.loss(logits, answers, advantage, 0.02)
    net.backward(logits)
    torch.cuda.synchronize()
    cpu = lambda x: x.double().cpu()  # noqa: E731
    # the formulas of the backward pass, in 64 bits, with the activations that were kept
    saved = []
    for codes, scales in net.saved:
        v = torch.empty(codes.shape, device="cuda")
        glr.glr_checkpoint_unpack(codes, scales, v)
        saved.append(cpu(v))
    n1, z, n2 = saved
    E, W1, W2, W3 = (cpu(w) for w in net.W)
    per_node = lambda x: x.view(nodes, per, -1)  # noqa: E731
    lp = torch.log_softmax(before, 1)
    p, ent = lp.exp(), -(lp.exp() * lp).sum(1, keepdim=True)
    a, t, k = cpu(advantage)[:, None], answers.cpu(), tokens.cpu()
    one = torch.zeros_like(p)
    ok = t >= 0
    one[ok, t[ok]] = 1.0
    dl = (-a * (one - p) * ok[:, None].double() + 0.02 * p * (lp + ent)) / per
    dn2, dW3 = dl @ W3, per_node(dl).transpose(1, 2) @ per_node(n2)
    dh1, dg2 = ref.norm_grad(dn2, cpu(net.h[1]), cpu(net.rstd[1]), cpu(net.g[1]), None, nodes)
    dz = (dh1 @ W2) * ref.act_slope(z, "silu")
    dW2 = per_node(dh1).transpose(1, 2) @ per_node(z * torch.sigmoid(z))
    dn1, dW1 = dz @ W1, per_node(dz).transpose(1, 2) @ per_node(n1)
    dh0, dg1 = ref.norm_grad(dn1, cpu(net.h[0]), cpu(net.rstd[0]), cpu(net.g[0]), dh1, nodes)
    dE, _, _ = ref.embedding_grad(dh0, k, nodes, vocab, net.scale)
    for got, want in zip([*net.dW, *net.dg], (dE, dW1, dW2, dW3, dg1, dg2)):
        for g, w in zip(got, want):
            assert torch.isfinite(g).all()
            assert float((cpu(g) - w).abs().max()) <= 2.0 ** -12 * float(w.abs().max())
    net.close()


def test_gradients_are_the_loss_slope():
    """Along a direction in all weights, the gradients give the slope of the loss (by differences in 64 bits) but for what
    8 bits of the activations change: a code is off by half a step, at most 1/127 of its block's largest element and at
    random from one to the next, so a slope summed over thousands of elements moves by far less than 2 %."""
    net, tokens, answers, advantage = _case(2, 200, 64, 96, 64)
    logits = net.forward(tokens)
    net.loss(logits, answers, advantage, 0.02)
    net.backward(logits)
    gen = torch.Generator().manual_seed(4)
    weights = [w.double().cpu() for w in (*net.W, *net.g)]
    grads = [torch.stack([g.double().cpu() for g in gs]).sum(0) for gs in (*net.dW, *net.dg)]
    # the gradient's own direction, a tenth of it at random
    way = [g / g.norm() + 0.1 * torch.randn(g.shape, generator=gen, dtype=torch.float64) / g.numel() ** 0.5 for g in grads]
    f = lambda e: float(_loss64(net, *(w + e * v for w, v in zip(weights, way)), tokens.cpu(), answers.cpu(),  # noqa: E731
                                advantage.double().cpu(), 0.02).sum())
    slope = sum(float((g * v).sum()) for g, v in zip(grads, way))
    assert abs((f(1e-5) - f(-1e-5)) / 2e-5 - slope) <= 0.02 * abs(slope)
    net.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_it_runs(dtype):
    from examples import tokens as ex
    losses = ex.train(3, vocab=120, d=64, hidden=96, nodes=2, rows=64, dtype=dtype)
    assert len(losses) == 3 and all(x == x and abs(x) < 1e3 for x in losses)
