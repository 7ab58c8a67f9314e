"""A small language model trained through the library alone, from tokens to the compressed step, with its activations kept
in 8 bits for the backward pass.

    python -m examples.tokens [--steps 40] [--dtype bf16]

    h0 = s E[token],  n1 = norm(h0),  z = W1 n1,  h1 = h0 + W2 silu(z),  n2 = norm(h1),  logits = W3 n2

with the rows split between N data-parallel nodes.  It raises the log-probabilities of answers by their advantage, with a
bonus for the entropy.  One step is

    glr_embedding                the rows of E
    glr_norm                     both norms, the residual's addition in the second; n1 and n2 in 8 bits
    glr_linear                   three layers; glr_checkpoint_pack keeps z in 8 bits
    glr_token_logp               log-probabilities and entropies of the logits
    glr_token_logp_grad          the logits' gradient, in their place
    glr_linear_grad_checkpoint   each layer's backward pass, its input from the 8 bits
    glr_norm_grad                the norms', with the gradient that passes by
    glr_embedding_grad           every node's gradient of E
    glr_step_group               GreedyLore: N gradients of each matrix compressed, averaged and applied

Nothing of the forward pass but h0 and h1 is kept in the layers' own type.  Tokens, answers and advantages are synthetic.
"""
from __future__ import annotations

import argparse

import torch

import paper_2507_08784_gb300 as glr

__all__ = ["Model", "train", "main"]


class Model:
    """Weights in fp32, their copies of the compute dtype, one GreedyLore handle a matrix."""

    def __init__(self, vocab: int, d: int, hidden: int, nodes: int, rank: int, *, dtype=torch.bfloat16, lr: float = 0.002, seed: int = 0):
        gen = torch.Generator("cuda").manual_seed(seed)
        shapes = ((vocab, d), (hidden, d), (d, hidden), (vocab, d))              # E, W1, W2, W3
        self.nodes, self.dtype, self.lr, self.scale = nodes, dtype, lr, float(d) ** 0.5
        self.master = [torch.randn(m, n, device="cuda", generator=gen) * n ** -0.5 for m, n in shapes]
        self.gain = [torch.ones(d, device="cuda") for _ in range(2)]
        self.W = [w.to(dtype) for w in self.master]
        self.g = [w.to(dtype) for w in self.gain]
        gd = torch.bfloat16 if dtype == torch.bfloat16 else torch.float32
        self.dW = [[torch.empty(m, n, device="cuda", dtype=gd) for _ in range(nodes)] for m, n in shapes]
        self.dg = [[torch.empty(d, device="cuda") for _ in range(nodes)] for _ in range(2)]
        self.handles = [glr.GreedyLore(m, n, min(rank, m, n), nodes, tau=10, optimizer="adam", lr=lr, beta1=0.9, beta2=0.99,
                                       grad_dtype="bf16" if gd == torch.bfloat16 else "f32") for m, n in shapes]

    def _new(self, rows: int, n: int) -> torch.Tensor:
        return torch.empty(rows, n, device="cuda", dtype=self.dtype)

    def _bits(self, rows: int, n: int):
        return (torch.empty(rows, n, device="cuda", dtype=torch.int8),
                torch.empty(rows, (n + 31) // 32, device="cuda", dtype=torch.uint8))

    def forward(self, tokens: torch.Tensor) -> torch.Tensor:
        """The logits of a row for each token; keeps what the backward pass reads."""
        (_, d), (hidden, _), (vocab, _) = self.W[0].shape, self.W[1].shape, self.W[3].shape
        rows, new = tokens.numel(), self._new
        self.tokens, self.h = tokens, [new(rows, d), new(rows, d)]
        self.rstd = [torch.empty(rows, device="cuda") for _ in range(2)]
        self.saved = [self._bits(rows, d), self._bits(rows, hidden), self._bits(rows, d)]       # n1, z, n2
        n, z, a, y, logits = new(rows, d), new(rows, hidden), new(rows, hidden), new(rows, d), new(rows, vocab)
        glr.glr_embedding(self.W[0], tokens, self.h[0], scale=self.scale)
        glr.glr_norm(self.h[0], n, weight=self.g[0], rstd=self.rstd[0], codes=self.saved[0][0], scales=self.saved[0][1])
        glr.glr_linear(n, self.W[1], a, act="silu", preact=z)
        glr.glr_checkpoint_pack(z, *self.saved[1])
        glr.glr_linear(a, self.W[2], y)
        glr.glr_norm(y, n, weight=self.g[1], residual=self.h[0], H=self.h[1], rstd=self.rstd[1], codes=self.saved[2][0],
                     scales=self.saved[2][1])
        glr.glr_linear(n, self.W[3], logits)
        return logits

    def backward(self, dlogits: torch.Tensor) -> None:
        """Every node's gradients from those of its rows' logits."""
        rows = dlogits.shape[0]
        (_, d), (hidden, _) = self.W[0].shape, self.W[1].shape
        dn, dh, dz = self._new(rows, d), self._new(rows, d), self._new(rows, hidden)
        glr.glr_linear_grad_checkpoint(dlogits, *self.saved[2], W=self.W[3], dX=dn, dW=self.dW[3])
        glr.glr_norm_grad(dn, self.h[1], self.rstd[1], dh, weight=self.g[1], dweight=self.dg[1])
        glr.glr_linear_grad_checkpoint(dh, *self.saved[1], W=self.W[2], dX=dz, dW=self.dW[2], act="silu")
        glr.glr_linear_grad_checkpoint(dz, *self.saved[0], W=self.W[1], dX=dn, dW=self.dW[1])
        glr.glr_norm_grad(dn, self.h[0], self.rstd[0], dh, weight=self.g[0], residual=dh, dweight=self.dg[0])
        glr.glr_embedding_grad(dh, self.tokens, self.dW[0], scale=self.scale)

    def loss(self, logits: torch.Tensor, answers: torch.Tensor, advantage: torch.Tensor, bonus: float) -> torch.Tensor:
        """Leaves the gradient where the logits were; returns the nodes' mean of -advantage logp - bonus entropy."""
        rows = logits.shape[0]
        logp, lse, entropy = (torch.empty(rows, device="cuda") for _ in range(3))
        glr.glr_token_logp(logits, tokens=answers, logp=logp, lse=lse, entropy=entropy)
        share = self.nodes / rows                             # each node's loss is its rows' mean
        glr.glr_token_logp_grad(logits, lse, logits, tokens=answers, dlogp=-share * advantage, entropy=entropy,
                                dentropy=torch.full_like(entropy, -share * bonus))
        return -(advantage * logp + bonus * entropy).mean()

    def step(self) -> None:
        glr.glr_step_group(self.handles, self.dW, self.master)
        for gain, grads in zip(self.gain, self.dg):           # vectors are averaged as they are
            gain -= self.lr * torch.stack(grads).mean(0)
        for to, w in zip(self.W + self.g, self.master + self.gain):
            to.copy_(w)

    def close(self) -> None:
        for h in self.handles:
            h.close()


def train(steps: int = 40, *, vocab: int = 512, d: int = 128, hidden: int = 384, nodes: int = 4, rows: int = 512, rank: int = 8,
          dtype=torch.bfloat16, seed: int = 0):
    """The losses of `steps` steps on one synthetic batch: rows tokens, an answer and an advantage for each."""
    gen = torch.Generator("cuda").manual_seed(seed + 1)
    model = Model(vocab, d, hidden, nodes, rank, dtype=dtype, seed=seed)
    tokens, answers = (torch.randint(0, vocab, (rows,), device="cuda", generator=gen) for _ in range(2))
    advantage = 0.5 + torch.rand(rows, device="cuda", generator=gen)
    losses = []
    try:
        for _ in range(steps):
            logits = model.forward(tokens)
            losses.append(float(model.loss(logits, answers, advantage, 0.01)))
            model.backward(logits)
            model.step()
    finally:
        model.close()
    return losses


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=40)
    p.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = p.parse_args()
    losses = train(a.steps, dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    for t in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {t:4d}  loss {losses[t]:.4f}")
    print(f"step {len(losses) - 1:4d}  loss {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
