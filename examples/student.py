"""A small student network trained through the library alone: layers, a loss on the logits, every node's gradients
and the compressed step.

    python -m examples.student --loss distill|preference|policy [--steps 60] [--dtype bf16]

The student is a feed-forward block and a head over fixed features, y = x + W2 silu(W1 x + b1) + b2, logits = W3 y,
with its rows split between N data-parallel nodes.  One step is

    glr_linear              three layers, the activation and the residual in their epilogues
    glr_distill_loss        (or glr_preference_loss, glr_policy_loss) the loss and its gradient, over the logits
    glr_linear_grad_weight  every node's gradient of a layer, as the compressed step takes it
    glr_linear_grad_input   the gradient below a layer, the activation's slope in its epilogue
    glr_step_group          GreedyLore: N gradients compressed, averaged and applied to the fp32 weights

Features, teacher and answers are synthetic.
"""
from __future__ import annotations

import argparse

import torch

import paper_2507_08784_gb300 as glr

__all__ = ["Student", "Distill", "Preference", "Policy", "train", "main"]


class Student:
    """Weights in fp32, their copies of the compute dtype, one GreedyLore handle a matrix."""

    def __init__(self, d: int, hidden: int, vocab: int, nodes: int, rank: int, *, dtype=torch.bfloat16, lr: float = 0.0005,
                 seed: int = 0):
        gen = torch.Generator("cuda").manual_seed(seed)
        shapes = ((hidden, d), (d, hidden), (vocab, d))
        self.nodes, self.dtype, self.lr = nodes, dtype, lr
        self.master = [torch.randn(m, n, device="cuda", generator=gen) * n ** -0.5 for m, n in shapes]
        self.bias = [torch.zeros(m, device="cuda") for m, _ in shapes[:2]]
        self.W = [w.to(dtype) for w in self.master]
        self.b = [b.to(dtype) for b in self.bias]
        gd = torch.bfloat16 if dtype == torch.bfloat16 else torch.float32
        self.dW = [[torch.empty(m, n, device="cuda", dtype=gd) for _ in range(nodes)] for m, n in shapes]
        self.db = [[torch.empty(m, device="cuda", dtype=gd) for _ in range(nodes)] for m, _ in shapes[:2]]
        self.handles = [glr.GreedyLore(m, n, min(rank, m, n), nodes, tau=10, optimizer="adam", lr=lr, beta1=0.9, beta2=0.99,
                                       grad_dtype="bf16" if gd == torch.bfloat16 else "f32") for m, n in shapes]

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """The logits of the rows of x; keeps what the backward pass reads."""
        (h, d), vocab, rows = self.W[0].shape, self.W[2].shape[0], x.shape[0]
        new = lambda n: torch.empty(rows, n, device="cuda", dtype=self.dtype)  # noqa: E731
        self.x, self.z, self.a, self.y, logits = x, new(h), new(h), new(d), new(vocab)
        glr.glr_linear(x, self.W[0], self.a, bias=self.b[0], act="silu", preact=self.z)
        glr.glr_linear(self.a, self.W[1], self.y, bias=self.b[1], residual=x)
        glr.glr_linear(self.y, self.W[2], logits)
        return logits

    def backward(self, dlogits: torch.Tensor) -> None:
        """Every node's gradients from those of its rows' logits."""
        dy, dz = torch.empty_like(self.y), torch.empty_like(self.z)
        glr.glr_linear_grad_weight(dlogits, self.y, self.dW[2])
        glr.glr_linear_grad_input(dlogits, self.W[2], dy)
        glr.glr_linear_grad_weight(dy, self.a, self.dW[1], db=self.db[1])
        glr.glr_linear_grad_input(dy, self.W[1], dz, preact=self.z, act="silu")
        glr.glr_linear_grad_weight(dz, self.x, self.dW[0], db=self.db[0])

    def step(self) -> None:
        glr.glr_step_group(self.handles, self.dW, self.master)
        for bias, grads in zip(self.bias, self.db):           # vectors are averaged as they are
            bias -= self.lr * torch.stack(grads).float().mean(0)
        for to, w in zip(self.W + self.b, self.master + self.bias):
            to.copy_(w)

    def close(self) -> None:
        for h in self.handles:
            h.close()


def _outputs(*sizes: int):
    return [torch.empty(n, device="cuda") for n in sizes]


class Distill:
    """A teacher's 16 largest logits a row, its first choice as label."""

    def __init__(self, student: Student, x: torch.Tensor, teacher: torch.Tensor):
        rows, self.nodes = x.shape[0], student.nodes
        top = (x.float() @ teacher.T).topk(min(16, teacher.shape[0]))
        self.teacher, self.ids, self.labels = top.values.contiguous(), top.indices.int(), top.indices[:, 0].contiguous()
        self.weight = torch.full((rows,), self.nodes / rows, device="cuda")     # each node's loss is its rows' mean
        self.loss, self.row = _outputs(1, rows)

    def __call__(self, logits: torch.Tensor) -> torch.Tensor:
        """Leaves the gradient where the logits were, and returns the nodes' mean loss."""
        glr.glr_distill_loss(logits, self.teacher, self.ids, loss=self.loss, row_loss=self.row, dlogits=logits,
                             labels=self.labels, weight=self.weight, temperature=2.0, soft=4.0, hard=0.5)
        return self.loss / self.nodes


class Preference:
    """Pairs of answers of 8 tokens: the teacher's choices against tokens at random, relative to the student at the start."""

    length = 8

    def __init__(self, student: Student, x: torch.Tensor, teacher: torch.Tensor):
        rows, self.nodes = x.shape[0], student.nodes
        if rows % (2 * self.length * self.nodes):
            raise ValueError(f"rows must be a multiple of {2 * self.length * self.nodes}")
        pairs, gen = rows // (2 * self.length), torch.Generator("cuda").manual_seed(1)
        chosen = (x.float() @ teacher.T).argmax(1)
        random = torch.randint(0, teacher.shape[0], (rows,), device="cuda", generator=gen)
        rejected = torch.arange(rows, device="cuda") // self.length % 2 == 1
        self.tokens = torch.where(rejected, random, chosen)
        self.offsets = torch.arange(0, rows + 1, self.length, device="cuda")
        self.weight = torch.full((pairs,), self.nodes / pairs, device="cuda")
        self.out = dict(zip(("loss", "pair_loss", "seq_logp", "row_logp", "workspace"),
                            _outputs(1, pairs, 2 * pairs, rows, 4 * rows + 16 * pairs + 1024)))
        glr.glr_preference_loss(student.forward(x), self.tokens, self.offsets, **self.out)
        self.ref = self.out["seq_logp"].clone()

    def __call__(self, logits: torch.Tensor) -> torch.Tensor:
        glr.glr_preference_loss(logits, self.tokens, self.offsets, dlogits=logits, ref_logp=self.ref, weight=self.weight,
                                beta=0.1, **self.out)
        return self.out["loss"] / self.nodes


class Policy:
    """Tokens drawn from the student at the start, rewarded where the teacher ranks them among its 16 first."""

    def __init__(self, student: Student, x: torch.Tensor, teacher: torch.Tensor):
        rows, self.nodes = x.shape[0], student.nodes
        logits, best = student.forward(x), x.float() @ teacher.T
        gen = torch.Generator("cuda").manual_seed(2)
        self.tokens = torch.multinomial(torch.softmax(logits.float(), 1), 1, generator=gen)[:, 0].contiguous()
        rank = (best > best.gather(1, self.tokens[:, None])).sum(1)
        reward = (rank < 16).float()
        self.advantage = ((reward - reward.mean()) / (reward.std() + 1e-6)).contiguous()
        self.weight = torch.full((rows,), self.nodes / rows, device="cuda")
        self.out = dict(zip(("loss", "row_loss", "logp"), _outputs(1, rows, rows)))
        glr.glr_policy_loss(logits, self.tokens, torch.zeros_like(self.advantage), self.advantage, **self.out)
        self.old = self.out["logp"].clone()

    def __call__(self, logits: torch.Tensor) -> torch.Tensor:
        glr.glr_policy_loss(logits, self.tokens, self.old, self.advantage, dlogits=logits, ref_logp=self.old, weight=self.weight,
                            kl=0.02, **self.out)
        return self.out["loss"] / self.nodes


LOSSES = {"distill": Distill, "preference": Preference, "policy": Policy}


def train(kind: str, *, steps: int = 60, d: int = 256, hidden: int = 512, vocab: int = 1000, nodes: int = 4, rows: int = 512,
          rank: int = 16, dtype=torch.bfloat16, lr: float = 0.0005, seed: int = 0):
    """`steps` steps on one batch of features (rows of all nodes together); the losses, one of each step, on the device."""
    student = Student(d, hidden, vocab, nodes, rank, dtype=dtype, lr=lr, seed=seed)
    gen = torch.Generator("cuda").manual_seed(seed + 1)
    x = torch.randn(rows, d, device="cuda", generator=gen).to(dtype)
    teacher = torch.randn(vocab, d, device="cuda", generator=gen) * 3 * d ** -0.5
    loss = LOSSES[kind](student, x, teacher)
    losses = []
    for _ in range(steps):
        logits = student.forward(x)
        losses.append(loss(logits))
        student.backward(logits)                              # the loss left its gradient there
        student.step()
    glr.glr_operator_status()
    student.close()
    return torch.cat(losses)


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--loss", choices=sorted(LOSSES), default="distill")
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--nodes", type=int, default=4)
    p.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = p.parse_args()
    losses = train(a.loss, steps=a.steps, nodes=a.nodes, dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32).tolist()
    for t in range(0, a.steps, max(1, a.steps // 10)):
        print(f"step {t:4d}  {a.loss} loss {losses[t]:.4f}")
    print(f"step {a.steps - 1:4d}  {a.loss} loss {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
