"""Data-parallel training of a token table with compressed pushes and pulls.

Two workers and a server, in one process on one GPU.  Every step each worker
  looks up the rows of its tokens in its bf16 copy of the table, scaled;
  predicts the next token from them (a linear layer, by torch);
  forms the gradient of the table from the tokens' gradients;
  clips all gradients by their global norm, into fp32;
  compresses them with error feedback (3LC).
The server adds up the workers' streams, takes a step of plain gradient
descent on its fp32 weights and compresses the model's change; the workers add
the decoded change to their copies.

    python examples/embedding_training.py [--steps 40]
"""
import argparse
import math
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1802_07389_amd import tlc  # noqa: E402

ROWS, DIM, TOKENS, WORKERS = 1024, 128, 2048, 2
SPARSITY = 1.0     # 3LC's s
RATE, MAX_NORM = 20.0, 0.1
SCALE = math.sqrt(DIM)
PADDING = 0        # id of the padding token


class Worker:
    def __init__(self, model, seed):
        n = sum(p.numel() for p in model)
        self.model = [p.clone() for p in model]  # fp32 copies that pulls are added to
        self.ctx = tlc.TrainContext(max_tokens=TOKENS, max_rows=ROWS, max_dim=DIM, max_tensors=2)
        self.codec = tlc.Context(max_n=n, max_tensors=2)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.table_grad = torch.empty(ROWS, DIM, device="cuda")
        self.out = torch.empty(DIM, ROWS, device="cuda", dtype=torch.bfloat16)
        self.clipped = [torch.empty_like(p) for p in model]
        self.residual = [torch.zeros_like(p) for p in model]

    def tokens(self):
        """Sequences that count upwards from a random token, with padded tails."""
        start = torch.randint(1, ROWS, (TOKENS // 64, 1), device="cuda", generator=self.gen)
        ids = (start + torch.arange(65, device="cuda")) % (ROWS - 1) + 1
        ids[:, 56:] = PADDING
        return ids[:, :-1].contiguous(), ids[:, 1:]

    def push(self):
        """One step; returns the loss and the compressed gradients."""
        ids, target = self.tokens()
        h = self.ctx.embedding(self.model[0], ids, scale=SCALE, dtype=torch.bfloat16)
        h.requires_grad_(True)
        w = self.out.copy_(self.model[1]).detach().requires_grad_(True)
        loss = F.cross_entropy((h.view(-1, DIM) @ w).float(), target.reshape(-1),
                               ignore_index=PADDING)
        loss.backward()
        self.ctx.embedding_grad(h.grad, ids, self.table_grad, scale=SCALE, padding_id=PADDING)
        self.norm = self.ctx.clip_grad_norm([self.table_grad, w.grad], MAX_NORM,
                                            outs=self.clipped)
        self.ctx.sync()
        return loss.detach(), self.codec.compress_batch(self.clipped, self.residual, SPARSITY)

    def pull(self, streams):
        self.codec.decompress_batch([c for c, _ in streams], [m for _, m in streams], self.model,
                                    accumulate=True)


class Server:
    def __init__(self, model):
        n = sum(p.numel() for p in model)
        self.model = model
        self.codec = tlc.Context(max_n=WORKERS * n, max_tensors=WORKERS)
        self.total = [torch.empty_like(p) for p in model]
        self.residual = [torch.zeros_like(p) for p in model]

    def step(self, pushes):
        """Adds up the pushes; returns the compressed change of the model."""
        for k, total in enumerate(self.total):
            self.codec.decompress_sum([p[k][0] for p in pushes], [p[k][1] for p in pushes], total)
        self.codec.sync()
        changes = [t.mul_(-RATE / WORKERS) for t in self.total]
        for p, c in zip(self.model, changes):
            p.add_(c)
        return self.codec.compress_batch(changes, self.residual, SPARSITY)


def train(steps=40, report=print):
    """Runs the loop; returns the losses and the bytes sent per value."""
    g = torch.Generator(device="cuda").manual_seed(0)
    model = [torch.randn(ROWS, DIM, device="cuda", generator=g) / DIM,
             torch.randn(DIM, ROWS, device="cuda", generator=g) / DIM]
    workers = [Worker(model, 1 + k) for k in range(WORKERS)]
    server = Server(model)
    values = sum(p.numel() for p in model)
    losses, sent = [], 0
    for step in range(steps):
        pushed = [w.push() for w in workers]
        losses.append(sum(float(loss) for loss, _ in pushed) / WORKERS)
        streams = server.step([p for _, p in pushed])
        for w in workers:
            w.pull(streams)
            w.codec.sync()
        sent += sum(c.numel() for c, _ in streams) * WORKERS
        sent += sum(c.numel() for _, p in pushed for c, _ in p)
        if step % 10 == 0 or step == steps - 1:
            norm = max(float(w.norm.norm) for w in workers)
            report(f"step {step}: loss {losses[-1]:.4f}, largest norm {norm:.3f}")
    return losses, sent / (steps * 2 * WORKERS * values)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=40)
    losses, share = train(ap.parse_args().steps)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}; {8 * share:.3f} bits a value on the wire "
          f"(fp32: 32)")


if __name__ == "__main__":
    main()
