"""Distributed training of a small head with compressed gradients, all of it through the library: M workers, each with a batch of its own, learn from
a teacher's top logits; their gradients are the rows that the compression takes, and the server's aggregate updates the model.

    y = layer_norm(x),  a = gelu(y W1^T + b1),  h = a W2^T + b2 + x,  s = h W3^T,  loss = distillation(s, teacher)

Per worker and step: forward, backward, weight gradients straight into the worker's row of the gradient matrix; then one compression of all rows
(adaptive Top-k ladder) and one aggregate with the update x <- x - eta * update.  Run: python examples/distill_head.py [steps]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_05508_amd as P  # noqa: E402


class Head:
    """Weights of the head as one fp32 vector (what the server updates) and, for the products, in the compute type."""

    def __init__(self, width: int, hidden: int, vocab: int, dtype=torch.bfloat16, seed: int = 0):
        self.width, self.hidden, self.vocab, self.dtype = width, hidden, vocab, dtype
        self.shapes = {"norm": (width,), "norm_bias": (width,), "w1": (hidden, width), "b1": (hidden,), "w2": (width, hidden), "b2": (width,), "w3": (vocab, width)}
        self.count = sum(torch.Size(s).numel() for s in self.shapes.values())
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.x = torch.empty(self.count, device="cuda").normal_(0.0, 0.5 * width ** -0.5, generator=gen)
        t = self.tensors(self.x)
        t["norm"].fill_(1.0)
        for name in ("norm_bias", "b1", "b2"):
            t[name].zero_()

    def tensors(self, row: torch.Tensor):
        """The tensors of a flat row, one behind the other."""
        out, at = {}, 0
        for name, shape in self.shapes.items():
            n = torch.Size(shape).numel()
            out[name] = row[at:at + n].view(shape)
            at += n
        return out

    def weights(self):
        """What a step computes with: matrices in the compute type, vectors in fp32."""
        return {name: t.to(self.dtype) if t.dim() == 2 else t for name, t in self.tensors(self.x).items()}


def worker_step(head: Head, w, x: torch.Tensor, t_idx: torch.Tensor, t_val: torch.Tensor, temperature: float, row: torch.Tensor) -> torch.Tensor:
    """Forward and backward pass of one worker on its batch x [n, width]; its gradient goes into `row`.  Returns the losses of the batch."""
    n = x.shape[0]
    g = head.tensors(row)
    y, stats = P.mlmc_layer_norm(x, w["norm"], w["norm_bias"], with_stats=True)
    z = torch.empty((n, head.hidden), dtype=head.dtype, device=x.device)
    a = P.mlmc_linear(y, w["w1"], w["b1"], act=P.MLMC_ACT_GELU, z=z)
    h = P.mlmc_linear(a, w["w2"], w["b2"], residual=x)
    s = P.mlmc_linear(h, w["w3"])
    loss, ds = P.mlmc_distill(s, t_idx, t_val, temperature, scale=1.0 / n, dlogits=s)      # the gradient in the logits' place
    P.mlmc_linear_wgrad(ds, h, g["w3"])
    dh = P.mlmc_linear_dgrad(ds, w["w3"])
    P.mlmc_linear_wgrad(dh, a, g["w2"], g["b2"])
    dz = P.mlmc_linear_dgrad(dh, w["w2"], act=P.MLMC_ACT_GELU, z=z, dx=z)
    P.mlmc_linear_wgrad(dz, y, g["w1"], g["b1"])
    dy = P.mlmc_linear_dgrad(dz, w["w1"])
    P.mlmc_layer_norm_backward(dy, x, w["norm"], stats, g["norm"], g["norm_bias"], dx=dy)  # of x itself nobody asks here: in place
    return loss


def teacher_batch(gen: torch.Generator, teacher: torch.Tensor, n: int, top: int, dtype):
    """A batch and the teacher's top logits for it; a tenth of the rows is padding, without a teacher."""
    x = torch.empty((n, teacher.shape[1]), device="cuda").normal_(generator=gen)
    val, idx = torch.topk(x @ teacher.t(), top, dim=1)
    pad = torch.rand(n, device="cuda", generator=gen) < 0.1
    return x.to(dtype), torch.where(pad[:, None], -1, idx).to(torch.int32), val


def train(steps: int = 40, workers: int = 4, batch: int = 64, width: int = 256, hidden: int = 512, vocab: int = 1000, top: int = 16, eta: float = 0.5,
          temperature: float = 2.0, dtype=torch.bfloat16, seed: int = 0):
    """Mean losses of the steps."""
    head = Head(width, hidden, vocab, dtype, seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    teacher = torch.empty((vocab, width), device="cuda").normal_(0.0, 2.0 * width ** -0.5, generator=gen)
    batches = [teacher_batch(gen, teacher, batch, top, dtype) for _ in range(workers)]
    levels = 6
    plan = P.Plan(P.MLMC_TOPK, workers, head.count, P.MLMC_F32, [head.count >> (levels - l) for l in range(levels + 1)], None)
    message = P.SparseMessage(plan, with_norms=True)
    rows = torch.zeros((workers, head.count), device="cuda")                               # the gradient matrix
    losses = []
    for step in range(steps):
        w = head.weights()
        losses.append(torch.stack([worker_step(head, w, *batches[i], temperature, rows[i]).mean() for i in range(workers)]).mean())
        P.mlmc_compress_topk(plan, rows, seed=seed, step=step, out=message)
        P.mlmc_aggregate_update(plan, message, 1.0 / workers, eta, head.x)
    assert plan.status() == 0
    return [float(v) for v in losses]


if __name__ == "__main__":
    got = train(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
    for k in range(0, len(got), max(1, len(got) // 10)):
        print("step %4d  loss %.4f" % (k, got[k]))
    print("step %4d  loss %.4f" % (len(got) - 1, got[-1]))
