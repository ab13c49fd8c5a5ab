"""Distributed training of a small residual head whose teacher answers in 8 bits, all of it through the library: the teacher's weights are brought into 8 bits once; per batch its norm gives 8 bits,
its products take them, and the top alternatives of its logits are what the students learn from.  A student drops a part of its branch (the mask is made again in the backward pass), adds it to
the stream and normalises by the root mean square; its gradient goes into its row of the gradient matrix, which is compressed, aggregated and applied.

    teacher:  h = x,  y = rms_norm(h) in 8 bits,  a = gelu(y W1^T) -> 8 bits,  h = a W2^T + h,  s = rms_norm(h) in 8 bits W3^T,  answers = top alternatives of log softmax s
    student:  b = x W1^T,  h = x + dropout(gelu b W2^T),  s = rms_norm(h) W3^T,  loss = distillation(s, answers)

Run: python examples/teach_head.py [steps]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_05508_amd as P  # noqa: E402


class Teacher:
    """Weights in 8 bits with a scale for every row."""

    def __init__(self, width: int, hidden: int, vocab: int, seed: int = 0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.norms = [torch.empty(width, device="cuda").normal_(1.0, 0.1, generator=gen) for _ in range(2)]
        self.w1, self.w2, self.w3 = (P.mlmc_quantize(torch.empty((n, k), device="cuda").normal_(0.0, std * k ** -0.5, generator=gen))
                                     for n, k, std in ((hidden, width, 1.0), (width, hidden, 1.0), (vocab, width, 2.0)))

    def logits(self, x: torch.Tensor) -> torch.Tensor:
        y = P.mlmc_rms_norm(x, self.norms[0], with_y=False, with_q=True)
        a = P.mlmc_linear_q8(y.q, y.scale, *self.w1, act=P.MLMC_ACT_GELU)
        h = P.mlmc_rms_norm(P.mlmc_linear_q8(*P.mlmc_quantize(a), *self.w2), self.norms[1], residual=x, with_y=False, with_q=True)
        return P.mlmc_linear_q8(h.q, h.scale, *self.w3)

    def answers(self, x: torch.Tensor, top: int, tokens: torch.Tensor | None = None) -> P.TokenLogprobs:
        """The top alternatives and their log probabilities, the entropy, and the log probabilities of given tokens."""
        return P.mlmc_token_logprobs(self.logits(x), tokens, top=top, with_entropy=True)


class Student:
    """Weights as one fp32 vector (what the server updates) and, for the products, in the compute type."""

    def __init__(self, width: int, hidden: int, vocab: int, dtype=torch.bfloat16, seed: int = 1):
        self.dtype = dtype
        self.shapes = {"w1": (hidden, width), "w2": (width, hidden), "norm": (width,), "w3": (vocab, width)}
        self.count = sum(torch.Size(s).numel() for s in self.shapes.values())
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.x = torch.empty(self.count, device="cuda").normal_(0.0, 0.5 * width ** -0.5, generator=gen)
        self.tensors(self.x)["norm"].fill_(1.0)

    def tensors(self, row: torch.Tensor):
        """The tensors of a flat row, one behind the other."""
        out, at = {}, 0
        for name, shape in self.shapes.items():
            n = torch.Size(shape).numel()
            out[name] = row[at:at + n].view(shape)
            at += n
        return out

    def weights(self):
        return {name: t.to(self.dtype) if t.dim() == 2 else t for name, t in self.tensors(self.x).items()}


def worker_step(student: Student, w, x: torch.Tensor, answers: P.TokenLogprobs, temperature: float, p: float, seed: int, step: int, worker: int, row: torch.Tensor) -> torch.Tensor:
    """Forward and backward pass of one worker on its batch x [n, width]; its gradient goes into `row`.  Returns the losses of the batch."""
    n = x.shape[0]
    g = student.tensors(row)
    z = torch.empty((n, w["w1"].shape[0]), dtype=x.dtype, device=x.device)
    a = P.mlmc_linear(x, w["w1"], act=P.MLMC_ACT_GELU, z=z)
    b = P.mlmc_linear(a, w["w2"])
    h = P.mlmc_dropout(b, p, seed, step, stream=worker, residual=x)
    y = P.mlmc_rms_norm(h, w["norm"], with_rstd=True)
    s = P.mlmc_linear(y.y, w["w3"])
    loss, ds = P.mlmc_distill(s, answers.top_idx, answers.top_logprob, temperature, scale=1.0 / n, dlogits=s)
    P.mlmc_linear_wgrad(ds, y.y, g["w3"])
    dy = P.mlmc_linear_dgrad(ds, w["w3"])
    dh = P.mlmc_rms_norm_backward(dy, h, w["norm"], y.rstd, g["norm"], dx=dy)
    db = P.mlmc_dropout(dh, p, seed, step, stream=worker, y=dh)          # the same mask; of x itself nobody asks here
    P.mlmc_linear_wgrad(db, a, g["w2"])
    dz = P.mlmc_linear_dgrad(db, w["w2"], act=P.MLMC_ACT_GELU, z=z, dx=z)
    P.mlmc_linear_wgrad(dz, x, g["w1"])
    return loss


def train(steps: int = 40, workers: int = 4, batch: int = 64, width: int = 256, hidden: int = 512, vocab: int = 1000, top: int = 16, eta: float = 0.5,
          temperature: float = 2.0, p: float = 0.1, dtype=torch.bfloat16, seed: int = 0):
    """Mean losses of the steps."""
    teacher, student = Teacher(width, hidden, vocab, seed), Student(width, hidden, vocab, dtype, seed + 1)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 2)
    batches = [torch.empty((batch, width), device="cuda").normal_(generator=gen).to(torch.bfloat16) for _ in range(workers)]
    answers = [teacher.answers(x, top) for x in batches]
    levels = 6
    plan = P.Plan(P.MLMC_TOPK, workers, student.count, P.MLMC_F32, [student.count >> (levels - l) for l in range(levels + 1)], None)
    message = P.SparseMessage(plan, with_norms=True)
    rows = torch.zeros((workers, student.count), device="cuda")                                # the gradient matrix
    losses = []
    for step in range(steps):
        w = student.weights()
        losses.append(torch.stack([worker_step(student, w, batches[i].to(dtype), answers[i], temperature, p, seed, step, i, rows[i]).mean() for i in range(workers)]).mean())
        P.mlmc_compress_topk(plan, rows, seed=seed, step=step, out=message)
        P.mlmc_aggregate_update(plan, message, 1.0 / workers, eta, student.x)
    assert plan.status() == 0
    return [float(v) for v in losses]


if __name__ == "__main__":
    got = train(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
    for k in range(0, len(got), max(1, len(got) // 10)):
        print("step %4d  loss %.4f" % (k, got[k]))
    print("step %4d  loss %.4f" % (len(got) - 1, got[-1]))
