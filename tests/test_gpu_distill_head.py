"""The example that trains a head with compressed gradients: a worker's gradient row against automatic differentiation of the same head in 64
bits, and the loss falls."""
import math
import os
import sys

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
import distill_head as E  # noqa: E402

pytestmark = pytest.mark.gpu


def reference(head, row, x, t_idx, t_val, temperature):
    """Losses and gradient of the mean loss, in 64 bits on the CPU."""
    p = {k: v.detach().cpu().double().requires_grad_(True) for k, v in head.tensors(row).items()}
    x = x.cpu().double()
    mean = x.mean(1, keepdim=True)
    y = (x - mean) / ((x - mean).pow(2).mean(1, keepdim=True) + 1e-5).sqrt() * p["norm"] + p["norm_bias"]
    z = y @ p["w1"].t() + p["b1"]
    a = 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    s = (a @ p["w2"].t() + p["b2"] + x) @ p["w3"].t()
    log_p = torch.log_softmax(s / temperature, 1)
    idx, val = t_idx.cpu().long(), t_val.cpu().double()
    live = (idx >= 0).any(1)
    log_q = torch.log_softmax(val / temperature, 1)
    loss = temperature ** 2 * (log_q.exp() * (log_q - log_p.gather(1, idx.clamp(min=0)))).sum(1)
    loss = torch.where(live, loss, torch.zeros(()).double())
    loss.mean().backward()
    return loss.detach(), torch.cat([p[k].grad.reshape(-1) for k in head.shapes])


def test_worker_gradient_matches_automatic_differentiation():
    """fp32: every stage rounds by 2^-24 and sums of up to 1000 terms follow one another; 1e-5 of a tensor's largest entry is over a hundred
    such roundings in each of the six stages."""
    head = E.Head(96, 200, 333, torch.float32, seed=3)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    teacher = torch.empty((333, 96), device="cuda").normal_(0.0, 0.2, generator=gen)
    x, t_idx, t_val = E.teacher_batch(gen, teacher, 37, 8, torch.float32)
    row = torch.full((head.count,), float("nan"), device="cuda")
    loss = E.worker_step(head, head.weights(), x, t_idx, t_val, 2.0, row)
    want_loss, want = reference(head, head.x, x, t_idx, t_val, 2.0)
    assert np.abs(loss.cpu().double().numpy() - want_loss.numpy()).max() < 1e-5 * want_loss.abs().max()
    for name, g in head.tensors(row).items():
        w = head.tensors(want)[name]
        assert (g.cpu().double() - w).abs().max() <= 1e-5 * w.abs().max(), name


def test_training_lowers_the_loss():
    losses = E.train(steps=30)
    print(losses, flush=True)
    assert all(math.isfinite(v) for v in losses)
    assert np.mean(losses[-5:]) < 0.8 * losses[0]
    assert E.train(steps=5) == losses[:5]     # the same bits from run to run
