"""Layer norm, linear layer and distillation loss at sizes whose definition in 64 bits runs on the GPU: many rows, long rows, several rounds of a
workgroup, every tile and every way of the linear layer.  Bounds as in test_gpu_worker.py (U is the rounding of fp32; a sum's error is U times the additions that a
term passes through times the sum of the terms' magnitudes)."""
import numpy as np
import pytest
import torch

import paper_2507_05508_amd as P
from test_gpu_worker import ACT, DT, U, UO, same

pytestmark = pytest.mark.gpu


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def normal(gen, n, d, dtype="f32", std=1.0, mean=0.0, pad=0, shift=0):
    """A matrix of normal entries, `shift` entries into a buffer of NaN, `pad` of them between its rows."""
    buf = torch.full((n * (d + pad) + shift,), float("nan"), dtype=DT[dtype], device="cuda")
    t = torch.as_strided(buf, (n, d), (d + pad, 1), shift)
    t.copy_(torch.empty((n, d), device="cuda").normal_(mean, std, generator=gen))
    return t


def check(name, got, want, tol, u=0.0):
    """|got - want| <= tol + u (|want| + tol), entry by entry."""
    off = (got.double() - want).abs_().sub_(tol)
    if u:
        off -= u * (want.abs() + tol)
    assert bool((off <= 0).all()), f"{name}: {float(off.max())} over its bound"


def norm_forward_bounds(x, w, b, eps):
    """y, mean, rstd and the bounds of their errors, the formulas of test_gpu_worker.norm_bounds."""
    d = x.shape[1]
    a = d / 64 + 64
    mean = x.sum(1, keepdim=True) / d
    diff = x - mean
    rstd = 1.0 / ((diff * diff).sum(1, keepdim=True) / d + eps).sqrt()
    dm = a * U * x.abs().sum(1, keepdim=True) / d + U * mean.abs()
    dd = dm + U * diff.abs()
    var = rstd ** -2 - eps
    dv = (2 * diff.abs() * dd + dd ** 2).sum(1, keepdim=True) / d + (a + 4) * U * (var + eps)
    dr = 0.5 * dv * rstd ** 3 + 4 * U * rstd
    h = diff * rstd
    dy = (dd * rstd + diff.abs() * dr + 2 * U * h.abs()) * w.abs() + 2 * U * ((h * w).abs() + b.abs())
    return h * w + b, mean[:, 0], rstd[:, 0], 1.01 * dy, 1.01 * dm[:, 0], 1.01 * dr[:, 0]


def norm_backward_bounds(dy, x, w, stats):
    """dx, dweight, dbias and the bounds of test_gpu_worker.test_layer_norm_backward."""
    n, d = x.shape
    a = d / 64 + 64
    mean, rstd = stats.double()[:, :1], stats.double()[:, 1:]
    h = (x - mean) * rstd
    c = dy * w
    dx = rstd * (c - c.sum(1, keepdim=True) / d - h * ((c * h).sum(1, keepdim=True) / d))
    dw, db = (dy * h).sum(0), dy.sum(0)
    tol_dw, tol_db = (n + 11) * U * (dy * h).abs().sum(0), (n + 8) * U * dy.abs().sum(0)
    h, c = h.abs(), c.abs()
    cm, ch = c.sum(1, keepdim=True) / d, (c * h).sum(1, keepdim=True) / d
    return dx, dw, db, rstd * (a * U * cm + h * (a + 4) * U * ch + 8 * U * (c + cm + h * ch)), tol_dw, tol_db


def norm_case(n, d, dtype, seed):
    gen = generator(seed)
    return (normal(gen, n, d, dtype, 2.0, 0.7), normal(gen, n, d, dtype, 0.1, 0.02), torch.empty(d, device="cuda").normal_(1.0, 0.3, generator=gen),
            torch.empty(d, device="cuda").normal_(0.0, 0.5, generator=gen))


# ---- sizes past what one launch of a workgroup a row takes ------------------------------------------------------------
def test_layer_norm_of_more_rows_than_a_launch_has_workgroups():
    n, d = (1 << 24) + 3, 4
    x, dy, w, b = norm_case(n, d, "f32", 1)
    y, stats = P.mlmc_layer_norm(x, w, b, with_stats=True)
    want, mean, rstd, ty, tm, tr = norm_forward_bounds(x.double(), w.double(), b.double(), 1e-5)
    check("mean", stats[:, 0], mean, tm)
    check("rstd", stats[:, 1], rstd, tr)
    check("y", y, want, ty, U)
    del want, ty, y
    dw, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    dx = P.mlmc_layer_norm_backward(dy, x, w, stats, dw, db)
    want, want_w, want_b, tol, tol_w, tol_b = norm_backward_bounds(dy.double(), x.double(), w.double(), stats)
    check("dx", dx, want, tol, U)
    check("dweight", dw, want_w, tol_w, U)
    check("dbias", db, want_b, tol_b, U)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_of_more_rows_than_a_launch_has_workgroups(dtype):
    n, v, temp = (1 << 24) + 3, 5, 2.0
    gen = generator(2)
    s = normal(gen, n, v, dtype, 2.0)
    at = torch.randint(0, v, (n, 1), device="cuda", generator=gen, dtype=torch.int32)
    loss, ds = P.mlmc_distill(s, at, torch.zeros((n, 1), device="cuda"), temp, scale=0.25)
    # one entry a teacher: q is 1 (the bounds of test_gpu_worker.distill_bounds with that)
    z = s.double()
    arg = (z.max(1, keepdim=True).values - z) / temp
    log_p = -arg - torch.exp(-arg).sum(1, keepdim=True).log()
    p = log_p.exp()
    rel = U * (4 * arg + 4 * (p * arg).sum(1, keepdim=True) + v / 64 + 80)
    hot = torch.zeros_like(p).scatter_(1, at.long(), 1.0)
    check("dlogits", ds, 0.25 * temp * (p - hot), 0.25 * temp * (p * rel + hot * U * 81 + 4 * U * (p + hot)), UO[dtype])
    log_p, arg, rel = (t.gather(1, at.long())[:, 0] for t in (log_p, arg, rel))
    check("loss", loss, -temp * temp * log_p, temp * temp * (arg * 6 * U + rel + 81 * U + 4 * U * log_p.abs() + (81 + 9) * U * log_p.abs()) + 4 * U * temp * temp * log_p.abs())


def test_layer_norm_backward_of_more_columns_than_a_launch_has_workgroups():
    """One row: dweight and dbias have one term each, the same bits as elementary operations give."""
    d = (1 << 28) + 65
    gen = generator(3)
    x, dy = normal(gen, 1, d, "bf16"), normal(gen, 1, d, "bf16", 0.1)
    stats = torch.tensor([[0.25, 1.5]], device="cuda")
    dw, db = torch.full((d,), 7.0, device="cuda"), torch.full((d,), 7.0, device="cuda")
    P.mlmc_layer_norm_backward(dy, x, None, stats, dw, db)
    assert torch.equal(db, dy[0].float())
    assert torch.equal(dw, (x[0].float() - 0.25) * 1.5 * dy[0].float())
