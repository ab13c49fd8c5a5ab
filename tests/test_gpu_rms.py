"""Root-mean-square norm, its gradient, and rows in 8 bits on the GPU against the definitions in 64 bits (oracle/worker.py).

Tolerances are bounds: U = 2^-24 is the rounding of fp32, a 16-bit output adds 2^-8 of itself.  No order used passes a term of a sum over d entries through more than d / 64 + 64 additions,
nor one of a column over n rows through more than n + 8.  The sum of the squares has terms of one sign, so that its relative error is that number times U, and that of the root half of it."""
import numpy as np
import pytest
import torch

import paper_2507_05508_amd as P
from gpu_util import launched
from oracle import worker as O
from test_gpu_worker import DT, U, UO, f64, near, out_like, rows, untouched, vec

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
SIZES = [  # rows, width, pad, shift
    (1, 1, 0, 0), (3, 2, 1, 1), (2, 7, 0, 0), (5, 8, 0, 0), (5, 63, 0, 0), (4, 64, 0, 0), (7, 65, 3, 1), (33, 256, 0, 0), (9, 257, 0, 3), (3, 511, 2, 0), (17, 1000, 8, 8),
    (130, 1024, 0, 0), (2, 2047, 0, 0), (5, 2056, 0, 0), (4, 4096, 8, 0), (3, 4099, 5, 2), (2, 8191, 0, 0), (1, 8192, 0, 0), (3, 16384, 0, 0), (2, 16400, 0, 8), (2, 20001, 0, 1),
    (1000, 24, 0, 0), (2100, 96, 0, 0), (515, 1536, 0, 0),
]


def eight_like(n, d, pad=0, shift=0):
    buf = torch.full((n * (d + pad) + shift + 64,), 77, dtype=torch.uint8, device="cuda")
    return torch.as_strided(buf, (n, d), (d + pad, 1), shift).view(E4M3), buf


def untouched_eight(buf, t):
    mask = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(mask, t.shape, t.stride(), t.storage_offset()).fill_(False)
    assert bool((buf[mask] == 77).all())


def relative(d):
    """Of y, before its rounding: half the sum's, the roundings of s (twice), of the mean, of eps, of the root and of two products."""
    return (0.5 * (d / 64 + 64 + 6) + 10) * U


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad,shift", SIZES)
def test_rms_norm(n, d, pad, shift, dtype):
    print(f"rms_norm n={n} d={d} pad={pad} shift={shift} {dtype}", flush=True)
    rng = np.random.default_rng(n * 7919 + d)
    x, x64 = rows(rng, n, d, dtype, pad, shift, std=2.0, mean=0.3)
    r, r64 = rows(rng, n, d, dtype, 0, 0, std=3.0)
    w, w64 = vec(rng, d, 1.0, 0.3)
    rel = relative(d)
    for residual, s64 in ((None, x64), (r, x64 + r64)):
        want, rstd = O.rms_norm(s64, w64, 1e-3)
        y, buf = out_like(n, d, dtype, pad, shift)
        q, qbuf = eight_like(n, d, pad, shift)
        got = P.mlmc_rms_norm(x, w, residual, eps=1e-3, y=y, q=q, with_rstd=True)
        near("rstd", got.rstd, rstd, rel * rstd)
        near("y", y, want, (rel + UO[dtype] * (1 + rel)) * np.abs(want))
        untouched(buf, y)
        untouched_eight(qbuf, q)
        most = np.abs(want).max(axis=1) / 448
        near("scale", got.scale, most, (rel + 2 * U) * most)
        v = want / f64(got.scale)[:, None]
        near("q", q.float(), v, np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10) * (1 + rel) + (rel + 2 * U) * np.abs(v))
        if residual is None:
            assert got.sum is None
        else:
            near("sum", got.sum, s64, UO[dtype] * np.abs(s64))
        alone = P.mlmc_rms_norm(x, w, residual, eps=1e-3, with_y=False, with_q=True)      # the same whatever else is asked for
        assert alone.y is None and torch.equal(alone.q.float(), q.float()) and torch.equal(alone.scale, got.scale)
        assert torch.equal(P.mlmc_rms_norm(x, w, residual, eps=1e-3).y, y)
    both = P.mlmc_rms_norm(x, w, r, eps=1e-3, y=x, sum=r)      # the norm in the place of x, the stream in its own
    assert torch.equal(x, got.y) and torch.equal(r, got.sum) and both.y is x


@pytest.mark.parametrize("grad_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad,shift", SIZES)
def test_rms_norm_backward(n, d, pad, shift, dtype, grad_dtype):
    print(f"rms_norm_backward n={n} d={d} pad={pad} shift={shift} {dtype} {grad_dtype}", flush=True)
    rng = np.random.default_rng(n * 31 + d)
    s, s64 = rows(rng, n, d, dtype, pad, shift, std=2.0)
    dy, dy64 = rows(rng, n, d, dtype, 0, 0, std=0.1)
    other, other64 = rows(rng, n, d, dtype, pad, 0, std=0.1)
    w, w64 = vec(rng, d, 1.0, 0.3)
    rstd = torch.from_numpy((1 / np.sqrt((s64 ** 2).mean(1) + 1e-5)).astype(np.float32)).cuda()
    r64 = f64(rstd)
    a = d / 64 + 64
    h, c = np.abs(s64 * r64[:, None]), np.abs(dy64 * w64)
    mean = (c * h).mean(1, keepdims=True)
    # h: 1 rounding, c: 1; the mean of the products: (a + 4) U of the magnitudes' mean; then three operations
    tol = 1.01 * U * r64[:, None] * (5 * c + h * ((a + 4) * mean + 5 * mean))
    for residual, res64 in ((None, None), (other, other64)):
        want, dw64 = O.rms_norm_backward(dy64, s64, w64, r64, res64)
        dx, buf = out_like(n, d, dtype, pad, shift)
        dw = torch.full((d + 2,), 77.0, dtype=DT[grad_dtype], device="cuda")
        P.mlmc_rms_norm_backward(dy, s, w, rstd, dw[1:d + 1], residual=residual, dx=dx)
        t = tol if res64 is None else tol + U * (np.abs(want) + np.abs(res64))
        near("dx", dx, want, t + UO[dtype] * (np.abs(want) + t))
        untouched(buf, dx)
        tw = 1.01 * (n + 10) * U * (np.abs(dy64) * h).sum(0)
        near("dweight", dw[1:d + 1], dw64, tw + UO[grad_dtype] * (np.abs(dw64) + tw))
        assert dw[0] == 77.0 and dw[-1] == 77.0
        assert torch.equal(P.mlmc_rms_norm_backward(dy, s, w, rstd, residual=residual), dx)      # without the weight's
    for k in range(3):      # dx in the place of an input
        t = [dy.clone(), s.clone(), other.clone()]
        again = torch.empty_like(dw)
        P.mlmc_rms_norm_backward(t[0], t[1], w, rstd, again[1:d + 1], residual=t[2], dx=t[k])
        assert torch.equal(t[k], dx) and torch.equal(again[1:d + 1], dw[1:d + 1])


def test_few_rows_need_no_second_launch():
    """What one workgroup has is written by it; more leave partial sums that are joined."""
    for n, d, more in ((16, 300, set()), (17, 300, {"k_norm_join"}), (1, 9000, set()), (1, 20000, {"k_rms_columns"}), (2, 20000, {"k_rms_columns", "k_norm_join"})):
        s, dw = torch.ones((n, d), device="cuda"), torch.zeros(d, device="cuda")
        assert launched(lambda: P.mlmc_rms_norm_backward(s, s, None, s[:, 0].contiguous(), dw)) == {"k_rms_backward"} | more
        assert (P.mlmc_rms_norm_workspace(n, d) == 0) == ("k_norm_join" not in more) and bool((dw == n).all())


def test_rms_norm_without_rows_weight_or_residual():
    x = torch.empty((0, 16), device="cuda")
    r = P.mlmc_rms_norm(x, with_q=True, with_rstd=True)
    assert r.y.shape == (0, 16) and r.q.shape == (0, 16) and r.scale.shape == (0,)
    dw = torch.full((16,), 3.0, device="cuda")
    P.mlmc_rms_norm_backward(x, x, None, torch.empty(0, device="cuda"), dw)
    assert bool((dw == 0).all())
    rng = np.random.default_rng(1)
    x, x64 = rows(rng, 6, 333)
    want, _ = O.rms_norm(x64, None, 1e-5)
    near("y", P.mlmc_rms_norm(x).y, want, (relative(333) + U) * np.abs(want))


@pytest.mark.parametrize("d", [40, 5000, 20000])
def test_rms_norm_of_special_rows(d):
    x = torch.zeros((6, d), device="cuda")
    x[1, 3] = float("nan")
    x[2, 3] = float("inf")
    x[3] = 2.0
    x[4, 0] = 1e-30
    x[5] = 1e30      # the sum of the squares is infinite: r is 0
    r = P.mlmc_rms_norm(x, eps=1e-5, with_q=True, with_rstd=True)
    assert bool((r.y[0] == 0).all()) and r.scale[0] == 2.0 ** -100 and bool((r.q[0].float() == 0).all())
    assert bool(r.y[1].isnan().all()) and bool(r.scale[1].isnan()) and bool(r.q[1].float().isnan().all())
    assert bool(r.y[2, 3].isnan()) and bool((r.y[2, 4:] == 0).all()) and bool(r.scale[2].isnan()) and bool(r.q[2].float().isnan().all())
    assert abs(float(r.y[3, 7]) - 2.0 / (4 + 1e-5) ** 0.5) < 1e-5 and bool((r.q[3].float() == 448).all())
    assert bool((r.y[5] == 0).all()) and r.rstd[5] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad,shift", SIZES)
def test_quantize_to_the_bit(n, d, pad, shift, dtype):
    """The scale is the fp32 quotient.  An entry of 16 bits goes to the nearest value, ties to even: 448 x / max is a quotient of small whole numbers, and next to a tie it is one.  One of 32 bits goes to the
    nearest or, within a rounding of fp32 (2^-23 with what the product leaves) of the middle of two, to the other."""
    print(f"quantize n={n} d={d} pad={pad} shift={shift} {dtype}", flush=True)
    rng = np.random.default_rng(n + d)
    x, x64 = rows(rng, n, d, dtype, pad, shift, std=0.02)
    q, buf = eight_like(n, d, pad, shift)
    got, scale = P.mlmc_quantize(x, q=q)
    assert got is q
    untouched_eight(buf, q)
    want, s64 = O.quantize(x64)
    assert np.array_equal(scale.cpu().numpy(), np.maximum(np.abs(x64).max(1).astype(np.float32) / np.float32(448), np.float32(2.0 ** -100)))
    have = q.float().cpu().double().numpy()
    if dtype == "bf16":
        assert np.array_equal(have, want)
    else:
        v = x64 * 448 / np.abs(x64).max(1, keepdims=True)
        assert ((have == want) | (have == O.e4m3(v * (1 + 2.0 ** -23))) | (have == O.e4m3(v * (1 - 2.0 ** -23)))).all()


@pytest.mark.parametrize("d", [5, 100, 17000])
def test_quantize_special_rows(d):
    x = torch.zeros((5, d), device="cuda")
    x[1, 2] = float("nan")
    x[2, 2] = -float("inf")
    x[3] = 3.4e38
    x[4] = 2.0 ** -100
    q, scale = P.mlmc_quantize(x)
    assert bool((q[0].float() == 0).all()) and scale[0] == 2.0 ** -100 and bool(scale[1:3].isnan().all()) and bool(q[1:3].float().isnan().all())
    assert bool((q[3].float() == 448).all()) and bool((q[4].float() == 1).all())
    assert bool((q[0].view(torch.uint8) == 0).all()) and q.stride(0) % 16 == 0
