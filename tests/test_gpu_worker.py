"""Layer norm, linear layer and distillation loss on the GPU against the definitions in 64 bits (oracle/worker.py).

Tolerances are bounds and not fitted.  U = 2^-24 is the rounding of fp32, the unit of every operation inside; an output of
16 bits adds 2^-8 of itself.  A sum of n terms in any order, held in fp32, is off by at most (additions that a term passes
through) U sum |terms|; no order used passes a term through more than n / 64 + 64 of them where 64 lanes share a sum, and
n + 8 where one lane has it (a column over rows, an entry of a product)."""
import numpy as np
import pytest
import torch

import paper_2507_05508_amd as P
from gpu_util import launched
from oracle import worker as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
UO = {"f32": U, "bf16": 2.0 ** -8}
ACT = {"none": P.MLMC_ACT_NONE, "relu": P.MLMC_ACT_RELU, "gelu": P.MLMC_ACT_GELU}


def rows(rng, n, d, dtype="f32", pad=0, shift=0, std=1.0, mean=0.0):
    """A matrix on the GPU, cut out of a larger buffer of NaN (`shift` entries in, `pad` more in a row), and its values in 64 bits."""
    buf = torch.full((n * (d + pad) + shift,), float("nan"), dtype=DT[dtype], device="cuda")
    t = torch.as_strided(buf, (n, d), (d + pad, 1), shift)
    t.copy_(torch.from_numpy(rng.normal(mean, std, (n, d)).astype(np.float32)))
    return t, f64(t)


def f64(t):
    return t.detach().cpu().double().numpy()


def vec(rng, d, mean, std):
    v = rng.normal(mean, std, d).astype(np.float32)
    return torch.from_numpy(v).cuda(), v.astype(np.float64)


def near(name, got, want, tol):
    got = f64(got)
    off = np.where(np.isnan(want), 0.0, np.abs(got - want) - tol)
    assert (np.isnan(got) == np.isnan(want)).all(), name
    assert (off <= 0).all(), f"{name}: {off.max()} over a bound of {np.broadcast_to(tol, off.shape).reshape(-1)[off.argmax()]}"


def out_like(n, d, dtype, pad=0, shift=0):
    buf = torch.full((n * (d + pad) + shift + 64,), 77.0, dtype=DT[dtype], device="cuda")
    return torch.as_strided(buf, (n, d), (d + pad, 1), shift), buf


def untouched(buf, t):
    """Nothing around the matrix was written."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(mask, t.shape, t.stride(), t.storage_offset()).fill_(False)
    assert bool((buf[mask] == 77.0).all())


# ---- layer norm -------------------------------------------------------------------------------------------------------
NORM = [  # rows, width, pad, shift
    (1, 1, 0, 0), (3, 2, 1, 1), (5, 63, 0, 0), (4, 64, 0, 0), (7, 65, 3, 1), (2, 127, 1, 0), (33, 256, 0, 0), (9, 257, 0, 3), (3, 511, 2, 0),
    (17, 1000, 8, 8), (130, 1024, 0, 0), (2, 2047, 0, 0), (5, 2056, 0, 0), (4, 4096, 8, 0), (3, 4099, 5, 2), (2, 8191, 0, 0), (1, 8192, 0, 0), (3, 16384, 0, 0), (2, 16400, 0, 8),
    (2, 20001, 0, 1), (1, 40000, 0, 0), (2, 70001, 3, 0), (1000, 24, 0, 0), (515, 320, 0, 0), (300, 1536, 0, 0),
]


def norm_bounds(x, w, b, eps):
    """Bounds of |y|'s, mean's and rstd's errors before the output's rounding."""
    d = x.shape[1]
    a = d / 64 + 64
    y, mean, rstd = O.layer_norm(x, w, b, eps)
    dm = a * U * np.abs(x).mean(1) + U * np.abs(mean)
    diff = np.abs(x - mean[:, None])
    dd = dm[:, None] + U * diff                                   # of x - mean
    var = (diff ** 2).mean(1)
    dv = (2 * diff * dd + dd ** 2).mean(1) + (a + 4) * U * (var + eps)
    dr = 0.5 * dv * rstd ** 3 + 4 * U * rstd                        # to first order; dv / (var + eps) is far below 1 in these cases
    h = diff * rstd[:, None]
    dy = (dd * rstd[:, None] + diff * dr[:, None] + 2 * U * h) * np.abs(w) + 2 * U * (np.abs(h * w) + np.abs(b))
    return y, mean, rstd, 1.01 * dy, 1.01 * dm, 1.01 * dr


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad,shift", NORM)
def test_layer_norm(n, d, pad, shift, dtype):
    print(f"layer_norm n={n} d={d} pad={pad} shift={shift} {dtype}", flush=True)
    rng = np.random.default_rng(n * 7919 + d)
    x, x64 = rows(rng, n, d, dtype, pad, shift, std=2.0, mean=0.7)
    w, w64 = vec(rng, d, 1.0, 0.3)
    b, b64 = vec(rng, d, 0.0, 0.5)
    y, buf = out_like(n, d, dtype, pad, shift)
    _, stats = P.mlmc_layer_norm(x, w, b, eps=1e-3, y=y, with_stats=True)
    want, mean, rstd, dy, dm, dr = norm_bounds(x64, w64, b64, 1e-3)
    near("mean", stats[:, 0], mean, dm)
    near("rstd", stats[:, 1], rstd, dr)
    near("y", y, want, dy + UO[dtype] * (np.abs(want) + dy))
    untouched(buf, y)
    again = P.mlmc_layer_norm(x, w, b, eps=1e-3)
    assert torch.equal(again, y)
    P.mlmc_layer_norm(x, w, b, eps=1e-3, y=x)      # in place
    assert torch.equal(x, y)


def test_layer_norm_without_weight_and_bias():
    rng = np.random.default_rng(1)
    x, x64 = rows(rng, 6, 333, "f32")
    want, _, _, dy, _, _ = norm_bounds(x64, np.ones(333), np.zeros(333), 1e-5)
    near("y", P.mlmc_layer_norm(x), want, dy + U * np.abs(want))


@pytest.mark.parametrize("d", [65, 1024, 5000, 40000])
def test_layer_norm_far_from_zero(d):
    """Rows whose mean is a thousand times their spread keep their variance."""
    rng = np.random.default_rng(d)
    x, x64 = rows(rng, 3, d, "f32", std=1.0, mean=1000.0)
    want, mean, rstd, dy, dm, dr = norm_bounds(x64, np.ones(d), np.zeros(d), 1e-5)
    y, stats = P.mlmc_layer_norm(x, with_stats=True)
    near("rstd", stats[:, 1], rstd, dr)
    near("y", y, want, dy + U * np.abs(want))


@pytest.mark.parametrize("d", [1, 64, 1000, 9000, 40000])
def test_layer_norm_of_equal_entries_and_of_nan(d):
    x = torch.full((4, d), 2.5, device="cuda")
    x[2, d // 2] = float("nan")
    b = torch.arange(d, dtype=torch.float32, device="cuda")
    y = P.mlmc_layer_norm(x, None, b)
    assert torch.equal(y[0], b) and torch.equal(y[1], b) and torch.equal(y[3], b) and bool(torch.isnan(y[2]).all())


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad,shift", NORM)
def test_layer_norm_backward(n, d, pad, shift, dtype, grad):
    print(f"layer_norm_backward n={n} d={d} pad={pad} shift={shift} {dtype} {grad}", flush=True)
    rng = np.random.default_rng(n * 104729 + d)
    x, x64 = rows(rng, n, d, dtype, pad, shift, std=2.0, mean=0.7)
    dy, dy64 = rows(rng, n, d, dtype, pad + 1, shift, std=0.1, mean=0.02)
    w, w64 = vec(rng, d, 1.0, 0.3)
    _, stats = P.mlmc_layer_norm(x, w, None, with_stats=True)
    mean, rstd = f64(stats).T                                      # the backward pass takes them as they are
    dx, buf = out_like(n, d, dtype, pad, shift)
    row = torch.full((2 * d + 3,), 77.0, dtype=DT[grad], device="cuda")
    dw, db = row[1:1 + d], row[2 + d:2 + 2 * d]
    P.mlmc_layer_norm_backward(dy, x, w, stats, dw, db, dx=dx)
    want, dw_want, db_want = O.layer_norm_backward(dy64, x64, w64, mean, rstd)
    a = d / 64 + 64
    h = np.abs((x64 - mean[:, None]) * rstd[:, None])
    c = np.abs(dy64 * w64)
    dcm = (a * U * c.mean(1))[:, None]
    dch = ((a + 4) * U * (c * h).mean(1))[:, None]
    cm, ch = c.mean(1, keepdims=True), (c * h).mean(1, keepdims=True)
    tol = rstd[:, None] * (dcm + h * dch + 8 * U * (c + cm + h * ch))
    near("dx", dx, want, tol + UO[dtype] * (np.abs(want) + tol))
    untouched(buf, dx)
    tol = (n + 8 + 3) * U * np.abs(dy64 * h).sum(0)
    near("dweight", dw, dw_want, tol + UO[grad] * (np.abs(dw_want) + tol))
    tol = (n + 8) * U * np.abs(dy64).sum(0)
    near("dbias", db, db_want, tol + UO[grad] * (np.abs(db_want) + tol))
    assert float(row[0]) == 77 and float(row[1 + d]) == 77 and float(row[2 + 2 * d]) == 77
    # once more: the same bits; without the sums; in place
    keep = row.clone()
    assert torch.equal(P.mlmc_layer_norm_backward(dy, x, w, stats, dw, db), dx) and torch.equal(row, keep)
    assert torch.equal(P.mlmc_layer_norm_backward(dy, x, w, stats), dx)
    P.mlmc_layer_norm_backward(dy, x, w, stats, None, db, dx=dy)
    assert torch.equal(dy, dx) and torch.equal(row, keep)


def test_layer_norm_no_rows():
    x = torch.empty((0, 100), device="cuda")
    dw, db = torch.full((100,), 5.0, device="cuda"), torch.full((100,), 5.0, device="cuda")
    y, stats = P.mlmc_layer_norm(x, with_stats=True)
    dx = P.mlmc_layer_norm_backward(x, x, None, stats, dw, db)
    assert y.shape == (0, 100) and dx.shape == (0, 100) and not dw.any() and not db.any()


def slopes(f, x, at, h):
    """Central differences of the 64-bit forward direction at some entries."""
    got = []
    for i in at:
        keep = x[i]
        x[i] = keep + h
        up = f()
        x[i] = keep - h
        down = f()
        x[i] = keep
        got.append((up - down) / (2 * h))
    return np.array(got)


def test_gradients_against_differences():
    """The kernels' gradients are the slopes of the definitions' forward direction (differences in 64 bits; h^2 terms under 1e-7)."""
    rng = np.random.default_rng(5)
    some = [(0, 0), (1, 7), (2, 36), (3, 99)]
    x, x64 = rows(rng, 4, 100)
    w, w64 = vec(rng, 100, 1.0, 0.2)
    r, r64 = rows(rng, 4, 100)
    _, stats = P.mlmc_layer_norm(x, w, None, with_stats=True)
    dw, db = torch.empty(100, device="cuda"), torch.empty(100, device="cuda")
    dx = f64(P.mlmc_layer_norm_backward(r, x, w, stats, dw, db))
    f = lambda: float((O.layer_norm(x64, w64, None, 1e-5)[0] * r64).sum())  # noqa: E731
    assert np.abs(slopes(f, x64, some, 1e-4) - [dx[i] for i in some]).max() < 2e-5
    assert np.abs(slopes(f, w64, [0, 50, 99], 1e-4) - f64(dw)[[0, 50, 99]]).max() < 2e-5
    # gelu(x) W^T through its input, weight and bias
    u, u64 = rows(rng, 4, 100)
    wt, wt64 = rows(rng, 30, 100, std=0.1)
    r, r64 = rows(rng, 4, 30)
    g = lambda: float((O.linear(O.act(u64, "gelu"), wt64)[0] * r64).sum())  # noqa: E731
    dx = f64(P.mlmc_linear_dgrad(r, wt, act=ACT["gelu"], z=u))
    assert np.abs(slopes(g, u64, some, 1e-4) - [dx[i] for i in some]).max() < 2e-5
    act = torch.from_numpy(O.act(u64, "gelu").astype(np.float32)).cuda()
    dwt = torch.empty((30, 100), device="cuda")
    P.mlmc_linear_wgrad(r, act, dwt)
    at = [(0, 0), (29, 99), (3, 64)]
    assert np.abs(slopes(g, wt64, at, 1e-4) - [f64(dwt)[i] for i in at]).max() < 2e-5
    # the loss
    s, s64 = rows(rng, 4, 100)
    idx = np.stack([rng.permutation(100)[:5] for _ in range(4)])
    val = rng.normal(0, 2, (4, 5))
    _, ds = P.mlmc_distill(s, torch.from_numpy(idx.astype(np.int32)).cuda(), torch.from_numpy(val.astype(np.float32)).cuda(), temperature=2.0)
    val = val.astype(np.float32).astype(np.float64)
    q = lambda: float(O.distill(s64, idx, val, 2.0)[0].sum())  # noqa: E731
    assert np.abs(slopes(q, s64, some + [(0, idx[0, 0]), (3, idx[3, 4])], 1e-4) - [f64(ds)[i] for i in some + [(0, idx[0, 0]), (3, idx[3, 4])]]).max() < 2e-5


# ---- linear layer -----------------------------------------------------------------------------------------------------
LINEAR = [  # rows, outputs, inputs, pad, shift
    (1, 1, 1, 0, 0), (1, 5, 3, 1, 1), (2, 64, 64, 0, 0), (1, 256, 512, 0, 0), (3, 300, 1000, 8, 8), (4, 1000, 520, 0, 0), (8, 96, 2048, 0, 0), (15, 130, 65, 0, 0),
    (16, 256, 384, 0, 0), (17, 128, 128, 0, 0), (31, 33, 129, 3, 1), (32, 512, 1024, 0, 0), (33, 257, 640, 0, 0), (60, 70, 80, 0, 0), (64, 64, 4096, 0, 0), (65, 200, 72, 8, 0), (127, 255, 31, 0, 0),
    (128, 128, 256, 0, 0), (129, 130, 257, 5, 3), (200, 136, 264, 0, 8), (256, 256, 512, 0, 0), (257, 513, 96, 0, 0), (300, 264, 520, 8, 0), (512, 768, 320, 0, 0), (1000, 40, 56, 0, 0), (520, 1032, 264, 0, 0),
    (700, 8, 1500, 0, 0), (2100, 300, 100, 0, 0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,m,k,pad,shift", LINEAR)
def test_linear(n, m, k, pad, shift, dtype):
    print(f"linear n={n} m={m} k={k} pad={pad} shift={shift} {dtype}", flush=True)
    rng = np.random.default_rng(n * 31 + m * 7 + k)
    x, x64 = rows(rng, n, k, dtype, pad, shift)
    w, w64 = rows(rng, m, k, dtype, pad, shift, std=k ** -0.5)
    b, b64 = vec(rng, m, 0.0, 0.3)
    res, res64 = rows(rng, n, m, dtype, pad, shift)
    size = np.abs(x64) @ np.abs(w64).T
    tol_v = (k + 2) * U * (size + np.abs(b64))
    for kind, use_b, use_r, use_z in (("none", False, False, False), ("gelu", True, True, True), ("relu", True, False, True), ("none", True, True, False)):
        y, buf = out_like(n, m, dtype, pad, shift)
        z, zbuf = out_like(n, m, dtype, pad + 1, shift) if use_z else (None, None)
        P.mlmc_linear(x, w, b if use_b else None, act=ACT[kind], residual=res if use_r else None, z=z, y=y)
        want, z_want = O.linear(x64, w64, b64 if use_b else None, kind, res64 if use_r else None)
        # both activations have slopes of at most 1.13; gelu itself is computed to 8 U of |v| + 1e-7 (erf's own error, where it cancels)
        tol = 1.13 * tol_v + (8 * U * np.abs(z_want) + 1e-7 * np.abs(z_want) if kind == "gelu" else 0) + 2 * U * (np.abs(want) + np.abs(res64))
        near(f"y {kind}", y, want, tol + UO[dtype] * (np.abs(want) + tol))
        untouched(buf, y)
        if use_z:
            near(f"z {kind}", z, z_want, tol_v + UO[dtype] * (np.abs(z_want) + tol_v))
            untouched(zbuf, z)
    # twice the same bits; the output in the residual's place
    assert torch.equal(P.mlmc_linear(x, w, b, residual=res), y)
    P.mlmc_linear(x, w, b, residual=res, y=res)
    assert torch.equal(res, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,m,k,pad,shift", LINEAR)
def test_linear_dgrad(n, m, k, pad, shift, dtype):
    print(f"linear_dgrad n={n} m={m} k={k} pad={pad} shift={shift} {dtype}", flush=True)
    rng = np.random.default_rng(n * 37 + m * 11 + k)
    dy, dy64 = rows(rng, n, m, dtype, pad, shift, std=0.1)
    w, w64 = rows(rng, m, k, dtype, pad, shift, std=k ** -0.5)
    z, z64 = rows(rng, n, k, dtype, pad, shift)
    res, res64 = rows(rng, n, k, dtype, pad, shift)
    tol_v = (m + 2) * U * (np.abs(dy64) @ np.abs(w64))
    v = np.abs(dy64 @ w64)
    for kind, use_r in (("none", False), ("gelu", True), ("relu", False), ("none", True)):
        dx, buf = out_like(n, k, dtype, pad, shift)
        P.mlmc_linear_dgrad(dy, w, act=ACT[kind], z=z if kind != "none" else None, residual=res if use_r else None, dx=dx)
        want = O.linear_dgrad(dy64, w64, kind, z64, res64 if use_r else None)
        tol = 1.13 * tol_v + 2e-6 * v + 2 * U * (np.abs(want) + np.abs(res64))   # the slope of gelu: a few roundings of terms below 1
        near(f"dx {kind}", dx, want, tol + UO[dtype] * (np.abs(want) + tol))
        untouched(buf, dx)
    P.mlmc_linear_dgrad(dy, w, residual=res, dx=res)   # in the residual's place
    assert torch.equal(res, dx)
    dx = P.mlmc_linear_dgrad(dy, w, act=ACT["gelu"], z=z)
    P.mlmc_linear_dgrad(dy, w, act=ACT["gelu"], z=z, dx=z)   # in z's place
    assert torch.equal(z, dx)


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,m,k,pad,shift", LINEAR)
def test_linear_wgrad(n, m, k, pad, shift, dtype, grad):
    print(f"linear_wgrad n={n} m={m} k={k} pad={pad} shift={shift} {dtype} {grad}", flush=True)
    rng = np.random.default_rng(n * 41 + m * 13 + k)
    dy, dy64 = rows(rng, n, m, dtype, pad, shift, std=0.1, mean=0.01)
    x, x64 = rows(rng, n, k, dtype, pad, shift)
    row = torch.full((m * k + m + 3,), 77.0, dtype=DT[grad], device="cuda")   # a worker's row, the tensors at odd places
    dw, db = row[1:1 + m * k].view(m, k), row[2 + m * k:2 + m * k + m]
    P.mlmc_linear_wgrad(dy, x, dw, db)
    dw_want, db_want = O.linear_wgrad(dy64, x64)
    tol = (n + 8) * U * (np.abs(dy64).T @ np.abs(x64))
    near("dweight", dw, dw_want, tol + UO[grad] * (np.abs(dw_want) + tol))
    tol = (n + 8) * U * np.abs(dy64).sum(0)
    near("dbias", db, db_want, tol + UO[grad] * (np.abs(db_want) + tol))
    assert float(row[0]) == 77 and float(row[1 + m * k]) == 77 and float(row[2 + m * k + m]) == 77
    wide, buf = out_like(m, k, grad, 5, 1)                        # rows of the gradient apart
    P.mlmc_linear_wgrad(dy, x, wide)
    assert torch.equal(wide, dw)
    untouched(buf, wide)
    keep = row.clone()
    P.mlmc_linear_wgrad(dy, x, dw, db)
    assert torch.equal(row, keep)


def test_linear_no_rows():
    x, w = torch.empty((0, 40), device="cuda"), torch.zeros((30, 40), device="cuda")
    dw, db = torch.full((30, 40), 5.0, device="cuda"), torch.full((30,), 5.0, device="cuda")
    assert P.mlmc_linear(x, w).shape == (0, 30) and P.mlmc_linear_dgrad(torch.empty((0, 30), device="cuda"), w).shape == (0, 40)
    P.mlmc_linear_wgrad(torch.empty((0, 30), device="cuda"), x, dw, db)
    assert not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,m,k", [(2, 70, 130), (40, 70, 130), (300, 264, 520)])
def test_linear_inf_and_nan_stay_in_their_row_and_column(n, m, k, dtype):
    """What lies outside a matrix (the buffers hold NaN there) and what a tile pads with zeros never reaches an output."""
    rng = np.random.default_rng(9)
    x, _ = rows(rng, n, k, dtype, 3, 1)
    w, _ = rows(rng, m, k, dtype, 3, 1)
    x[1, k - 1] = float("inf")
    w[5, 0] = float("nan")
    y = P.mlmc_linear(x, w)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[1, :] = True
    want[:, 5] = True
    assert torch.equal(bad, want)


# ---- distillation -----------------------------------------------------------------------------------------------------
DISTILL = [  # rows, vocabulary, top, pad, shift, temperature
    (1, 1, 1, 0, 0, 1.0), (3, 2, 3, 1, 1, 2.0), (4, 63, 5, 0, 0, 1.0), (2, 64, 64, 0, 0, 4.0), (5, 257, 1, 3, 1, 0.5), (130, 1000, 16, 0, 0, 2.0), (3, 1024, 100, 8, 8, 1.0),
    (2, 4099, 300, 5, 2, 2.0), (300, 2056, 8, 0, 0, 1.0), (3, 8192, 32, 0, 0, 2.0), (2, 16391, 1024, 0, 0, 3.0), (600, 5000, 20, 0, 0, 1.0), (4, 32768, 32, 0, 0, 2.0), (1, 50021, 64, 0, 3, 1.0), (3, 65536, 10, 0, 0, 1.0), (2, 65544, 10, 8, 0, 1.0),
    (1, 131072, 64, 0, 0, 2.0), (2, 131077, 5, 0, 0, 1.0), (1, 200003, 33, 0, 0, 1.0), (1, 270000, 7, 0, 0, 2.0),
    (270, 40000, 12, 0, 0, 1.0), (513, 33000, 3, 0, 0, 2.0),
]


def teacher(rng, n, v, top, pads=True):
    """Indices, distinct except for a few, and values; some entries are padding, some rows have none but padding."""
    idx = rng.integers(0, v, (n, top))
    val = rng.normal(0, 2.0, (n, top)).astype(np.float32)
    if pads:
        idx[rng.random((n, top)) < 0.1] = -1
        val[idx < 0] = np.nan
        if n > 2:
            idx[1] = -1
            val[2, :] = -np.inf
        if n > 3 and top > 1:
            val[3, 0] = -np.inf
            idx[3, 1] = idx[3, -1]
    return idx, val


def distill_bounds(s, idx, val, temp, dloss, scale):
    n, v = s.shape
    loss, grad = O.distill(s, idx, val, temp, dloss, scale)
    m = s.max(1, keepdims=True)
    arg = np.abs(s - m) / temp
    p = np.exp(-arg)
    p /= p.sum(1, keepdims=True)
    mean_arg = (p * arg).sum(1, keepdims=True)
    rel_p = U * (4 * arg + 4 * mean_arg + v / 64 + 80)             # of p: its argument's roundings, the sum's, exp and divide
    here = idx >= 0
    t = np.where(here, val, -np.inf).astype(np.float64)
    top = np.where(np.isfinite(t.max(1)), t.max(1), 0.0)[:, None]
    targ = np.where(np.isfinite(t), np.abs(t - top) / temp, 0.0)
    rel_q = U * (8 * targ.max(1, keepdims=True) + idx.shape[1] + 80)
    q = np.zeros((n, v))
    for i in range(n):
        e = np.where(np.isfinite(t[i]), np.exp(-targ[i]), 0.0)
        if e.sum() > 0:
            np.add.at(q[i], idx[i][here[i]], (e / e.sum())[here[i]])
    w = np.abs(scale * temp * (np.ones(n) if dloss is None else dloss))[:, None]
    tol_grad = w * (p * rel_p + q * rel_q + 4 * U * (p + q))
    logs = np.zeros(n)
    for i in range(n):
        j = idx[i][here[i]]
        logs[i] = (q[i][j] * (arg[i][j] * 6 * U + rel_p[i][j] + rel_q[i] + 4 * U * (np.abs(np.log(p[i][j])) + np.abs(np.log(np.maximum(q[i][j], 1e-300)))))).sum() + \
            (q[i][j] * (rel_q[i] + (idx.shape[1] + 8) * U) * (np.abs(np.log(p[i][j])) + np.abs(np.log(np.maximum(q[i][j], 1e-300))))).sum()
    return loss, grad, temp * temp * logs + 4 * U * np.abs(loss), tol_grad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v,top,pad,shift,temp", DISTILL)
def test_distill(n, v, top, pad, shift, temp, dtype):
    print(f"distill n={n} v={v} top={top} pad={pad} shift={shift} T={temp} {dtype}", flush=True)
    rng = np.random.default_rng(n + v * 3 + top)
    s, s64 = rows(rng, n, v, dtype, pad, shift, std=2.0)
    idx, val = teacher(rng, n, v, top)
    dloss = rng.uniform(0.5, 2.0, n).astype(np.float32)
    if n > 4:
        dloss[4] = 0.0
    ti, tv = torch.from_numpy(idx.astype(np.int32)).cuda(), torch.from_numpy(val).cuda()
    ds, buf = out_like(n, v, dtype, pad, shift)
    status = torch.full((1,), 99, dtype=torch.int32, device="cuda")
    loss, _ = P.mlmc_distill(s, ti, tv, temperature=temp, dloss=torch.from_numpy(dloss).cuda(), scale=0.25, dlogits=ds, dev_status=status)
    want, grad, tol_loss, tol = distill_bounds(s64, idx, val.astype(np.float64), temp, dloss.astype(np.float64), 0.25)
    near("loss", loss, want, tol_loss)
    near("dlogits", ds, grad, tol + UO[dtype] * (np.abs(grad) + tol))
    assert int(status) == 0
    untouched(buf, ds)
    alone, none = P.mlmc_distill(s, ti, tv, temperature=temp, grad=False)
    assert none is None
    near("the loss alone", alone, want, tol_loss)
    again, g2 = P.mlmc_distill(s, ti, tv, temperature=temp, dloss=torch.from_numpy(dloss).cuda(), scale=0.25)
    assert torch.equal(again, loss) and torch.equal(g2, ds)
    P.mlmc_distill(s, ti, tv, temperature=temp, dloss=torch.from_numpy(dloss).cuda(), scale=0.25, dlogits=s)   # in place
    assert torch.equal(s, ds)


SHAPES = [(3, 100), (3, 5000), (300, 5000), (2, 40000), (300, 40000), (2, 140000), (1, 270000)]   # the ways a row may be taken


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", SHAPES)
def test_distill_masked_rows_are_not_read(n, v, dtype):
    print(f"distill masked n={n} v={v} {dtype}", flush=True)
    s = torch.full((n, v), float("nan"), dtype=DT[dtype], device="cuda")
    ds = torch.full_like(s, 3.0)
    idx = torch.full((n, 4), -1, dtype=torch.int32, device="cuda")
    loss, _ = P.mlmc_distill(s, idx, torch.full((n, 4), float("nan"), device="cuda"), dlogits=ds)
    assert not loss.any() and not ds.any()
    idx[:, 1:3] = 5
    loss, _ = P.mlmc_distill(s, idx, torch.full((n, 4), float("-inf"), device="cuda"), dlogits=ds)
    assert not loss.any() and not ds.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", SHAPES)
def test_distill_special_values(n, v, dtype):
    print(f"distill special n={n} v={v} {dtype}", flush=True)
    rng = np.random.default_rng(8)
    lowest = torch.finfo(DT[dtype]).min
    base, _ = rows(rng, n, v, dtype)
    s = base.clone()
    s[0, 7] = float("-inf")            # masked entries of the vocabulary
    s[0, 9:50] = lowest
    idx = torch.zeros((n, 3), dtype=torch.int32, device="cuda")
    idx[:] = torch.tensor([3, 60, 90], dtype=torch.int32)
    val = torch.zeros((n, 3), device="cuda")
    loss, ds = P.mlmc_distill(s, idx, val)
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(ds).all()) and not ds[0, 7] and not ds[0, 9:50].any()
    s[0, 60] = float("-inf")           # the student rules out what the teacher wants
    assert float(P.mlmc_distill(s, idx, val)[0][0]) == float("inf")
    s = torch.full_like(base, lowest)  # every entry the type's lowest value: uniform
    loss, ds = P.mlmc_distill(s, idx, torch.full_like(val, torch.finfo(torch.float32).min))
    assert np.abs(f64(loss) - (np.log(v) - np.log(3))).max() < 1e-5 * np.log(v) + 1e-6 * (v / 64)
    if n > 1:
        s = base.clone()
        s[1, v - 1] = float("nan")
        loss, ds = P.mlmc_distill(s, idx, val)
        assert bool(torch.isnan(loss[1])) and bool(torch.isnan(ds[1]).all()) and int(torch.isnan(loss).sum()) == 1 and int(torch.isnan(ds).sum()) == v
        d = torch.ones(n, device="cuda")
        d[1] = 0.0                     # a weight of zero: no gradient, whatever the logits
        _, ds = P.mlmc_distill(s, idx, val, dloss=d)
        assert not ds[1].any() and bool(ds[0].any())
        s[1, v - 1] = float("inf")
        assert bool(torch.isnan(P.mlmc_distill(s, idx, val)[0][1]))


@pytest.mark.parametrize("n,v", SHAPES)
def test_distill_index_out_of_range(n, v):
    print(f"distill out of range n={n} v={v}", flush=True)
    rng = np.random.default_rng(8)
    s, _ = rows(rng, n, v)
    idx = torch.zeros((n, 2), dtype=torch.int32, device="cuda")
    idx[n - 1, 1] = v
    val = torch.zeros((n, 2), device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, ds = P.mlmc_distill(s, idx, val, dev_status=status)
    assert int(status) == P.MLMC_DEV_RANGE and bool(torch.isnan(loss[n - 1])) and not ds[n - 1].any()
    assert n == 1 or (bool(torch.isfinite(loss[:n - 1]).all()) and bool(ds[0].any()))
    idx[n - 1, 1] = 2 ** 31 - 1
    P.mlmc_distill(s, idx, val, dev_status=status)
    assert int(status) == P.MLMC_DEV_RANGE
    idx[n - 1, 1] = -2 ** 31
    P.mlmc_distill(s, idx, val, dev_status=status)
    assert int(status) == 0


def test_distill_no_rows():
    status = torch.full((1,), 99, dtype=torch.int32, device="cuda")
    loss, ds = P.mlmc_distill(torch.empty((0, 50), device="cuda"), torch.empty((0, 3), dtype=torch.int32, device="cuda"), torch.empty((0, 3), device="cuda"), dev_status=status)
    assert loss.shape == (0,) and ds.shape == (0, 50) and int(status) == 0


# ---- streams, graphs, memory ------------------------------------------------------------------------------------------
def step(x, w1, w2, t_idx, t_val, nw, row, buf):
    """A small head, forward and backward, with the caller's buffers; weight gradients into `row`."""
    n, k = x.shape
    m, v = w1.shape[0], w2.shape[0]
    P.mlmc_layer_norm(x, nw, None, y=buf["h"], stats=buf["stats"])
    P.mlmc_linear(buf["h"], w1, None, act=ACT["gelu"], z=buf["z"], y=buf["a"], ws=buf["ws"])
    P.mlmc_linear(buf["a"], w2, y=buf["s"], ws=buf["ws"])
    P.mlmc_distill(buf["s"], t_idx, t_val, 2.0, scale=1.0 / n, loss=buf["loss"], dlogits=buf["s"], ws=buf["ws"])
    dw1, dw2, dnw = row[:m * k].view(m, k), row[m * k:m * k + v * m].view(v, m), row[m * k + v * m:]
    P.mlmc_linear_wgrad(buf["s"], buf["a"], dw2, ws=buf["ws"])
    P.mlmc_linear_dgrad(buf["s"], w2, act=ACT["gelu"], z=buf["z"], dx=buf["z"], ws=buf["ws"])
    P.mlmc_linear_wgrad(buf["z"], buf["h"], dw1, ws=buf["ws"])
    P.mlmc_linear_dgrad(buf["z"], w1, dx=buf["h"], ws=buf["ws"])
    P.mlmc_layer_norm_backward(buf["h"], x, nw, buf["stats"], dnw, None, dx=buf["h"], ws=buf["ws"])


def head(n=24, k=136, m=264, v=1003, dtype="bf16"):
    rng = np.random.default_rng(3)
    x, w1, w2 = rows(rng, n, k, dtype)[0], rows(rng, m, k, dtype, std=0.1)[0], rows(rng, v, m, dtype, std=0.1)[0]
    idx, val = teacher(rng, n, v, 8, pads=False)
    need = max(P.mlmc_layer_norm_workspace(n, k), P.mlmc_linear_workspace(n, m, k), P.mlmc_linear_workspace(n, v, m), P.mlmc_distill_workspace(n, v, 8), 256)
    e = lambda *s: torch.empty(s, dtype=DT[dtype], device="cuda")  # noqa: E731
    buf = {"h": e(n, k), "z": e(n, m), "a": e(n, m), "s": e(n, v), "stats": torch.empty((n, 2), device="cuda"), "loss": torch.empty(n, device="cuda"),
           "ws": torch.empty(need, dtype=torch.uint8, device="cuda")}
    row = torch.zeros(m * k + v * m + k, device="cuda")
    return (x, w1, w2, torch.from_numpy(idx.astype(np.int32)).cuda(), torch.from_numpy(val).cuda(), torch.ones(k, device="cuda"), row, buf)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_step_in_a_graph_and_on_another_stream(dtype):
    args = head(dtype=dtype)
    x, row, buf = args[0], args[6], args[7]
    step(*args)
    torch.cuda.synchronize()
    want, loss = row.clone(), buf["loss"].clone()
    assert bool(torch.isfinite(want).all()) and bool(want.any())
    before = torch.cuda.memory_allocated()
    row.zero_()
    step(*args)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() == before      # nothing is allocated where everything is given
    assert torch.equal(row, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        row.zero_()
        step(*args)
        got = row.clone()
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*args)
    x2 = x.clone()
    for k in range(4):
        x.copy_(x2 * (1.0 + k))
        row.zero_()
        step(*args)
        torch.cuda.synchronize()
        eager, el = row.clone(), buf["loss"].clone()
        row.zero_()
        buf["loss"].zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(row, eager) and torch.equal(buf["loss"], el)
        if k == 0:
            assert torch.equal(row, want) and torch.equal(el, loss)


def test_the_librarys_own_kernels_run():
    names = launched(lambda: step(*head()))
    assert names and all(n.startswith(("k_norm", "k_linear", "k_distill")) for n in names), names


# ---- sizes that take the other ways -----------------------------------------------------------------------------------
def test_linear_large_tiles():
    """Products large enough for the largest tile, the contraction ending inside a step; the definition on the GPU in 64 bits."""
    n, m, k = 4072, 4088, 4040
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    make = lambda r, c, std: torch.empty((r, c), device="cuda").normal_(0.0, std, generator=gen).to(torch.bfloat16)  # noqa: E731
    x, w, dy, z, res = make(n, k, 1.0), make(m, k, k ** -0.5), make(n, m, 0.1), make(n, k, 1.0), make(n, m, 1.0)
    b = torch.empty(m, device="cuda").normal_(0.0, 0.3, generator=gen)

    def check(name, got, want, tol):
        off = (got.double() - want).abs() - tol
        assert bool((off <= 0).all()), f"{name}: {float(off.max())}"

    X, W, D, Z, R = (t.double() for t in (x, w, dy, z, res))
    v = X @ W.t().contiguous() + b.double()
    tol_v = (k + 2) * U * (X.abs() @ W.abs().t().contiguous() + b.double().abs())
    zo = torch.empty((n, m), dtype=torch.bfloat16, device="cuda")
    y = P.mlmc_linear(x, w, b, act=ACT["gelu"], residual=res, z=zo)
    want = 0.5 * v * torch.erfc(-v / 2 ** 0.5) + R
    tol = 1.13 * tol_v + (8 * U + 1e-7) * v.abs() + 2 * U * (want.abs() + R.abs())
    check("y", y, want, tol + UO["bf16"] * (want.abs() + tol))
    check("z", zo, v, tol_v + UO["bf16"] * (v.abs() + tol_v))
    dx = P.mlmc_linear_dgrad(dy, w, act=ACT["gelu"], z=z)
    v = D @ W
    want = v * (0.5 * torch.erfc(-Z / 2 ** 0.5) + Z * torch.exp(-0.5 * Z * Z) * (2 * np.pi) ** -0.5)
    tol = 1.13 * (m + 2) * U * (D.abs() @ W.abs()) + 2e-6 * v.abs() + 2 * U * want.abs()
    check("dx", dx, want, tol + UO["bf16"] * (want.abs() + tol))
    dw, db = torch.empty((m, k), device="cuda"), torch.empty(m, device="cuda")
    P.mlmc_linear_wgrad(dy, x, dw, db)
    check("dweight", dw, D.t().contiguous() @ X, (n + 9) * U * (D.abs().t().contiguous() @ X.abs()))
    check("dbias", db, D.sum(0), (n + 9) * U * D.abs().sum(0))


def test_offsets_past_32_bits():
    """Rows two to the 28 entries apart: the last of 20 begins 10 GB behind the first."""
    n, d, far = 20, 200, (1 << 28) + 3
    rng = np.random.default_rng(4)
    big = torch.empty(far * (n - 1) + d, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(big, (n, d), (far, 1), 0)
    near_, x64 = rows(rng, n, d, "bf16")
    x.copy_(near_)
    w, w64 = vec(rng, d, 1.0, 0.2)
    y, stats = P.mlmc_layer_norm(x, w, with_stats=True)
    assert torch.equal(y, P.mlmc_layer_norm(near_, w))
    dy, dy64 = rows(rng, n, d, "bf16")
    dw, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    dx = P.mlmc_layer_norm_backward(dy, x, w, stats, dw, db)
    dw2 = torch.empty_like(dw)
    assert torch.equal(dx, P.mlmc_layer_norm_backward(dy, near_, w, stats, dw2)) and torch.equal(dw, dw2)
    wt, wt64 = rows(rng, 72, d, "bf16", std=0.1)
    for k in (3, n):                                               # the way of few rows and the tiles
        out = torch.as_strided(big, (k, 72), (far, 1), d - 72)
        keep = out.clone()
        want = x64[:k] @ wt64.T
        tol = (d + 2) * U * (np.abs(x64[:k]) @ np.abs(wt64).T)
        got = P.mlmc_linear(x[:k], wt)
        near("y", got, want, tol + UO["bf16"] * (np.abs(want) + tol))
        other = torch.as_strided(torch.empty(far * (k - 1) + 72, dtype=torch.bfloat16, device="cuda"), (k, 72), (far, 1), 0)
        P.mlmc_linear(x[:k], wt, y=other)
        assert torch.equal(other, got) and torch.equal(out, keep)
        del other
    g = torch.empty((72, d), device="cuda")
    dz, dz64 = rows(rng, n, 72, "bf16")
    P.mlmc_linear_wgrad(dz, x, g)
    near("dweight", g, dz64.T @ x64, (n + 8) * U * (np.abs(dz64).T @ np.abs(x64)))
    idx, val = teacher(rng, n, d, 5, pads=False)
    ti, tv = torch.from_numpy(idx.astype(np.int32)).cuda(), torch.from_numpy(val).cuda()
    loss, ds = P.mlmc_distill(near_, ti, tv)
    loss2, _ = P.mlmc_distill(x, ti, tv, dlogits=x)
    assert torch.equal(loss, loss2) and torch.equal(ds, x)


@pytest.mark.parametrize("dtype,n", [("f32", 130), ("bf16", 250)])
def test_distill_long_rows_in_groups(dtype, n):
    """Rows too long for a workgroup, and more of them than one launch takes: the ends of the groups against the definition."""
    v = 270_001
    rng = np.random.default_rng(6)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    s = torch.empty((n, v), device="cuda").normal_(0.0, 2.0, generator=gen).to(DT[dtype])
    idx, val = teacher(rng, n, v, 6)
    ti, tv = torch.from_numpy(idx.astype(np.int32)).cuda(), torch.from_numpy(val).cuda()
    loss, ds = P.mlmc_distill(s, ti, tv, 2.0, scale=0.25)
    for i in (0, 1, 2, 3, 92, 93, 94, n - 65, n - 64, n - 1):
        want, grad, tol_loss, tol = distill_bounds(f64(s[i:i + 1]), idx[i:i + 1], val[i:i + 1].astype(np.float64), 2.0, None, 0.25)
        near(f"loss {i}", loss[i:i + 1], want, tol_loss)
        near(f"dlogits {i}", ds[i:i + 1], grad, tol + UO[dtype] * (np.abs(grad) + tol))
    P.mlmc_distill(s, ti, tv, 2.0, scale=0.25, dlogits=s)
    bits = torch.int32 if dtype == "f32" else torch.int16          # (one row's teacher has a NaN)
    assert torch.equal(s.view(bits), ds.view(bits))


@pytest.mark.parametrize("n,v", SHAPES)
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_distill_nan_and_inf_among_the_teachers_values(n, v, what):
    """The row's loss and its gradient at the teacher's indices are NaN, all else is as without."""
    print(f"distill teacher {what} n={n} v={v}", flush=True)
    rng = np.random.default_rng(8)
    s, s64 = rows(rng, n, v)
    idx = np.tile(np.array([3, 60, 90]), (n, 1))
    val = rng.normal(0, 1, (n, 3)).astype(np.float32)
    val[n - 1, 1] = what
    loss, ds = P.mlmc_distill(s, torch.from_numpy(idx.astype(np.int32)).cuda(), torch.from_numpy(val).cuda())
    for i in {0, n - 1}:
        want, grad = O.distill(s64[i:i + 1], idx[i:i + 1], val[i:i + 1].astype(np.float64), 1.0)
        assert np.isnan(want[0]) == (i == n - 1) and np.isnan(grad).sum() == (3 if i == n - 1 else 0)
        p = np.exp(s64[i] - s64[i].max())
        near(f"dlogits {i}", ds[i:i + 1], grad, (p / p.sum() + 1)[None] * U * (v / 64 + 200))
    assert int(torch.isnan(loss).sum()) == 1 and bool(torch.isnan(loss[n - 1]))


@pytest.mark.parametrize("n,m,k,pad,shift", [(130, 70, 130, 2, 2), (70, 258, 194, 0, 0), (33, 6, 2, 0, 6), (300, 130, 4, 2, 2), (2, 2, 1000, 0, 2), (515, 262, 134, 4, 4)])
def test_linear_of_rows_that_begin_at_four_bytes(n, m, k, pad, shift):
    for dtype in ("bf16", "f32"):
        test_linear(n, m, k, pad, shift, dtype)
        test_linear_dgrad(n, m, k, pad, shift, dtype)
        test_linear_wgrad(n, m, k, pad, shift, dtype, "bf16")


@pytest.mark.parametrize("n,m,k", [(1, 48, 9000), (3, 40, 20000), (16, 16, 20003)])
def test_linear_few_rows_few_outputs_long_contraction(n, m, k):
    for dtype in ("bf16", "f32"):
        test_linear(n, m, k, 0, 0, dtype)
        test_linear(n, m, k, 3, 1, dtype)


def same(name, a, b):
    """Equal entry by entry, NaN with NaN."""
    assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.where(torch.isnan(a), 0.0, a), torch.where(torch.isnan(b), 0.0, b)), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(1, 8), (17, 24), (500, 320), (4099, 512), (3, 520), (2051, 1000), (5, 1500), (1027, 2048), (3, 2056), (515, 4096), (7, 8191), (5, 16384), (3, 5), (4, 16400)])
def test_layer_norm_backward_in_the_place_of_x(n, d, dtype):
    """dx in the place of x, or of dy, with an Inf in the last row's gradient: its dx is not finite, and dweight and dbias are those of a call with a dx of its own, where a single
    column is not finite."""
    print(f"layer_norm_backward in place n={n} d={d} {dtype}", flush=True)
    rng = np.random.default_rng(n + d)
    x, _ = rows(rng, n, d, dtype)
    dy, _ = rows(rng, n, d, dtype, std=0.1)
    dy[n - 1, d // 2] = float("inf")
    w, _ = vec(rng, d, 1.0, 0.3)
    _, stats = P.mlmc_layer_norm(x, w, None, with_stats=True)
    dw, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    dx = P.mlmc_layer_norm_backward(dy, x, w, stats, dw, db)
    assert not bool(torch.isfinite(dx[n - 1]).any()) and bool(torch.isfinite(dx[:n - 1]).all())
    off = (~torch.isfinite(dw)).nonzero().flatten().tolist()
    assert off == [d // 2] and (~torch.isfinite(db)).nonzero().flatten().tolist() == [d // 2]
    for place in ("x", "dy"):
        x2, dy2 = x.clone(), dy.clone()
        dw2, db2 = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        P.mlmc_layer_norm_backward(dy2, x2, w, stats, dw2, db2, dx=x2 if place == "x" else dy2)
        same("dx in " + place, x2 if place == "x" else dy2, dx)
        same("dweight, dx in " + place, dw2, dw)
        same("dbias, dx in " + place, db2, db)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,m", [(3, 8), (40, 8), (40, 4096)])      # a tile, and one in parts with a join
def test_activations_at_infinity(n, m, dtype):
    """Where the activation is a straight line already, infinity is on it: the slope of gelu and relu is 1 at +Inf and 0 at -Inf, gelu(-Inf) = 0; NaN stays NaN (the slope of relu
    is a comparison, 0 there)."""
    top = float(torch.finfo(DT[dtype]).max)
    z = torch.tensor([float("inf"), -float("inf"), float("nan"), top, -top, 1e30, -1e30, 70.0, -70.0, 0.0], device="cuda").to(DT[dtype])
    k = z.numel()
    dy = torch.zeros((n, m), dtype=DT[dtype], device="cuda")
    dy[:, 0] = 2.0
    w = torch.zeros((m, k), dtype=DT[dtype], device="cuda")
    w[0] = 1.0
    for kind, at_zero in (("gelu", 1.0), ("relu", 0.0)):
        dx = P.mlmc_linear_dgrad(dy, w, act=ACT[kind], z=z.expand(n, k).contiguous())
        want = torch.tensor([2.0, 0.0, float("nan") if kind == "gelu" else 0.0, 2.0, 0.0, 2.0, 0.0, 2.0, 0.0, at_zero], device="cuda").to(DT[dtype])
        same("dx " + kind, dx, want.expand(n, k))
    x, one = z[:, None].contiguous(), torch.ones((1, 1), dtype=DT[dtype], device="cuda")
    for kind in ("gelu", "relu"):
        y = P.mlmc_linear(x, one, act=ACT[kind])[:, 0]
        same("y " + kind, y, torch.tensor([float("inf"), 0.0, float("nan"), top, 0.0, 1e30, 0.0, 70.0, 0.0, 0.0], device="cuda").to(DT[dtype]))


def test_gelu_of_32_bits_is_as_exact_as_its_roundings():
    """A product with one is exact, so that only gelu and its slope round.  In units of U and relative to the term: erfc 32 (16 ulp, the most that it may be off), its argument's two roundings
    2 (z^2 + 1) of the tail; the exponential 6, its argument's z^2 / 2, the products 4.  Near zero, where most entries are, no more than elementary operations with erf are off."""
    one = torch.ones((1, 1), device="cuda")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    normal = torch.empty(1 << 18, device="cuda").normal_(generator=gen)
    z = torch.cat((normal, torch.linspace(-12, 12, 100001, device="cuda")))[:, None].contiguous()
    Z = z.double()
    phi, density = 0.5 * torch.erfc(-Z / 2 ** 0.5), torch.exp(-0.5 * Z * Z) / (2 * np.pi) ** 0.5
    tail = U * (35 + 2 * (Z * Z + 1)) * phi
    for n in (16, z.shape[0]):                                     # the way of few rows and the tiles
        y = P.mlmc_linear(z[:n], one, act=ACT["gelu"]).double()
        off = (y - (Z * phi)[:n]).abs() - (tail * Z.abs() + 1e-37)[:n]
        assert bool((off <= 0).all()), float(off.max())
    slope = P.mlmc_linear_dgrad(torch.ones_like(z), one, act=ACT["gelu"], z=z).double()
    want = phi + Z * density
    off = (slope - want).abs() - (tail + U * (Z * Z / 2 + 10) * (Z * density).abs() + U * want.abs() + 1e-37)
    assert bool((off <= 0).all()), float(off.max())
    near_, n = z[:1 << 18], 1 << 18
    erf = torch.erf(near_ * 0.5 ** 0.5)
    rms = lambda v: float(v.pow(2).mean().sqrt())  # noqa: E731
    assert rms(y[:n] - (Z * phi)[:n]) <= rms((0.5 * near_ * (1 + erf)).double() - (Z * phi)[:n])
    plain = 0.5 * (1 + erf) + near_ * torch.exp(-0.5 * near_ * near_) * (2 * np.pi) ** -0.5
    assert rms(slope[:n] - want[:n]) <= rms(plain.double() - want[:n])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [5, 13, 15, 41, 60, 448, 832, 960, 1920, 2624, 3008, 3264, 3520, 4032, 8064, 13000, 20001])
def test_layer_norm_of_equal_entries_is_the_bias(d, dtype):
    """The sums of these entries are exact and so is their quotient by the width: the mean is the entry itself, and the row the bias, at widths too whose reciprocal rounds."""
    b = torch.arange(d, dtype=torch.float32, device="cuda") % 251
    for v in (1.0, 2.5, 1000.0):
        y, stats = P.mlmc_layer_norm(torch.full((3, d), v, dtype=DT[dtype], device="cuda"), None, b, with_stats=True)
        assert bool((stats[:, 0] == v).all()), (v, stats)
        assert torch.equal(y, b.to(DT[dtype]).expand(3, d)), v


@pytest.mark.parametrize("n,v", SHAPES)
def test_distill_at_temperatures_near_zero(n, v):
    """The softmaxes are one entry each then, and the loss is T (greatest logit - logit at the teacher's greatest), with the roundings of a difference, a product and q; the squares of
    these temperatures are no numbers of fp32."""
    print(f"distill cold n={n} v={v}", flush=True)
    rng = np.random.default_rng(11)
    s, s64 = rows(rng, n, v, std=2.0)
    idx = np.tile(np.array([3, 60, 90]), (n, 1))
    val = np.tile(np.array([0.5, 2.0, -1.0], dtype=np.float32), (n, 1))
    for t in (1e-12, 1e-20, 1e-25, 1e-30, 1e-36):
        t = float(np.float32(t))
        loss, ds = P.mlmc_distill(s, torch.from_numpy(idx.astype(np.int32)).cuda(), torch.from_numpy(val).cuda(), temperature=t)
        want = t * (s64.max(1) - s64[:, 60])
        near(f"loss {t}", loss, want, 8 * U * want)
        grad = np.zeros((n, v))
        grad[np.arange(n), s64.argmax(1)] = t
        grad[:, 60] -= t
        near(f"dlogits {t}", ds, grad, 8 * U * np.abs(grad))
