"""Layer norm, linear layer and distillation loss at sizes whose definition in 64 bits runs on the GPU: many rows, long rows, several rounds of a
workgroup, every tile and every way of the linear layer.  Bounds as in test_gpu_worker.py (U is the rounding of fp32; a sum's error is U times the additions that a
term passes through times the sum of the terms' magnitudes)."""
import re

import numpy as np
import pytest
import torch

import paper_2507_05508_amd as P
from test_gpu_worker import ACT, DT, U, UO, out_like, untouched

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


# ---- layer norm, more rows than the workgroups take at once -----------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(8197, 320), (4099, 1000), (2051, 1536), (1030, 4096), (515, 8191), (515, 16384)])
def test_layer_norm_in_rounds(n, d, dtype):
    """Two rounds of rows and a part of a third for every number of threads that share a row: the rows fetched ahead, the LDS that rounds take in turn, dweight and dbias
    added up over the rounds; in place as well."""
    print(f"layer_norm rounds n={n} d={d} {dtype}", flush=True)
    x, dy, w, b = norm_case(n, d, dtype, n + d)
    y, stats = P.mlmc_layer_norm(x, w, b, with_stats=True)
    want, mean, rstd, ty, tm, tr = norm_forward_bounds(x.double(), w.double(), b.double(), 1e-5)
    check("mean", stats[:, 0], mean, tm)
    check("rstd", stats[:, 1], rstd, tr)
    check("y", y, want, ty, UO[dtype])
    dw, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    dx = P.mlmc_layer_norm_backward(dy, x, w, stats, dw, db)
    want, want_w, want_b, tol, tol_w, tol_b = norm_backward_bounds(dy.double(), x.double(), w.double(), stats)
    check("dx", dx, want, tol, UO[dtype])
    check("dweight", dw, want_w, tol_w, U)
    check("dbias", db, want_b, tol_b, U)
    for place in ("x", "dy"):
        x2, dy2 = x.clone(), dy.clone()
        dw2, db2 = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        P.mlmc_layer_norm_backward(dy2, x2, w, stats, dw2, db2, dx=x2 if place == "x" else dy2)
        assert torch.equal(x2 if place == "x" else dy2, dx) and torch.equal(dw2, dw) and torch.equal(db2, db), place
    x2 = x.clone()
    P.mlmc_layer_norm(x2, w, b, y=x2)
    assert torch.equal(x2, y)


# ---- linear layer, every tile and every way ---------------------------------------------------------------------------
# rows, outputs, inputs, type, pad, shift: between them every tile (32, 64, 128, 256 rows) meets every way to LDS (registers, chunks, words), whole and in parts of the contraction, with
# neither, either and both of its operands copied to aligned rows, in each of the three directions that the plan has it for.
TILES = [
    (17, 8, 8, "f32", 0, 0), (17, 8, 8, "f32", 3, 1), (17, 8, 8, "bf16", 0, 0), (17, 8, 8, "bf16", 3, 1), (17, 8, 8, "bf16", 2, 2), (17, 8, 613, "bf16", 0, 0),
    (17, 8, 20001, "bf16", 3, 1), (17, 257, 1024, "bf16", 0, 0), (1000, 8, 1030, "f32", 0, 0), (1000, 8, 1030, "bf16", 0, 0), (1000, 1030, 8, "bf16", 3, 1),
    (515, 8, 2048, "f32", 0, 0), (1000, 8, 2048, "bf16", 0, 0), (1000, 8, 2048, "bf16", 3, 1), (1000, 2048, 8, "bf16", 0, 0), (1000, 2048, 8, "bf16", 2, 2),
    (1000, 4095, 8, "f32", 0, 0), (1000, 4095, 8, "bf16", 0, 0), (1000, 4095, 8, "bf16", 3, 1), (2048, 4095, 8, "bf16", 2, 2), (4097, 4096, 8, "f32", 0, 0),
    (4097, 4098, 8, "f32", 3, 1), (300, 257, 4096, "bf16", 2, 2), (300, 1030, 1024, "f32", 0, 0), (4097, 1024, 130, "bf16", 0, 0), (515, 2048, 1024, "f32", 0, 0),
    (2048, 4096, 257, "bf16", 0, 0), (1000, 1024, 4095, "f32", 0, 0), (4096, 4095, 257, "bf16", 0, 0), (4097, 130, 8192, "bf16", 0, 0),
    (4097, 130, 8192, "bf16", 3, 1), (4097, 136, 8192, "bf16", 2, 2), (8192, 8192, 136, "bf16", 0, 0), (4097, 136, 20000, "bf16", 0, 0),
    (1000, 4098, 4098, "bf16", 0, 0), (1000, 8, 4095, "bf16", 0, 0), (17, 1024, 4095, "bf16", 0, 0), (17, 4095, 1024, "bf16", 0, 0), (17, 512, 8192, "f32", 0, 0),
    (17, 1024, 4096, "bf16", 0, 0), (17, 1024, 4096, "bf16", 3, 1), (17, 1024, 4096, "bf16", 2, 2), (4097, 257, 136, "bf16", 0, 0), (20003, 2048, 8, "bf16", 3, 1),
    (20003, 2048, 8, "bf16", 2, 2), (4096, 4096, 257, "bf16", 0, 0), (515, 4095, 4096, "bf16", 0, 0), (8192, 130, 8192, "bf16", 0, 0),
    (200, 4096, 20000, "bf16", 0, 0), (4097, 4098, 1024, "bf16", 0, 0), (8192, 8192, 257, "bf16", 0, 0), (4096, 1030, 4095, "bf16", 0, 0),
    (20003, 512, 2048, "f32", 0, 0), (20003, 136, 8192, "bf16", 0, 0), (300, 4095, 20000, "bf16", 3, 1), (515, 4096, 20001, "bf16", 0, 0),
    (1000, 4095, 8, "f32", 3, 1), (4097, 8, 2048, "f32", 3, 1), (1000, 2049, 4095, "bf16", 0, 0),
]
MET = {}


def tiles_of(call):
    """The call's result, and which kernels it launched: (tile's rows, way, "parts" if it was joined, "copied" if an operand was)."""
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        out = call()
        torch.cuda.synchronize()
    names = [e.key for e in prof.key_averages()]
    for name in names:
        m = re.search(r"k_linear_tile<\d, (\d), \d, (\d), \d, (?:true|false), (?:true|false), (\d)>", name)
        if m:
            rows, way = 32 * int(m[1]) * int(m[2]), ("registers", "chunks", "words")[int(m[3])]
            return out, (rows, way, any("k_linear_join" in k for k in names), any("k_linear_pack" in k for k in names))
    return out, None


@pytest.mark.parametrize("n,m,k,dtype,pad,shift", TILES)
def test_linear_tiles(n, m, k, dtype, pad, shift):
    print(f"linear tiles n={n} m={m} k={k} {dtype} pad={pad} shift={shift}", flush=True)
    gen = generator(n + m + k)
    x, w = normal(gen, n, k, dtype, 1.0, 0.0, pad, shift), normal(gen, m, k, dtype, k ** -0.5, 0.0, pad, shift)
    dy, z, res = normal(gen, n, m, dtype, 0.1, 0.01, pad, shift), normal(gen, n, k, dtype, 1.0, 0.0, pad, shift), normal(gen, n, m, dtype, 1.0, 0.0, pad, shift)
    b = torch.empty(m, device="cuda").normal_(0.0, 0.3, generator=gen)
    X, W, D = x.double(), w.double(), dy.double()
    met = MET.setdefault((n, m, k, dtype, pad, shift), {})
    # forward
    y, buf = out_like(n, m, dtype, pad, shift)
    zo, zbuf = out_like(n, m, dtype, pad, shift)
    _, met["forward"] = tiles_of(lambda: P.mlmc_linear(x, w, b, act=ACT["gelu"], residual=res, z=zo, y=y))
    v = X @ W.t().contiguous() + b.double()
    tol_v = (k + 2) * U * (X.abs() @ W.abs().t().contiguous() + b.double().abs())
    check("z", zo, v, tol_v, UO[dtype])
    want = 0.5 * v * torch.erfc(-v / 2 ** 0.5) + res.double()
    check("y", y, want, 1.13 * tol_v + (8 * U + 1e-7) * v.abs() + 2 * U * (want.abs() + res.double().abs()), UO[dtype])
    untouched(buf, y)
    untouched(zbuf, zo)
    del v, tol_v, want, buf, zbuf, y, zo
    # input gradient
    dx, buf = out_like(n, k, dtype, pad, shift)
    _, met["input"] = tiles_of(lambda: P.mlmc_linear_dgrad(dy, w, act=ACT["gelu"], z=z, dx=dx))
    v, Z = D @ W, z.double()
    want = v * (0.5 * torch.erfc(-Z / 2 ** 0.5) + Z * torch.exp(-0.5 * Z * Z) * (2 * np.pi) ** -0.5)
    check("dx", dx, want, 1.13 * (m + 2) * U * (D.abs() @ W.abs()) + 2e-6 * v.abs() + 2 * U * want.abs(), UO[dtype])
    untouched(buf, dx)
    P.mlmc_linear_dgrad(dy, w, act=ACT["gelu"], z=z, dx=z)        # in z's place
    assert torch.equal(z, dx)
    del v, Z, want, buf, dx
    # weight gradient, at an odd place of a row
    row = torch.full((m * k + m + 3,), 77.0, device="cuda")
    dw, db = row[1:1 + m * k].view(m, k), row[2 + m * k:2 + m * k + m]
    _, met["weight"] = tiles_of(lambda: P.mlmc_linear_wgrad(dy, x, dw, db))
    check("dweight", dw, D.t().contiguous() @ X, (n + 9) * U * (D.abs().t().contiguous() @ X.abs()))
    check("dbias", db, D.sum(0), (n + 9) * U * D.abs().sum(0))
    assert float(row[0]) == 77 and float(row[1 + m * k]) == 77 and float(row[2 + m * k + m]) == 77
    dw16, db16 = torch.empty((m, k), dtype=torch.bfloat16, device="cuda"), torch.empty(m, dtype=torch.bfloat16, device="cuda")
    P.mlmc_linear_wgrad(dy, x, dw16, db16)
    assert torch.equal(dw16, dw.to(torch.bfloat16)) and torch.equal(db16, db.to(torch.bfloat16))


def test_linear_tiles_are_all_met():
    """The sizes above reach what they are there for (the plan's costs may change)."""
    if len(MET) < len(TILES) or not any(any(v.values()) for v in MET.values()):
        pytest.skip("needs the tests above, and the profiler's names of their kernels")
    for dtype in ("f32", "bf16"):
        for part in ("forward", "input", "weight"):
            met = {v[part] for key, v in MET.items() if key[3] == dtype}
            want = {(t, way, parts, False) for t in (32, 64, 128) for way in (("chunks", "words") if dtype == "f32" else ("registers", "chunks", "words")) for parts in (False, True)}
            if dtype == "bf16":
                want |= {(256, "chunks", parts, copied) for parts in (False, True) for copied in (False, True)}
                want |= {(t, "chunks", False, True) for t in (64, 128)}
            assert want <= met, (dtype, part, want - met)
