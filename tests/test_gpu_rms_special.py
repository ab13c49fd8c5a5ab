"""Root-mean-square norm with weights and roots that are no numbers of fp32, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2507_05508_amd as P
from oracle import worker as O
from test_gpu_rms import relative
from test_gpu_worker import U, UO, f64, rows, vec

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def same(got, want, rel):
    """Infinities and NaN in the same places, numbers within their bound."""
    got = f64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), (np.isnan(got).sum(), np.isnan(want).sum())
    inf = np.isinf(want)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(got[inf], want[inf])
    ok = np.isfinite(want)
    assert (np.abs(got[ok] - want[ok]) <= rel * np.abs(want[ok])).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [5, 40, 700, 1500, 3001, 5000, 9000, 20000])
def test_infinite_weights(d, dtype):
    """s r w is infinite where w is, NaN where s is 0 there; the other columns are what they are."""
    rng = np.random.default_rng(d)
    x, x64 = rows(rng, 6, d, dtype)
    r, r64 = rows(rng, 6, d, dtype)
    w, w64 = vec(rng, d, 1.0, 0.3)
    for j, v in ((0, INF), (2, -INF), (3, NAN), (d - 1, INF)):
        w[j] = w64[j] = v
    x[1, 2] = x64[1, 2] = 0.0
    x[2, 0] = x64[2, 0] = 1e-30
    rel = relative(d)
    with np.errstate(invalid="ignore"):
        want, _ = O.rms_norm(x64, w64, 1e-5)
        both, _ = O.rms_norm(x64 + r64, w64, 1e-5)
    out = rel + UO[dtype] * (1 + rel)
    same(P.mlmc_rms_norm(x, w).y, want, out)
    got = P.mlmc_rms_norm(x, w, r, with_q=True)
    same(got.y, both, out)
    assert bool(got.scale.isnan().all()) and bool(got.q.float().isnan().all())      # a row with an infinity has no 8 bits


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [5, 40, 5000, 9000, 20000])
def test_squares_below_fp32(d, dtype):
    """eps = 0 and squares whose fp32 sum is 0: the root is infinite, and y the product with it; a row of zeros is NaN."""
    x = torch.zeros((3, d), device="cuda")
    x[1] = 1e-30
    x[1, 1] = -1e-30
    x[2] = 0.5
    got = P.mlmc_rms_norm(x.to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype]), eps=0.0, with_rstd=True)
    y = got.y.float()
    assert bool(y[0].isnan().all()) and bool((got.rstd[:2] == INF).all())
    assert y[1, 1] == -INF and bool((y[1, 2:] == INF).all()) and y[1, 0] == INF
    assert bool(((y[2] - 1.0).abs() <= relative(d) + U).all())
