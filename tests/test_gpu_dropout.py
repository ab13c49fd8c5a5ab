"""Dropout on the GPU against the definition (oracle/worker.py): the mask bit for bit, the values within two roundings of fp32 (of the scale and of the product) and the output's own."""
import numpy as np
import pytest
import torch

import paper_2507_05508_amd as P
from oracle import worker as O
from test_gpu_worker import DT, U, UO, f64, near, out_like, rows, untouched

pytestmark = pytest.mark.gpu
SIZES = [  # rows, width, pad, shift
    (1, 1, 0, 0), (3, 2, 1, 1), (2, 7, 0, 0), (5, 8, 0, 0), (5, 9, 0, 1), (4, 64, 0, 0), (7, 65, 3, 1), (33, 256, 0, 0), (9, 257, 0, 3), (17, 1000, 8, 8), (3, 2056, 0, 0), (2, 4099, 5, 2),
    (300, 16, 0, 0), (1, 20001, 0, 1), (700, 24, 1, 0),
]
SEED = 0xFEDCBA9876543210


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad,shift", SIZES)
def test_dropout(n, d, pad, shift, dtype):
    print(f"dropout n={n} d={d} pad={pad} shift={shift} {dtype}", flush=True)
    rng = np.random.default_rng(n * 7919 + d)
    x, x64 = rows(rng, n, d, dtype, pad, shift)
    r, r64 = rows(rng, n, d, dtype, shift, pad, std=3.0)
    for p in (0.1, 0.5):
        least = int(np.floor(p * 65536 + 0.5))
        keep = O.dropout_keep(n, d, least, SEED, 5, 17, row0=1000)
        scaled = np.where(keep, x64 / (1 - least / 65536), 0.0)
        y, buf = out_like(n, d, dtype, pad, shift)
        assert P.mlmc_dropout(x, p, SEED, 5, stream=17, row0=1000, y=y) is y
        untouched(buf, y)
        near("y", y, scaled, (2 * U + UO[dtype] * (1 + 2 * U)) * np.abs(scaled))
        assert np.array_equal(f64(y) != 0, keep & (x64 != 0))
        z = P.mlmc_dropout(x, p, SEED, 5, stream=17, row0=1000, residual=r)
        t = 2 * U * np.abs(scaled) + U * np.abs(scaled + r64)
        near("sum", z, scaled + r64, t + UO[dtype] * (np.abs(scaled + r64) + t))
        assert torch.equal(z[torch.from_numpy(~keep).cuda()], r[torch.from_numpy(~keep).cuda()])      # what is dropped leaves the residual as it was
        for k in range(2):      # in the place of x, of the residual
            t = [x.clone(), r.clone()]
            P.mlmc_dropout(t[0], p, SEED, 5, stream=17, row0=1000, residual=t[1], y=t[k])
            assert torch.equal(t[k], z)


def test_dropout_of_all_numbers_it_takes():
    """The ends of step, stream and row0, and a seed past 64 bits, which is taken modulo 2^64."""
    x = torch.ones((2, 40), device="cuda")
    for seed, step, stream, row0 in ((0, 0, 0, 0), ((1 << 64) - 1, (1 << 32) - 1, (1 << 32) - 1, (1 << 32) - 2), (1 << 63, 1, 2, 1 << 31)):
        y = P.mlmc_dropout(x, 0.5, seed, step, stream=stream, row0=row0)
        assert np.array_equal(f64(y) != 0, O.dropout_keep(2, 40, 32768, seed, step, stream, row0))
    assert torch.equal(P.mlmc_dropout(x, 0.5, 7, 1), P.mlmc_dropout(x, 0.5, 7 + (1 << 64), 1))


def test_dropout_shares():
    """p of 0 drops nothing, the smallest p that is not 0 one in 65536, the greatest all but one: the mean stays."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.empty((257, 1003), device="cuda").normal_(generator=gen)
    assert torch.equal(P.mlmc_dropout(x, 0.0, 1, 2), x) and torch.equal(P.mlmc_dropout(x, 2.0 ** -18, 1, 2), x)
    ones = torch.ones((4096, 4096), device="cuda")      # 2^24 entries
    for p in (2.0 ** -16, 0.1, 0.3, 1 - 2.0 ** -16):
        y = P.mlmc_dropout(ones, p, 3, 4)
        least = int(p * 65536 + 0.5)
        share, q = float((y == 0).double().mean()), least / 65536
        assert abs(share - q) <= 6 * (q * (1 - q) / ones.numel()) ** 0.5, (p, share)
        assert y.max() == np.float32(65536 / (65536 - least))


def test_dropout_drops_infinities():
    x = torch.full((8, 512), float("inf"), device="cuda")
    x[::2] = float("nan")
    r = torch.ones_like(x)
    keep = torch.from_numpy(O.dropout_keep(8, 512, 32768, 1, 2, 0)).cuda()
    y, z = P.mlmc_dropout(x, 0.5, 1, 2), P.mlmc_dropout(x, 0.5, 1, 2, residual=r)
    assert bool((y[~keep] == 0).all()) and bool((z[~keep] == 1).all()) and not bool(y[keep].isfinite().any()) and not bool(z[keep].isfinite().any())


def test_dropout_is_the_same_for_every_type_cut_and_launch():
    """A large matrix, cut into rows and columns, of either type: the mask is that of the place."""
    ones = torch.ones((3001, 4104), device="cuda")
    whole = P.mlmc_dropout(ones, 0.25, SEED, 9, stream=1)
    assert torch.equal(P.mlmc_dropout(ones.bfloat16(), 0.25, SEED, 9, stream=1) != 0, whole != 0)
    assert torch.equal(P.mlmc_dropout(ones[:, :1001], 0.25, SEED, 9, stream=1), whole[:, :1001])
    parts = torch.cat([P.mlmc_dropout(ones[i:i + 700], 0.25, SEED, 9, stream=1, row0=i) for i in range(0, 3001, 700)])
    assert torch.equal(parts, whole)
    at = [0, 1499, 3000]
    for i in at:
        assert np.array_equal(f64(whole[i:i + 1]) != 0, O.dropout_keep(1, 4104, 16384, SEED, 9, 1, row0=i))
    thin = P.mlmc_dropout(torch.ones((70001, 8), device="cuda"), 0.25, SEED, 9)      # more rows than workgroups along them
    assert np.array_equal(f64(thin[70000:]) != 0, O.dropout_keep(1, 8, 16384, SEED, 9, 0, row0=70000))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropout_gradient(dtype):
    """The same call on the gradient, with one that comes by another way; and against differences: the call is linear in x."""
    rng = np.random.default_rng(2)
    dy, dy64 = rows(rng, 37, 301, dtype)
    other, other64 = rows(rng, 37, 301, dtype)
    dx = P.mlmc_dropout(dy, 0.3, 5, 6, stream=7, residual=other)
    least = int(0.3 * 65536 + 0.5)
    want = np.where(O.dropout_keep(37, 301, least, 5, 6, 7), dy64 / (1 - least / 65536), 0.0) + other64
    t = 3 * U * (np.abs(want) + np.abs(other64))
    near("dx", dx, want, t + UO[dtype] * (np.abs(want) + t))
    if dtype == "f32":
        x, _ = rows(rng, 37, 301)
        up, down = (P.mlmc_dropout(x + h * dy, 0.3, 5, 6, stream=7).double() for h in (1.0, -1.0))
        slope = P.mlmc_dropout(dy, 0.3, 5, 6, stream=7).double()
        off = ((up - down) / 2 - slope).abs()
        assert bool((off <= 8 * U * (x.abs() + dy.abs()).double() / 0.69).all())      # x +- dy is rounded, and each product
