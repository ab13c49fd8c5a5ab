"""gelu in the epilogue of the linear layer of 8-bit matrices, entry by entry: small whole numbers and scales that are powers of two give what gelu is applied to exactly.

gelu's error with U = 2^-24, of 16-bit results: the tail of the normal distribution by formula 7.1.26 of Abramowitz and Stegun is off by 0.75e-7; its polynomial and reciprocal round by 8 U, the two
products and the exponential by 2 U of at most 1/2 each, the exponential's argument by z^2 U of the tail, which is below 0.2 U: 11 U in all, times |z|.  A rounding of fp32 for the last step and one for the residual, and
2^-8 for the 16-bit result."""
import pytest
import torch

import paper_2507_05508_amd as P
from gpu_util import launched
from test_gpu_linear_q8 import whole
from test_gpu_worker import U, out_like, untouched

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,m,k,pad,shift", [
    (1, 4096, 4096, 0, 0), (16, 100, 1000, 8, 0), (5, 33, 64, 0, 0), (40, 129, 130, 0, 0), (129, 257, 1023, 0, 0), (128, 128, 8192, 0, 0), (513, 1025, 2049, 0, 0), (1000, 640, 4096, 0, 4),
    (4096, 4096, 4096, 0, 0), (4000, 4001, 4112, 0, 0), (4000, 4002, 4111, 1, 0), (3841, 4090, 4224, 16, 0), (2049, 2305, 1025, 3, 1), (8190, 5000, 1920, 0, 0),
])
def test_gelu_by_entry(n, m, k, pad, shift):
    print(f"gelu n={n} m={m} k={k} pad={pad} shift={shift}", flush=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n + m + k)
    x, w = whole(gen, n, k, pad, shift), whole(gen, m, k, 0 if k % 2 else pad, shift)
    half = round(2 * k ** 0.5).bit_length()      # results of a few units: products have a mean square of 16
    xs, ws = (torch.exp2(torch.randint(-1, 2, (c,), device="cuda", generator=gen).float() - e) for c, e in ((n, half), (m, 0)))
    bias = torch.randint(-8, 9, (m,), device="cuda", generator=gen).float() / 8
    residual = (torch.randint(-16, 17, (n, m), device="cuda", generator=gen) / 8).to(torch.bfloat16)
    z = (x.to(torch.float64) @ w.to(torch.float64).t().contiguous()) * xs.double()[:, None] * ws.double() + bias.double()
    assert torch.equal(z, z.float().double())    # a number of fp32
    g = 0.5 * z * torch.erfc(-z / 2 ** 0.5)
    off = z.abs() * (0.75e-7 + 11 * U) + U * g.abs()
    for r in (None, residual):
        y, buf = out_like(n, m, "bf16", pad, shift)
        P.mlmc_linear_q8(x, xs, w, ws, bias, act=P.MLMC_ACT_GELU, residual=r, y=y)
        want = g if r is None else g + r.double()
        tol = off if r is None else off + U * want.abs()
        over = (y.double() - want).abs() - (tol + 2.0 ** -8 * (want.abs() + tol) + 2.0 ** -134)
        at = int(over.argmax())
        assert bool((over <= 0).all()), (float(over.max()), divmod(at, m), float(z.flatten()[at]), float(y.flatten()[at]))
        untouched(buf, y)
    if n * m >= 1 << 24 and k >= 4096:
        assert "k_linear_q8" in launched(lambda: P.mlmc_linear_q8(x, xs, w, ws, bias, act=P.MLMC_ACT_GELU))
