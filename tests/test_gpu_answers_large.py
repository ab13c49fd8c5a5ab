"""Root-mean-square norm, 8 bits, dropout and log probabilities where offsets pass 32 bits, and with more rows than a launch has: what the call gives the last rows is, bit for bit, what it gives them
alone, which the other tests compare with the definitions."""
import pytest
import torch

import paper_2507_05508_amd as P

pytestmark = pytest.mark.gpu


def big(n, d, dtype=torch.bfloat16, tail=3):
    """A matrix whose last `tail` rows alone are normal: the rest repeats one row."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n + d)
    t = torch.empty((n, d), dtype=dtype, device="cuda")
    t[:] = torch.empty(d, device="cuda").normal_(generator=gen).to(dtype)
    t[-tail:] = torch.empty((tail, d), device="cuda").normal_(generator=gen).to(dtype)
    return t


@pytest.mark.parametrize("n,d", [(270000, 16384), (2200000, 2048), (60000, 80000), (20000000, 4)])
def test_norm_quantize_dropout(n, d):
    """Over 2^32 entries in rows of registers and wide rows; more short rows than a launch has."""
    print(f"n={n} d={d}", flush=True)
    x = big(n, d)
    w = torch.ones(d, device="cuda")
    r = P.mlmc_rms_norm(x, w, with_q=True, with_rstd=True)
    s = P.mlmc_rms_norm(x[-3:], w, with_q=True, with_rstd=True)
    assert torch.equal(r.y[-3:], s.y) and torch.equal(r.q[-3:].view(torch.uint8), s.q.view(torch.uint8)) and torch.equal(r.scale[-3:], s.scale) and torch.equal(r.rstd[-3:], s.rstd)
    assert torch.equal(r.y[0], r.y[-4] if n > 4 else r.y[0])
    del r
    q, c = P.mlmc_quantize(x)
    q2, c2 = P.mlmc_quantize(x[-3:])
    assert torch.equal(q[-3:].view(torch.uint8), q2.view(torch.uint8)) and torch.equal(c[-3:], c2)
    del q
    y = P.mlmc_dropout(x, 0.3, 1, 2, stream=3)
    assert torch.equal(y[-3:], P.mlmc_dropout(x[-3:], 0.3, 1, 2, stream=3, row0=n - 3))
    del y
    rstd = torch.ones(n, device="cuda")
    dx = P.mlmc_rms_norm_backward(x, x, w, rstd, dx=None)
    assert torch.equal(dx[-3:], P.mlmc_rms_norm_backward(x[-3:], x[-3:], w, rstd[-3:]))


def test_log_probabilities():
    n, v = 40000, 131072      # 5.2e9 logits, more rows than a launch
    x = big(n, v)
    tokens = torch.full((n, 1), v - 1, dtype=torch.int32, device="cuda")
    r = P.mlmc_token_logprobs(x, tokens, top=9, with_entropy=True, with_stats=True)
    s = P.mlmc_token_logprobs(x[-3:], tokens[-3:], top=9, with_entropy=True, with_stats=True)
    for a, b in zip(r, s):
        assert torch.equal(a[-3:], b)
    assert bool((r.top_idx[:-3] == r.top_idx[0]).all())
    g = torch.ones((n, 1), device="cuda")
    last = x[-3:].clone()
    d = P.mlmc_token_logprobs_backward(x, r.stats, tokens, g, dlogits=x)
    assert torch.equal(d[-3:], P.mlmc_token_logprobs_backward(last, s.stats, tokens[-3:], g[-3:]))
    assert torch.equal(d[0], d[-4])


def test_many_short_rows_of_log_probabilities():
    x = big(1000000, 7, torch.float32)
    r = P.mlmc_token_logprobs(x, top=2, with_entropy=True)
    s = P.mlmc_token_logprobs(x[-3:], top=2, with_entropy=True)
    assert torch.equal(r.top_idx[-3:], s.top_idx) and torch.equal(r.entropy[-3:], s.entropy) and bool((r.top_idx[:-3] == r.top_idx[0]).all())


@pytest.mark.parametrize("n,m,k", [(1200000, 64, 4096), (1100000, 4096, 64), (40000, 1 << 17, 32)])
def test_linear_q8(n, m, k):
    """Operands and results past 2^32 entries: small whole numbers, whose sums are exact in any order."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.zeros((n, k), dtype=torch.float8_e4m3fn, device="cuda")
    x[-5:] = torch.randint(-3, 4, (5, k), device="cuda", generator=gen).to(torch.float8_e4m3fn)
    x[0] = x[-1]
    w = torch.randint(-3, 4, (m, k), device="cuda", generator=gen).to(torch.float8_e4m3fn)
    one, ones = torch.ones(n, device="cuda"), torch.ones(m, device="cuda")
    y = P.mlmc_linear_q8(x, one, w, ones)
    assert torch.equal(y[-5:], P.mlmc_linear_q8(x[-5:], one[-5:], w, ones)) and torch.equal(y[0], y[-1]) and not bool(y[1:-5].any())
