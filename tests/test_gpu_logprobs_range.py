"""Log probabilities of logits as large as their type has them, at temperatures as large, against the definitions in 64 bits: differences of logits pass the range of fp32, and over the temperature they are
ordinary numbers.

Bounds as in tests/test_gpu_logprobs.py, U = 2^-24: an argument of the exponential is off by A U |x| (difference, scaling, and the rounding of 1 / T, which is at most 4 U where it is subnormal: 6 U in all),
the exponential by 2 U more; log S by 302 U + A U E|x| + 2 U, a log probability by that and (A + 2) U |x| + U |log p|, the entropy by log S's times 1 + E|x|, A U (E|x| + E x^2) and 305 U E|x|."""
import numpy as np
import pytest
import torch

import paper_2507_05508_amd as P
from oracle import worker as O
from test_gpu_worker import DT, U, UO, f64, near

pytestmark = pytest.mark.gpu
A = 6


def make(v, dtype, seed):
    rng = np.random.default_rng(seed)
    s = rng.uniform(-3.3e38, 3.3e38, (6, v))
    s[1, :] = -3.3e38
    s[1, v // 2] = 3.3e38                # all of the row as far below as there is
    s[2] = np.where(np.arange(v) % 3 == 0, -3.3e38, 2.5e38)
    s[3] = rng.normal(0, 3, v)           # nothing of the kind
    s[4] = rng.uniform(-3.3e38, 0.0, v)
    s[4, 0] = 2e31                       # a greatest logit that is far from the range itself, and the lowest there is
    s[4, 1] = -3.4028234663852886e38 if dtype == "f32" else -3.3895313892515355e38
    s[5, ::2] = -np.inf
    t = torch.from_numpy(s.astype(np.float32)).to(DT[dtype]).cuda()
    return rng, t, f64(t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temperature", [2.5e37, 1e38, 3.4e38])
@pytest.mark.parametrize("v", [2, 7, 700, 9000, 16390, 33000, 140000])
def test_differences_past_the_range(v, temperature, dtype):
    print(f"differences past the range v={v} T={temperature} {dtype}", flush=True)
    rng, logits, s = make(v, dtype, v)
    temperature = float(np.float32(temperature))
    tokens = np.stack([np.full(6, 0), np.full(6, v - 1), np.full(6, v // 2), rng.integers(0, v, 6)], 1)
    top = min(9, v)
    for rows in (6, 600):      # the same rows often enough for the other way
        if rows == 600 and not (8192 < v < 40000):
            continue
        big = logits.repeat(rows // 6, 1)
        got = P.mlmc_token_logprobs(big, torch.from_numpy(tokens).int().cuda().repeat(rows // 6, 1), top=top, temperature=temperature, with_entropy=True, with_stats=True)
        want, h, idx, val, stats = O.token_logprobs(s, tokens, top, temperature)
        x = np.abs((s - s.max(1, keepdims=True)) / temperature)
        p = np.exp(-x) / np.exp(-x).sum(1, keepdims=True)
        live = np.where(p > 0, x, 0.0)
        ex, exx = (p * live).sum(1), (p * live * live).sum(1)
        t_s = 1.01 * U * (304 + A * ex)
        t_h = 1.01 * (t_s * (1 + ex) + U * (A * (ex + exx) + 305 * ex) + 4 * U * (1 + ex))

        def bound(log_p):
            return np.where(np.isfinite(log_p), t_s[:, None] + (A + 3) * U * np.abs(np.where(np.isfinite(log_p), log_p, 0.0)), 0.0)

        def close(name, have, need):
            have = f64(have)[-6:]
            gone = np.isinf(need)
            assert np.array_equal(np.isinf(have), gone), name
            near(name, torch.from_numpy(np.where(gone, 0.0, have)), np.where(gone, 0.0, need), bound(need))
        close("logprob", got.logprob, want)
        close("top", got.top_logprob, val)
        assert np.array_equal(got.top_idx[-6:].cpu().numpy(), idx)
        near("entropy", got.entropy[-6:], h, t_h)
        # the gradient, of sizes that fp32 has after the division by the temperature
        g, e = (rng.normal(0, 1e37, tokens.shape)).astype(np.float32), (rng.normal(0, 1e37, 6)).astype(np.float32)
        grad = P.mlmc_token_logprobs_backward(logits, got.stats[-6:].contiguous(), torch.from_numpy(tokens).int().cuda(), torch.from_numpy(g).cuda(),
                                              dentropy=torch.from_numpy(e).cuda(), temperature=temperature)
        need = O.token_logprobs_backward(s, tokens, g.astype(np.float64), None, None, e, temperature)
        log_p = -x - np.log(np.exp(-x).sum(1, keepdims=True))
        far = np.where(p > 0, x, 0.0)
        apart = np.abs(np.where(p > 0, log_p, 0.0) + h[:, None])
        rel = t_s[:, None] + U * (A * far + 8)
        weights = np.abs(g.astype(np.float64)).sum(1, keepdims=True) / temperature
        hm = np.abs(e.astype(np.float64))[:, None] / temperature
        tol = p * (weights * (rel + 20 * U) + hm * (apart * (rel + 10 * U) + t_s[:, None] + t_h[:, None] + U * (A * far + np.abs(h)[:, None] + 8)))
        hit = np.zeros_like(s)
        for k in range(tokens.shape[1]):
            hit[np.arange(6), tokens[:, k]] += np.abs(g[:, k].astype(np.float64)) / temperature
        tol = 1.01 * (tol + 12 * U * hit + 6 * U * np.abs(need))
        near("dlogits", grad, need, tol + UO[dtype] * (np.abs(need) + tol))


def test_the_smallest_temperatures():
    """A temperature at which nothing but the greatest logit counts, where twice its inverse is no number of fp32."""
    s = torch.tensor([[3e38, -3e38, 3e38, 1.0], [0.0, 1e-38, 2e-38, -1e-38]], device="cuda")
    t = 5e-39
    r = P.mlmc_token_logprobs(s, top=4, temperature=t, with_entropy=True)
    assert r.top_idx.tolist() == [[0, 2, 3, 1], [2, 1, 0, 3]]
    assert np.allclose(f64(r.top_logprob[0, :2]), -np.log(2), atol=1e-6) and bool((r.top_logprob[0, 2:] == -float("inf")).all()) and abs(float(r.entropy[0]) - np.log(2)) < 1e-6
    want = O.token_logprobs(f64(s), np.zeros((2, 0), int), 4, float(np.float32(t)))
    # subnormal logits and their differences have 2^-149 to the step, 1 / T 24 bits: |x| up to 6 is off by 6 2^-149 / 2e-38 and a few roundings
    assert (np.abs(f64(r.top_logprob[1]) - want[3][1]) <= 1e-6 * 6 + 304 * U).all()
