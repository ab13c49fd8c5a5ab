"""Alternatives at temperatures below 1, of rows with one logit far above the others, flat ones and ordinary ones, in one launch and in two; tables with more places than there are alternatives.

The order of the alternatives does not depend on the temperature; their log probabilities are compared within the bounds of tests/test_gpu_logprobs.py."""
import numpy as np
import pytest
import torch

import paper_2507_05508_amd as P
from gpu_util import launched
from oracle import worker as O
from test_gpu_logprobs import forward_bounds
from test_gpu_worker import DT, U, f64, near

pytestmark = pytest.mark.gpu


def make(n, v, dtype):
    rng = np.random.default_rng(n + v)
    s = rng.normal(0, 2.5, (n, v)).astype(np.float32)
    for i in range(n):
        k = i % 4
        if k == 0:
            s[i, rng.integers(v)] += 20.0
        elif k == 1:
            s[i] *= 0.1
        elif k == 2:
            s[i, rng.integers(v, size=3)] += 12.0
    t = torch.from_numpy(s).to(DT[dtype]).cuda()
    return t, f64(t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temperature", [0.05, 0.2, 0.7])
@pytest.mark.parametrize("n,v", [(600, 5000), (4, 9000), (520, 15000), (520, 16390), (4, 33000), (4, 131072), (5, 262147)])
def test_alternatives_below_1(n, v, temperature, dtype):
    print(f"alternatives n={n} v={v} T={temperature} {dtype}", flush=True)
    logits, s = make(n, v, dtype)
    assert len(launched(lambda: P.mlmc_token_logprobs(logits, top=20))) == (2 if P.mlmc_token_logprobs_workspace(n, v, 20) and (dtype == "f32" or v > (32768 if n <= 512 else 16384)) else 1)
    m = min(n, 40)
    temperature = float(np.float32(temperature))
    log_p = (s[:m] - s[:m].max(1, keepdims=True)) / temperature
    log_p -= np.log(np.exp(log_p).sum(1, keepdims=True))
    t_s, t_h, _ = forward_bounds(s[:m], temperature, log_p)
    plain = P.mlmc_token_logprobs(logits, top=128)
    for top in (1, 20, 64, 128):
        got = P.mlmc_token_logprobs(logits, top=top, temperature=temperature, with_entropy=True)
        _, h, idx, val, _ = O.token_logprobs(s[:m], np.zeros((m, 0), int), top, temperature)
        assert np.array_equal(got.top_idx[:m].cpu().numpy(), idx)
        assert torch.equal(got.top_idx, plain.top_idx[:, :top])      # whatever the temperature
        near("top", got.top_logprob[:m], val, t_s[:, None] + 8 * U * np.abs(val))
        near("entropy", got.entropy[:m], h, t_h + U * np.abs(h))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v,top,barred", [(3, 2, 5, 0), (5, 64, 128, 0), (700, 100, 128, 0), (4, 9000, 128, 8950), (520, 16390, 64, 16380), (4, 140000, 128, 139900)])
def test_places_without_an_alternative(n, v, top, barred, dtype):
    """More places than a row has logits above -Inf: those that it has are compared, the others hold -1 and -Inf."""
    logits, _ = make(n, v, dtype)
    if barred:
        logits[:, torch.randperm(v, generator=torch.Generator().manual_seed(v))[:barred].cuda()] = -float("inf")
    m = min(n, 40)
    s = f64(logits[:m])
    got = P.mlmc_token_logprobs(logits, top=top)
    _, _, idx, val, _ = O.token_logprobs(s, np.zeros((m, 0), int), top, 1.0)
    assert np.array_equal(got.top_idx[:m].cpu().numpy(), idx)
    gone = idx < 0
    assert gone.sum() == m * (top - (v - barred)) and (f64(got.top_logprob[:m])[gone] == -np.inf).all()
    with np.errstate(invalid="ignore", divide="ignore"):
        log_p = s - s.max(1, keepdims=True)
        log_p -= np.log(np.exp(log_p).sum(1, keepdims=True))
        t_s, _, _ = forward_bounds(s, 1.0, log_p)
    there = np.where(gone, 0.0, val)
    near("top", torch.where(got.top_logprob[:m] == -float("inf"), 0.0, got.top_logprob[:m]), there, t_s[:, None] + 8 * U * np.abs(there))
