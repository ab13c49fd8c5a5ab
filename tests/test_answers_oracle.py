"""The definitions of oracle/worker.py for root-mean-square norm, 8 bits, dropout and log probabilities: against differences of their own forward direction, and against closed forms."""
import math

import numpy as np
import pytest
import torch

from oracle import worker as O
from test_worker_oracle import close, differences


def test_rms_norm_gradient_is_the_slope():
    rng = np.random.default_rng(0)
    s, w, r = rng.normal(0.2, 1.0, (3, 7)), rng.normal(1, 0.2, 7), rng.normal(0, 1, (3, 7))
    f = lambda: float((O.rms_norm(s, w, 1e-5)[0] * r).sum())  # noqa: E731
    ds, dw = O.rms_norm_backward(r, s, w, O.rms_norm(s, w, 1e-5)[1])
    close(ds, differences(f, s))
    close(dw, differences(f, w))
    other = rng.normal(0, 1, (3, 7))
    close(O.rms_norm_backward(r, s, w, O.rms_norm(s, w, 1e-5)[1], other)[0], ds + other)


def test_rms_norm_of_equal_entries():
    y, rstd = O.rms_norm(np.full((2, 5), 3.0), None, 0.0)
    assert np.allclose(y, 1.0, atol=1e-15) and np.allclose(rstd, 1 / 3, atol=1e-15)


def test_e4m3_is_torchs():
    """Every value, the middles between neighbours (ties) and what lies next to them."""
    v = O.E4M3
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20), -mid, [448.0]])
    assert np.array_equal(O.e4m3(x), torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy())
    assert np.isnan(O.e4m3(np.array([np.nan]))).all()


def test_quantize():
    q, scale = O.quantize(np.array([[448.0, -1.0, 0.0], [0.0, 0.0, 0.0], [1.0, np.inf, 2.0], [np.nan, 1.0, 1.0]]))
    assert np.array_equal(q[0], [448.0, -1.0, 0.0]) and scale[0] == 1.0 and scale[1] == 2.0 ** -100 and (q[1] == 0).all()
    assert np.isnan(q[2:]).all() and np.isnan(scale[2:]).all()


def test_dropout_keeps_its_share_and_nothing_else():
    keep = O.dropout_keep(40, 203, 16384, seed=7 << 33 | 5, step=3, stream=9)     # a quarter dropped
    assert abs(keep.mean() - 0.75) < 5 * math.sqrt(0.75 * 0.25 / keep.size)
    assert np.array_equal(O.dropout_keep(7, 203, 16384, 7 << 33 | 5, 3, 9, row0=33), keep[33:])      # a part of the rows
    assert np.array_equal(O.dropout_keep(40, 17, 16384, 7 << 33 | 5, 3, 9), keep[:, :17])
    for other in (dict(seed=5), dict(step=4), dict(stream=8)):
        assert not np.array_equal(O.dropout_keep(40, 203, 16384, **{**dict(seed=7 << 33 | 5, step=3, stream=9), **other}), keep)
    x = np.arange(1.0, 8121.0).reshape(40, 203)
    y = O.dropout(x, 0.25, 7 << 33 | 5, 3, 9, residual=-x)
    assert np.allclose(y, np.where(keep, x / 0.75, 0.0) - x)
    assert O.dropout_keep(3, 9, 0, 1, 2, 3).all()


@pytest.mark.parametrize("temperature", [1.0, 2.0])
def test_log_probabilities_gradient_is_the_slope(temperature):
    rng = np.random.default_rng(3)
    s = rng.normal(0, 2, (3, 6))
    tokens = np.array([[1, 1, -1], [5, 0, 7], [-1, -1, -1]])
    g, h = rng.normal(0, 1, (3, 3)), np.array([0.3, 0.0, -0.2])
    top_idx = O.token_logprobs(s, tokens, 2, temperature)[2]
    a = rng.normal(0, 1, (3, 2))

    def f():
        logprob, entropy, _, top_logprob, _ = O.token_logprobs(s, np.where(tokens == 7, -1, tokens), 2, temperature)
        return float((logprob * g).sum() + (entropy * h).sum() + (top_logprob * a).sum())
    close(O.token_logprobs_backward(s, tokens, g, top_idx, a, h, temperature), differences(f, s))


def test_log_probabilities():
    logits = np.array([[0.0, 0.0, 0.0, 0.0], [-math.inf, 2.0, 2.0, -math.inf], [-math.inf] * 4, [1.0, math.nan, 0.0, 0.0], [0.0, math.inf, 0.0, 0.0]])
    logprob, h, idx, top, stats = O.token_logprobs(logits, np.array([[2, -1, 4]] * 5), 3, 1.0)
    assert np.allclose(logprob[0, :2], [-math.log(4), 0.0]) and np.isnan(logprob[0, 2]) and np.isclose(h[0], math.log(4))
    assert list(idx[0]) == [0, 1, 2] and list(idx[1]) == [1, 2, -1] and top[1, 2] == -math.inf and np.isclose(h[1], math.log(2))
    assert (idx[2:] == -1).all() and np.isnan(top[2:]).all() and np.isnan(h[2:]).all() and (logprob[:, 1] == 0).all()
