"""More of a worker's step next to the compression, and what its teacher answers with: root-mean-square norm with the residual's
addition and an output in 8 bits, matrices in 8 bits with a scale for every row and the product of two of them, dropout whose mask
is made again instead of stored, and log probabilities of given tokens with entropy and the top alternatives, which are the entries
that a student's distillation loss takes.

A case is one call.  `run` computes it in its plain form, elementary torch operations in 32 bits rounded once at the end, or,
where `own` is set, by the framework's entry points.  Eight bits are e4m3 (torch.float8_e4m3fn): an entry stands for its value times
the scale of its row.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ("none", "relu", "gelu")
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
LEAST_SCALE = 2.0 ** -100     # of a row of 8 bits: zeros and rows next to them
EPS = 1e-5
MOST_ROWS = 1 << 27           # rows x width of the largest norm, dropout and matrix to be rounded
MOST_PRODUCT = 1 << 37        # rows x outputs x inputs of the largest product
MOST_LOGITS = 1 << 28         # rows x vocabulary of the largest table of logits, in 16 bits; of 32-bit ones half


def _rms(name, rows, width, dtype="bf16", residual=True, eight=False, backward=False, grad_dtype="f32", pad=0):
    """residual: added to x before the norm, the sum is an output (in the backward pass: a gradient that comes to the sum by another
    way); eight: the normalised rows come in 8 bits; pad: entries between the end of a row and the next one's start."""
    return {"name": name, "op": "rms", "rows": rows, "width": width, "dtype": dtype, "residual": residual, "eight": eight,
            "backward": backward, "grad_dtype": grad_dtype, "pad": pad}


def _quantize(name, rows, width, dtype="bf16", pad=0):
    return {"name": name, "op": "quantize", "rows": rows, "width": width, "dtype": dtype, "pad": pad}


def _linear(name, rows, outputs, inputs, act="none", residual=False, pad=0):
    """Results and residual have 16 bits; pad: entries (of 8 bits) behind a row of x."""
    return {"name": name, "op": "linear_q8", "rows": rows, "outputs": outputs, "inputs": inputs, "dtype": "bf16", "act": act,
            "residual": residual, "pad": pad}


def _dropout(name, rows, width, p, dtype="bf16", residual=False, pad=0):
    """residual: added to what is kept.  Without it the call is the backward pass as well: the same mask on the gradient."""
    return {"name": name, "op": "dropout", "rows": rows, "width": width, "p": p, "dtype": dtype, "residual": residual, "pad": pad}


def _logprobs(name, rows, vocab, given, top, dtype="bf16", temperature=1.0, masked=0.0, barred=0.0, backward=False, entropy=True):
    """given: tokens of a row whose log probabilities are asked for; top: alternatives; masked: share of the rows without a token
    (padding); barred: share of the vocabulary that a row may not answer with (logits of -Inf); entropy: its gradient too."""
    return {"name": name, "op": "logprobs", "rows": rows, "vocab": vocab, "given": given, "top": top, "dtype": dtype,
            "temperature": temperature, "masked": masked, "barred": barred, "backward": backward, "entropy": entropy}


def listed():
    return [
        # a few sequences' next tokens: latency is the time
        _rms("rms_tokens", 4, 4096),
        # a teacher's batch: the norm in front of a product in 8 bits
        _rms("rms_eight", 8192, 4096, eight=True),
        # the largest: the gradient of wide fp32 rows of an odd width, cut from a wider buffer, the weight's into an fp32 row
        _rms("rms_backward_wide_f32", 16381, 8191, dtype="f32", backward=True, pad=5),
        # a layer's weight brought into 8 bits, as when a model is loaded or has been updated
        _quantize("quantize_weight", 4096, 4096),
        # fp32 rows of an odd width
        _quantize("quantize_ragged_f32", 1021, 5003, dtype="f32", pad=3),
        # one token through one layer: the weight is read once
        _linear("linear_q8_token", 1, 4096, 4096, residual=True),
        # a batch through the layer that widens
        _linear("linear_q8_batch", 8192, 4096, 4096, act="gelu"),
        # a training batch: a branch dropped and added to the stream that goes past it
        _dropout("dropout_residual", 8192, 4096, 0.1, residual=True),
        # the gradient of a small fp32 layer of odd sizes: the mask once more
        _dropout("dropout_ragged_f32", 1021, 4099, 0.25, dtype="f32", pad=5),
        # the next tokens of a few sequences with their alternatives: rows are fewer than the workgroups that the chip holds
        _logprobs("logprobs_few", 4, 131072, 1, 20),
        # a teacher's answers over a batch, the entries that a student learns from
        _logprobs("logprobs_teacher", 2048, 131072, 1, 64, masked=0.1),
        # the gradient of a batch's log probabilities with a term for the entropy
        _logprobs("logprobs_backward", 4096, 32768, 1, 0, masked=0.1, backward=True),
    ]


def _size(rng, lo, hi):
    """Spread over the logarithm; a third each multiples of 64, of 8, and any whole number."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    unit = rng.choice((64, 8, 1))
    return max(lo, min(hi, int(round(v / unit)) * unit)) if v >= 4 * unit else max(lo, min(hi, int(round(v))))


def draw(rng):
    op = rng.choice(("rms", "rms", "quantize", "linear_q8", "linear_q8", "dropout", "dropout", "logprobs", "logprobs", "logprobs"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    pad = rng.choice((0, 0, 5, 8))
    if op == "linear_q8":
        outputs, inputs = _size(rng, 128, 8192), _size(rng, 128, 8192)
        rows = _size(rng, 1, max(1, min(16384, MOST_PRODUCT // (outputs * inputs))))
        c = _linear("", rows, outputs, inputs, rng.choice(ACTS), rng.random() < 0.5, rng.choice((0, 0, 5, 16)))
    elif op == "logprobs":
        vocab = _size(rng, 1000, 262144)
        rows = _size(rng, 1, min(8192, MOST_LOGITS // vocab // (2 if dtype == "f32" else 1)))
        backward = rng.random() < 0.35
        c = _logprobs("", rows, vocab, rng.choice((1, 1, 1, 4, 7)), rng.choice((0, 5, 20, 64, 128)), dtype, rng.choice((1.0, 1.0, 2.0, 0.7)),
                      rng.choice((0.0, 0.1)), rng.choice((0.0, 0.0, 0.5)), backward, rng.random() < 0.6)
    else:
        width = _size(rng, 64, 16384)
        rows = _size(rng, 1, min(32768, MOST_ROWS // width))
        if op == "rms":
            backward = rng.random() < 0.4
            c = _rms("", rows, width, dtype, rng.random() < 0.7, not backward and rng.random() < 0.5, backward, rng.choice(("f32", "bf16")), pad)
        elif op == "quantize":
            c = _quantize("", rows, width, dtype, pad)
        else:
            c = _dropout("", rows, width, rng.choice((0.05, 0.1, 0.25, 0.5)), dtype, rng.random() < 0.5, pad)
    del c["name"]
    return c


def _normal(gen, rows, width, dtype, pad=0, std=1.0):
    """[rows][width] normal entries, cut from a buffer with `pad` entries more in a row."""
    t = torch.empty((rows, width + pad), dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen)
    return t.to(DTYPES[dtype])[:, :width]


def _normal_e4m3(gen, rows, width, std, pad=0):
    """Normal rows in 8 bits, as a file of weights has them: entries and the scale of every row, rows `pad` entries apart."""
    t = torch.empty((rows, width), dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen)
    scale = t.abs().amax(dim=1) / E4M3_MAX
    q = torch.empty((rows, width + pad), dtype=torch.uint8, device="cuda").view(E4M3)[:, :width]
    q.copy_((t / scale[:, None]).to(E4M3))
    return q, scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s, op = {"case": case}, case["op"]
    if op == "rms":
        n, d, dt, pad = case["rows"], case["width"], case["dtype"], case["pad"]
        s["weight"] = torch.empty(d, device="cuda").normal_(1.0, 0.2, generator=gen)
        s["x"] = _normal(gen, n, d, dt, pad, std=1.5)
        s["residual"] = None
        if case["backward"]:     # x is the sum that the forward pass has stored
            s["dy"] = _normal(gen, n, d, dt, pad, std=1e-3)
            if case["residual"]:
                s["residual"] = _normal(gen, n, d, dt, pad, std=1e-3)
            s["rstd"] = torch.rsqrt(s["x"].float().pow(2).mean(dim=1) + EPS)
            s["dweight"] = torch.zeros(d, dtype=DTYPES[case["grad_dtype"]], device="cuda")
        elif case["residual"]:
            s["residual"] = _normal(gen, n, d, dt, pad, std=4.0)
    elif op == "quantize":
        s["x"] = _normal(gen, case["rows"], case["width"], case["dtype"], case["pad"], std=0.02)
    elif op == "linear_q8":
        n, m, k = case["rows"], case["outputs"], case["inputs"]
        s["x"], s["x_scale"] = _normal_e4m3(gen, n, k, 1.0, case["pad"])
        s["weight"], s["weight_scale"] = _normal_e4m3(gen, m, k, k ** -0.5)
        s["bias"] = torch.empty(m, device="cuda").normal_(0.0, 0.1, generator=gen)
        s["residual"] = _normal(gen, n, m, case["dtype"]) if case["residual"] else None
    elif op == "dropout":
        s["x"] = _normal(gen, case["rows"], case["width"], case["dtype"], case["pad"])
        s["residual"] = _normal(gen, case["rows"], case["width"], case["dtype"], case["pad"], std=4.0) if case["residual"] else None
        s["seed"], s["step"], s["stream"] = seed * 0x9E3779B97F4A7C15 % (1 << 64), 1000 + seed % 100000, seed % 97
    else:
        n, v, given, top = case["rows"], case["vocab"], case["given"], case["top"]
        logits = torch.empty((n, v), dtype=torch.float32, device="cuda").normal_(0.0, 2.5, generator=gen)
        tokens = torch.randint(0, v, (n, given), device="cuda", generator=gen)
        logits.scatter_add_(1, tokens[:, :1], torch.full((n, 1), 8.0, device="cuda"))       # a likely token and others
        if case["barred"]:
            bar = torch.rand((n, v), device="cuda", generator=gen) < case["barred"]
            bar.scatter_(1, tokens[:, :1], False)
            logits.masked_fill_(bar, -math.inf)
        s["logits"] = logits.to(DTYPES[case["dtype"]])
        gone = torch.rand(n, device="cuda", generator=gen) < case["masked"]
        s["tokens"] = torch.where(gone[:, None], -1, tokens).to(torch.int32)
        if case["backward"]:
            z = s["logits"].float() / case["temperature"]
            log_p = torch.log_softmax(z, dim=1)
            h = torch.where(log_p > -math.inf, -log_p.exp() * log_p, 0.0).sum(dim=1)
            s["stats"] = torch.stack((s["logits"].float().max(dim=1).values, -log_p.max(dim=1).values, h), dim=1)  # greatest, log of the sum, entropy
            keep = (~gone).float()
            s["dlogprob"] = torch.empty((n, given), device="cuda").normal_(0.0, 1.0 / n, generator=gen) * keep[:, None]
            s["dentropy"] = torch.full((n,), 0.01 / n, device="cuda") * keep if case["entropy"] else None
            s["top_idx"] = s["dtop"] = None
            if top:
                s["top_idx"] = torch.topk(s["logits"], top, dim=1).indices.to(torch.int32)
                s["dtop"] = torch.empty((n, top), device="cuda").normal_(0.0, 0.1 / n, generator=gen) * keep[:, None]
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _to_eight(y):
    """Entries in 8 bits and the scale of every row."""
    scale = torch.clamp(y.abs().amax(dim=1) / E4M3_MAX, min=LEAST_SCALE)
    return (y / scale[:, None]).to(E4M3), scale


def _plain_rms(s, case):
    x, w, dt = s["x"].float(), s["weight"], s["x"].dtype
    if case["backward"]:
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        h = x * rstd
        c = dy * w
        dx = rstd * (c - h * (c * h).mean(dim=1, keepdim=True))
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        return {"dx": dx.to(dt), "dweight": (dy * h).sum(dim=0).to(s["dweight"].dtype)}
    out = {}
    if s["residual"] is not None:
        x = x + s["residual"].float()
        out["sum"] = x.to(dt)
    rstd = torch.rsqrt((x * x).mean(dim=1) + EPS)
    y = x * rstd[:, None] * w
    out["rstd"] = rstd
    if case["eight"]:
        out["q"], out["scale"] = _to_eight(y)
    else:
        out["y"] = y.to(dt)
    return out


def _plain_quantize(s, case):
    q, scale = _to_eight(s["x"].float())
    return {"q": q, "scale": scale}


def _plain_linear(s, case):
    z = (s["x"].float() @ s["weight"].float().t()) * (s["x_scale"][:, None] * s["weight_scale"]) + s["bias"]
    y = _act(z, case["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(DTYPES[case["dtype"]])}


LOW = 0xFFFFFFFF


def _philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 of counters and a key of 32-bit words (in 64-bit integers, whose products wrap): four tensors of words."""
    for r in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & LOW) ^ c1 ^ k0, b & LOW, ((a >> 32) & LOW) ^ c3 ^ k1, a & LOW
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    return c0, c1, c2, c3


def _plain_dropout(s, case):
    n, d = s["x"].shape
    group = torch.arange((d + 7) // 8, device="cuda")[None, :] + 1          # eight entries of a row have a counter
    row = torch.arange(n, device="cuda")[:, None]
    start = torch.zeros((n, group.shape[1]), dtype=torch.int64, device="cuda")
    words = torch.stack(_philox(start + s["step"], start + s["stream"], start + row, start + group, s["seed"] & LOW, s["seed"] >> 32), dim=-1)
    halves = torch.stack((words & 0xFFFF, words >> 16), dim=-1).reshape(n, -1)[:, :d]
    least = int(case["p"] * 65536 + 0.5)
    y = torch.where(halves >= least, s["x"].float() * (65536.0 / (65536 - least)), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(s["x"].dtype)}


def _plain_logprobs(s, case):
    n, v = s["logits"].shape
    temp, top = case["temperature"], case["top"]
    z = s["logits"].float() / temp
    live = s["tokens"] >= 0
    at = s["tokens"].clamp(min=0).long()
    if case["backward"]:
        log_p = z - s["stats"][:, :1] / temp - s["stats"][:, 1:2]
        p = torch.exp(log_p)
        g = torch.where(live, s["dlogprob"], 0.0)
        d = -p * g.sum(dim=1, keepdim=True)
        if s["dtop"] is not None:
            d = d - p * s["dtop"].sum(dim=1, keepdim=True)
            d = d.scatter_add(1, s["top_idx"].long(), s["dtop"])
        if s["dentropy"] is not None:
            d = d - s["dentropy"][:, None] * torch.where(p > 0, p * (log_p + s["stats"][:, 2:]), 0.0)
        return {"dlogits": (d.scatter_add(1, at, g) / temp).to(s["logits"].dtype)}
    z = z - z.max(dim=1, keepdim=True).values
    e = torch.exp(z)
    total = e.sum(dim=1, keepdim=True)
    log_p = z - torch.log(total)
    out = {"logprob": torch.where(live, log_p.gather(1, at), 0.0),
           "entropy": -torch.where(e > 0, e * log_p, 0.0).sum(dim=1) / total[:, 0]}
    if top:      # equal logits: the lowest index first, by keys of which no two are equal
        bits = (s["logits"].float() + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        key = order * (1 << 32) + (LOW - torch.arange(v, device="cuda"))
        idx = torch.topk(key, top, dim=1).indices
        val = log_p.gather(1, idx)
        out["top_idx"], out["top_logprob"] = torch.where(val > -math.inf, idx, -1).to(torch.int32), val
    return out


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _own(s, case):
    import paper_2507_05508_amd as P
    op = case["op"]
    if op == "rms":
        if case["backward"]:
            dx = P.mlmc_rms_norm_backward(s["dy"], s["x"], s["weight"], s["rstd"], s["dweight"], residual=s["residual"])
            return {"dx": dx, "dweight": s["dweight"]}
        r = P.mlmc_rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS, with_y=not case["eight"], with_q=case["eight"], with_rstd=True)
        out = {"rstd": r.rstd}
        if r.sum is not None:
            out["sum"] = r.sum
        return out | ({"q": r.q, "scale": r.scale} if case["eight"] else {"y": r.y})
    if op == "quantize":
        q, scale = P.mlmc_quantize(s["x"])
        return {"q": q, "scale": scale}
    if op == "linear_q8":
        act = {"none": P.MLMC_ACT_NONE, "relu": P.MLMC_ACT_RELU, "gelu": P.MLMC_ACT_GELU}[case["act"]]
        return {"y": P.mlmc_linear_q8(s["x"], s["x_scale"], s["weight"], s["weight_scale"], s["bias"], act=act, residual=s["residual"])}
    if op == "dropout":
        return {"y": P.mlmc_dropout(s["x"], case["p"], s["seed"], s["step"], stream=s["stream"], residual=s["residual"])}
    if case["backward"]:
        return {"dlogits": P.mlmc_token_logprobs_backward(s["logits"], s["stats"], s["tokens"], s["dlogprob"], top_idx=s["top_idx"], dtop=s["dtop"],
                                                          dentropy=s["dentropy"], temperature=case["temperature"])}
    r = P.mlmc_token_logprobs(s["logits"], s["tokens"], top=case["top"], temperature=case["temperature"], with_entropy=True)
    out = {"logprob": r.logprob, "entropy": r.entropy}
    return out | ({"top_idx": r.top_idx, "top_logprob": r.top_logprob} if case["top"] else {})


def run(state):
    case = state["case"]
    if own:
        return _own(state, case)
    return {"rms": _plain_rms, "quantize": _plain_quantize, "linear_q8": _plain_linear, "dropout": _plain_dropout,
            "logprobs": _plain_logprobs}[case["op"]](state, case)


def work(case):
    e, op = 2 if case["dtype"] == "bf16" else 4, case["op"]
    if op == "linear_q8":
        n, m, k = case["rows"], case["outputs"], case["inputs"]
        return {"bytes": n * k + m * k + (1 + case["residual"]) * n * m * e + 4 * (n + 2 * m), "flops": 2 * n * m * k}
    if op == "logprobs":
        n, v = case["rows"], case["vocab"]
        if case["backward"]:
            return {"bytes": 2 * n * v * e + n * (12 + 8 * case["given"] + 8 * case["top"] + 4 * case["entropy"]), "flops": 8 * n * v}
        return {"bytes": n * v * e + n * (8 * case["given"] + 4 + 8 * case["top"]), "flops": 6 * n * v}
    n, d = case["rows"], case["width"]
    if op == "rms":
        if case["backward"]:
            return {"bytes": (3 + case["residual"]) * n * d * e + 4 * n + 4 * d + d * (2 if case["grad_dtype"] == "bf16" else 4), "flops": 10 * n * d}
        read = (1 + 2 * case["residual"]) * n * d * e       # x, the residual, the sum
        return {"bytes": read + n * d * (1 if case["eight"] else e) + n * (8 if case["eight"] else 4) + 4 * d, "flops": 6 * n * d}
    if op == "quantize":
        return {"bytes": n * d * (e + 1) + 4 * n, "flops": 3 * n * d}
    return {"bytes": (2 + case["residual"]) * n * d * e, "flops": 25 * n * d}     # a generator's word takes 10 rounds of 10 operations


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _grid_e4m3(y):
    """The nearest value of three bits behind the point and exponents from -6 on, ties to even."""
    _, e = torch.frexp(y)
    step = torch.exp2((torch.clamp(e.double() - 1.0, min=-6.0) - 3.0))
    return torch.round(y / step) * step


def _eight_exact(y):
    scale = torch.maximum(y.abs().max(dim=1).values / 448.0, torch.full((), LEAST_SCALE, dtype=torch.float64, device="cuda"))
    return _grid_e4m3(y.div(scale[:, None])), scale


def _mul32(a, b):
    """High and low word of the product of 32-bit words, by halves: no partial product passes 2^63."""
    a1, a0, b1, b0 = a >> 16, a & 65535, b >> 16, b & 65535
    mid = a1 * b0 + (a0 * b0 >> 16)
    low_mid = (mid & 65535) + a0 * b1
    return a1 * b1 + (mid >> 16) + (low_mid >> 16), ((low_mid & 65535) << 16) + (a0 * b0 & 65535)


def _kept(n, d, least, seed, step, stream):
    blocks = -(-d // 8)
    i = torch.arange(n * blocks, device="cuda")
    state = [torch.full_like(i, step), torch.full_like(i, stream), i // blocks, i % blocks + 1]
    key = [seed % (1 << 32), seed // (1 << 32)]
    for _ in range(10):
        h0, l0 = _mul32(state[0], 0xD2511F53)
        h1, l1 = _mul32(state[2], 0xCD9E8D57)
        state = [h1 ^ state[1] ^ key[0], l1, h0 ^ state[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    kept = torch.empty((n * blocks, 8), dtype=torch.bool, device="cuda")
    for k in range(8):
        kept[:, k] = (state[k // 2] >> (16 * (k % 2))) % 65536 >= least
    return kept.view(n, blocks * 8)[:, :d]


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "quantize":
        q, scale = _eight_exact(s["x"].double())
        return {"q": q, "scale": scale}
    if op == "rms":
        x, w, d = s["x"].double(), s["weight"].double(), case["width"]
        rest = None if s["residual"] is None else s["residual"].double()
        if case["backward"]:
            dy, r = s["dy"].double(), s["rstd"].double()[:, None]
            dweight = (dy * x * r).sum(0)
            a = dy.mul_(w)
            slope = (a * x).sum(1, keepdim=True) / d
            dx = a.mul_(r).sub_(x.mul_(slope * r ** 3))
            return {"dx": dx if rest is None else dx.add_(rest), "dweight": dweight}
        out = {}
        if rest is not None:
            x = out["sum"] = x + rest
        r = 1.0 / torch.sqrt(x.pow(2).sum(1) / d + EPS)
        out["rstd"] = r
        y = x * w * r[:, None]
        if case["eight"]:
            out["q"], out["scale"] = _eight_exact(y)
        else:
            out["y"] = y
        return out
    if op == "linear_q8":
        x = s["x"].to(torch.float64) * s["x_scale"].double()[:, None]
        w = s["weight"].to(torch.float64) * s["weight_scale"].double()[:, None]
        z = torch.addmm(s["bias"].double(), x, w.t().contiguous())
        if case["act"] == "relu":
            z = torch.where(z > 0, z, 0.0)
        elif case["act"] == "gelu":
            z = z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
        return {"y": z if s["residual"] is None else z + s["residual"].double()}
    if op == "dropout":
        n, d = s["x"].shape
        least = math.floor(case["p"] * 65536 + 0.5)
        y = s["x"].double() * _kept(n, d, least, s["seed"], s["step"], s["stream"]) / (1.0 - least / 65536)
        return {"y": y if s["residual"] is None else y + s["residual"].double()}
    n, v, temp, top = case["rows"], case["vocab"], case["temperature"], case["top"]
    live, at = s["tokens"] >= 0, s["tokens"].long().clamp_min(0)
    if case["backward"]:
        greatest, log_sum, h = (c[:, None] for c in s["stats"].double().unbind(1))
        log_p = (s["logits"].double() - greatest) / temp - log_sum
        p = log_p.exp()
        g = s["dlogprob"].double() * live
        d = torch.zeros((n, v), dtype=torch.float64, device="cuda")
        rows = torch.arange(n, device="cuda")[:, None]
        d.index_put_((rows.expand_as(at), at), g, accumulate=True)
        total = g.sum(1, keepdim=True)
        if s["dtop"] is not None:
            idx = s["top_idx"].long()
            d.index_put_((rows.expand_as(idx), idx), s["dtop"].double(), accumulate=True)
            total = total + s["dtop"].double().sum(1, keepdim=True)
        d.sub_(p * total)
        if s["dentropy"] is not None:
            d.sub_(p * log_p.add_(h).clamp_min_(-1e300) * s["dentropy"].double()[:, None])
        return {"dlogits": d.div_(temp)}
    log_p = torch.log_softmax(s["logits"].double() / temp, dim=1)
    out = {"logprob": torch.where(live, log_p.gather(1, at), 0.0), "entropy": torch.special.entr(log_p.exp()).sum(1)}
    if top:
        idx = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True).indices[:, :top]
        val = log_p.gather(1, idx)
        out["top_idx"], out["top_logprob"] = torch.where(torch.isinf(val), -1, idx), val
    return out
