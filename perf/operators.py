"""The work of one worker's training step next to the compression: layer norm, the matrix product with bias, activation and
residual in its epilogue, and the distillation loss from a teacher's top logits, each in its directions.

A case is one call.  `run` computes it in its plain form, elementary torch operations in 32 bits rounded once at the end, or,
where `own` is set, by the framework's entry points.  Weight gradients are written where a worker keeps them: into its row
of the gradient matrix that the compression reads, at the tensor's place in it.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ("none", "relu", "gelu")
MOST_NORM = 1 << 27           # rows x width of the largest norm
MOST_PRODUCT = 1 << 37        # rows x outputs x inputs of the largest product of 16-bit entries; of 32-bit ones a 32nd
MOST_LOGITS = 1 << 27         # rows x vocabulary of the largest loss


def _norm(name, rows, width, dtype="bf16", grad_dtype="f32", backward=False, pad=0):
    """pad: entries between the end of a row and the next one's start."""
    return {"name": name, "op": "norm", "rows": rows, "width": width, "dtype": dtype, "grad_dtype": grad_dtype,
            "backward": backward, "pad": pad}


def _linear(name, rows, outputs, inputs, dtype="bf16", part="forward", act="none", residual=False, grad_dtype="f32", pad=0, place=0):
    """part: forward, dgrad (gradient of the input) or wgrad (of weight and bias); place: where the weight's gradient
    begins in the worker's row."""
    return {"name": name, "op": "linear", "rows": rows, "outputs": outputs, "inputs": inputs, "dtype": dtype, "part": part,
            "act": act, "residual": residual, "grad_dtype": grad_dtype, "pad": pad, "place": place}


def _distill(name, rows, vocab, top, dtype="bf16", temperature=1.0, masked=0.0, grad=True):
    """top: entries of a row's teacher; masked: share of the rows that have no teacher (padding tokens); grad: with the
    gradient, as in training, or the loss alone."""
    return {"name": name, "op": "distill", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "temperature": temperature,
            "masked": masked, "grad": grad}


def listed():
    return [
        # a few sequences' next tokens: latency is the time
        _norm("norm_tokens", 4, 4096),
        # the activations of a training batch, forward
        _norm("norm_forward", 16384, 1024),
        # the same batch's backward pass, the weight's gradient into an fp32 row
        _norm("norm_backward", 16384, 1024, backward=True),
        # the largest: wide fp32 rows, of an odd width, cut from a wider buffer
        _norm("norm_backward_wide_f32", 16381, 8191, dtype="f32", backward=True, pad=5),
        # one token through one layer: the weight is read once
        _linear("linear_token", 1, 4096, 4096, residual=True),
        # a training batch through the layer that widens, activation in the epilogue
        _linear("linear_forward", 8192, 4096, 4096, act="gelu"),
        # its gradient with respect to the input, through the activation before it; a ragged number of rows
        _linear("linear_dgrad", 4001, 4096, 4096, part="dgrad", act="gelu"),
        # its gradient with respect to weight and bias, at an odd place of the worker's row
        _linear("linear_wgrad", 8192, 4096, 1024, part="wgrad", place=4097),
        # a small fp32 layer of odd sizes
        _linear("linear_ragged_f32", 1000, 2049, 1537, dtype="f32", act="relu", residual=True, pad=3),
        # a few rows of a large vocabulary: rows are fewer than the workgroups that the chip holds
        _distill("distill_few_rows", 4, 131072, 64, temperature=2.0),
        # a training batch
        _distill("distill_train", 4096, 32768, 32, temperature=2.0, masked=0.1),
        # an odd vocabulary in fp32
        _distill("distill_ragged_f32", 1021, 50021, 100, dtype="f32", masked=0.1),
    ]


def _size(rng, lo, hi):
    """Spread over the logarithm; a third each multiples of 64, of 8, and any whole number."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    unit = rng.choice((64, 8, 1))
    return max(lo, min(hi, int(round(v / unit)) * unit)) if v >= 4 * unit else max(lo, min(hi, int(round(v))))


def draw(rng):
    op = rng.choice(("norm", "norm", "linear", "linear", "linear", "distill", "distill"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "norm":
        width = _size(rng, 64, 16384)
        rows = _size(rng, 1, min(32768, MOST_NORM // width))
        c = _norm("", rows, width, dtype, rng.choice(("f32", "bf16")), rng.random() < 0.6, rng.choice((0, 0, 5, 8)))
    elif op == "linear":
        outputs, inputs = _size(rng, 128, 8192), _size(rng, 128, 8192)
        most = MOST_PRODUCT if dtype == "bf16" else MOST_PRODUCT // 32
        rows = _size(rng, 1, max(1, min(16384, most // (outputs * inputs))))
        part = rng.choice(("forward", "forward", "dgrad", "wgrad"))
        c = _linear("", rows, outputs, inputs, dtype, part, "none" if part == "wgrad" else rng.choice(ACTS),
                    part != "wgrad" and rng.random() < 0.5, rng.choice(("f32", "bf16")), rng.choice((0, 0, 3, 8)),
                    rng.choice((0, 8, 4097)) if part == "wgrad" else 0)
    else:
        vocab = _size(rng, 1000, 262144)
        rows = _size(rng, 1, min(8192, MOST_LOGITS // vocab // (2 if dtype == "f32" else 1)))
        c = _distill("", rows, vocab, _size(rng, 1, 256), dtype, rng.choice((1.0, 2.0, 4.0)), rng.choice((0.0, 0.1)), rng.random() < 0.8)
    del c["name"]
    return c


def _rows(gen, rows, width, dtype, pad, std=1.0, mean=0.0):
    """[rows][width] normal entries, cut from a buffer with `pad` entries more in a row."""
    t = torch.empty((rows, width + pad), dtype=torch.float32, device="cuda")
    t.normal_(mean, std, generator=gen)
    return t.to(DTYPES[dtype])[:, :width]


def _gradient_row(count, place, dtype):
    """A worker's row of the gradient matrix; the tensors of the case begin at `place`."""
    return torch.zeros(place + count, dtype=DTYPES[dtype], device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    if case["op"] == "norm":
        n, d = case["rows"], case["width"]
        s["x"] = _rows(gen, n, d, case["dtype"], case["pad"], std=1.5, mean=0.3)
        s["weight"] = torch.empty(d, device="cuda").normal_(1.0, 0.2, generator=gen)
        s["bias"] = torch.empty(d, device="cuda").normal_(0.0, 0.2, generator=gen)
        if case["backward"]:
            s["dy"] = _rows(gen, n, d, case["dtype"], case["pad"], std=1e-3)
            x = s["x"].float()
            var, mean = torch.var_mean(x, dim=1, unbiased=False)
            s["stats"] = torch.stack((mean, (var + 1e-5).rsqrt()), dim=1)
            row = _gradient_row(2 * d, 0, case["grad_dtype"])
            s["dweight"], s["dbias"] = row[:d], row[d:]
    elif case["op"] == "linear":
        n, m, k, dt, pad = case["rows"], case["outputs"], case["inputs"], case["dtype"], case["pad"]
        if case["part"] != "wgrad":
            s["weight"] = _rows(gen, m, k, dt, 0, std=k ** -0.5)
        if case["part"] == "forward":
            s["x"] = _rows(gen, n, k, dt, pad)
            s["bias"] = torch.empty(m, device="cuda").normal_(0.0, 0.1, generator=gen)
            s["residual"] = _rows(gen, n, m, dt, pad) if case["residual"] else None
            if case["act"] != "none":
                s["z"] = torch.empty((n, m), dtype=DTYPES[dt], device="cuda")
        elif case["part"] == "dgrad":
            s["dy"] = _rows(gen, n, m, dt, pad, std=1e-3)
            s["z"] = _rows(gen, n, k, dt, pad) if case["act"] != "none" else None
            s["residual"] = _rows(gen, n, k, dt, pad, std=1e-3) if case["residual"] else None
        else:
            s["dy"] = _rows(gen, n, m, dt, pad, std=1e-3)
            s["x"] = _rows(gen, n, k, dt, pad)
            row = _gradient_row(m * k + m, case["place"], case["grad_dtype"])[case["place"]:]
            s["dweight"], s["dbias"] = row[:m * k].view(m, k), row[m * k:]
    else:
        n, v, top = case["rows"], case["vocab"], case["top"]
        teacher = _rows(gen, n, v, "f32", 0, std=2.0)
        logits = teacher * 0.7
        logits += _rows(gen, n, v, "f32", 0, std=1.0)
        s["logits"] = logits.to(DTYPES[case["dtype"]])
        s["t_val"], at = torch.topk(teacher, top, dim=1)
        masked = torch.rand(n, device="cuda", generator=gen) < case["masked"]
        s["t_idx"] = torch.where(masked[:, None], -1, at).to(torch.int32)
        s["scale"] = 1.0 / n
    return s


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_norm(s, case):
    x, w = s["x"].float(), s["weight"]
    if not case["backward"]:
        mean = x.mean(dim=1, keepdim=True)
        x = x - mean
        rstd = torch.rsqrt((x * x).mean(dim=1, keepdim=True) + 1e-5)
        y = x * rstd * w + s["bias"]
        return {"y": y.to(s["x"].dtype), "stats": torch.cat((mean, rstd), dim=1)}
    dy = s["dy"].float()
    mean, rstd = s["stats"][:, :1], s["stats"][:, 1:]
    xh = (x - mean) * rstd
    c = dy * w
    dx = rstd * (c - c.mean(dim=1, keepdim=True) - xh * (c * xh).mean(dim=1, keepdim=True))
    g = s["dweight"].dtype
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xh).sum(dim=0).to(g), "dbias": dy.sum(dim=0).to(g)}


def _plain_linear(s, case):
    act = case["act"]
    if case["part"] == "forward":
        z = s["x"].float() @ s["weight"].float().t() + s["bias"]
        y = _act(z, act)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        out = {"y": y.to(s["x"].dtype)}
        if act != "none":
            out["z"] = z.to(s["x"].dtype)
        return out
    dy = s["dy"].float()
    if case["part"] == "dgrad":
        dx = dy @ s["weight"].float()
        if act != "none":
            dx = dx * _act_slope(s["z"].float(), act)
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        return {"dx": dx.to(s["dy"].dtype)}
    g = s["dweight"].dtype
    return {"dweight": (dy.t() @ s["x"].float()).to(g), "dbias": dy.sum(dim=0).to(g)}


def _plain_distill(s, case):
    temp, scale = case["temperature"], s["scale"]
    z = s["logits"].float() / temp
    here = s["t_idx"] >= 0
    live = here.any(dim=1, keepdim=True)
    at = s["t_idx"].clamp(min=0).long()
    t = torch.where(here, s["t_val"] / temp, -math.inf)
    t = torch.where(live, t - t.max(dim=1, keepdim=True).values, 0.0)
    e = torch.where(here, torch.exp(t), 0.0)
    total = torch.where(live, e.sum(dim=1, keepdim=True), 1.0)
    q = e / total
    log_q = t - torch.log(total)
    z = z - z.max(dim=1, keepdim=True).values
    ez = torch.exp(z)
    sum_z = ez.sum(dim=1, keepdim=True)
    log_p = z.gather(1, at) - torch.log(sum_z)
    loss = temp * temp * torch.where(q > 0, q * (log_q - log_p), 0.0).sum(dim=1)
    if not case["grad"]:
        return {"loss": loss}
    d = torch.where(live, ez / sum_z, 0.0)
    d = d.scatter_add(1, at, -q) * (temp * scale)
    return {"loss": loss, "dlogits": d.to(s["logits"].dtype)}


def _own(s, case):
    import paper_2507_05508_amd as P
    if case["op"] == "norm":
        if not case["backward"]:
            y, stats = P.mlmc_layer_norm(s["x"], s["weight"], s["bias"], eps=1e-5, with_stats=True)
            return {"y": y, "stats": stats}
        dx = P.mlmc_layer_norm_backward(s["dy"], s["x"], s["weight"], s["stats"], s["dweight"], s["dbias"])
        return {"dx": dx, "dweight": s["dweight"], "dbias": s["dbias"]}
    if case["op"] == "linear":
        act = {"none": P.MLMC_ACT_NONE, "relu": P.MLMC_ACT_RELU, "gelu": P.MLMC_ACT_GELU}[case["act"]]
        if case["part"] == "forward":
            z = s.get("z")
            y = P.mlmc_linear(s["x"], s["weight"], s["bias"], act=act, residual=s["residual"], z=z)
            return {"y": y} if z is None else {"y": y, "z": z}
        if case["part"] == "dgrad":
            return {"dx": P.mlmc_linear_dgrad(s["dy"], s["weight"], act=act, z=s["z"], residual=s["residual"])}
        P.mlmc_linear_wgrad(s["dy"], s["x"], s["dweight"], s["dbias"])
        return {"dweight": s["dweight"], "dbias": s["dbias"]}
    loss, dlogits = P.mlmc_distill(s["logits"], s["t_idx"], s["t_val"], temperature=case["temperature"], scale=s["scale"],
                                   grad=case["grad"])
    return {"loss": loss} if dlogits is None else {"loss": loss, "dlogits": dlogits}


def run(state):
    case = state["case"]
    if own:
        return _own(state, case)
    return {"norm": _plain_norm, "linear": _plain_linear, "distill": _plain_distill}[case["op"]](state, case)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    g = 2 if case.get("grad_dtype") == "bf16" else 4
    if case["op"] == "norm":
        n, d = case["rows"], case["width"]
        if case["backward"]:
            return {"bytes": 3 * n * d * e + 8 * n + 4 * d + 2 * d * g, "flops": 14 * n * d}
        return {"bytes": 2 * n * d * e + 8 * n + 8 * d, "flops": 8 * n * d}
    if case["op"] == "linear":
        n, m, k = case["rows"], case["outputs"], case["inputs"]
        more = (case["act"] != "none") + case["residual"]
        if case["part"] == "forward":
            b = (n * k + m * k + (1 + more) * n * m) * e + 4 * m
        elif case["part"] == "dgrad":
            b = (n * m + m * k + (1 + more) * n * k) * e
        else:
            b = (n * m + n * k) * e + (m * k + m) * g
        return {"bytes": b, "flops": 2 * n * m * k}
    n, v, top = case["rows"], case["vocab"], case["top"]
    return {"bytes": n * v * e * (2 if case["grad"] else 1) + n * (8 * top + 4), "flops": (8 if case["grad"] else 4) * n * v}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x, w, n = s["x"].double(), s["weight"].double(), case["width"]
        if not case["backward"]:
            mean = x.sum(1) / n
            x = x.sub_(mean[:, None])
            rstd = 1.0 / torch.sqrt(x.pow(2).sum(1) / n + 1e-5)
            return {"y": torch.addcmul(s["bias"].double(), x.mul_(rstd[:, None]), w), "stats": torch.stack((mean, rstd), 1)}
        mean, rstd = s["stats"].double().unbind(1)
        xh = x.sub_(mean[:, None]).mul_(rstd[:, None])
        dy = s["dy"].double()
        dweight, dbias = (dy * xh).sum(0), dy.sum(0)
        a = dy.mul_(w)
        a_mean = a.sum(1) / n
        slope = (a * xh).sum(1) / n
        a = a.sub_(a_mean[:, None]).sub_(xh.mul_(slope[:, None])).mul_(rstd[:, None])
        return {"dx": a, "dweight": dweight, "dbias": dbias}
    if case["op"] == "linear":
        if case["part"] == "wgrad":
            dy = s["dy"].double()
            return {"dweight": torch.matmul(dy.t().contiguous(), s["x"].double()), "dbias": dy.sum(0)}
        name = "x" if case["part"] == "forward" else "dy"
        weight = s["weight"].double()
        z = torch.matmul(s[name].double(), weight.t().contiguous() if name == "x" else weight)
        rest = 0.0 if s["residual"] is None else s["residual"].double()
        half_up = math.sqrt(2.0)
        if name == "x":
            z = z + s["bias"].double()
            if case["act"] == "none":
                return {"y": z + rest}
            gate = (z > 0).double() if case["act"] == "relu" else 0.5 * torch.erfc(-z / half_up)
            return {"y": z * gate + rest, "z": z}
        if case["act"] == "relu":
            z = z * (s["z"] > 0).double()
        elif case["act"] == "gelu":
            u = s["z"].double()
            z = z * (0.5 * torch.erfc(-u / half_up) + u * torch.exp(-u * u / 2.0) / math.sqrt(2.0 * math.pi))
        return {"dx": z + rest}
    temp, n = case["temperature"], case["rows"]
    log_p = torch.log_softmax(s["logits"].double() / temp, dim=1)
    live = s["t_idx"][:, 0] >= 0
    at = s["t_idx"].long() * live[:, None]
    log_q = torch.log_softmax(s["t_val"].double() / temp, dim=1)
    q = torch.exp(log_q) * live[:, None]
    loss = temp ** 2 * (q * (log_q - torch.gather(log_p, 1, at))).sum(1)
    if not case["grad"]:
        return {"loss": loss}
    d = torch.exp(log_p) * live[:, None]
    rows = torch.arange(n, device="cuda")[:, None].expand_as(at)
    d.index_put_((rows, at), -q, accumulate=True)
    return {"loss": loss, "dlogits": d * (temp * s["scale"])}
