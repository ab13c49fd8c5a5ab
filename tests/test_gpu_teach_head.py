"""Norms, 8 bits, dropout, log probabilities and the losses together, as examples/teach_head.py runs them: the teacher's answers against 64 bits, a student's gradient against automatic
differentiation with the mask of the definition, the whole as a graph, on another stream and with workspaces of the caller's."""
import math
import os
import sys

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
import paper_2507_05508_amd as P  # noqa: E402
import teach_head as E  # noqa: E402
from oracle import worker as O  # noqa: E402

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().cpu().double().numpy()


def batch(n, width, seed, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.empty((n, width), device="cuda").normal_(generator=gen).to(dtype)


def test_teacher_answers():
    """Its logits within what four roundings to 8 bits (2^-4 each, of a half or so of every sum) leave of the exact ones; the answers are those of the logits, entry by entry."""
    teacher, x = E.Teacher(96, 200, 333), batch(37, 96, 5)
    s = teacher.logits(x)
    w1, w2, w3 = (f64(q.float()) * f64(c)[:, None] for q, c in (teacher.w1, teacher.w2, teacher.w3))
    y = O.rms_norm(f64(x), f64(teacher.norms[0]), 1e-5)[0]
    h = O.linear(O.linear(y, w1, kind="gelu")[0], w2)[0] + f64(x)
    want = O.linear(O.rms_norm(h, f64(teacher.norms[1]), 1e-5)[0], w3)[0]
    assert np.linalg.norm(f64(s) - want) <= 4 * 2.0 ** -4 * np.linalg.norm(want)
    tokens = torch.arange(37, dtype=torch.int32, device="cuda")
    a = teacher.answers(x, 8, tokens)
    logprob, entropy, idx, val, _ = O.token_logprobs(f64(s), tokens.cpu().numpy()[:, None], 8, 1.0)
    assert np.array_equal(a.top_idx.cpu().numpy(), idx)
    for got, right in ((a.logprob, logprob[:, 0]), (a.entropy, entropy), (a.top_logprob, val)):
        assert np.abs(f64(got) - right).max() < 1e-5 * 30      # 400 roundings of 2^-24 of magnitudes up to 12


def reference(student, row, x, answers, temperature, keep, scale):
    """Losses and gradient of the mean loss, in 64 bits on the CPU."""
    p = {k: v.detach().cpu().double().requires_grad_(True) for k, v in student.tensors(row).items()}
    x = x.cpu().double()
    b = x @ p["w1"].t()
    a = 0.5 * b * (1 + torch.erf(b / math.sqrt(2)))
    h = x + (a @ p["w2"].t()) * torch.from_numpy(keep) * scale
    s = h / (h.pow(2).mean(1, keepdim=True) + 1e-5).sqrt() * p["norm"] @ p["w3"].t()
    log_p = torch.log_softmax(s / temperature, 1)
    idx, log_q = answers.top_idx.cpu().long(), torch.log_softmax(answers.top_logprob.cpu().double() / temperature, 1)
    loss = temperature ** 2 * (log_q.exp() * (log_q - log_p.gather(1, idx))).sum(1)
    loss.mean().backward()
    return loss.detach(), torch.cat([p[k].grad.reshape(-1) for k in student.shapes])


def test_student_gradient_matches_automatic_differentiation():
    """fp32: every stage rounds by 2^-24 and sums of up to 1000 terms follow one another; 1e-5 of a tensor's largest entry is over a hundred such roundings in each of the six stages."""
    teacher, student = E.Teacher(96, 200, 333), E.Student(96, 200, 333, torch.float32)
    x = batch(37, 96, 5)
    answers = teacher.answers(x, 8)
    row = torch.full((student.count,), float("nan"), device="cuda")
    loss = E.worker_step(student, student.weights(), x.float(), answers, 2.0, 0.25, 11, 3, 2, row)
    keep = O.dropout_keep(37, 96, 16384, 11, 3, 2)
    want_loss, want = reference(student, student.x, x, answers, 2.0, keep, 1 / 0.75)
    assert np.abs(f64(loss) - want_loss.numpy()).max() < 1e-5 * want_loss.abs().max()
    for name, g in student.tensors(row).items():
        w = student.tensors(want)[name]
        assert (g.cpu().double() - w).abs().max() <= 1e-5 * w.abs().max(), name


def test_example_runs_and_repeats():
    losses = E.train(steps=6)
    assert all(math.isfinite(v) for v in losses)
    assert E.train(steps=3) == losses[:3]     # the same bits from run to run


def run(teacher, student, x, row, seed=11):
    answers = teacher.answers(x, 20)
    loss = E.worker_step(student, student.weights(), x, answers, 2.0, 0.25, seed, 3, 2, row)
    r = P.mlmc_token_logprobs(teacher.logits(x), answers.top_idx[:, :1].contiguous(), top=5, with_entropy=True, with_stats=True)
    d = P.mlmc_token_logprobs_backward(teacher.logits(x), r.stats, answers.top_idx[:, :1].contiguous(), r.logprob, r.top_idx, r.top_logprob, r.entropy)
    return loss, answers, r, d


def flat(out):
    loss, answers, r, d = out
    return [loss, *(t for t in answers if t is not None), *(t for t in r if t is not None), d]


def test_as_a_graph():
    """Captured once and replayed with new inputs in the same place, eager work in between: every replay has the eager result's bits.  Two graphs that take turns, each with memory of its own."""
    teacher, student = E.Teacher(256, 512, 9000), E.Student(256, 512, 9000)
    for attempt in range(2):
        run(teacher, student, batch(130, 256, 1), torch.zeros(student.count, device="cuda"))
    torch.cuda.synchronize()
    graphs = []
    for k in range(2):
        x, row = batch(130, 256, 20 + k), torch.zeros(student.count, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run(teacher, student, x, row)
        graphs.append((graph, x, row, out))
    for k in range(6):
        graph, x, row, out = graphs[k % 2]
        new = batch(130, 256, 100 + k)
        x.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in flat(out)] + [row.clone()]
        eager_row = torch.zeros_like(row)
        want = flat(run(teacher, student, new, eager_row)) + [eager_row]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g, w), k


def test_on_another_stream():
    teacher, student = E.Teacher(256, 512, 9000), E.Student(256, 512, 9000)
    x, row = batch(130, 256, 1), torch.zeros(student.count, device="cuda")
    want = flat(run(teacher, student, x, row))
    other_row = torch.zeros_like(row)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = flat(run(teacher, student, x, other_row))
    torch.cuda.current_stream().wait_stream(side)
    for g, w in zip(got + [other_row], want + [row]):
        assert torch.equal(g, w)


def test_workspaces_of_the_caller():
    """Of exactly the size asked for, filled with NaN before; 16 bytes are refused."""
    x, logits = batch(50, 9000, 3), batch(50, 40000, 3)
    tokens = torch.zeros((50, 1), dtype=torch.int32, device="cuda")
    q, s = P.mlmc_quantize(batch(128, 8192, 4))
    dy, rstd, dw = batch(50, 9000, 5), torch.ones(50, device="cuda"), torch.zeros(9000, device="cuda")
    calls = ((lambda ws: P.mlmc_token_logprobs(logits, tokens, top=7, with_entropy=True, ws=ws)[:4], P.mlmc_token_logprobs_workspace(50, 40000, 7)),
             (lambda ws: (P.mlmc_linear_q8(q, s, q, s, ws=ws),), P.mlmc_linear_q8_workspace(128, 128, 8192)),
             (lambda ws: (P.mlmc_rms_norm_backward(dy, x, None, rstd, dw, ws=ws), dw.clone()), P.mlmc_rms_norm_workspace(50, 9000)))
    for call, need in calls:
        assert need > 0
        want = call(None)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        for g, w in zip(call(ws), want):
            assert torch.equal(g, w)
        with pytest.raises(P.MlmcError):
            call(ws[:16])
