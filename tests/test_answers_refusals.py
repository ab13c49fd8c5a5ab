"""Arguments that root-mean-square norm, 8-bit matrices, dropout and log probabilities refuse, on the host: nothing is launched."""
import ctypes as C

import pytest
import torch

import paper_2507_05508_amd as P

OK, EINVAL = 0, P.binding.MLMC_EINVAL
BUF = (C.c_char * 8192)()
A = (C.addressof(BUF) + 255) // 256 * 256   # stands for a device pointer: every call here is refused, or has no rows
INF, NAN = float("inf"), float("nan")


def rms(**k):
    a = dict(x=A, ldx=8, res=None, ldr=0, rows=2, d=8, dtype=0, weight=None, eps=1e-5, sum=None, lds=0, y=A, ldy=8, q=None, ldq=0, scale=None, rstd=None)
    a.update(k)
    return P.lib().mlmc_rms_norm(*a.values(), None)


def rms_backward(**k):
    a = dict(dy=A, lddy=8, s=A, lds=8, rows=2, d=8, dtype=0, weight=None, rstd=A, res=None, ldr=0, dx=A, lddx=8, dw=A, gd=0, ws=A, wsb=1 << 20)
    a.update(k)
    return P.lib().mlmc_rms_norm_backward(*a.values(), None)


def quantize(**k):
    a = dict(x=A, ldx=8, rows=2, d=8, dtype=0, q=A, ldq=8, scale=A)
    a.update(k)
    return P.lib().mlmc_quantize(*a.values(), None)


def linear(**k):
    a = dict(x=A, ldx=8, xs=A, w=A, ldw=8, wsc=A, rows=2, m=4, k=8, bias=None, act=0, res=None, ldr=0, y=A, ldy=4, ws=A, wsb=1 << 40)
    a.update(k)
    return P.lib().mlmc_linear_q8(*a.values(), None)


def dropout(**k):
    a = dict(x=A, ldx=8, rows=2, d=8, dtype=0, p=0.5, seed=1, step=2, stream=3, row0=0, res=None, ldr=0, y=A, ldy=8)
    a.update(k)
    return P.lib().mlmc_dropout(*a.values(), None)


def logprobs(**k):
    a = dict(s=A, ldl=8, rows=2, v=8, dtype=0, tok=A, given=1, top=2, temp=1.0, lp=A, h=None, idx=A, val=A, stats=None, st=None, ws=A, wsb=1 << 40)
    a.update(k)
    return P.lib().mlmc_token_logprobs(*a.values(), None)


def logprobs_backward(**k):
    a = dict(s=A, ldl=8, rows=2, v=8, dtype=0, stats=A, tok=A, given=1, g=A, idx=A, top=2, a=A, h=None, temp=1.0, ds=A, ldd=8)
    a.update(k)
    return P.lib().mlmc_token_logprobs_backward(*a.values(), None)


@pytest.mark.parametrize("call,bad", [
    (rms, dict(rows=-1)), (rms, dict(rows=1 << 31)), (rms, dict(d=0)), (rms, dict(dtype=2)), (rms, dict(ldx=7)), (rms, dict(ldy=7)), (rms, dict(res=A, ldr=7)),
    (rms, dict(sum=A, lds=8)), (rms, dict(res=A, ldr=8, sum=A, lds=7)), (rms, dict(eps=-1.0)), (rms, dict(eps=NAN)), (rms, dict(eps=INF)), (rms, dict(y=None)),
    (rms, dict(q=A, ldq=8)), (rms, dict(q=A, ldq=7, scale=A)), (rms, dict(x=None)), (rms, dict(x=A + 2)), (rms, dict(dtype=1, x=A + 1)), (rms, dict(weight=A + 1)),
    (rms, dict(rstd=A + 2)), (rms, dict(res=A, ldr=8, sum=A, lds=8, y=A)), (rms, dict(q=A, ldq=8, scale=A + 1)), (rms, dict(res=A + 2, ldr=8)),
    (rms_backward, dict(rstd=None)), (rms_backward, dict(dx=None)), (rms_backward, dict(lddx=7)), (rms_backward, dict(lddy=7)), (rms_backward, dict(lds=7)),
    (rms_backward, dict(res=A, ldr=7)), (rms_backward, dict(res=A + 1, ldr=8)), (rms_backward, dict(gd=2)), (rms_backward, dict(dw=A + 2)), (rms_backward, dict(gd=1, dw=A + 1)),
    (rms_backward, dict(rows=200, ws=None)), (rms_backward, dict(rows=200, ws=A + 64)), (rms_backward, dict(rows=200, wsb=8)), (rms_backward, dict(s=None)),
    (quantize, dict(rows=-1)), (quantize, dict(d=0)), (quantize, dict(ldx=7)), (quantize, dict(ldq=7)), (quantize, dict(dtype=2)), (quantize, dict(q=None)), (quantize, dict(scale=None)),
    (quantize, dict(x=A + 2)), (quantize, dict(scale=A + 2)),
    (linear, dict(rows=-1)), (linear, dict(m=0)), (linear, dict(k=0)), (linear, dict(k=(1 << 21) + 1, ldx=1 << 22, ldw=1 << 22)), (linear, dict(ldx=7)), (linear, dict(ldw=7)),
    (linear, dict(ldy=3)), (linear, dict(act=3)), (linear, dict(xs=None)), (linear, dict(wsc=None)), (linear, dict(xs=A + 1)), (linear, dict(x=None)), (linear, dict(y=A + 1)),
    (linear, dict(bias=A + 2)), (linear, dict(res=A, ldr=3)), (linear, dict(res=A + 1, ldr=4)), (linear, dict(rows=512, m=512, k=8192, ldx=8192, ldw=8192, ldy=512, ws=None, wsb=0)),
    (dropout, dict(rows=-1)), (dropout, dict(d=0)), (dropout, dict(ldx=7)), (dropout, dict(ldy=7)), (dropout, dict(res=A, ldr=7)), (dropout, dict(p=-0.1)), (dropout, dict(p=1.0)),
    (dropout, dict(p=1 - 2.0 ** -17)), (dropout, dict(p=NAN)), (dropout, dict(step=1 << 32)), (dropout, dict(row0=-1)), (dropout, dict(row0=(1 << 32) - 1)), (dropout, dict(dtype=2)),
    (dropout, dict(row0=(1 << 63) - 1)), (dropout, dict(x=A + 1)), (dropout, dict(y=None)),
    (logprobs, dict(v=0)), (logprobs, dict(v=(1 << 20) + 1, ldl=1 << 22)), (logprobs, dict(ldl=7)), (logprobs, dict(given=129)), (logprobs, dict(top=129)), (logprobs, dict(top=-1)),
    (logprobs, dict(given=-1)), (logprobs, dict(temp=0.0)), (logprobs, dict(temp=INF)), (logprobs, dict(temp=1e-45)), (logprobs, dict(tok=None)), (logprobs, dict(lp=None)),
    (logprobs, dict(idx=None)), (logprobs, dict(val=A + 1)), (logprobs, dict(h=A + 2)), (logprobs, dict(stats=A + 1)), (logprobs, dict(st=A + 1)), (logprobs, dict(s=A + 2)),
    (logprobs, dict(v=131072, ldl=131072, ws=None)), (logprobs, dict(v=131072, ldl=131072, wsb=64)),
    (logprobs_backward, dict(stats=None)), (logprobs_backward, dict(ldd=7)), (logprobs_backward, dict(g=None)), (logprobs_backward, dict(a=None)), (logprobs_backward, dict(tok=A + 2)),
    (logprobs_backward, dict(idx=None)), (logprobs_backward, dict(ds=None)), (logprobs_backward, dict(h=A + 1)), (logprobs_backward, dict(temp=NAN)), (logprobs_backward, dict(top=129)),
])
def test_refused(call, bad):
    assert call(**bad) == EINVAL


def test_no_rows_is_no_work():
    assert rms(rows=0, x=None, y=None) == OK
    assert rms_backward(rows=0, dy=None, s=None, rstd=None, dx=None, dw=None, ws=None, wsb=0) == OK
    assert quantize(rows=0, x=None, q=None, scale=None) == OK
    assert linear(rows=0, x=None, xs=None, y=None) == OK
    assert dropout(rows=0, x=None, y=None, row0=1 << 32) == OK
    assert logprobs(rows=0, s=None, tok=None, lp=None, idx=None, val=None, ws=None) == OK
    assert logprobs_backward(rows=0, s=None, stats=None, tok=None, g=None, idx=None, a=None, ds=None) == OK


def test_workspace_of_refused_sizes_is_zero():
    for f, a in ((P.mlmc_rms_norm_workspace, (-1, 8)), (P.mlmc_rms_norm_workspace, (1, 0)), (P.mlmc_linear_q8_workspace, (1, 0, 1)), (P.mlmc_linear_q8_workspace, (-1, 1, 1)),
                 (P.mlmc_token_logprobs_workspace, (1, 0, 1)), (P.mlmc_token_logprobs_workspace, (1, 8, 129)), (P.mlmc_token_logprobs_workspace, (1, (1 << 20) + 1, 1))):
        assert f(*a) == 0


def test_binding_refuses():
    x = torch.zeros(2, 8)
    q, s = x.to(torch.float8_e4m3fn), torch.zeros(2)
    for f in (lambda: P.mlmc_rms_norm(x), lambda: P.mlmc_rms_norm_backward(x, x, None, s), lambda: P.mlmc_quantize(x), lambda: P.mlmc_linear_q8(q, s, q, s),
              lambda: P.mlmc_dropout(x, 0.5, 1, 2), lambda: P.mlmc_token_logprobs(x), lambda: P.mlmc_token_logprobs_backward(x, torch.zeros(2, 3))):
        with pytest.raises(P.MlmcError):      # host tensors
            f()
