"""Arguments that the calls of a worker's own step refuse, on the host: nothing is launched."""
import ctypes as C

import pytest
import torch

import paper_2507_05508_amd as P

OK, EINVAL = 0, P.binding.MLMC_EINVAL
BUF = (C.c_char * 8192)()
A = (C.addressof(BUF) + 255) // 256 * 256   # stands for a device pointer: every call here is refused, or has no rows


def norm(**k):
    a = dict(x=A, ldx=8, rows=2, d=8, dtype=0, weight=None, bias=None, eps=1e-5, y=A, ldy=8, stats=None)
    a.update(k)
    return P.lib().mlmc_layer_norm(*a.values(), None)


def norm_backward(**k):
    a = dict(dy=A, lddy=8, x=A, ldx=8, rows=2, d=8, dtype=0, weight=None, stats=A, dx=A, lddx=8, dw=A, db=A, gd=0, ws=A, wsb=1 << 20)
    a.update(k)
    return P.lib().mlmc_layer_norm_backward(*a.values(), None)


def linear(**k):
    a = dict(x=A, ldx=8, w=A, ldw=8, rows=2, m=4, k=8, dtype=0, bias=None, act=0, res=None, ldr=0, z=None, ldz=0, y=A, ldy=4, ws=A, wsb=1 << 40)
    a.update(k)
    return P.lib().mlmc_linear(*a.values(), None)


def dgrad(**k):
    a = dict(dy=A, lddy=4, w=A, ldw=8, rows=2, m=4, k=8, dtype=0, act=0, z=None, ldz=0, res=None, ldr=0, dx=A, lddx=8, ws=A, wsb=1 << 40)
    a.update(k)
    return P.lib().mlmc_linear_dgrad(*a.values(), None)


def wgrad(**k):
    a = dict(dy=A, lddy=4, x=A, ldx=8, rows=2, m=4, k=8, dtype=0, dw=A, lddw=8, db=None, gd=0, ws=A, wsb=1 << 40)
    a.update(k)
    return P.lib().mlmc_linear_wgrad(*a.values(), None)


def distill(**k):
    a = dict(s=A, ldl=8, rows=2, v=8, dtype=0, idx=A, val=A, top=2, temp=1.0, dloss=None, scale=1.0, loss=A, ds=None, ldd=0, st=None, ws=A, wsb=1 << 40)
    a.update(k)
    return P.lib().mlmc_distill(*a.values(), None)


@pytest.mark.parametrize("call,bad", [
    (norm, dict(rows=-1)), (norm, dict(rows=1 << 31)), (norm, dict(d=0)), (norm, dict(d=1 << 31, ldx=1 << 31, ldy=1 << 31)), (norm, dict(dtype=2)), (norm, dict(ldx=7)),
    (norm, dict(ldy=7)), (norm, dict(eps=-1.0)), (norm, dict(eps=float("nan"))), (norm, dict(eps=float("inf"))), (norm, dict(x=None)),
    (norm, dict(y=None)), (norm, dict(x=A + 2)), (norm, dict(dtype=1, x=A + 1)), (norm, dict(weight=A + 2)), (norm, dict(bias=A + 1)), (norm, dict(stats=A + 2)),
    (norm_backward, dict(stats=None)), (norm_backward, dict(dx=None)), (norm_backward, dict(lddx=7)), (norm_backward, dict(lddy=7)),
    (norm_backward, dict(gd=3)), (norm_backward, dict(dw=A + 2)), (norm_backward, dict(gd=1, db=A + 1)), (norm_backward, dict(ws=None)),
    (norm_backward, dict(ws=A + 64)), (norm_backward, dict(wsb=8)),
    (linear, dict(rows=-1)), (linear, dict(m=0)), (linear, dict(k=0)), (linear, dict(k=(1 << 21) + 1, ldx=1 << 22, ldw=1 << 22)), (linear, dict(ldx=7)), (linear, dict(ldw=7)),
    (linear, dict(ldy=3)), (linear, dict(act=3)), (linear, dict(dtype=-1)), (linear, dict(res=A, ldr=3)), (linear, dict(z=A, ldz=3)), (linear, dict(y=None)),
    (linear, dict(bias=A + 1)), (linear, dict(w=A + 2)), (linear, dict(dtype=1, z=A + 1, ldz=4)),
    (dgrad, dict(act=2, z=None, ldz=8)), (dgrad, dict(act=2, z=A, ldz=7)), (dgrad, dict(lddx=7)), (dgrad, dict(lddy=3)), (dgrad, dict(res=A, ldr=7)), (dgrad, dict(dx=None)),
    (wgrad, dict(dw=None)), (wgrad, dict(dw=None, rows=0)), (wgrad, dict(gd=2)), (wgrad, dict(lddw=7)), (wgrad, dict(db=A + 2)), (wgrad, dict(x=None)),
    (distill, dict(top=0)), (distill, dict(top=1025)), (distill, dict(v=0)), (distill, dict(ldl=7)), (distill, dict(ds=A, ldd=7)), (distill, dict(temp=0.0)),
    (distill, dict(temp=-1.0)), (distill, dict(temp=float("nan"))), (distill, dict(temp=float("inf"))), (distill, dict(temp=1e-45)), (distill, dict(loss=None)),
    (distill, dict(idx=None)), (distill, dict(val=None)), (distill, dict(idx=A + 1)), (distill, dict(dloss=A + 2)), (distill, dict(st=A + 1)), (distill, dict(s=A + 2)),
])
def test_refused(call, bad):
    assert call(**bad) == EINVAL


def test_no_rows_is_no_work():
    assert norm(rows=0, x=None, y=None) == OK
    assert norm_backward(rows=0, dy=None, x=None, dx=None, stats=None, dw=None, db=None, ws=None, wsb=0) == OK
    assert linear(rows=0, x=None, y=None) == OK
    assert dgrad(rows=0, dy=None, dx=None) == OK
    assert distill(rows=0, s=None, idx=None, val=None, loss=None) == OK


def test_workspace_of_refused_sizes_is_zero():
    for f, a in ((P.mlmc_layer_norm_workspace, (-1, 8)), (P.mlmc_layer_norm_workspace, (1, 0)), (P.mlmc_linear_workspace, (1, 0, 1)),
                 (P.mlmc_linear_workspace, (-1, 1, 1)), (P.mlmc_distill_workspace, (1, 1, 0)), (P.mlmc_distill_workspace, (1, 0, 1))):
        assert f(*a) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros(2, 8)
    for f in (lambda: P.mlmc_layer_norm(x), lambda: P.mlmc_linear(x, x), lambda: P.mlmc_linear_dgrad(x, x), lambda: P.mlmc_linear_wgrad(x, x, x),
              lambda: P.mlmc_distill(x, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1))):
        with pytest.raises(P.MlmcError):
            f()
