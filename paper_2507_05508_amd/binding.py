"""ctypes binding of libmlmc.so: the same entry points as include/mlmc.h, taking torch CUDA tensors.

Argument marshalling only -- every step of the method runs in the HIP kernels of the library.  torch is
used for device memory and for the current stream.  There is no CPU fallback: if the library has not
been built (python -m paper_2507_05508_amd.build) loading fails with an error.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import NamedTuple, Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmlmc.so")

MLMC_OK, MLMC_EINVAL, MLMC_ENOMEM, MLMC_EHIP, MLMC_ELIMIT = 0, 1, 2, 3, 4
MLMC_STATIC_SCRATCH_BYTES = 1 << 20
MLMC_DEV_CAPACITY, MLMC_DEV_NONFINITE, MLMC_DEV_INTERNAL, MLMC_DEV_REDONE, MLMC_DEV_RANGE = 1, 2, 4, 8, 16
MLMC_F32, MLMC_BF16 = 0, 1
MLMC_TOPK, MLMC_BITS, MLMC_FBITS, MLMC_STOPK, MLMC_VBITS, MLMC_RTN = 0, 1, 2, 3, 4, 5
MLMC_ACT_NONE, MLMC_ACT_RELU, MLMC_ACT_GELU = 0, 1, 2
MLMC_MAX_SLEVELS = 65536
MLMC_MAX_TEACHER = 1024
MLMC_MAX_ANSWERS = 128
MLMC_TILE = 4096
MLMC_MAX_LEVELS = 32

EXPORTS = ["mlmc_plan", "mlmc_plan_destroy", "mlmc_plan_set_sampling", "mlmc_plan_set_staging", "mlmc_plan_set_overlap", "mlmc_plan_num_tiles", "mlmc_plan_chunk", "mlmc_plan_num_planes", "mlmc_geometric_p",
           "mlmc_status_string", "mlmc_level_norms", "mlmc_compress_topk", "mlmc_compress_bits", "mlmc_compress_bits_static", "mlmc_compress_rtn", "mlmc_aggregate", "mlmc_aggregate_update", "mlmc_message_bits",
           "mlmc_layer_norm", "mlmc_layer_norm_workspace", "mlmc_layer_norm_backward", "mlmc_linear", "mlmc_linear_workspace", "mlmc_linear_dgrad", "mlmc_linear_wgrad",
           "mlmc_distill", "mlmc_distill_workspace", "mlmc_rms_norm", "mlmc_rms_norm_workspace", "mlmc_rms_norm_backward", "mlmc_quantize", "mlmc_linear_q8", "mlmc_linear_q8_workspace",
           "mlmc_dropout", "mlmc_token_logprobs", "mlmc_token_logprobs_workspace", "mlmc_token_logprobs_backward",
           "mlmc_profile_enable", "mlmc_profile_reset", "mlmc_profile_num_kernels", "mlmc_profile_kernel_name",
           "mlmc_profile_get"]

_lib = None


class MlmcError(RuntimeError):
    pass


def lib():
    """The loaded library (loads on first use; raises if it was not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise MlmcError(f"{LIB_PATH} is missing: build it with `python -m paper_2507_05508_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u64, dbl_p = C.c_void_p, C.c_int, C.c_int64, C.c_uint64, C.POINTER(C.c_double)
        L.mlmc_plan.restype = C.c_int
        L.mlmc_plan.argtypes = [C.POINTER(vp), i32, i32, i64, i32, i32, C.POINTER(i64), dbl_p,
                                C.POINTER(C.c_size_t), C.POINTER(i64)]
        L.mlmc_plan_destroy.restype = None
        L.mlmc_plan_destroy.argtypes = [vp]
        L.mlmc_plan_set_sampling.restype = C.c_int
        L.mlmc_plan_set_sampling.argtypes = [vp, i32]
        L.mlmc_plan_set_staging.restype = C.c_int
        L.mlmc_plan_set_staging.argtypes = [vp, i32]
        L.mlmc_plan_set_overlap.restype = C.c_int
        L.mlmc_plan_set_overlap.argtypes = [vp, i32]
        L.mlmc_plan_num_tiles.restype = i64
        L.mlmc_plan_num_tiles.argtypes = [vp]
        L.mlmc_plan_chunk.restype = i64
        L.mlmc_plan_chunk.argtypes = [vp]
        L.mlmc_plan_num_planes.restype = i32
        L.mlmc_plan_num_planes.argtypes = [vp]
        L.mlmc_geometric_p.restype = C.c_int
        L.mlmc_geometric_p.argtypes = [i32, dbl_p]
        L.mlmc_status_string.restype = C.c_char_p
        L.mlmc_status_string.argtypes = [i32]
        L.mlmc_level_norms.restype = C.c_int
        L.mlmc_level_norms.argtypes = [vp, vp, i64, vp, vp, vp, vp]
        L.mlmc_compress_topk.restype = C.c_int
        L.mlmc_compress_topk.argtypes = [vp, vp, i64, vp, i32, u64, u64, vp, vp, vp, vp, i64, vp, vp, vp, vp, vp]
        L.mlmc_compress_bits.restype = C.c_int
        L.mlmc_compress_bits.argtypes = [vp, vp, i64, u64, u64, vp, vp, vp, vp, vp, vp]
        L.mlmc_compress_rtn.restype = C.c_int
        L.mlmc_compress_rtn.argtypes = [vp, vp, i64, u64, u64, vp, vp, vp, vp, vp, vp, vp]
        L.mlmc_compress_bits_static.restype = C.c_int
        L.mlmc_compress_bits_static.argtypes = [vp, vp, i64, u64, u64, vp, vp, vp, vp, vp]
        L.mlmc_aggregate.restype = C.c_int
        L.mlmc_aggregate.argtypes = [vp, vp, vp, vp, vp, i64, vp, vp, vp, C.c_float, vp, vp, vp]
        L.mlmc_aggregate_update.restype = C.c_int
        L.mlmc_aggregate_update.argtypes = [vp, vp, vp, vp, vp, i64, vp, vp, vp, C.c_float, C.c_float, vp, vp, vp, vp]
        L.mlmc_message_bits.restype = C.c_int
        L.mlmc_message_bits.argtypes = [vp, vp, vp, vp]
        f32, sz = C.c_float, C.c_size_t
        for name, args in (("mlmc_layer_norm_workspace", [i64, i64]), ("mlmc_linear_workspace", [i64, i64, i64, i32, i32]), ("mlmc_distill_workspace", [i64, i64, i32]),
                           ("mlmc_rms_norm_workspace", [i64, i64]), ("mlmc_linear_q8_workspace", [i64, i64, i64]), ("mlmc_token_logprobs_workspace", [i64, i64, i32])):
            getattr(L, name).restype = sz
            getattr(L, name).argtypes = args
        for name, args in (("mlmc_layer_norm", [vp, i64, i64, i64, i32, vp, vp, f32, vp, i64, vp, vp]),
                           ("mlmc_layer_norm_backward", [vp, i64, vp, i64, i64, i64, i32, vp, vp, vp, i64, vp, vp, i32, vp, sz, vp]),
                           ("mlmc_linear", [vp, i64, vp, i64, i64, i64, i64, i32, vp, i32, vp, i64, vp, i64, vp, i64, vp, sz, vp]),
                           ("mlmc_linear_dgrad", [vp, i64, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp, sz, vp]),
                           ("mlmc_linear_wgrad", [vp, i64, vp, i64, i64, i64, i64, i32, vp, i64, vp, i32, vp, sz, vp]),
                           ("mlmc_distill", [vp, i64, i64, i64, i32, vp, vp, i32, f32, vp, f32, vp, vp, i64, vp, vp, sz, vp]),
                           ("mlmc_rms_norm", [vp, i64, vp, i64, i64, i64, i32, vp, f32, vp, i64, vp, i64, vp, i64, vp, vp, vp]),
                           ("mlmc_rms_norm_backward", [vp, i64, vp, i64, i64, i64, i32, vp, vp, vp, i64, vp, i64, vp, i32, vp, sz, vp]),
                           ("mlmc_quantize", [vp, i64, i64, i64, i32, vp, i64, vp, vp]),
                           ("mlmc_linear_q8", [vp, i64, vp, vp, i64, vp, i64, i64, i64, vp, i32, vp, i64, vp, i64, vp, sz, vp]),
                           ("mlmc_dropout", [vp, i64, i64, i64, i32, C.c_double, u64, u64, C.c_uint32, i64, vp, i64, vp, i64, vp]),
                           ("mlmc_token_logprobs", [vp, i64, i64, i64, i32, vp, i32, i32, f32, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
                           ("mlmc_token_logprobs_backward", [vp, i64, i64, i64, i32, vp, vp, i32, vp, vp, i32, vp, vp, f32, vp, i64, vp])):
            getattr(L, name).restype = C.c_int
            getattr(L, name).argtypes = args
        L.mlmc_profile_enable.restype = None
        L.mlmc_profile_enable.argtypes = [i32]
        L.mlmc_profile_reset.restype = None
        L.mlmc_profile_reset.argtypes = []
        L.mlmc_profile_num_kernels.restype = i32
        L.mlmc_profile_num_kernels.argtypes = []
        L.mlmc_profile_kernel_name.restype = C.c_char_p
        L.mlmc_profile_kernel_name.argtypes = [i32]
        L.mlmc_profile_get.restype = C.c_int
        L.mlmc_profile_get.argtypes = [i32, dbl_p, C.POINTER(i64)]
        _lib = L
    return _lib


def mlmc_profile_enable(on: bool):
    lib().mlmc_profile_enable(int(bool(on)))


def mlmc_profile_reset():
    lib().mlmc_profile_reset()


def mlmc_profile_get():
    """{kernel name: (total device ms, launches)} since the last reset (waits for the recorded events)."""
    out = {}
    for i in range(lib().mlmc_profile_num_kernels()):
        ms, n = C.c_double(), C.c_int64()
        _check(lib().mlmc_profile_get(i, C.byref(ms), C.byref(n)), "mlmc_profile_get")
        if n.value:
            out[lib().mlmc_profile_kernel_name(i).decode()] = (ms.value, n.value)
    return out


def _check(rc: int, what: str):
    if rc != MLMC_OK:
        raise MlmcError(f"{what}: {lib().mlmc_status_string(rc).decode()}")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream():
    # the handle of torch.cuda.current_stream(), without the object around it (2.7 us of a call, 0.2 this way)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def mlmc_geometric_p(L: int):
    buf = (C.c_double * L)()
    _check(lib().mlmc_geometric_p(L, buf), "mlmc_geometric_p")
    return list(buf)


class Plan:
    """Host plan + the device workspace and status word the calls need (allocated once, reused)."""

    def __init__(self, kind: int, M: int, d: int, dtype: int, ladder: Sequence[int],
                 p_fixed: Optional[Sequence[float]], device="cuda:0", allocate: bool = True):
        if kind == MLMC_STOPK:   # ladder = [s]: segments of s entries of the sorted row, L = ceil(d / s) levels
            self.s = int(ladder[0])
            L = -(-d // self.s) if self.s >= 1 else 0
            self.ladder = [min(self.s * l, d) for l in range(L + 1)] if 1 <= L <= MLMC_MAX_SLEVELS else [self.s]
            lad = (C.c_int64 * 1)(self.s)
        else:
            L = len(ladder) - 1
            self.ladder = [int(x) for x in ladder]
            lad = (C.c_int64 * (L + 1))(*self.ladder)
        self.kind, self.M, self.d, self.dtype, self.L = kind, M, d, dtype, L
        self.p_fixed = None if p_fixed is None else [float(x) for x in p_fixed]
        pf = None if p_fixed is None else (C.c_double * L)(*self.p_fixed)
        handle, wsb, cap = C.c_void_p(), C.c_size_t(), C.c_int64()
        rc = lib().mlmc_plan(C.byref(handle), kind, M, d, dtype, L, lad, pf, C.byref(wsb), C.byref(cap))
        _check(rc, "mlmc_plan")
        self.handle = handle
        self.workspace_bytes = wsb.value
        self.sparse_capacity_worst = cap.value
        self.num_tiles = lib().mlmc_plan_num_tiles(handle)
        self.num_planes = lib().mlmc_plan_num_planes(handle)
        self.chunk = lib().mlmc_plan_chunk(handle)
        self.device = torch.device(device)
        self.ws = None
        self.dev_status = None
        if allocate:
            self.ws = torch.empty(self.workspace_bytes + 256, dtype=torch.uint8, device=self.device)
            assert self.ws.data_ptr() % 256 == 0
            self.dev_status = torch.zeros(1, dtype=torch.int32, device=self.device)

    def close(self):
        if getattr(self, "handle", None):
            lib().mlmc_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_sampling(self, shift: int):
        """Histogram sampling of the threshold search: one block out of 2^shift (run time only, never results)."""
        _check(lib().mlmc_plan_set_sampling(self.handle, int(shift)), "mlmc_plan_set_sampling")

    def set_staging(self, enable: bool):
        """Stage the drawn band's members during the selection read (run time only, never results)."""
        _check(lib().mlmc_plan_set_staging(self.handle, int(bool(enable))), "mlmc_plan_set_staging")

    def set_overlap(self, enable: bool):
        """Run the second read of unstaged rows on the plan's side stream, beside the assembly of the other rows' messages
        (run time only, never results)."""
        _check(lib().mlmc_plan_set_overlap(self.handle, int(bool(enable))), "mlmc_plan_set_overlap")

    def status(self, informational: bool = False) -> int:
        """Device status bits of the last call (synchronises).  MLMC_DEV_REDONE is not an error and is only
        reported when `informational` is set."""
        s = int(self.dev_status.item())
        return s if informational else s & ~MLMC_DEV_REDONE


def mlmc_plan(kind, M, d, dtype, ladder, p_fixed=None, device="cuda:0", allocate=True) -> Plan:
    return Plan(kind, M, d, dtype, ladder, p_fixed, device, allocate)


def _check_g(plan: Plan, g: torch.Tensor):
    want = torch.float32 if plan.dtype == MLMC_F32 else torch.bfloat16
    if g.dtype != want or g.dim() != 2 or g.shape[0] != plan.M or g.shape[1] != plan.d or g.stride(1) != 1 or not g.is_cuda:
        raise MlmcError(f"g must be a CUDA {want} tensor [M={plan.M}, d={plan.d}] with unit inner stride")
    return g.stride(0)


def mlmc_level_norms(plan: Plan, g: torch.Tensor, norms: Optional[torch.Tensor] = None) -> torch.Tensor:
    ld = _check_g(plan, g)
    if norms is None:
        norms = torch.empty((plan.M, plan.L), dtype=torch.float64, device=g.device)
    rc = lib().mlmc_level_norms(plan.handle, _ptr(g), ld, _ptr(norms), _ptr(plan.dev_status), _ptr(plan.ws), _stream())
    _check(rc, "mlmc_level_norms")
    return norms


class SparseMessage:
    """Device buffers of one mlmc_compress_topk call (reused across steps when passed back in)."""

    def __init__(self, plan: Plan, capacity: Optional[int] = None, with_norms: bool = False):
        dev = plan.device
        self.capacity = plan.sparse_capacity_worst if capacity is None else int(capacity)
        self.level = torch.empty(plan.M, dtype=torch.int32, device=dev)
        self.row_off = torch.empty(plan.M + 1, dtype=torch.int64, device=dev)
        self.idx = torch.empty(max(self.capacity, 1), dtype=torch.int32, device=dev)   # uint32 payload
        self.val = torch.empty(max(self.capacity, 1), dtype=torch.float32, device=dev)
        self.tile_off = torch.empty((plan.M, plan.num_tiles + 1), dtype=torch.int32, device=dev)
        self.norms = torch.empty((plan.M, plan.L), dtype=torch.float64, device=dev) if with_norms else None


def mlmc_compress_topk(plan: Plan, g: torch.Tensor, seed: int, step: int, p: Optional[torch.Tensor] = None,
                       p_is_norms: bool = False, out: Optional[SparseMessage] = None) -> SparseMessage:
    ld = _check_g(plan, g)
    if out is None:
        out = SparseMessage(plan, with_norms=(plan.p_fixed is None and p is None))
    if p is not None and (p.dtype != torch.float64 or tuple(p.shape) != (plan.M, plan.L) or not p.is_contiguous()):
        raise MlmcError("p must be a contiguous float64 CUDA tensor [M, L]")
    rc = lib().mlmc_compress_topk(plan.handle, _ptr(g), ld, _ptr(p), int(bool(p_is_norms)), seed, step,
                                  _ptr(out.level), _ptr(out.row_off), _ptr(out.idx), _ptr(out.val), out.capacity,
                                  _ptr(out.tile_off), _ptr(out.norms), _ptr(plan.dev_status), _ptr(plan.ws), _stream())
    _check(rc, "mlmc_compress_topk")
    return out


class BitsMessage:
    def __init__(self, plan: Plan):
        dev = plan.device
        self.nwords = (plan.d + 63) // 64
        self.level = torch.empty(plan.M, dtype=torch.int32, device=dev)
        # per row: the scale exponent (MLMC_BITS), the bits of the largest entry (MLMC_VBITS), or, for MLMC_RTN, two
        # words: the bits of c and of the coefficient
        self.scale_exp = torch.empty((plan.M, 2) if plan.kind == MLMC_RTN else (plan.M,), dtype=torch.int32, device=dev)
        self.norms = torch.empty((plan.M, plan.L), dtype=torch.float64, device=dev) if plan.kind == MLMC_RTN else None
        self.planes = torch.zeros((plan.M, plan.num_planes, self.nwords), dtype=torch.int64, device=dev)  # uint64 payload


def mlmc_compress_bits(plan: Plan, g: torch.Tensor, seed: int, step: int, out: Optional[BitsMessage] = None) -> BitsMessage:
    ld = _check_g(plan, g)
    if out is None:
        out = BitsMessage(plan)
    rc = lib().mlmc_compress_bits(plan.handle, _ptr(g), ld, seed, step, _ptr(out.level), _ptr(out.scale_exp),
                                  _ptr(out.planes), _ptr(plan.dev_status), _ptr(plan.ws), _stream())
    _check(rc, "mlmc_compress_bits")
    return out


def mlmc_compress_rtn(plan: Plan, g: torch.Tensor, seed: int, step: int, out: Optional[BitsMessage] = None) -> BitsMessage:
    ld = _check_g(plan, g)
    if out is None:
        out = BitsMessage(plan)
    rc = lib().mlmc_compress_rtn(plan.handle, _ptr(g), ld, seed, step, _ptr(out.level), _ptr(out.scale_exp), _ptr(out.planes),
                                 _ptr(out.norms), _ptr(plan.dev_status), _ptr(plan.ws), _stream())
    _check(rc, "mlmc_compress_rtn")
    return out


def mlmc_compress_bits_static(plan: Plan, g: torch.Tensor, seed: int, step: int, out: BitsMessage,
                              dev_status: torch.Tensor) -> BitsMessage:
    """mlmc_compress_bits without a workspace (the library's static device scratch).  `out` and `dev_status` are
    the caller's: this call allocates nothing."""
    ld = _check_g(plan, g)
    rc = lib().mlmc_compress_bits_static(plan.handle, _ptr(g), ld, seed, step, _ptr(out.level), _ptr(out.scale_exp),
                                         _ptr(out.planes), _ptr(dev_status), _stream())
    _check(rc, "mlmc_compress_bits_static")
    return out


def mlmc_aggregate(plan: Plan, msg, alpha: float, out: Optional[torch.Tensor] = None, use_tile_off: bool = True) -> torch.Tensor:
    if out is None:
        out = torch.empty(plan.d, dtype=torch.float32, device=plan.device)
    if plan.kind in (MLMC_TOPK, MLMC_STOPK):
        rc = lib().mlmc_aggregate(plan.handle, None, _ptr(msg.row_off), _ptr(msg.idx), _ptr(msg.val), msg.capacity,
                                  _ptr(msg.tile_off) if use_tile_off else None, None, None, float(alpha), _ptr(out),
                                  _ptr(plan.ws), _stream())
    else:
        rc = lib().mlmc_aggregate(plan.handle, _ptr(msg.level), None, None, None, 0, None, _ptr(msg.scale_exp),
                                  _ptr(msg.planes), float(alpha), _ptr(out), _ptr(plan.ws), _stream())
    _check(rc, "mlmc_aggregate")
    return out


def mlmc_aggregate_update(plan: Plan, msg, alpha: float, eta: float, x: torch.Tensor, out: Optional[torch.Tensor] = None,
                          use_tile_off: bool = True) -> torch.Tensor:
    """x <- x - eta * (alpha * sum of the workers' messages), in place; `out` (optional) also receives the update."""
    if x.dtype != torch.float32 or x.numel() != plan.d or not x.is_contiguous() or not x.is_cuda:
        raise MlmcError("x must be a contiguous float32 CUDA tensor [d]")
    if plan.kind in (MLMC_TOPK, MLMC_STOPK):
        rc = lib().mlmc_aggregate_update(plan.handle, None, _ptr(msg.row_off), _ptr(msg.idx), _ptr(msg.val), msg.capacity,
                                         _ptr(msg.tile_off) if use_tile_off else None, None, None, float(alpha), float(eta),
                                         _ptr(x), _ptr(out), _ptr(plan.ws), _stream())
    else:
        rc = lib().mlmc_aggregate_update(plan.handle, _ptr(msg.level), None, None, None, 0, None, _ptr(msg.scale_exp),
                                         _ptr(msg.planes), float(alpha), float(eta), _ptr(x), _ptr(out), _ptr(plan.ws), _stream())
    _check(rc, "mlmc_aggregate_update")
    return x


def mlmc_message_bits(plan: Plan, msg, bits: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Bits per worker that the message `msg` of this plan takes on the wire (int64 tensor [M])."""
    if bits is None:
        bits = torch.empty(plan.M, dtype=torch.int64, device=plan.device)
    _check(lib().mlmc_message_bits(plan.handle, _ptr(msg.level), _ptr(bits), _stream()), "mlmc_message_bits")
    return bits



# ---- a worker's own step and its teacher: norms, linear layers, dropout, distillation loss, log probabilities of tokens --
# None of these calls is recorded by autograd: they read the values of their tensors, whether these require gradients or not, what they return requires none, and the gradients
# are the calls that compute them.
_DTYPE = {torch.float32: MLMC_F32, torch.bfloat16: MLMC_BF16}


def _elsewhere(t: torch.Tensor) -> bool:
    """Not on the current CUDA device (asked without torch.cuda's check that CUDA is initialised: a CUDA tensor has done that)."""
    at = t.get_device()
    return at < 0 or at != torch._C._cuda_getDevice()


def _matrix(t: torch.Tensor, name: str, dtype=None, n: int = -1, d: int = -1) -> int:
    """Row distance of a matrix on the current device with unit inner stride ([n, d] of dtype where given); raises for anything else."""
    try:
        rows, cols = t.shape
        r, c = t.stride()
    except ValueError:
        raise MlmcError(f"{name} must be a matrix") from None
    if (t.dtype is not dtype and (dtype is not None or t.dtype not in _DTYPE)) or (n >= 0 and rows != n) or (d >= 0 and cols != d):
        raise MlmcError(f"{name} must be of " + ("float32 or bfloat16" if dtype is None else str(dtype)) + f" and have the size that the others give it (it is {rows} x {cols})")
    at = t.get_device()
    if at < 0 or at != torch._C._cuda_getDevice():     # _elsewhere, without the call
        raise MlmcError(f"{name} is not on the current CUDA device")
    if (c != 1 and cols > 1) or (r < cols and rows > 1):
        raise MlmcError(f"{name} must have unit inner stride and rows that do not overlap")
    return r if rows > 1 and r > cols else cols


def _vector(t: Optional[torch.Tensor], name: str, d: int, dtype=torch.float32):
    if t is None:
        return None
    at = t.get_device()
    if t.dtype is not dtype or t.dim() != 1 or t.numel() != d or not t.is_contiguous() or at < 0 or at != torch._C._cuda_getDevice():
        raise MlmcError(f"{name} must be a contiguous tensor of {dtype}, [{d}], on the current CUDA device")
    return t.data_ptr()


def _table(t: torch.Tensor, name: str, n: int, d: int, dtype):
    if t.dtype is not dtype or t.dim() != 2 or t.shape[0] != n or t.shape[1] != d or not t.is_contiguous() or _elsewhere(t):
        raise MlmcError(f"{name} must be a contiguous tensor of {dtype}, [{n}, {d}], on the current CUDA device")
    return t.data_ptr()


def _scratch(ws: Optional[torch.Tensor], need: int, like: torch.Tensor):
    """The caller's workspace (address, bytes, tensor), or one of this call from torch's allocator, on the current stream."""
    if ws is None:
        if need == 0:
            return None, 0, None
        ws = like.new_empty(need, dtype=torch.uint8)
    elif ws.dtype is not torch.uint8 or not ws.is_contiguous() or _elsewhere(ws):
        raise MlmcError("ws must be a contiguous tensor of torch.uint8 on the current CUDA device")
    return ws.data_ptr(), ws.numel(), ws


@functools.lru_cache(maxsize=4096)
def mlmc_layer_norm_workspace(rows: int, d: int) -> int:
    return lib().mlmc_layer_norm_workspace(rows, d)


@functools.lru_cache(maxsize=4096)
def mlmc_linear_workspace(rows: int, outputs: int, inputs: int, call: int = 0, dtype: int = -1) -> int:
    """Bytes for mlmc_linear (1), mlmc_linear_dgrad (2), mlmc_linear_wgrad (3) or any of them (0), of matrices of dtype or of either (-1)."""
    return lib().mlmc_linear_workspace(rows, outputs, inputs, call, dtype)


@functools.lru_cache(maxsize=4096)
def mlmc_distill_workspace(rows: int, vocab: int, top: int) -> int:
    return lib().mlmc_distill_workspace(rows, vocab, top)


def mlmc_layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                    y: Optional[torch.Tensor] = None, with_stats: bool = False, stats: Optional[torch.Tensor] = None):
    """y, or (y, stats) if the statistics for the backward pass are asked for (with_stats, or a tensor [rows, 2] that receives them).  Not recorded by autograd: the gradient is
    mlmc_layer_norm_backward."""
    ldx = _matrix(x, "x")
    dtype = x.dtype
    n, d = x.shape
    if y is None:
        y, ldy = x.new_empty((n, d)), d
    else:
        ldy = _matrix(y, "y", dtype, n, d)
    if stats is not None:
        _table(stats, "stats", n, 2, torch.float32)
    elif with_stats:
        stats = torch.empty((n, 2), dtype=torch.float32, device=x.device)
    rc = lib().mlmc_layer_norm(x.data_ptr(), ldx, n, d, _DTYPE[dtype], _vector(weight, "weight", d), _vector(bias, "bias", d), eps,
                               y.data_ptr(), ldy, None if stats is None else stats.data_ptr(), _stream())
    if rc:
        _check(rc, "mlmc_layer_norm")
    return y if stats is None else (y, stats)


def mlmc_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], stats: torch.Tensor,
                             dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                             dx: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dx; dweight and dbias ([d], fp32 or bf16 alike, for instance parts of a row of the gradient matrix) are written in place."""
    ldx = _matrix(x, "x")
    dtype = x.dtype
    n, d = x.shape
    if dx is None:
        dx, lddx = x.new_empty((n, d)), d
    else:
        lddx = _matrix(dx, "dx", dtype, n, d)
    g, need = torch.float32, 0
    if dweight is not None or dbias is not None:
        g = (dbias if dweight is None else dweight).dtype
        if g not in _DTYPE:
            raise MlmcError("dweight and dbias must be of float32 or bfloat16")
        need = mlmc_layer_norm_workspace(n, d)
    p, nbytes, ws = _scratch(ws, need, x)
    rc = lib().mlmc_layer_norm_backward(dy.data_ptr(), _matrix(dy, "dy", dtype, n, d), x.data_ptr(), ldx, n, d, _DTYPE[dtype],
                                        _vector(weight, "weight", d), _table(stats, "stats", n, 2, torch.float32), dx.data_ptr(), lddx,
                                        _vector(dweight, "dweight", d, g), _vector(dbias, "dbias", d, g), _DTYPE[g], p, nbytes, _stream())
    if rc:
        _check(rc, "mlmc_layer_norm_backward")
    return dx


def mlmc_linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, act: int = MLMC_ACT_NONE,
                residual: Optional[torch.Tensor] = None, z: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y = act(x weight^T + bias) + residual; z, if given, receives what act is applied to.  Not recorded by autograd: the gradients are mlmc_linear_dgrad and mlmc_linear_wgrad."""
    ldx = _matrix(x, "x")
    dtype = x.dtype
    n, k = x.shape
    ldw = _matrix(weight, "weight", dtype, -1, k)
    m = weight.shape[0]
    if y is None:
        y, ldy = x.new_empty((n, m)), m
    else:
        ldy = _matrix(y, "y", dtype, n, m)
    p, nbytes, ws = _scratch(ws, mlmc_linear_workspace(n, m, k, 1, _DTYPE[dtype]), x)
    rc = lib().mlmc_linear(x.data_ptr(), ldx, weight.data_ptr(), ldw, n, m, k, _DTYPE[dtype], _vector(bias, "bias", m), act,
                           None if residual is None else residual.data_ptr(), 0 if residual is None else _matrix(residual, "residual", dtype, n, m),
                           None if z is None else z.data_ptr(), 0 if z is None else _matrix(z, "z", dtype, n, m),
                           y.data_ptr(), ldy, p, nbytes, _stream())
    if rc:
        _check(rc, "mlmc_linear")
    return y


def mlmc_linear_dgrad(dy: torch.Tensor, weight: torch.Tensor, act: int = MLMC_ACT_NONE, z: Optional[torch.Tensor] = None,
                      residual: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                      ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dx = (dy weight) act'(z) + residual, z being what the activation in front of the layer was applied to."""
    lddy = _matrix(dy, "dy")
    dtype = dy.dtype
    n, m = dy.shape
    ldw = _matrix(weight, "weight", dtype, m)
    k = weight.shape[1]
    if act != MLMC_ACT_NONE and z is None:
        raise MlmcError("the gradient of an activation needs z")
    if dx is None:
        dx, lddx = dy.new_empty((n, k)), k
    else:
        lddx = _matrix(dx, "dx", dtype, n, k)
    p, nbytes, ws = _scratch(ws, mlmc_linear_workspace(n, m, k, 2, _DTYPE[dtype]), dy)
    rc = lib().mlmc_linear_dgrad(dy.data_ptr(), lddy, weight.data_ptr(), ldw, n, m, k, _DTYPE[dtype], act,
                                 None if z is None else z.data_ptr(), 0 if z is None else _matrix(z, "z", dtype, n, k),
                                 None if residual is None else residual.data_ptr(), 0 if residual is None else _matrix(residual, "residual", dtype, n, k),
                                 dx.data_ptr(), lddx, p, nbytes, _stream())
    if rc:
        _check(rc, "mlmc_linear_dgrad")
    return dx


def mlmc_linear_wgrad(dy: torch.Tensor, x: torch.Tensor, dweight: torch.Tensor, dbias: Optional[torch.Tensor] = None,
                      ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dweight = dy^T x and, if given, dbias = sum over rows of dy, written in place (fp32 or bf16 alike)."""
    lddy = _matrix(dy, "dy")
    dtype = dy.dtype
    n, m = dy.shape
    ldx = _matrix(x, "x", dtype, n)
    k = x.shape[1]
    lddw = _matrix(dweight, "dweight", None, m, k)
    p, nbytes, ws = _scratch(ws, mlmc_linear_workspace(n, m, k, 3, _DTYPE[dtype]), dy)
    rc = lib().mlmc_linear_wgrad(dy.data_ptr(), lddy, x.data_ptr(), ldx, n, m, k, _DTYPE[dtype], dweight.data_ptr(), lddw,
                                 _vector(dbias, "dbias", m, dweight.dtype), _DTYPE[dweight.dtype], p, nbytes, _stream())
    if rc:
        _check(rc, "mlmc_linear_wgrad")
    return dweight


def mlmc_distill(logits: torch.Tensor, t_idx: torch.Tensor, t_val: torch.Tensor, temperature: float = 1.0,
                 dloss: Optional[torch.Tensor] = None, scale: float = 1.0, grad: bool = True, loss: Optional[torch.Tensor] = None,
                 dlogits: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """(loss of every row, scale * dloss times its gradient in the logits); the second is None if neither `grad` nor `dlogits` asks for it.
    dlogits may be the logits themselves.  Not recorded by autograd: the gradient is the one returned.  dev_status (int32 [1]), if given, receives MLMC_DEV_RANGE for an index outside the vocabulary."""
    ldl = _matrix(logits, "logits")
    dtype = logits.dtype
    n, v = logits.shape
    if t_idx.dim() != 2:
        raise MlmcError("t_idx must be a matrix")
    top = t_idx.shape[1]
    ldd = 0
    if dlogits is not None:
        ldd = _matrix(dlogits, "dlogits", dtype, n, v)
    elif grad:
        dlogits, ldd = logits.new_empty((n, v)), v
    if loss is None:
        loss = torch.empty(n, dtype=torch.float32, device=logits.device)
    p, nbytes, ws = _scratch(ws, mlmc_distill_workspace(n, v, top), logits)
    rc = lib().mlmc_distill(logits.data_ptr(), ldl, n, v, _DTYPE[dtype], _table(t_idx, "t_idx", n, top, torch.int32), _table(t_val, "t_val", n, top, torch.float32),
                            top, temperature, _vector(dloss, "dloss", n), scale, _vector(loss, "loss", n),
                            None if dlogits is None else dlogits.data_ptr(), ldd, _vector(dev_status, "dev_status", 1, torch.int32), p, nbytes, _stream())
    if rc:
        _check(rc, "mlmc_distill")
    return loss, dlogits


class RmsNorm(NamedTuple):
    """What mlmc_rms_norm was asked for; None in the other places."""
    y: Optional[torch.Tensor]
    sum: Optional[torch.Tensor]
    rstd: Optional[torch.Tensor]
    q: Optional[torch.Tensor]
    scale: Optional[torch.Tensor]


class TokenLogprobs(NamedTuple):
    """What mlmc_token_logprobs was asked for; None in the other places."""
    logprob: Optional[torch.Tensor]
    entropy: Optional[torch.Tensor]
    top_idx: Optional[torch.Tensor]
    top_logprob: Optional[torch.Tensor]
    stats: Optional[torch.Tensor]


_E4M3 = torch.float8_e4m3fn


def _eight_bits(n: int, d: int, like: torch.Tensor):
    """A matrix of 8 bits whose rows begin at multiples of 16 bytes, which the product of such matrices reads fastest, and its row distance."""
    ld = (d + 15) // 16 * 16
    return torch.empty_strided((n, d), (ld, 1), dtype=_E4M3, device=like.device), ld


def _same(x: torch.Tensor, n: int, d: int) -> torch.Tensor:
    return torch.empty_like(x) if x.is_contiguous() else x.new_empty(n, d)     # the former takes less time


def _or_none(t: Optional[torch.Tensor], name: str, dtype, n: int, d: int):
    """Address and row distance of a matrix that may be absent."""
    return (None, 0) if t is None else (t.data_ptr(), _matrix(t, name, dtype, n, d))


@functools.lru_cache(maxsize=4096)
def mlmc_rms_norm_workspace(rows: int, d: int) -> int:
    return lib().mlmc_rms_norm_workspace(rows, d)


@functools.lru_cache(maxsize=4096)
def mlmc_linear_q8_workspace(rows: int, outputs: int, inputs: int) -> int:
    return lib().mlmc_linear_q8_workspace(rows, outputs, inputs)


@functools.lru_cache(maxsize=4096)
def mlmc_token_logprobs_workspace(rows: int, vocab: int, top: int) -> int:
    return lib().mlmc_token_logprobs_workspace(rows, vocab, top)


def mlmc_rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, eps: float = 1e-5,
                  with_y: bool = True, with_rstd: bool = False, with_q: bool = False, y: Optional[torch.Tensor] = None,
                  sum: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
                  scale: Optional[torch.Tensor] = None) -> RmsNorm:
    """The norm of x + residual: in x's type (y), in 8 bits (q, float8_e4m3fn, and the scale of every row), or both; with a residual the sum as well.  Tensors that are given receive
    what is asked for.  Not recorded by autograd: the gradient is mlmc_rms_norm_backward."""
    ldx = _matrix(x, "x")
    dtype = x.dtype
    n, d = x.shape
    p_r = p_s = p_y = p_q = p_scale = p_rstd = None     # what the call makes itself needs no check
    ldr = lds = ldy = ldq = 0
    if residual is not None:
        p_r, ldr = residual.data_ptr(), _matrix(residual, "residual", dtype, n, d)
        if sum is None:
            sum, lds = _same(x, n, d), d
        else:
            lds = _matrix(sum, "sum", dtype, n, d)
        p_s = sum.data_ptr()
    elif sum is not None:
        raise MlmcError("sum is an output of a norm with a residual")
    if y is not None:
        p_y, ldy = y.data_ptr(), _matrix(y, "y", dtype, n, d)
    elif with_y:
        y, ldy = _same(x, n, d), d
        p_y = y.data_ptr()
    if q is not None or with_q:
        if q is None:
            q, ldq = _eight_bits(n, d, x)
        else:
            ldq = _matrix(q, "q", _E4M3, n, d)
        p_q = q.data_ptr()
        if scale is None:
            scale = x.new_empty(n, dtype=torch.float32)
            p_scale = scale.data_ptr()
        else:
            p_scale = _vector(scale, "scale", n)
    elif scale is not None:
        raise MlmcError("scale is that of q")
    elif y is None:
        raise MlmcError("neither y nor q is asked for")
    if rstd is not None:
        p_rstd = _vector(rstd, "rstd", n)
    elif with_rstd:
        rstd = x.new_empty(n, dtype=torch.float32)
        p_rstd = rstd.data_ptr()
    rc = lib().mlmc_rms_norm(x.data_ptr(), ldx, p_r, ldr, n, d, _DTYPE[dtype], _vector(weight, "weight", d), eps, p_s, lds, p_y, ldy, p_q, ldq, p_scale, p_rstd, _stream())
    if rc:
        _check(rc, "mlmc_rms_norm")
    return RmsNorm(y, sum, rstd, q, scale)


def mlmc_rms_norm_backward(dy: torch.Tensor, s: torch.Tensor, weight: Optional[torch.Tensor], rstd: torch.Tensor, dweight: Optional[torch.Tensor] = None,
                           residual: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of x and of the forward call's residual alike; s: the sum that the forward call stored (x where there was none); residual: a gradient that comes to the sum by
    another way; dweight ([d], fp32 or bf16, for instance a part of a row of the gradient matrix) is written in place."""
    lds = _matrix(s, "s")
    dtype = s.dtype
    n, d = s.shape
    if dx is None:
        dx, lddx = s.new_empty((n, d)), d
    else:
        lddx = _matrix(dx, "dx", dtype, n, d)
    g, need = torch.float32, 0
    if dweight is not None:
        g = dweight.dtype
        if g not in _DTYPE:
            raise MlmcError("dweight must be of float32 or bfloat16")
        need = mlmc_rms_norm_workspace(n, d)
    p, nbytes, ws = _scratch(ws, need, s)
    p_r, ldr = _or_none(residual, "residual", dtype, n, d)
    if rstd is None:
        raise MlmcError("the gradient needs rstd")
    rc = lib().mlmc_rms_norm_backward(dy.data_ptr(), _matrix(dy, "dy", dtype, n, d), s.data_ptr(), lds, n, d, _DTYPE[dtype], _vector(weight, "weight", d),
                                      _vector(rstd, "rstd", n), p_r, ldr, dx.data_ptr(), lddx, _vector(dweight, "dweight", d, g), _DTYPE[g], p, nbytes, _stream())
    if rc:
        _check(rc, "mlmc_rms_norm_backward")
    return dx


def mlmc_quantize(x: torch.Tensor, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None):
    """(q, scale): the rows of x in 8 bits (float8_e4m3fn) and the scale of every row."""
    ldx = _matrix(x, "x")
    n, d = x.shape
    if q is None:
        q, ldq = _eight_bits(n, d, x)
    else:
        ldq = _matrix(q, "q", _E4M3, n, d)
    if scale is None:
        scale = x.new_empty(n, dtype=torch.float32)
        p_scale = scale.data_ptr()
    else:
        p_scale = _vector(scale, "scale", n)
    rc = lib().mlmc_quantize(x.data_ptr(), ldx, n, d, _DTYPE[x.dtype], q.data_ptr(), ldq, p_scale, _stream())
    if rc:
        _check(rc, "mlmc_quantize")
    return q, scale


def mlmc_linear_q8(x: torch.Tensor, x_scale: torch.Tensor, weight: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
                   act: int = MLMC_ACT_NONE, residual: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                   ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y = act(x weight^T + bias) + residual in bfloat16, x and weight in 8 bits (float8_e4m3fn) with a scale for every row, as mlmc_rms_norm and mlmc_quantize give them."""
    ldx = _matrix(x, "x", _E4M3)
    n, k = x.shape
    ldw = _matrix(weight, "weight", _E4M3, -1, k)
    m = weight.shape[0]
    if x_scale is None or w_scale is None:
        raise MlmcError("matrices in 8 bits need their scales")
    if y is None:
        y, ldy = x.new_empty(n, m, dtype=torch.bfloat16), m
    else:
        ldy = _matrix(y, "y", torch.bfloat16, n, m)
    p, nbytes, ws = _scratch(ws, mlmc_linear_q8_workspace(n, m, k), x)
    p_r, ldr = _or_none(residual, "residual", torch.bfloat16, n, m)
    rc = lib().mlmc_linear_q8(x.data_ptr(), ldx, _vector(x_scale, "x_scale", n), weight.data_ptr(), ldw, _vector(w_scale, "w_scale", m), n, m, k,
                              _vector(bias, "bias", m), act, p_r, ldr, y.data_ptr(), ldy, p, nbytes, _stream())
    if rc:
        _check(rc, "mlmc_linear_q8")
    return y


def mlmc_dropout(x: torch.Tensor, p: float, seed: int, step: int, stream: int = 0, row0: int = 0, residual: Optional[torch.Tensor] = None,
                 y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """What is kept of x, over 1 - p, plus residual; the mask is a function of (seed, step, stream, row0 + row, column) and is not stored.  Not recorded by autograd: the gradient is the
    same call on the gradient of y, with the same numbers.  seed is taken modulo 2^64."""
    ldx = _matrix(x, "x")
    dtype = x.dtype
    n, d = x.shape
    if y is None:
        y, ldy = _same(x, n, d), d
    else:
        ldy = _matrix(y, "y", dtype, n, d)
    if not (0 <= step < 1 << 32 and 0 <= stream < 1 << 32 and 0 <= row0 <= 1 << 32):
        raise MlmcError("step, stream and row0 are numbers of 32 bits")
    p_r, ldr = _or_none(residual, "residual", dtype, n, d)
    rc = lib().mlmc_dropout(x.data_ptr(), ldx, n, d, _DTYPE[dtype], p, seed, step, stream, row0, p_r, ldr, y.data_ptr(), ldy, _stream())
    if rc:
        _check(rc, "mlmc_dropout")
    return y


def mlmc_token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, top: int = 0, temperature: float = 1.0, with_entropy: bool = False,
                        with_stats: bool = False, dev_status: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> TokenLogprobs:
    """Log probabilities of the tokens (int32 [rows] or [rows, given], -1: padding), the entropy and the `top` alternatives of every row, whose indices and log probabilities
    mlmc_distill takes as a teacher's entries.  Not recorded by autograd: the gradient is mlmc_token_logprobs_backward, which needs the stats.
    dev_status (int32 [1]), if given, receives MLMC_DEV_RANGE for a token outside the vocabulary."""
    ldl = _matrix(logits, "logits")
    n, v = logits.shape
    given, p_t, logprob = 0, None, None
    if tokens is not None:
        given = _given(tokens)
        p_t = _answers(tokens, "tokens", n, torch.int32)
        logprob = torch.empty_like(tokens, dtype=torch.float32)     # tokens are contiguous
    entropy = logits.new_empty(n, dtype=torch.float32) if with_entropy else None
    stats = logits.new_empty(n, 3, dtype=torch.float32) if with_stats else None
    top_idx = top_logprob = None
    if top > 0:
        top_logprob = logits.new_empty(n, top, dtype=torch.float32)
        top_idx = torch.empty_like(top_logprob, dtype=torch.int32)
    p, nbytes, ws = _scratch(ws, mlmc_token_logprobs_workspace(n, v, top), logits)
    rc = lib().mlmc_token_logprobs(logits.data_ptr(), ldl, n, v, _DTYPE[logits.dtype], p_t, given, top, temperature,
                                   None if logprob is None else logprob.data_ptr(), None if entropy is None else entropy.data_ptr(),
                                   None if top_idx is None else top_idx.data_ptr(), None if top_logprob is None else top_logprob.data_ptr(),
                                   None if stats is None else stats.data_ptr(), _vector(dev_status, "dev_status", 1, torch.int32), p, nbytes, _stream())
    if rc:
        _check(rc, "mlmc_token_logprobs")
    return TokenLogprobs(logprob, entropy, top_idx, top_logprob, stats)


def _given(tokens: torch.Tensor) -> int:
    if tokens.dim() not in (1, 2):
        raise MlmcError("tokens must be a vector or a matrix")
    return tokens.shape[1] if tokens.dim() == 2 else 1


def _answers(t: torch.Tensor, name: str, n: int, dtype):
    """Address of a table with a row for each row of the logits, [n] or [n, given]."""
    if t.dtype is not dtype or t.shape[0] != n or not t.is_contiguous() or _elsewhere(t):
        raise MlmcError(f"{name} must be a contiguous tensor of {dtype}, [{n}] or [{n}, given], on the current CUDA device")
    return t.data_ptr()


def mlmc_token_logprobs_backward(logits: torch.Tensor, stats: torch.Tensor, tokens: Optional[torch.Tensor] = None, dlogprob: Optional[torch.Tensor] = None,
                                 top_idx: Optional[torch.Tensor] = None, dtop: Optional[torch.Tensor] = None, dentropy: Optional[torch.Tensor] = None,
                                 temperature: float = 1.0, dlogits: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient in the logits of what mlmc_token_logprobs returned for them: dlogprob that of the tokens' log probabilities, dtop of the alternatives', dentropy of the entropies.
    dlogits may be the logits themselves."""
    ldl = _matrix(logits, "logits")
    dtype = logits.dtype
    n, v = logits.shape
    if (tokens is None) != (dlogprob is None) or (top_idx is None) != (dtop is None):
        raise MlmcError("tokens and dlogprob, top_idx and dtop come together")
    given = top = 0
    p_t = p_g = p_i = p_a = None
    if tokens is not None:
        given = _given(tokens)
        if dlogprob.shape != tokens.shape:
            raise MlmcError("dlogprob has the size of tokens")
        p_t, p_g = _answers(tokens, "tokens", n, torch.int32), _answers(dlogprob, "dlogprob", n, torch.float32)
    if top_idx is not None:
        if top_idx.dim() != 2:
            raise MlmcError("top_idx must be a matrix")
        top = top_idx.shape[1]
        p_i, p_a = _table(top_idx, "top_idx", n, top, torch.int32), _table(dtop, "dtop", n, top, torch.float32)
    if dlogits is None:
        dlogits, ldd = logits.new_empty((n, v)), v
    else:
        ldd = _matrix(dlogits, "dlogits", dtype, n, v)
    rc = lib().mlmc_token_logprobs_backward(logits.data_ptr(), ldl, n, v, _DTYPE[dtype], _table(stats, "stats", n, 3, torch.float32), p_t, given, p_g, p_i, top, p_a,
                                            _vector(dentropy, "dentropy", n), temperature, dlogits.data_ptr(), ldd, _stream())
    if rc:
        _check(rc, "mlmc_token_logprobs_backward")
    return dlogits
