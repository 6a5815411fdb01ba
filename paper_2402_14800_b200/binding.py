"""Thin ctypes binding of ``libmoe.so`` (see ``include/moe.h``).

Argument marshalling only: every step of the path runs in the library's CUDA
kernels.  Tensors are ``torch`` CUDA tensors used as device memory; the
library is given their ``data_ptr()``.  There is no CPU fallback: if the
library is missing or a call fails, a ``MoeError`` is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
from math import comb

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libmoe.so")

MOE_OK = 0
STATUS_NAMES = {
    0: "MOE_OK", -1: "MOE_ERR_INVALID_ARG", -2: "MOE_ERR_UNSUPPORTED_SHAPE", -3: "MOE_ERR_CUDA",
    -4: "MOE_ERR_OOM", -5: "MOE_ERR_DEVICE_TIMEOUT", -6: "MOE_ERR_ARCH",
}


class MoeError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__("%s: %s" % (STATUS_NAMES.get(code, str(code)), message))
        self.code = code


_lib = None


def load_library(path: str | None = None):
    """Load ``libmoe.so`` (built by ``python -m paper_2402_14800_b200.build``)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or _LIB_PATH
    if not os.path.exists(p):
        raise MoeError(-3, "%s not found: build it with `python -m paper_2402_14800_b200.build`" % p)
    lib = ctypes.CDLL(p)
    vp, ci, cf, u32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_uint32
    lib.moe_layer_create.restype = vp
    lib.moe_layer_create.argtypes = [vp, vp, vp, vp, ci, ci, ci, u32]
    lib.moe_layer_destroy.restype = None
    lib.moe_layer_destroy.argtypes = [vp]
    lib.moe_set_stream.argtypes = [vp, vp]
    lib.moe_layer_weight_bytes.restype = ctypes.c_size_t
    lib.moe_layer_weight_bytes.argtypes = [vp]
    lib.moe_layer_scratch_bytes.restype = ctypes.c_size_t
    lib.moe_layer_scratch_bytes.argtypes = [vp]
    lib.moe_layer_forward_kernel.restype = ctypes.c_char_p
    lib.moe_layer_forward_kernel.argtypes = [vp, ci]
    lib.moe_forward.argtypes = [vp, vp, ci, cf, vp, vp]
    lib.moe_forward_residual.argtypes = [vp, vp, ci, cf, vp, vp, vp]
    lib.moe_forward_host.argtypes = [vp, vp, ci, cf, vp]
    lib.moe_top2_distance.argtypes = [vp, vp, ci, vp]
    lib.moe_forward_topk.argtypes = [vp, vp, ci, ci, cf, vp, vp, vp, vp]
    lib.moe_routing_stats_layout.restype = ctypes.c_size_t
    lib.moe_routing_stats_layout.argtypes = [ci, ci, ctypes.POINTER(ctypes.c_size_t)]
    lib.moe_routing_stats_bytes.restype = ctypes.c_size_t
    lib.moe_routing_stats_bytes.argtypes = [ci, ci]
    lib.moe_calibrate_beta.argtypes = [vp, vp, ci, ctypes.POINTER(cf)]
    lib.moe_prune_search.argtypes = [vp, vp, ci, ci, ctypes.POINTER(cf), ctypes.POINTER(u32)]
    lib.moe_prune_search_multi.argtypes = [vp, vp, ci, ctypes.POINTER(ci), ci, ctypes.POINTER(cf),
                                           ctypes.POINTER(u32)]
    lib.moe_prune_search_progressive.argtypes = [vp, vp, vp, ci, ci, ctypes.POINTER(cf), ctypes.POINTER(u32)]
    lib.moe_num_subsets.restype = ctypes.c_long
    lib.moe_num_subsets.argtypes = [ci, ci]
    lib.moe_rmsnorm.argtypes = [vp, ci, ci, cf, vp, vp]
    lib.moe_add_rmsnorm.argtypes = [vp, vp, vp, ci, ci, cf, ci, vp, vp, vp, vp]
    lib.moe_add_rmsnorm_e4m3.argtypes = [vp, vp, vp, ci, ci, cf, ci, ci, vp, vp, vp, vp]
    lib.moe_add_rmsnorm_backward_workspace.restype = ctypes.c_size_t
    lib.moe_add_rmsnorm_backward_workspace.argtypes = [ci, ci]
    lib.moe_add_rmsnorm_backward.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, vp, vp, vp, ctypes.c_size_t, vp]
    cs = ctypes.c_size_t
    lib.moe_ffn_saved_bytes.restype = cs
    lib.moe_ffn_saved_bytes.argtypes = [ci, ci]
    lib.moe_ffn_forward_workspace.restype = cs
    lib.moe_ffn_forward_workspace.argtypes = [ci, ci, ci]
    lib.moe_ffn_backward_workspace.restype = cs
    lib.moe_ffn_backward_workspace.argtypes = [ci, ci, ci]
    lib.moe_ffn_forward.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, vp, vp, vp, cs, vp]
    lib.moe_ffn_backward.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, vp, vp, vp, vp, vp, cs, vp]
    lib.moe_stack_forward.argtypes = [ctypes.POINTER(vp), ci, vp, ci, ctypes.POINTER(cf), cf, vp]
    lib.moe_coselection.argtypes = [vp, vp, ci, ctypes.POINTER(ctypes.c_int32)]
    lib.moe_frequency_subset.restype = u32
    lib.moe_frequency_subset.argtypes = [ctypes.POINTER(ctypes.c_int32), ci, ci]
    lib.moe_device_status.argtypes = [vp]
    lib.moe_layer_share_scratch.argtypes = [vp, vp]
    lib.moe_profile_enable.argtypes = [vp, ci]
    lib.moe_profile_read.argtypes = [vp, ctypes.POINTER(cf), ctypes.POINTER(ci)]
    lib.moe_calibrate_beta_noalloc.argtypes = [vp, vp, ci, ci, ci, vp, ctypes.POINTER(cf)]
    lib.moe_reserve.argtypes = [vp, ci]
    lib.moe_test_wait_expiry.argtypes = [vp, ctypes.c_uint, ci]
    lib.moe_test_wait_expiry_pair.argtypes = [vp, ctypes.c_uint, ci]
    lib.moe_test_large_batch.argtypes = [vp, ci, ci]
    lib.moe_test_host_slabs.argtypes = [vp, ci]
    lib.moe_test_operators_expiry.argtypes = [ctypes.c_uint, vp]
    lib.moe_test_hold.argtypes = [ctypes.c_uint, vp]
    lib.moe_test_fail_occupancy.argtypes = [ci]
    lib.moe_test_ffn_plan.argtypes = [ci, ci, ci, ci, ci, ctypes.POINTER(ci)]
    lib.moe_test_ffn_deal.argtypes = [ci, ci, ci, ci, ci, ctypes.POINTER(ci), ci, ctypes.POINTER(ci)]
    lib.moe_test_set_free_bytes_limit.restype = None
    lib.moe_test_set_free_bytes_limit.argtypes = [ctypes.c_longlong]
    lib.moe_last_error.restype = ctypes.c_char_p
    if path is None:
        _lib = lib
    return lib


def last_error() -> str:
    return load_library().moe_last_error().decode()


def _check(rc: int):
    if rc != MOE_OK:
        raise MoeError(rc, last_error())


def _dev_bf16(t: torch.Tensor, shape=None) -> torch.Tensor:
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous()):
        raise MoeError(-1, "expected a contiguous bf16 CUDA tensor")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise MoeError(-1, "shape %s, expected %s" % (tuple(t.shape), tuple(shape)))
    return t


def routing_stats_layout(T: int, E: int):
    offs = (ctypes.c_size_t * 7)()
    total = load_library().moe_routing_stats_layout(T, E, offs)
    return int(total), [int(o) for o in offs]


def num_subsets(E: int, r: int) -> int:
    return int(load_library().moe_num_subsets(E, r))


class RoutingStats:
    """Device buffer for the routing record of one ``moe_forward`` call, with typed views."""

    def __init__(self, T: int, E: int, device):
        self.T, self.E = T, E
        total, o = routing_stats_layout(T, E)
        self.buf = torch.zeros(max(total, 16), dtype=torch.uint8, device=device)
        b = self.buf
        self.idx = b[o[0]:o[0] + T * 8].view(torch.int32).view(T, 2)
        self.wn = b[o[1]:o[1] + T * 8].view(torch.float32).view(T, 2)
        self.ratio = b[o[2]:o[2] + T * 4].view(torch.float32)
        self.skipped = b[o[3]:o[3] + T]
        self.count = b[o[4]:o[4] + E * 8].view(torch.int32).view(E, 2)
        self.n_skipped = b[o[5]:o[5] + 4].view(torch.int32)
        self.n_experts_touched = b[o[6]:o[6] + 4].view(torch.int32)


class MoeLayer:
    """One MoE layer restricted to the experts of ``kept_mask`` (``moe_layer_create``)."""

    def __init__(self, W_gate, W1, W3, W2, kept_mask: int | None = None):
        lib = load_library()
        E, h = W_gate.shape
        f = W1.shape[1]
        _dev_bf16(W_gate, (E, h)); _dev_bf16(W1, (E, f, h)); _dev_bf16(W3, (E, f, h)); _dev_bf16(W2, (E, h, f))
        self.h, self.f, self.E = h, f, E
        self.kept_mask = (1 << E) - 1 if kept_mask is None else int(kept_mask)
        self.device = W_gate.device
        with torch.cuda.device(self.device):
            self._h = lib.moe_layer_create(W_gate.data_ptr(), W1.data_ptr(), W3.data_ptr(), W2.data_ptr(),
                                           h, f, E, self.kept_mask)
        if not self._h:
            raise MoeError(-1, last_error())
        self.set_stream(torch.cuda.current_stream(self.device))

    def close(self):
        if getattr(self, "_h", None):
            load_library().moe_layer_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_stream(self, stream: torch.cuda.Stream):
        _check(load_library().moe_set_stream(self._h, ctypes.c_void_p(stream.cuda_stream)))

    def share_scratch(self, owner: "MoeLayer | None"):
        """Run out of ``owner``'s scratch buffers (``moe_layer_share_scratch``)."""
        _check(load_library().moe_layer_share_scratch(self._h, owner._h if owner is not None else None))

    def reserve(self, T_max: int):
        """``moe_reserve``: grow the scratch for any forward batch of up to ``T_max`` tokens now."""
        _check(load_library().moe_reserve(self._h, int(T_max)))

    @property
    def weight_bytes(self) -> int:
        return int(load_library().moe_layer_weight_bytes(self._h))

    @property
    def scratch_bytes(self) -> int:
        return int(load_library().moe_layer_scratch_bytes(self._h))

    def forward_kernel(self, T: int) -> str:
        """Name of the kernel that does the gate/up products of a forward call of T tokens."""
        return load_library().moe_layer_forward_kernel(self._h, T).decode()

    def forward(self, x, beta: float = 0.0, y=None, stats: RoutingStats | None = None, residual=None):
        """``moe_forward`` / ``moe_forward_residual``; returns y."""
        T = x.shape[0]
        _dev_bf16(x, (T, self.h))
        if y is None:
            y = torch.empty_like(x)
        _dev_bf16(y, (T, self.h))
        sp = stats.buf.data_ptr() if stats is not None else None
        lib = load_library()
        if residual is None:
            _check(lib.moe_forward(self._h, x.data_ptr(), T, beta, y.data_ptr(), sp))
        else:
            _dev_bf16(residual, (T, self.h))
            _check(lib.moe_forward_residual(self._h, x.data_ptr(), T, beta, residual.data_ptr(),
                                            y.data_ptr(), sp))
        return y

    def forward_topk(self, x, k: int, beta: float = 0.0, y=None, record: bool = False):
        """``moe_forward_topk``; with ``record`` also returns (idx[T,k] i32, wn[T,k] f32, n_active[T] i32)."""
        T = x.shape[0]
        _dev_bf16(x, (T, self.h))
        if y is None:
            y = torch.empty_like(x)
        idx = wn = na = None
        if record:
            idx = torch.empty((T, max(k, 1)), dtype=torch.int32, device=x.device)
            wn = torch.empty((T, max(k, 1)), dtype=torch.float32, device=x.device)
            na = torch.empty((T,), dtype=torch.int32, device=x.device)
        _check(load_library().moe_forward_topk(
            self._h, x.data_ptr(), T, k, beta, y.data_ptr(),
            idx.data_ptr() if record else None, wn.data_ptr() if record else None,
            na.data_ptr() if record else None))
        return (y, idx, wn, na) if record else y

    def top2_distance(self, x):
        """``moe_top2_distance``: fp32 CUDA tensor [T] of ||E_e0(x) - E_e1(x)||_2."""
        T = x.shape[0]
        _dev_bf16(x, (T, self.h))
        out = torch.empty((T,), dtype=torch.float32, device=x.device)
        _check(load_library().moe_top2_distance(self._h, x.data_ptr(), T, out.data_ptr()))
        return out

    def forward_host(self, x_host: torch.Tensor, beta: float, y_host: torch.Tensor):
        """``moe_forward_host``: x_host, y_host are host bf16 tensors (pinned or not)."""
        T = x_host.shape[0]
        assert x_host.dtype == torch.bfloat16 and y_host.dtype == torch.bfloat16
        assert not x_host.is_cuda and not y_host.is_cuda and x_host.is_contiguous() and y_host.is_contiguous()
        _check(load_library().moe_forward_host(self._h, x_host.data_ptr(), T, beta, y_host.data_ptr()))
        return y_host

    def calibrate_beta(self, x) -> float:
        T = x.shape[0]
        _dev_bf16(x, (T, self.h))
        out = ctypes.c_float(0)
        _check(load_library().moe_calibrate_beta(self._h, x.data_ptr(), T, ctypes.byref(out)))
        return float(out.value)

    def prune_search(self, x_calib, r: int):
        """``moe_prune_search``; returns (losses list of C(E, r) floats, best_subset bitmask)."""
        T = x_calib.shape[0]
        _dev_bf16(x_calib, (T, self.h))
        n = comb(self.E, r) if 0 <= r <= self.E else 1
        losses = (ctypes.c_float * max(n, 1))()
        best = ctypes.c_uint32(0)
        _check(load_library().moe_prune_search(self._h, x_calib.data_ptr(), T, r, losses, ctypes.byref(best)))
        return list(losses)[:n], int(best.value)

    def prune_search_multi(self, x_calib, rs):
        """``moe_prune_search_multi``: one evaluation of the experts, one enumeration per subset
        size in ``rs``; returns a list of (losses, best_subset) in the order of ``rs``."""
        T = x_calib.shape[0]
        _dev_bf16(x_calib, (T, self.h))
        rs = [int(r) for r in rs]
        ns = [comb(self.E, r) if 0 <= r <= self.E else 1 for r in rs]
        losses = (ctypes.c_float * max(sum(ns), 1))()
        best = (ctypes.c_uint32 * max(len(rs), 1))()
        r_arr = (ctypes.c_int * max(len(rs), 1))(*rs)
        _check(load_library().moe_prune_search_multi(self._h, x_calib.data_ptr(), T, r_arr, len(rs),
                                                     losses, best))
        out, o = [], 0
        for i, n in enumerate(ns):
            out.append((list(losses[o:o + n]), int(best[i])))
            o += n
        return out

    def coselection(self, x):
        """``moe_coselection``: E x E list of lists, counts[a][b] = tokens with top-2 (a, b)."""
        T = x.shape[0]
        _dev_bf16(x, (T, self.h))
        buf = (ctypes.c_int32 * (self.E * self.E))()
        _check(load_library().moe_coselection(self._h, x.data_ptr(), T, buf))
        return [[int(buf[a * self.E + b]) for b in range(self.E)] for a in range(self.E)]

    def frequency_subset(self, counts, r: int) -> int:
        """``moe_frequency_subset``: the activation-frequency baseline's kept mask."""
        flat = [int(v) for row in counts for v in row]
        buf = (ctypes.c_int32 * len(flat))(*flat)
        return int(load_library().moe_frequency_subset(buf, self.E, r))

    def profile_enable(self, on: bool = True):
        _check(load_library().moe_profile_enable(self._h, int(bool(on))))

    def profile_read(self):
        """Returns (stage_ms[4] summed over the recorded calls, number of calls)."""
        ms = (ctypes.c_float * 4)()
        n = ctypes.c_int(0)
        _check(load_library().moe_profile_read(self._h, ms, ctypes.byref(n)))
        return [float(v) for v in ms], int(n.value)

    def prune_search_progressive(self, x_pruned, F_ref, r: int):
        """``moe_prune_search_progressive``: F_ref is a contiguous fp32 CUDA tensor [T, h]."""
        T = x_pruned.shape[0]
        _dev_bf16(x_pruned, (T, self.h))
        if not (F_ref.is_cuda and F_ref.dtype == torch.float32 and F_ref.is_contiguous()
                and tuple(F_ref.shape) == (T, self.h)):
            raise MoeError(-1, "F_ref must be a contiguous fp32 CUDA tensor of shape [T, h]")
        n = comb(self.E, r) if 0 <= r <= self.E else 1
        losses = (ctypes.c_float * max(n, 1))()
        best = ctypes.c_uint32(0)
        _check(load_library().moe_prune_search_progressive(self._h, x_pruned.data_ptr(), F_ref.data_ptr(),
                                                           T, r, losses, ctypes.byref(best)))
        return list(losses)[:n], int(best.value)

    def device_status(self) -> int:
        return int(load_library().moe_device_status(self._h))


def calibrate_beta_noalloc(W_gate_kept, x, stream=None) -> float:
    """``moe_calibrate_beta_noalloc``: the beta median without any device allocation by the
    library (scratch is a fixed array inside it; at most 16384 tokens).  ``W_gate_kept`` holds
    the router rows of the kept experts, ``x`` the calibration tokens."""
    r, h = W_gate_kept.shape
    T = x.shape[0]
    _dev_bf16(W_gate_kept)
    _dev_bf16(x, (T, h))
    st = stream or torch.cuda.current_stream(x.device)
    out = ctypes.c_float(0)
    _check(load_library().moe_calibrate_beta_noalloc(W_gate_kept.data_ptr(), x.data_ptr(), T, h, r,
                                                     ctypes.c_void_p(st.cuda_stream), ctypes.byref(out)))
    return float(out.value)


def rmsnorm(x, eps: float = 1e-5, out=None, stream=None):
    T, h = x.shape
    _dev_bf16(x)
    if out is None:
        out = torch.empty_like(x)
    st = stream or torch.cuda.current_stream(x.device)
    _check(load_library().moe_rmsnorm(x.data_ptr(), T, h, eps, out.data_ptr(), ctypes.c_void_p(st.cuda_stream)))
    return out


# Operators on the caller's own tensors: no handle, scratch from torch's allocator on the call's stream.  They read and
# write memory and leave no autograd graph: what requires a gradient gets none through them, the backward passes
# are calls of their own.

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


# a tenth of the time of torch.cuda.current_stream().cuda_stream, but a private name that not every torch has
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _operand(name, t, dtype, shape, index):
    """Address of a contiguous tensor of this type and shape on this device; None for None."""
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == index and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    raise MoeError(-1, "%s must be a contiguous %s tensor of shape %s on cuda:%d, got %s" % (
        name, dtype, tuple(shape), index,
        "%s %s on %s, strides %s" % (t.dtype, tuple(t.shape), t.device, t.stride()) if isinstance(t, torch.Tensor)
        else type(t).__name__))


def _on_device_of(x, dims, stream, body, *args):
    """body(device index, stream handle, *args) with the device of ``x`` current; memory that it takes from torch's
    allocator belongs to the stream that it launches on."""
    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dim() == dims and x.dtype in DTYPES and x.is_contiguous()):
        raise MoeError(-1, "expected a contiguous %d-dimensional CUDA tensor of bf16, fp16 or fp32" % dims)
    index = x.get_device()
    if stream is not None:
        if stream.device_index != index:
            raise MoeError(-1, "the stream is on cuda:%d, the tensors on cuda:%d" % (stream.device_index, index))
        with torch.cuda.stream(stream):  # makes the stream's device current too
            return body(index, stream.cuda_stream, *args)
    if torch.cuda.current_device() == index:
        return body(index, _raw_stream(index), *args)
    with torch.cuda.device(index):
        return body(index, _raw_stream(index), *args)


def _output(name, t, like, index, dtype=None):
    """(address, tensor) of an output of ``like``'s shape, a new tensor where the caller gave none."""
    if t is None:
        t = torch.empty_like(like) if dtype is None else torch.empty_like(like, dtype=dtype)
        return t.data_ptr(), t
    return _operand(name, t, dtype or like.dtype, like.shape, index), t


def _sum_buffer(x, residual, s, index):
    """Address of s (a new tensor where the caller gave none), and s itself."""
    if residual is None:
        if s is not None:
            raise MoeError(-1, "without a residual s is x itself")
        return None, x
    return _output("s", s, x, index)


def add_rmsnorm(x, residual=None, gain=None, eps: float = 1e-5, out=None, s=None, rstd=None, stream=None):
    """``moe_add_rmsnorm``: s = x + residual (in their type), out = s / sqrt(mean(s^2) + eps) * gain.

    x, residual, out, s [T, h] bf16, fp16 or fp32, gain [h] of the same type (None: 1).  Without a residual
    s is x.  ``rstd``: an fp32 tensor [T] that receives 1 / sqrt(...) for the backward pass.
    Returns (out, s)."""
    return _on_device_of(x, 2, stream, _add_rmsnorm, x, residual, gain, eps, out, s, rstd)


def _add_rmsnorm(index, st, x, residual, gain, eps, out, s, rstd):
    T, h = shape = x.shape
    dt = x.dtype
    rp, gp = _operand("residual", residual, dt, shape, index), _operand("gain", gain, dt, (h,), index)
    tp = _operand("rstd", rstd, torch.float32, (T,), index)
    sp, s = _sum_buffer(x, residual, s, index)
    op, out = _output("out", out, x, index)
    _check(load_library().moe_add_rmsnorm(x.data_ptr(), rp, gp, T, h, eps, DTYPES[dt], op, sp, tp, st))
    return out, s


def add_rmsnorm_e4m3(x, residual=None, gain=None, eps: float = 1e-5, group: int = 0, q=None, scales=None, s=None,
                     stream=None):
    """``moe_add_rmsnorm_e4m3``: the norm of ``add_rmsnorm`` in 8 bits.  q [T, h] float8_e4m3fn and fp32
    ``scales``, one a row ([T, 1], group 0) or one for each 128 columns ([T, h / 128], group 128);
    q * scales is the normalised value.  Returns (q, scales, s)."""
    return _on_device_of(x, 2, stream, _add_rmsnorm_e4m3, x, residual, gain, eps, group, q, scales, s)


def _add_rmsnorm_e4m3(index, st, x, residual, gain, eps, group, q, scales, s):
    T, h = shape = x.shape
    dt = x.dtype
    rp, gp = _operand("residual", residual, dt, shape, index), _operand("gain", gain, dt, (h,), index)
    sp, s = _sum_buffer(x, residual, s, index)
    qp, q = _output("q", q, x, index, torch.float8_e4m3fn)
    n = h // group if group > 0 else 1
    if scales is None:
        scales = x.new_empty((T, n), dtype=torch.float32)
    cp = _operand("scales", scales, torch.float32, (T, n), index)
    _check(load_library().moe_add_rmsnorm_e4m3(x.data_ptr(), rp, gp, T, h, eps, DTYPES[dt], group, qp, cp, sp, st))
    return q, scales, s


def add_rmsnorm_backward(d_out, s, rstd, gain=None, d_s=None, dx=None, dgain=None, stream=None):
    """``moe_add_rmsnorm_backward``: gradients of ``add_rmsnorm`` from its s and rstd.  ``d_s``: the gradient
    that reaches s along the residual stream (None: 0).  Returns (dx, dgain): dx belongs to x and to the
    residual alike; dgain is None without a gain."""
    return _on_device_of(d_out, 2, stream, _add_rmsnorm_backward, d_out, s, rstd, gain, d_s, dx, dgain)


@functools.lru_cache(maxsize=256)
def _norm_workspace(T: int, h: int, index: int) -> int:
    """Bytes of the backward pass's workspace on this device, which is current."""
    return int(load_library().moe_add_rmsnorm_backward_workspace(T, h))


def _add_rmsnorm_backward(index, st, d_out, s, rstd, gain, d_s, dx, dgain):
    T, h = shape = d_out.shape
    dt = d_out.dtype
    sp, ep = _operand("s", s, dt, shape, index), _operand("d_s", d_s, dt, shape, index)
    gp, tp = _operand("gain", gain, dt, (h,), index), _operand("rstd", rstd, torch.float32, (T,), index)
    xp, dx = _output("dx", dx, d_out, index)
    if gain is not None and dgain is None:
        dgain = torch.empty_like(gain)
    wp, n = None, 0
    if dgain is not None:
        n = _norm_workspace(T, h, index)
        ws = d_out.new_empty(n, dtype=torch.uint8)
        wp = ws.data_ptr()
    _check(load_library().moe_add_rmsnorm_backward(d_out.data_ptr(), ep, sp, tp, gp, T, h, DTYPES[dt], xp,
                                                   _operand("dgain", dgain, dt, (h,), index), wp, n, st))
    return dx, dgain


@functools.lru_cache(maxsize=256)
def _ffn_bytes(T: int, h: int, f: int, index: int):
    """(saved, forward workspace, backward workspace) in bytes on this device, which is current."""
    lib = load_library()
    return (int(lib.moe_ffn_saved_bytes(T, f)), int(lib.moe_ffn_forward_workspace(T, h, f)),
            int(lib.moe_ffn_backward_workspace(T, h, f)))


@functools.lru_cache(maxsize=256)
def _saved_bytes(T: int, f: int) -> int:
    return int(load_library().moe_ffn_saved_bytes(T, f))


def ffn_saved(T: int, f: int, device) -> torch.Tensor:
    """A buffer for what ``ffn_forward`` saves for ``ffn_backward`` (``moe_ffn_saved_bytes``)."""
    return torch.empty(_saved_bytes(T, f), dtype=torch.uint8, device=device)


def ffn_forward(x, W1, W3, W2, residual=None, y=None, saved=None, stream=None):
    """``moe_ffn_forward``: y = (silu(x W1^T) * (x W3^T)) W2^T [+ residual], bf16 or fp16.

    x, residual, y [T, h], W1, W3 [f, h], W2 [h, f].  ``saved``: a buffer of ``ffn_saved`` where
    ``ffn_backward`` is to follow.  Returns y."""
    return _on_device_of(x, 2, stream, _ffn_forward, x, W1, W3, W2, residual, y, saved)


def _ffn_sizes(x, W1):
    if not (isinstance(W1, torch.Tensor) and W1.dim() == 2):
        raise MoeError(-1, "W1 must be a matrix [f, h]")
    return x.shape[0], x.shape[1], W1.shape[0]


def _ffn_forward(index, st, x, W1, W3, W2, residual, y, saved):
    T, h, f = _ffn_sizes(x, W1)
    dt, shape = x.dtype, x.shape
    w1, w3 = _operand("W1", W1, dt, (f, h), index), _operand("W3", W3, dt, (f, h), index)
    w2, rp = _operand("W2", W2, dt, (h, f), index), _operand("residual", residual, dt, shape, index)
    n_saved, n, _ = _ffn_bytes(T, h, f, index)
    sp = _operand("saved", saved, torch.uint8, (n_saved,), index)
    yp, y = _output("y", y, x, index)
    ws = x.new_empty(n, dtype=torch.uint8)
    _check(load_library().moe_ffn_forward(x.data_ptr(), w1, w3, w2, rp, T, h, f, DTYPES[dt], yp, sp, ws.data_ptr(), n, st))
    return y


def ffn_backward(d_y, x, W1, W3, W2, saved, dx=None, dW1=None, dW3=None, dW2=None, stream=None):
    """``moe_ffn_backward``: gradients of ``ffn_forward`` from d_y and its ``saved`` buffer.
    Returns (dx, dW1, dW3, dW2); the residual's gradient is d_y itself."""
    return _on_device_of(x, 2, stream, _ffn_backward, d_y, x, W1, W3, W2, saved, dx, dW1, dW3, dW2)


def _ffn_backward(index, st, d_y, x, W1, W3, W2, saved, dx, dW1, dW3, dW2):
    T, h, f = _ffn_sizes(x, W1)
    dt, shape = x.dtype, x.shape
    dp = _operand("d_y", d_y, dt, shape, index)
    w1, w3 = _operand("W1", W1, dt, (f, h), index), _operand("W3", W3, dt, (f, h), index)
    n_saved, _, n = _ffn_bytes(T, h, f, index)
    w2, sp = _operand("W2", W2, dt, (h, f), index), _operand("saved", saved, torch.uint8, (n_saved,), index)
    (xp, dx), (p1, dW1) = _output("dx", dx, x, index), _output("dW1", dW1, W1, index)
    (p3, dW3), (p2, dW2) = _output("dW3", dW3, W3, index), _output("dW2", dW2, W2, index)
    ws = x.new_empty(n, dtype=torch.uint8)
    _check(load_library().moe_ffn_backward(dp, x.data_ptr(), w1, w3, w2, sp, T, h, f, DTYPES[dt], xp, p1, p3, p2,
                                           ws.data_ptr(), n, st))
    return dx, dW1, dW3, dW2


def operators_status(device=None) -> int:
    """``moe_operators_status`` of a device (None: the current one)."""
    with torch.cuda.device(device):
        return int(load_library().moe_operators_status())


def stack_forward(layers, x, betas=None, eps: float = 1e-5, y=None):
    """``moe_stack_forward``: x_{l+1} = x_l + MoE_l(RMSNorm(x_l)) over ``layers``."""
    T, h = x.shape
    _dev_bf16(x)
    if y is None:
        y = torch.empty_like(x)
    n = len(layers)
    arr = (ctypes.c_void_p * n)(*[l._h for l in layers])
    b = None
    if betas is not None:
        b = (ctypes.c_float * n)(*[float(v) for v in betas])
    _check(load_library().moe_stack_forward(arr, n, x.data_ptr(), T, b, eps, y.data_ptr()))
    return y
