"""ctypes binding over libhilberta.so: same names as the C ABI, marshalling only.

Tensors are torch CUDA tensors used as plain device memory; every step of the
path runs inside the library's kernels.  If the shared library is missing or
fails to load, every call raises -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhilberta.so")

OK = 0
ERR_INVALID, ERR_UNSUPPORTED, ERR_ARCH, ERR_CUDA, ERR_NOMEM, ERR_BUFFER, ERR_UNBOUND, ERR_TIMEOUT = (
    -1, -2, -3, -4, -5, -6, -7, -8)
BF16, FP32, FP8_E4M3 = 0, 1, 2
(EXPORT_HIL_D2T, EXPORT_HIL_T2D, EXPORT_PHYS2ORIG, EXPORT_ORIG2PHYS, EXPORT_SHARED_RUNS, EXPORT_WINDOWS,
 EXPORT_NNZ, EXPORT_INFO, EXPORT_LAUNCH_CLOCK, EXPORT_CUTS) = range(10)

# every symbol include/hilberta.h declares
SYMBOLS = (
    "hilberta_plan", "hilberta_plan_groups", "hilberta_plan_video", "hilberta_plan_destroy", "hilberta_trim",
    "hilberta_plan_export",
    "hilberta_plan_bind",
    "hilberta_forward", "hilberta_forward_unpermute", "hilberta_forward_fused", "hilberta_forward_lse",
    "hilberta_backward",
    "hilberta_backward_static", "hilberta_permute",
    "hilberta_unpermute",
    "hilberta_forward_host",
    "hilberta_layer_norm", "hilberta_layer_norm_backward", "hilberta_layer_norm_workspace", "hilberta_layer_norm_status",
    "hilberta_rotary", "hilberta_rotary_backward", "hilberta_rotary_frequencies",
    "hilberta_packed_forward", "hilberta_packed_backward", "hilberta_packed_workspace", "hilberta_packed_status",
    "hilberta_check_work_list", "hilberta_check_overlap", "hilberta_schedule_units", "hilberta_cut_schedule",
    "hilberta_check_shares",
    "hilberta_plan_status", "hilberta_selftest_timeout", "hilberta_selftest_layer_norm_timeout", "hilberta_launch_count", "hilberta_status_string", "hilberta_version",
    "hilberta_last_cuda_error",
)

ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BASE, ROTARY_BANDS = range(4)

_lib = None


class HilbertaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().hilberta_status_string(status).decode()
        if status == ERR_CUDA:
            msg += f" (cudaError {lib().hilberta_last_cuda_error()})"
        super().__init__(f"{where}: {msg} [{status}]")


def lib():
    """Load the C-ABI library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2509_26538_b200.build` "
            "(there is no CPU or PyTorch fallback)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    L.hilberta_plan.argtypes = [i32] * 6 + [ctypes.POINTER(vp)]
    L.hilberta_plan.restype = i32
    L.hilberta_plan_groups.argtypes = [i32] * 6 + [ctypes.POINTER(vp)]
    L.hilberta_plan_groups.restype = i32
    L.hilberta_plan_video.argtypes = [i32] * 8 + [ctypes.POINTER(vp)]
    L.hilberta_plan_video.restype = i32
    L.hilberta_plan_destroy.argtypes = [vp]
    L.hilberta_plan_destroy.restype = i32
    L.hilberta_trim.argtypes = []
    L.hilberta_trim.restype = sz
    L.hilberta_plan_export.argtypes = [vp, i32, vp, sz, ctypes.POINTER(sz)]
    L.hilberta_plan_export.restype = i32
    L.hilberta_plan_bind.argtypes = [vp, i32, i32, i32, i32, i64, i64, i64, f32]
    L.hilberta_plan_bind.restype = i32
    L.hilberta_forward.argtypes = [vp, vp, vp, vp, vp, vp]
    L.hilberta_forward.restype = i32
    L.hilberta_forward_unpermute.argtypes = [vp, vp, vp, vp, vp, vp]
    L.hilberta_forward_unpermute.restype = i32
    L.hilberta_forward_fused.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp]
    L.hilberta_forward_fused.restype = i32
    L.hilberta_forward_lse.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    L.hilberta_forward_lse.restype = i32
    L.hilberta_backward.argtypes = [vp] * 11
    L.hilberta_backward.restype = i32
    L.hilberta_backward_static.argtypes = [vp] * 11
    L.hilberta_backward_static.restype = i32
    L.hilberta_forward_host.argtypes = [vp, vp, vp, vp, vp, vp]
    L.hilberta_forward_host.restype = i32
    for name in ("hilberta_permute", "hilberta_unpermute"):
        f = getattr(L, name)
        f.argtypes = [vp, vp, vp, i32, i32, i32, vp]
        f.restype = i32
    L.hilberta_layer_norm.argtypes = [vp] * 6 + [i64, i32] + [i64] * 4 + [i32] * 3 + [f32, vp]
    L.hilberta_layer_norm.restype = i32
    L.hilberta_layer_norm_backward.argtypes = [vp] * 9 + [sz, i64, i32] + [i64] * 6 + [i32] * 3 + [vp]
    L.hilberta_layer_norm_backward.restype = i32
    L.hilberta_layer_norm_workspace.argtypes = [i64, i32, i64]
    L.hilberta_layer_norm_workspace.restype = sz
    L.hilberta_layer_norm_status.argtypes = []
    L.hilberta_layer_norm_status.restype = i32
    L.hilberta_selftest_layer_norm_timeout.argtypes = [vp]
    L.hilberta_selftest_layer_norm_timeout.restype = i32
    f64 = ctypes.c_double
    for name in ("hilberta_rotary", "hilberta_rotary_backward"):
        f = getattr(L, name)
        f.argtypes = [vp] * 5 + [i32] * 3 + [f64, vp] + [i32] * 5 + [vp, i64, vp]
        f.restype = i32
    L.hilberta_rotary_frequencies.argtypes = [vp, i32, f64, i32, f64, f64, f64, f64, vp]
    L.hilberta_rotary_frequencies.restype = i32
    L.hilberta_packed_forward.argtypes = [vp] * 6 + [i32] * 6 + [vp, i32, f32, vp]
    L.hilberta_packed_forward.restype = i32
    L.hilberta_packed_backward.argtypes = [vp] * 10 + [sz, vp] + [i32] * 6 + [vp, i32, f32, vp]
    L.hilberta_packed_backward.restype = i32
    L.hilberta_packed_workspace.argtypes = [i32, i32]
    L.hilberta_packed_workspace.restype = sz
    L.hilberta_packed_status.argtypes = []
    L.hilberta_packed_status.restype = i32
    L.hilberta_check_work_list.argtypes = [vp, i32, i32, i32, i32]
    L.hilberta_check_work_list.restype = i32
    i64, u64 = ctypes.c_int64, ctypes.c_uint64
    L.hilberta_check_overlap.argtypes = [u64, u64, i32, i32, i32, i64, i64, i64, i64]
    L.hilberta_check_overlap.restype = i32
    L.hilberta_schedule_units.argtypes = [i32, vp, vp, i32, i32, vp, vp, vp]
    L.hilberta_schedule_units.restype = i32
    L.hilberta_cut_schedule.argtypes = [vp, i32, vp, vp, i32, i32, vp, i32, i64, vp, vp, vp, i32, vp, vp]
    L.hilberta_cut_schedule.restype = i32
    L.hilberta_check_shares.argtypes = [vp, i32, vp, i32, i32]
    L.hilberta_check_shares.restype = i32
    L.hilberta_selftest_timeout.argtypes = [vp, vp]
    L.hilberta_selftest_timeout.restype = i32
    L.hilberta_plan_status.argtypes = [vp]
    L.hilberta_plan_status.restype = i32
    L.hilberta_launch_count.argtypes = []
    L.hilberta_launch_count.restype = ctypes.c_uint64
    L.hilberta_status_string.argtypes = [i32]
    L.hilberta_status_string.restype = ctypes.c_char_p
    L.hilberta_version.argtypes = []
    L.hilberta_version.restype = i32
    L.hilberta_last_cuda_error.argtypes = []
    L.hilberta_last_cuda_error.restype = i32
    _lib = L
    return L


def check_work_list(items, S: int, item_rows: int, block: int) -> int:
    """Status of hilberta_check_work_list for an [n, 10] int32 array of work items (host only)."""
    a = np.ascontiguousarray(items, dtype=np.int32).reshape(-1, 10)
    return int(lib().hilberta_check_work_list(a.ctypes.data, a.shape[0], int(S), int(item_rows), int(block)))


def check_overlap(a: int, b: int, batch: int, heads: int, S: int, stride_b: int, stride_h: int, stride_s: int,
                  row_bytes: int) -> bool:
    """hilberta_check_overlap: do two [batch, heads, S, row] tensors with these byte strides share a byte? (host only)"""
    return bool(lib().hilberta_check_overlap(int(a), int(b), int(batch), int(heads), int(S), int(stride_b),
                                             int(stride_h), int(stride_s), int(row_bytes)))


def schedule_units(cost, cost_two_heads, bh: int, n_cta: int):
    """hilberta_schedule_units (host only): (units [n, 3] int32, cta_begin [n_cta + 1] int32, largest load)."""
    c1 = np.ascontiguousarray(cost, dtype=np.int64)
    c2 = None if cost_two_heads is None else np.ascontiguousarray(cost_two_heads, dtype=np.int64)
    units = np.full((max(len(c1) * int(bh), 1), 3), -7, dtype=np.int32)
    begin = np.zeros(int(n_cta) + 1, dtype=np.int32)
    load = ctypes.c_int64(0)
    _check(lib().hilberta_schedule_units(len(c1), c1.ctypes.data, None if c2 is None else c2.ctypes.data, int(bh), int(n_cta),
                                         units.ctypes.data, begin.ctypes.data, ctypes.addressof(load)), "hilberta_schedule_units")
    return units[:begin[-1]], begin, int(load.value)


def cut_schedule(items, cost, cost_two_heads, bh: int, sm_count: int, clusters, block: int, merge_extra: int = 0):
    """hilberta_cut_schedule (host only): (cluster, cut items, CTAs, shares [cut items * cluster, 10], units [n, 3],
    cta_begin [CTAs + 1], largest load)."""
    a = np.ascontiguousarray(items, dtype=np.int32).reshape(-1, 10)
    n = a.shape[0]
    c1 = np.ascontiguousarray(cost, dtype=np.int64)
    c2 = None if cost_two_heads is None else np.ascontiguousarray(cost_two_heads, dtype=np.int64)
    cl = np.ascontiguousarray(clusters, dtype=np.int32)
    chosen, shares = np.zeros(3, dtype=np.int32), np.zeros((8 * n, 10), dtype=np.int32)
    units, begin = np.zeros((8 * n * int(bh), 3), dtype=np.int32), np.zeros(int(sm_count) + 1, dtype=np.int32)
    load = ctypes.c_int64(0)
    _check(lib().hilberta_cut_schedule(a.ctypes.data, n, c1.ctypes.data, None if c2 is None else c2.ctypes.data, int(bh),
                                       int(sm_count), cl.ctypes.data, int(block), int(merge_extra), chosen.ctypes.data,
                                       shares.ctypes.data, units.ctypes.data, len(units), begin.ctypes.data,
                                       ctypes.addressof(load)), "hilberta_cut_schedule")
    cluster, cut, n_cta = (int(x) for x in chosen)
    return cluster, cut, n_cta, shares[:cut * cluster], units[:begin[n_cta]], begin[:n_cta + 1], int(load.value)


def check_shares(items, shares, cluster: int, block: int) -> int:
    """Status of hilberta_check_shares for [n, 10] items and their [n * cluster, 10] shares (host only)."""
    a = np.ascontiguousarray(items, dtype=np.int32).reshape(-1, 10)
    b = np.ascontiguousarray(shares, dtype=np.int32).reshape(-1, 10)
    if len(b) != len(a) * int(cluster):
        raise ValueError("cluster shares for every item")
    return int(lib().hilberta_check_shares(a.ctypes.data, len(a), b.ctypes.data, int(cluster), int(block)))


def _check(status: int, where: str):
    if status != OK:
        raise HilbertaError(status, where)


_codes = {}   # torch dtype -> code, filled by the first call (torch is imported by whoever has tensors)


def _dtype_code(t) -> int:
    if not _codes:
        import torch
        _codes.update({torch.bfloat16: BF16, torch.float32: FP32, torch.float8_e4m3fn: FP8_E4M3})
    code = _codes.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return code


def _current_stream_ptr() -> int:
    """The handle of torch's current stream on the current device.  Asking for the bare handle takes 0.3 us;
    torch.cuda.current_stream() builds a Stream object around it, 3.4 us of a call of 8."""
    global _current_stream_ptr
    import torch
    ptr = int(torch.cuda.current_stream().cuda_stream)   # initialises torch's side of CUDA if need be
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is not None and device is not None and raw(device()) == ptr:
        _current_stream_ptr = lambda: raw(device())
    else:
        _current_stream_ptr = lambda: int(torch.cuda.current_stream().cuda_stream)
    return ptr


def _stream_ptr(stream) -> int:
    return _current_stream_ptr() if stream is None else int(stream.cuda_stream)


_EXPORT_NP = {
    EXPORT_HIL_D2T: (np.int32, None), EXPORT_HIL_T2D: (np.int32, None),
    EXPORT_PHYS2ORIG: (np.int32, None), EXPORT_ORIG2PHYS: (np.int32, None),
    EXPORT_SHARED_RUNS: (np.int32, 2), EXPORT_WINDOWS: (np.int32, 5),
    EXPORT_NNZ: (np.uint64, None), EXPORT_INFO: (np.int32, None), EXPORT_LAUNCH_CLOCK: (np.int32, None),
    EXPORT_CUTS: (np.int32, 3),
}


class Plan:
    """Owner of a hilberta_plan_t*.  Methods mirror the C entry points."""

    def __init__(self, H, W, tile, layer_offset, shared_region, n_text, groups=0, frames=1, shared_frames=0):
        """tile > 0: hilberta_plan; groups > 0 (tile ignored): hilberta_plan_groups;
        frames > 1: hilberta_plan_video (a frames x H x W volume)."""
        self._h = ctypes.c_void_p()
        if frames > 1:
            _check(lib().hilberta_plan_video(int(frames), int(H), int(W), int(tile), int(layer_offset),
                                             int(shared_region), int(shared_frames), int(n_text),
                                             ctypes.byref(self._h)), "hilberta_plan_video")
        elif groups:
            _check(lib().hilberta_plan_groups(int(H), int(W), int(groups), int(layer_offset), int(shared_region),
                                              int(n_text), ctypes.byref(self._h)), "hilberta_plan_groups")
        else:
            _check(lib().hilberta_plan(int(H), int(W), int(tile), int(layer_offset), int(shared_region),
                                       int(n_text), ctypes.byref(self._h)), "hilberta_plan")
        self.H, self.W, self.tile, self.n_text = int(H), int(W), int(tile), int(n_text)
        self.S = int(n_text) + int(frames) * int(H) * int(W)
        self._bound = None

    @property
    def handle(self) -> int:
        return self._h.value

    def destroy(self):
        if self._h is not None and self._h.value:
            lib().hilberta_plan_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def export(self, what: int) -> np.ndarray:
        need = ctypes.c_size_t()
        _check(lib().hilberta_plan_export(self._h, what, None, 0, ctypes.byref(need)), "hilberta_plan_export")
        dt, cols = _EXPORT_NP[what]
        buf = np.empty(need.value // np.dtype(dt).itemsize, dtype=dt)
        _check(lib().hilberta_plan_export(self._h, what, buf.ctypes.data, buf.nbytes, None),
               "hilberta_plan_export")
        return buf.reshape(-1, cols) if cols else buf

    def bind(self, batch, heads, head_dim, dtype, strides=(0, 0, 0), scale=0.0):
        _check(lib().hilberta_plan_bind(self._h, int(batch), int(heads), int(head_dim), int(dtype),
                                        int(strides[0]), int(strides[1]), int(strides[2]), float(scale)),
               "hilberta_plan_bind")
        self._bound = (int(batch), int(heads), int(head_dim), int(dtype), tuple(int(s) for s in strides))

    def bind_like(self, t, scale=0.0):
        """Bind to the shape and strides of a [B, heads, S, D] tensor."""
        B, Hh, S, D = t.shape
        if S != self.S or t.stride(3) != 1:
            raise ValueError("tensor does not match the plan")
        strides = (t.stride(0), t.stride(1), t.stride(2))
        if t.is_contiguous():
            strides = (0, 0, 0)
        self.bind(B, Hh, D, _dtype_code(t), strides, scale)

    def forward(self, q, k, v, out, stream=None):
        _check(lib().hilberta_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), self._h,
                                      _stream_ptr(stream)), "hilberta_forward")
        return out

    def forward_unpermute(self, q, k, v, out, stream=None):
        """Forward whose output lands in ORIGINAL token order (exit gather fused in)."""
        _check(lib().hilberta_forward_unpermute(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                                self._h, _stream_ptr(stream)), "hilberta_forward_unpermute")
        return out

    def forward_fused(self, q, k, v, out, in_original=True, out_original=True, stream=None):
        """Forward with the entry gather (q, k, v in ORIGINAL order) and / or the exit gather fused in."""
        _check(lib().hilberta_forward_fused(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), self._h,
                                            int(bool(in_original)), int(bool(out_original)), _stream_ptr(stream)),
               "hilberta_forward_fused")
        return out

    def forward_lse(self, q, k, v, out, lse, stream=None):
        """Forward that also writes the per-row log-sum-exp (fp32 [B, heads, S], physical order)."""
        _check(lib().hilberta_forward_lse(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                          lse.data_ptr(), self._h, _stream_ptr(stream)), "hilberta_forward_lse")
        return out, lse

    def backward(self, dout, q, k, v, out, lse, dq, dk, dv, stream=None):
        """dq, dk, dv from dout and the forward's inputs, output and lse (all physical order, bf16)."""
        _check(lib().hilberta_backward(dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                       lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), self._h,
                                       _stream_ptr(stream)), "hilberta_backward")
        return dq, dk, dv

    def backward_static(self, dout, q, k, v, out, lse, dq, dk, dv, stream=None):
        """backward() with the scratch in the library's fixed array: no allocation in the call."""
        _check(lib().hilberta_backward_static(dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                              out.data_ptr(), lse.data_ptr(), dq.data_ptr(), dk.data_ptr(),
                                              dv.data_ptr(), self._h, _stream_ptr(stream)),
               "hilberta_backward_static")
        return dq, dk, dv

    def forward_host(self, q, k, v, out, stream=None):
        """q, k, v, out: HOST tensors (pinned for asynchronous copies), original order."""
        for t in (q, k, v, out):
            if t.is_cuda or not t.is_contiguous():
                raise ValueError("forward_host wants contiguous host tensors")
        _check(lib().hilberta_forward_host(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), self._h,
                                           _stream_ptr(stream)), "hilberta_forward_host")
        return out

    def _gather(self, fn, name, src, dst, stream):
        if src.shape != dst.shape or src.dtype != dst.dtype:
            raise ValueError("src and dst must match")
        if not (src.is_contiguous() and dst.is_contiguous()):
            raise ValueError("contiguous tensors only")
        if src.dim() < 2 or src.shape[-2] != self.S:
            raise ValueError("expected [..., S, row_elems]")
        batch = 1
        for s in src.shape[:-2]:
            batch *= int(s)
        _check(fn(src.data_ptr(), dst.data_ptr(), self._h, batch, int(src.shape[-1]), _dtype_code(src),
                  _stream_ptr(stream)), name)
        return dst

    def permute(self, src, dst, stream=None):
        return self._gather(lib().hilberta_permute, "hilberta_permute", src, dst, stream)

    def unpermute(self, src, dst, stream=None):
        return self._gather(lib().hilberta_unpermute, "hilberta_unpermute", src, dst, stream)

    def status(self) -> int:
        return int(lib().hilberta_plan_status(self._h))


def hilberta_plan(H, W, tile, layer_offset, shared_region, n_text) -> Plan:
    return Plan(H, W, tile, layer_offset, shared_region, n_text)


def hilberta_forward(q, k, v, out, plan: Plan, stream=None):
    return plan.forward(q, k, v, out, stream)


def hilberta_permute(src, dst, plan: Plan, stream=None):
    return plan.permute(src, dst, stream)


def hilberta_unpermute(src, dst, plan: Plan, stream=None):
    return plan.unpermute(src, dst, stream)


# ---- operators of the block around the attention ---------------------------------------------------------------
# These calls take a few microseconds on the device, so their checks are written to cost little on the host.

_I64x6, _I64x8, _I64x16 = ctypes.c_int64 * 6, ctypes.c_int64 * 8, ctypes.c_int64 * 16


def _current_device() -> int:
    global _current_device
    import torch
    device = int(torch.cuda.current_device())   # initialises torch's side of CUDA if need be
    _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    return device


def _here(*tensors):
    """The tensors live on the current CUDA device (the library launches there)."""
    device = _current_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"tensor on {t.device}, the current device is cuda:{device}")


def _scratch(n, like, stream):
    """n bytes of torch's memory that belong to the stream of the call, so that they are reused in its order."""
    import torch
    if stream is None:
        return like.new_empty(n, dtype=torch.uint8)
    with torch.cuda.stream(stream):
        return like.new_empty(n, dtype=torch.uint8)


def _given(workspace):
    """Bytes of a workspace that the caller brings: the library takes them as one run."""
    if not workspace.is_contiguous():
        raise ValueError("workspace: contiguous")
    return workspace.nbytes


def _zero(t, stream):
    import torch
    if stream is None:
        t.zero_()
    else:
        with torch.cuda.stream(stream):
            t.zero_()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _row_stride(t, name):
    """The row stride of a [..., cols] tensor whose leading axes are one."""
    shape = t.shape
    if t.is_contiguous():
        return shape[-1]
    if t.dim() < 1 or (shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name}: the last axis has to be contiguous")
    rows, stride = 1, 0
    for n, st in zip(reversed(shape[:-1]), reversed(t.stride()[:-1])):
        if n == 1:
            continue
        if rows > 1 and st != rows * stride:
            raise ValueError(f"{name}: rows have to be evenly spaced")
        if rows == 1:
            stride = st
        rows *= n
    return stride if rows > 1 else shape[-1]


def _same_rows(a, b):
    """Do two tensors of one shape lie alike?  An axis of one element has any stride."""
    return all(n == 1 or i == j for n, i, j in zip(a.shape, a.stride(), b.stride()))


def _norm_weights(x, a, b):
    """(rows per group, row stride, dtype code) of weight and bias, or of their gradients: [cols] or [groups, cols]."""
    w = b if a is None else a
    if w is None:
        return 0, 0, _dtype_code(x)
    shape, stride, xshape = w.shape, w.stride(), x.shape
    cols = xshape[-1]
    if a is not None and b is not None and (b.shape != shape or b.dtype != w.dtype or (b.stride() != stride and not _same_rows(a, b))):
        raise ValueError("weight and bias (and their gradients): one shape, dtype and row stride")
    if shape[-1] != cols or (stride[-1] != 1 and cols > 1):
        raise ValueError("weights are [cols] or [groups, cols], the last axis contiguous")
    if len(shape) == 1:
        return 0, cols, _dtype_code(w)
    if len(shape) != 2 or len(xshape) < 2 or shape[0] != xshape[0]:
        raise ValueError("weights of a group of rows are [x.shape[0], cols]")
    groups = shape[0]
    per = x.numel() // (cols * groups) if groups and cols else 0
    return (0 if groups == 1 else per), stride[0], _dtype_code(w)


def _statistics(rows, device, *tensors):
    for t in tensors:
        if t is not None and (t.numel() != rows or _dtype_code(t) != FP32 or not t.is_contiguous() or t.get_device() != device):
            raise ValueError("mean and rstd: contiguous fp32 on the current device, one element for each row of x")


def layer_norm(x, weight, bias, y, mean=None, rstd=None, eps=1e-6, unit_offset=False, stream=None):
    """y = (x - mean) * rstd * (weight [+ 1]) + bias over the last axis of x [..., cols].

    weight, bias: None, [cols], or [x.shape[0], cols] (one row per sample).  mean, rstd: None or fp32 [...] to be
    written for layer_norm_backward.  y may be x."""
    shape = x.shape
    if y.shape != shape or y.dtype != x.dtype:
        raise ValueError("x and y must match")
    cols = shape[-1]
    sx = cols if x.is_contiguous() else _row_stride(x, "x")
    sy = cols if y.is_contiguous() else _row_stride(y, "y")
    rows = x.numel() // cols if cols else 0
    per, sw, wcode = _norm_weights(x, weight, bias)
    _here(x, y, weight, bias)
    _statistics(rows, x.get_device(), mean, rstd)
    status = lib().hilberta_layer_norm(x.data_ptr(), None if weight is None else weight.data_ptr(), None if bias is None else bias.data_ptr(),
                                       y.data_ptr(), None if mean is None else mean.data_ptr(), None if rstd is None else rstd.data_ptr(),
                                       rows, cols, per, sx, sy, sw, _dtype_code(x), wcode, 1 if unit_offset else 0, eps,
                                       _current_stream_ptr() if stream is None else int(stream.cuda_stream))
    if status:
        _check(status, "hilberta_layer_norm")
    return y, mean, rstd


def layer_norm_workspace(x, weight=None) -> int:
    """Bytes of workspace that layer_norm_backward needs for x and weight (or one of their gradients)."""
    cols = x.shape[-1]
    return int(lib().hilberta_layer_norm_workspace(x.numel() // max(cols, 1), cols, _norm_weights(x, weight, None)[0]))


def layer_norm_backward(dy, x, weight, mean, rstd, dx, dweight, dbias, unit_offset=False, workspace=None, stream=None):
    """Gradients of layer_norm into dx, dweight, dbias (any may be None, not all).  workspace: None (taken from torch's
    allocator) or a uint8 tensor of layer_norm_workspace() bytes."""
    shape, dtype = x.shape, x.dtype
    if dy.shape != shape or dy.dtype != dtype or (dx is not None and (dx.shape != shape or dx.dtype != dtype)):
        raise ValueError("dy, x and dx must match")
    if mean is None or rstd is None:
        raise ValueError("mean and rstd of the forward pass are needed")
    cols = shape[-1]
    sx = cols if x.is_contiguous() else _row_stride(x, "x")
    sdy = cols if dy.is_contiguous() else _row_stride(dy, "dy")
    sdx = cols if dx is None or dx.is_contiguous() else _row_stride(dx, "dx")
    rows = x.numel() // cols if cols else 0
    per, sw, wcode = _norm_weights(x, weight, None)
    L, sdw, ws_bytes = lib(), 0, 0 if workspace is None else _given(workspace)
    if dweight is not None or dbias is not None:
        gper, sdw, gcode = _norm_weights(x, dweight, dbias)
        if weight is not None and (gper != per or gcode != wcode):
            raise ValueError("a weight and its gradient: one shape and dtype")
        per, wcode = gper, gcode
        if workspace is None:
            ws_bytes = L.hilberta_layer_norm_workspace(rows, cols, per)
            if ws_bytes:
                workspace = _scratch(ws_bytes, x, stream)
    _here(x, dy, weight, dx, dweight, dbias, workspace)
    _statistics(rows, x.get_device(), mean, rstd)
    status = L.hilberta_layer_norm_backward(dy.data_ptr(), x.data_ptr(), _ptr(weight), mean.data_ptr(), rstd.data_ptr(), _ptr(dx),
                                            _ptr(dweight), _ptr(dbias), _ptr(workspace), ws_bytes,
                                            rows, cols, per, sdy, sx, sdx, sw, sdw, _dtype_code(x), wcode, 1 if unit_offset else 0,
                                            _stream_ptr(stream))
    if status:
        _check(status, "hilberta_layer_norm_backward")
    if not rows:   # how many groups there are without a row, the library cannot tell
        for g in (dweight, dbias):
            if g is not None and g.dim() == 2:
                _zero(g, stream)
    return dx, dweight, dbias


def layer_norm_status() -> int:
    """0, or ERR_TIMEOUT if a wait inside a backward kernel of the layer norm has given up since the last call; synchronises."""
    return int(lib().hilberta_layer_norm_status())


def rotary_frequencies(pairs, base=10000.0, scaling=ROTARY_PLAIN, scale=1.0, context=0.0, slow=1.0, fast=32.0):
    """(inv_freq, factor): `pairs` fp64 frequencies on the CPU and the factor that goes with them (host only)."""
    import torch
    f, factor = torch.empty(int(pairs), dtype=torch.float64), ctypes.c_double(1.0)
    _check(lib().hilberta_rotary_frequencies(f.data_ptr(), int(pairs), float(base), int(scaling), float(scale), float(context),
                                             float(slow), float(fast), ctypes.addressof(factor)), "hilberta_rotary_frequencies")
    return f, factor.value


_host_types = []   # torch's fp64 and int32, filled by the first call


def _rotary(fn, name, x, out, inv_freq, positions, axis, interleaved, factor, plan, stream):
    if not _host_types:
        import torch
        _host_types.extend((torch.float64, torch.int32))
    f64, int32 = _host_types
    shape, dtype = x.shape, x.dtype
    if len(shape) != 4 or out.shape != shape or out.dtype != dtype:
        raise ValueError("x and out: [batch, heads, S, head_dim], one shape and dtype")
    B, H, S, D = shape
    xb, xh, xs, xd = x.stride()
    ob, oh, os_, od = out.stride()
    if (xd != 1 or od != 1) and D > 1:
        raise ValueError("the head_dim axis has to be contiguous")
    if inv_freq.dtype != f64 or inv_freq.dim() != 1 or inv_freq.is_cuda or not inv_freq.is_contiguous():
        raise ValueError("inv_freq: contiguous fp64 [pairs] on the CPU")
    axes, pos_stride, pos = 1, 0, None
    if axis is not None and (axis.dtype != int32 or axis.is_cuda or axis.shape != inv_freq.shape or not axis.is_contiguous()):
        raise ValueError("axis: contiguous int32 [pairs] on the CPU")
    device = _current_device()
    if x.get_device() != device or out.get_device() != device:
        _here(x, out)
    if positions is not None:
        if positions.dtype != int32 or not positions.is_contiguous():
            raise ValueError("positions: contiguous int32")
        if positions.get_device() != device:
            _here(positions)
        ps = positions.shape
        if axis is not None:
            if not ps:
                raise ValueError("positions: [S, axes] or [batch, S, axes]")
            axes, ps = ps[-1], ps[:-1]
        if ps == (B, S):
            pos_stride = S
        elif ps != (S,):
            raise ValueError("positions: [S] or [batch, S], with an axis for each position axis if `axis` is given")
        pos = positions.data_ptr()
    status = fn(x.data_ptr(), out.data_ptr(), pos, inv_freq.data_ptr(), None if axis is None else axis.data_ptr(), inv_freq.numel(), axes,
                1 if interleaved else 0, factor, None if plan is None else plan._h, B, H, S, D, _dtype_code(x),
                _I64x6(xb, xh, xs, ob, oh, os_), pos_stride, _current_stream_ptr() if stream is None else int(stream.cuda_stream))
    if status:
        _check(status, name)
    return out


def rotary(x, out, inv_freq, positions=None, axis=None, interleaved=False, factor=1.0, plan=None, stream=None):
    """Rotary positions on x [batch, heads, S, head_dim] into out (x itself for in place).  positions: int32 [S] or
    [batch, S], with a last axis of position axes if `axis` (int32 [pairs] on the CPU) is given; None: the token's index.
    plan: x in ORIGINAL order, out in PHYSICAL order."""
    return _rotary(lib().hilberta_rotary, "hilberta_rotary", x, out, inv_freq, positions, axis, interleaved, factor, plan, stream)


def rotary_backward(dout, dx, inv_freq, positions=None, axis=None, interleaved=False, factor=1.0, plan=None, stream=None):
    """The gradient of rotary(): dx from dout; with a plan, dout in PHYSICAL and dx in ORIGINAL order."""
    return _rotary(lib().hilberta_rotary_backward, "hilberta_rotary_backward", dout, dx, inv_freq, positions, axis, interleaved,
                   factor, plan, stream)


def _packed_args(like_q, like_k, lse, cu_seqlens):
    """(total, heads, kv_heads, head_dim) of packed tensors, those of q's shape and those of k's, and all their strides."""
    if not _host_types:
        import torch
        _host_types.extend((torch.float64, torch.int32))
    q, k = like_q[0], like_k[0]
    qs, ks, dtype, strides = q.shape, k.shape, q.dtype, []
    if len(qs) != 3 or len(ks) != 3 or qs[0] != ks[0] or qs[2] != ks[2]:
        raise ValueError("packed tensors are [total, heads, head_dim] and [total, kv_heads, head_dim]")
    T, H, D = qs
    Hk, device = ks[1], _current_device()
    for ts, shape in ((like_q, qs), (like_k, ks)):
        for t in ts:
            if t.shape != shape or t.dtype != dtype:
                raise ValueError("packed tensors must match: one shape for q's kind and one for k's, one dtype")
            if t.get_device() != device:
                _here(t)
            strides += t.stride()
    if D > 1 and strides[2::3].count(1) * 3 != len(strides):
        raise ValueError("the head_dim axis has to be contiguous")
    if T <= 1 or H == 1 or Hk == 1:   # an axis of one element has any stride
        for i in range(0, len(strides), 3):
            heads = H if i < 3 * len(like_q) else Hk
            if heads == 1:
                strides[i + 1] = (D + 7) // 8 * 8
            if T <= 1:
                strides[i] = max(heads * strides[i + 1], 8)
    if lse is not None and (lse.shape != (H, T) or _dtype_code(lse) != FP32 or not lse.is_contiguous() or lse.get_device() != device):
        raise ValueError("lse: contiguous fp32 [heads, total] on the current device")
    if cu_seqlens.dtype != _host_types[1] or cu_seqlens.dim() != 1 or not cu_seqlens.is_contiguous() or cu_seqlens.numel() < 1:
        raise ValueError("cu_seqlens: contiguous int32 [sequences + 1]")
    if cu_seqlens.get_device() != device:
        _here(cu_seqlens)
    return T, H, Hk, D, strides


def packed_forward(q, k, v, out, cu_seqlens, lse=None, causal=True, scale=0.0, stream=None):
    """Attention within each of the sequences packed along the first axis: q, out [total, heads, head_dim], k, v
    [total, kv_heads, head_dim] bf16; cu_seqlens int32 [sequences + 1] on the device; lse None or fp32 [heads, total]."""
    T, H, Hk, D, st = _packed_args((q, out), (k, v), lse, cu_seqlens)
    status = lib().hilberta_packed_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), _ptr(lse), cu_seqlens.data_ptr(),
                                           cu_seqlens.numel() - 1, T, H, Hk, D, _dtype_code(q),
                                           _I64x8(st[0], st[1], st[6], st[7], st[9], st[10], st[3], st[4]), 1 if causal else 0, scale,
                                           _stream_ptr(stream))
    if status:
        _check(status, "hilberta_packed_forward")
    return out, lse


def packed_workspace(total, heads) -> int:
    """Bytes of workspace that packed_backward needs on the current device."""
    return int(lib().hilberta_packed_workspace(int(total), int(heads)))


def packed_backward(dout, q, k, v, out, lse, dq, dk, dv, cu_seqlens, causal=True, scale=0.0, workspace=None, stream=None):
    """Gradients of packed_forward into dq, dk, dv, from dout and the forward's inputs, output and lse.  workspace: None
    (taken from torch's allocator) or a uint8 tensor of packed_workspace() bytes."""
    if lse is None:
        raise ValueError("lse of the forward pass is needed")
    ws_bytes = 0 if workspace is None else _given(workspace)
    T, H, Hk, D, st = _packed_args((dout, q, out, dq), (k, v, dk, dv), lse, cu_seqlens)
    if workspace is None:
        ws_bytes = lib().hilberta_packed_workspace(T, H)
        workspace = _scratch(ws_bytes, q, stream)
    else:
        _here(workspace)
    status = lib().hilberta_packed_backward(dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                            dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), workspace.data_ptr(), ws_bytes,
                                            cu_seqlens.data_ptr(), cu_seqlens.numel() - 1, T, H, Hk, D, _dtype_code(q),
                                            _I64x16(st[0], st[1], st[3], st[4], st[12], st[13], st[15], st[16], st[6], st[7],
                                                    st[9], st[10], st[18], st[19], st[21], st[22]), 1 if causal else 0, scale, _stream_ptr(stream))
    if status:
        _check(status, "hilberta_packed_backward")
    return dq, dk, dv


def packed_status() -> int:
    """0, or ERR_TIMEOUT if a wait inside a packed attention kernel has given up since the last call; synchronises."""
    return int(lib().hilberta_packed_status())


def trim() -> int:
    """Give back the device memory that destroyed plans and replaced bindings have left behind; returns the bytes."""
    return int(lib().hilberta_trim())


def launch_count() -> int:
    return int(lib().hilberta_launch_count())


def version() -> int:
    return int(lib().hilberta_version())
