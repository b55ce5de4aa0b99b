"""ctypes binding of libmxnorm.so: same names as the C ABI, argument marshalling only.

Every step of the hot path runs in the CUDA kernels behind the C ABI; this module only turns
torch CUDA tensors into device pointers and sizes.  There is no CPU fallback: if the compiled
library is missing the import of this module fails.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmxnorm.so")

ROUND_RCEIL_POW2, ROUND_FLOOR_OCP, ROUND_RCEIL_MAX = 0, 1, 2
SCALES_ROWMAJOR, SCALES_SWIZZLE_128x4 = 0, 1
ROPE_HALVES, ROPE_PAIRS = 0, 1
OK = 0

EXPORTS = ("mxn_scale_bytes", "mxn_status_string", "mx_cast", "rmsnorm_mxfp8_fwd", "mxnorm_fwd",
           "mxnorm_nvfp4_fwd", "mxnorm_bwd", "mxnorm_bwd_workspace_bytes", "mxnorm_fwd_host",
           "mxnorm_fwd_host_workspace_bytes", "mxnorm_bwd_noalloc", "mxnorm_bwd_noalloc_max_scratch_bytes",
           "mxn_device_timeouts", "mxn_device_timeouts_reset", "mxn_selftest_bounded_wait", "mx_cast_fp4", "rmsnorm_mxfp4_fwd", "mxnorm_mxfp4_fwd",
           "mx_cast_transposed", "rmsnorm_nvfp4_fwd", "mxn_selftest_division", "mxn_selftest_dispatch",
           "mx_cast_e5m2", "mx_cast_transposed_e5m2", "mxnorm_postround_fwd",
           "mxnorm_add_fwd", "mx_cast_nvfp4", "mxn_device_bad_indices", "mxn_device_bad_indices_reset",
           "rmsnorm_rope_fwd", "rmsnorm_rope_bwd", "rmsnorm_rope_bwd_workspace_bytes", "mxkv_append", "mxkv_attention",
           "mxkv_attention_workspace_bytes")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2603_13180_b200.build` "
        "(the MXNorm path has no fallback implementation)")

lib = ctypes.CDLL(LIB_PATH)

_vp, _i64, _i32, _f32, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
lib.mxn_scale_bytes.argtypes = [_i64, _i64, _i32]
lib.mxn_scale_bytes.restype = _sz
lib.mxn_status_string.argtypes = [_i32]
lib.mxn_status_string.restype = ctypes.c_char_p
lib.mxn_device_timeouts.argtypes = [ctypes.POINTER(ctypes.c_uint)]
lib.mxn_device_timeouts.restype = _i32
lib.mxn_device_timeouts_reset.argtypes = []
lib.mxn_device_timeouts_reset.restype = _i32
lib.mxn_selftest_bounded_wait.argtypes = [ctypes.c_uint, _vp]
lib.mxn_selftest_bounded_wait.restype = _i32
lib.mxn_selftest_division.argtypes = [ctypes.POINTER(ctypes.c_ulonglong)]
lib.mxn_selftest_division.restype = _i32
lib.mxn_selftest_dispatch.argtypes = [_i64, ctypes.POINTER(ctypes.c_longlong), ctypes.POINTER(_i64), ctypes.POINTER(_i32)]
lib.mxn_selftest_dispatch.restype = _i32
lib.mx_cast.argtypes = [_vp, _i64, _i64, _i32, _vp, _vp, _i32, _i32, _vp]
lib.rmsnorm_mxfp8_fwd.argtypes = [_vp, _vp, _i64, _i64, _i32, _f32, _vp, _vp, _vp, _i32, _i32, _vp]
lib.mxnorm_fwd.argtypes = [_vp, _vp, _i64, _i64, _i32, _i32, _f32, _f32, _vp, _vp, _vp, _i32, _i32, _vp]
lib.mxnorm_nvfp4_fwd.argtypes = [_vp, _i64, _i64, _i32, _f32, _f32, _f32, _vp, _vp, _vp, _i32, _vp]
lib.mxnorm_bwd.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _vp, _i32, _vp, _vp, _sz, _vp]
lib.mxnorm_bwd_workspace_bytes.argtypes = [_i64, _i64]
lib.mxnorm_bwd_workspace_bytes.restype = _sz
lib.mxnorm_fwd_host.argtypes = [_vp, _i64, _i64, _i32, _i32, _f32, _f32, _vp, _vp, _vp, _i32, _i32, _vp, _sz, _vp]
lib.mxnorm_fwd_host_workspace_bytes.argtypes = [_i64, _i64, _i32, _i32]
lib.mxnorm_fwd_host_workspace_bytes.restype = _sz
lib.mx_cast_fp4.argtypes = [_vp, _i64, _i64, _i32, _vp, _vp, _i32, _vp]
lib.rmsnorm_mxfp4_fwd.argtypes = [_vp, _i64, _i64, _i32, _f32, _vp, _vp, _vp, _i32, _vp]
lib.mxnorm_mxfp4_fwd.argtypes = [_vp, _i64, _i64, _i32, _i32, _f32, _f32, _vp, _vp, _vp, _i32, _vp]
lib.mxnorm_add_fwd.argtypes = [_vp, _vp, _i64, _i64, _i32, _i32, _f32, _f32, _vp, _vp, _vp, _vp, _i32, _vp]
lib.mxnorm_postround_fwd.argtypes = [_vp, _i64, _i64, _i32, _f32, _vp, _vp, _vp, _i32, _vp]
lib.mx_cast_e5m2.argtypes = [_vp, _i64, _i64, _i32, _vp, _vp, _i32, _vp]
lib.mx_cast_transposed_e5m2.argtypes = [_vp, _i64, _i64, _vp, _vp, _i32, _vp]
lib.rmsnorm_nvfp4_fwd.argtypes = [_vp, _i64, _i64, _f32, _f32, _vp, _vp, _vp, _i32, _vp]
lib.mx_cast_nvfp4.argtypes = [_vp, _i64, _i64, _f32, _vp, _vp, _i32, _vp]
lib.mx_cast_transposed.argtypes = [_vp, _vp, _i64, _i64, _f32, _vp, _vp, _i32, _i32, _vp]
lib.mxnorm_bwd_noalloc.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _vp, _i32, _vp, _vp]
lib.mxnorm_bwd_noalloc_max_scratch_bytes.argtypes = []
lib.mxnorm_bwd_noalloc_max_scratch_bytes.restype = _sz
lib.mxn_device_bad_indices.argtypes = [ctypes.POINTER(ctypes.c_uint)]
lib.mxn_device_bad_indices_reset.argtypes = []
lib.rmsnorm_rope_fwd.argtypes = [_vp, _i64, _i32, _vp, _i64, _i32, _i64, _i32, _i32, _vp, _vp, _f32, _vp, _i64, _i32, _i32, _vp,
                                 _vp, _i64, _vp, _i64, _vp]
lib.rmsnorm_rope_bwd.argtypes = [_vp, _i64, _i32, _vp, _i64, _i32, _vp, _i64, _vp, _i64, _i64, _i32, _i32, _vp, _vp, _f32, _vp, _i64,
                                 _i32, _i32, _vp, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _sz, _vp]
lib.rmsnorm_rope_bwd_workspace_bytes.argtypes = [_i64, _i32, _i32, _i32]
lib.rmsnorm_rope_bwd_workspace_bytes.restype = _sz
lib.mxkv_append.argtypes = [_vp, _i64, _vp, _i64, _i64, _i32, _i32, _vp, _i64, _vp, _vp, _i64, _i64, _i32, _i32, _vp, _i64, _i32, _i32,
                            _vp, _vp, _vp, _vp, _vp]
lib.mxkv_attention.argtypes = [_vp, _i64, _i64, _i32, _i32, _i32, _vp, _i64, _i64, _vp, _i64, _vp, _i64, _i64, _i32, _i32, _vp, _vp, _vp,
                               _vp, _f32, _i32, _i64, _vp, _i64, _vp, _vp, _sz, _vp]
lib.mxkv_attention_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, _i32, _i32, _i32]
lib.mxkv_attention_workspace_bytes.restype = _sz
for _name in ("mx_cast", "rmsnorm_mxfp8_fwd", "mxnorm_fwd", "mxnorm_nvfp4_fwd", "mxnorm_bwd", "mxnorm_fwd_host",
              "mxnorm_bwd_noalloc", "mx_cast_fp4", "rmsnorm_mxfp4_fwd", "mxnorm_mxfp4_fwd",
           "mx_cast_transposed", "rmsnorm_nvfp4_fwd", "mxn_selftest_division", "mxn_selftest_dispatch",
           "mx_cast_e5m2", "mx_cast_transposed_e5m2", "mxnorm_postround_fwd",
           "mxnorm_add_fwd", "mx_cast_nvfp4", "mxn_device_bad_indices", "mxn_device_bad_indices_reset", "rmsnorm_rope_fwd",
           "rmsnorm_rope_bwd", "mxkv_append", "mxkv_attention"):
    getattr(lib, _name).restype = _i32


class MXNormError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def status_string(status: int) -> str:
    return lib.mxn_status_string(status).decode()


def _check(status: int, where: str):
    if status != OK:
        raise MXNormError(status, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def _dev(t: torch.Tensor, dtype, name: str):
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise ValueError(f"{name}: expected a contiguous CUDA tensor of {dtype}")
    return t


def device_timeouts() -> int:
    """Synchronises the device and returns how many bounded device-side waits have run out (0 = healthy)."""
    n = ctypes.c_uint(0)
    st = lib.mxn_device_timeouts(ctypes.byref(n))
    if st not in (OK, 7):
        raise MXNormError(st, "mxn_device_timeouts")
    return int(n.value)


def device_timeouts_reset() -> None:
    """Synchronises the device and sets the count of run-out waits back to 0."""
    _check(lib.mxn_device_timeouts_reset(), "mxn_device_timeouts_reset")


def selftest_bounded_wait(polls: int = 2000, stream=None) -> None:
    """Enqueues one warp whose bounded wait (on a barrier nobody completes) must run out after `polls` polls."""
    _check(lib.mxn_selftest_bounded_wait(polls, _stream(stream)), "mxn_selftest_bounded_wait")


def selftest_division() -> int:
    """Re-checks on the current device that the division shortcuts of the NVFP4 kernels equal IEEE division;
    returns the number of mismatching quotients (0)."""
    n = ctypes.c_ulonglong(0)
    _check(lib.mxn_selftest_division(ctypes.byref(n)), "mxn_selftest_division")
    return int(n.value)


def selftest_dispatch(max_D: int = 65536):
    """Host only: (number of accepted forward shapes and options without a compiled kernel, first such D, its case
    code); the count is expected to be 0."""
    n, d, c = ctypes.c_longlong(0), _i64(0), _i32(0)
    _check(lib.mxn_selftest_dispatch(max_D, ctypes.byref(n), ctypes.byref(d), ctypes.byref(c)), "mxn_selftest_dispatch")
    return int(n.value), int(d.value), int(c.value)


def scale_bytes(T: int, K: int, layout: int = SCALES_ROWMAJOR) -> int:
    return int(lib.mxn_scale_bytes(T, K, layout))


def alloc_outputs(T: int, D: int, block: int = 32, layout: int = SCALES_ROWMAJOR, nvfp4: bool = False,
                  device="cuda"):
    """Allocates (codes, scales, rms) for one forward call (torch owns the memory)."""
    codes = torch.empty((T, D // 2 if nvfp4 else D), dtype=torch.uint8, device=device)
    scales = torch.empty((scale_bytes(T, D // block, layout),), dtype=torch.uint8, device=device)
    rms = torch.empty((T,), dtype=torch.float32, device=device)
    return codes, scales, rms


def mx_cast(x, codes, scales, block=32, round=ROUND_RCEIL_POW2, layout=SCALES_ROWMAJOR, stream=None):
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.mx_cast(_ptr(x), T, D, block, _ptr(codes), _ptr(scales), round, layout, _stream(stream)), "mx_cast")


def rmsnorm_mxfp8_fwd(x, gain, codes, scales, rms_out=None, eps=0.0, block=32, round=ROUND_RCEIL_POW2,
                      layout=SCALES_ROWMAJOR, stream=None):
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.rmsnorm_mxfp8_fwd(_ptr(x), _ptr(gain), T, D, block, eps, _ptr(codes), _ptr(scales), _ptr(rms_out),
                                 round, layout, _stream(stream)), "rmsnorm_mxfp8_fwd")


def mxnorm_fwd(x, gain, codes, scales, rms_est_out=None, p=2, coef=0.0, eps=0.0, block=32,
               round=ROUND_RCEIL_POW2, layout=SCALES_ROWMAJOR, stream=None):
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.mxnorm_fwd(_ptr(x), _ptr(gain), T, D, block, p, coef, eps, _ptr(codes), _ptr(scales),
                          _ptr(rms_est_out), round, layout, _stream(stream)), "mxnorm_fwd")


def mxnorm_nvfp4_fwd(x, codes_packed, scales_e4m3, rms_est_out=None, p=2, coef=0.0, eps=0.0, global_scale=1.0,
                     layout=SCALES_ROWMAJOR, stream=None):
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.mxnorm_nvfp4_fwd(_ptr(x), T, D, p, coef, eps, global_scale, _ptr(codes_packed), _ptr(scales_e4m3),
                                _ptr(rms_est_out), layout, _stream(stream)), "mxnorm_nvfp4_fwd")


def mxnorm_bwd_workspace_bytes(T: int, D: int) -> int:
    return int(lib.mxnorm_bwd_workspace_bytes(T, D))


def mxnorm_bwd(x, grad_out, gain, rms, dx, dgain=None, workspace=None, stream=None):
    _dev(x, torch.bfloat16, "x")
    _dev(grad_out, torch.bfloat16, "grad_out")
    T, D = x.shape
    if dx.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("dx must be bf16 or fp32")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib.mxnorm_bwd(_ptr(x), _ptr(grad_out), _ptr(gain), _ptr(rms), T, D, _ptr(dx),
                          1 if dx.dtype == torch.float32 else 0, _ptr(dgain), _ptr(workspace), ws_bytes,
                          _stream(stream)), "mxnorm_bwd")


def mxnorm_fwd_host_workspace_bytes(T: int, D: int, block: int = 32, layout: int = SCALES_ROWMAJOR) -> int:
    return int(lib.mxnorm_fwd_host_workspace_bytes(T, D, block, layout))


def mxnorm_fwd_host(x_host, codes_host, scales_host, rms_est_host, workspace, p=2, coef=0.0, eps=0.0, block=32,
                    round=ROUND_RCEIL_POW2, layout=SCALES_ROWMAJOR, stream=None):
    """Host tensors in and out (pin them for asynchronous copies); `workspace` is a CUDA uint8 tensor."""
    if x_host.is_cuda or codes_host.is_cuda or scales_host.is_cuda or x_host.dtype != torch.bfloat16:
        raise ValueError("mxnorm_fwd_host takes host tensors (bf16 input)")
    T, D = x_host.shape
    _check(lib.mxnorm_fwd_host(_ptr(x_host), T, D, block, p, coef, eps, _ptr(codes_host), _ptr(scales_host),
                               _ptr(rms_est_host), round, layout, _ptr(workspace),
                               workspace.numel() * workspace.element_size(), _stream(stream)), "mxnorm_fwd_host")


def mxnorm_bwd_noalloc(x, grad_out, gain, rms, dx, dgain=None, stream=None):
    """mxnorm_bwd for callers that cannot allocate a workspace: the dgain partial sums use an 8 MiB array
    built into the library (shared by all calls on the device - do not overlap two calls).  Raises
    MXNormError(MXN_ERR_TOO_LARGE) when the problem would need more scratch than that."""
    _dev(x, torch.bfloat16, "x")
    _dev(grad_out, torch.bfloat16, "grad_out")
    T, D = x.shape
    if dx.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("dx must be bf16 or fp32")
    _check(lib.mxnorm_bwd_noalloc(_ptr(x), _ptr(grad_out), _ptr(gain), _ptr(rms), T, D, _ptr(dx),
                                  1 if dx.dtype == torch.float32 else 0, _ptr(dgain), _stream(stream)),
           "mxnorm_bwd_noalloc")


def mx_cast_fp4(x, codes_packed, scales, block=32, layout=SCALES_ROWMAJOR, stream=None):
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.mx_cast_fp4(_ptr(x), T, D, block, _ptr(codes_packed), _ptr(scales), layout, _stream(stream)), "mx_cast_fp4")


def rmsnorm_mxfp4_fwd(x, codes_packed, scales, rms_out=None, eps=0.0, block=32, layout=SCALES_ROWMAJOR, stream=None):
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.rmsnorm_mxfp4_fwd(_ptr(x), T, D, block, eps, _ptr(codes_packed), _ptr(scales), _ptr(rms_out), layout,
                                 _stream(stream)), "rmsnorm_mxfp4_fwd")


def mxnorm_mxfp4_fwd(x, codes_packed, scales, rms_est_out=None, p=2, coef=0.0, eps=0.0, block=32,
                     layout=SCALES_ROWMAJOR, stream=None):
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.mxnorm_mxfp4_fwd(_ptr(x), T, D, block, p, coef, eps, _ptr(codes_packed), _ptr(scales), _ptr(rms_est_out),
                                layout, _stream(stream)), "mxnorm_mxfp4_fwd")


def mx_cast_transposed(x, rms, codes_t, scales_t, eps=0.0, round=ROUND_RCEIL_POW2, layout=SCALES_ROWMAJOR, stream=None):
    """Column-wise MXCast of x * (1 / (rms + eps)) (rms may be None): codes_t [D, T], scales_t [D, T/32]."""
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.mx_cast_transposed(_ptr(x), _ptr(rms), T, D, eps, _ptr(codes_t), _ptr(scales_t), round, layout,
                                  _stream(stream)), "mx_cast_transposed")


def rmsnorm_nvfp4_fwd(x, codes_packed, scales_e4m3, rms_out=None, eps=0.0, global_scale=1.0, layout=SCALES_ROWMAJOR,
                      stream=None):
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.rmsnorm_nvfp4_fwd(_ptr(x), T, D, eps, global_scale, _ptr(codes_packed), _ptr(scales_e4m3), _ptr(rms_out),
                                 layout, _stream(stream)), "rmsnorm_nvfp4_fwd")


def mx_cast_nvfp4(x, codes_packed, scales_e4m3, global_scale=1.0, layout=SCALES_ROWMAJOR, stream=None):
    """NVFP4 cast without a normaliser (e.g. of a weight): E2M1 codes two per byte, E4M3 scales per 16 elements."""
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.mx_cast_nvfp4(_ptr(x), T, D, global_scale, _ptr(codes_packed), _ptr(scales_e4m3), layout, _stream(stream)),
           "mx_cast_nvfp4")


def mx_cast_e5m2(x, codes, scales, block=32, layout=SCALES_ROWMAJOR, stream=None):
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.mx_cast_e5m2(_ptr(x), T, D, block, _ptr(codes), _ptr(scales), layout, _stream(stream)), "mx_cast_e5m2")


def mx_cast_transposed_e5m2(x, codes_t, scales_t, layout=SCALES_ROWMAJOR, stream=None):
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.mx_cast_transposed_e5m2(_ptr(x), T, D, _ptr(codes_t), _ptr(scales_t), layout, _stream(stream)),
           "mx_cast_transposed_e5m2")


def mxnorm_postround_fwd(x, codes, scales, rms_est_out=None, eps=0.0, block=32, layout=SCALES_ROWMAJOR, stream=None):
    """MXNorm with the RMS estimated from power-of-two-rounded block absmaxes (the paper's ablation)."""
    _dev(x, torch.bfloat16, "x")
    T, D = x.shape
    _check(lib.mxnorm_postround_fwd(_ptr(x), T, D, block, eps, _ptr(codes), _ptr(scales), _ptr(rms_est_out), layout,
                                    _stream(stream)), "mxnorm_postround_fwd")


def mxnorm_add_fwd(x, residual, h_out, codes, scales, rms_est_out=None, p=2, coef=0.0, eps=0.0, block=32,
                   layout=SCALES_ROWMAJOR, stream=None):
    """h_out = bf16(x + residual) and MXNorm(h_out) in one pass (h_out may be x or residual itself)."""
    _dev(x, torch.bfloat16, "x")
    _dev(residual, torch.bfloat16, "residual")
    T, D = x.shape
    _check(lib.mxnorm_add_fwd(_ptr(x), _ptr(residual), T, D, block, p, coef, eps, _ptr(h_out), _ptr(codes), _ptr(scales),
                              _ptr(rms_est_out), layout, _stream(stream)), "mxnorm_add_fwd")


# ---- queries, keys and values around attention ----

def device_bad_indices() -> int:
    """Synchronises the device and returns how many indices in device memory were found out of range (0 = healthy)."""
    n = ctypes.c_uint(0)
    st = lib.mxn_device_bad_indices(ctypes.byref(n))
    if st not in (OK, 9):
        raise MXNormError(st, "mxn_device_bad_indices")
    return int(n.value)


def device_bad_indices_reset() -> None:
    """Synchronises the device and sets the count of indices found out of range back to 0."""
    _check(lib.mxn_device_bad_indices_reset(), "mxn_device_bad_indices_reset")


def _on_current_device(stream, first, *tensors):
    """Every tensor lies on the current device (calls enqueue there); returns the raw stream to enqueue on."""
    if not first.is_cuda:
        raise ValueError(f"expected CUDA tensors, not tensors on {first.device}")
    device = torch._C._cuda_getDevice()
    if first.get_device() != device:
        raise ValueError(f"tensors are on {first.device}, the current device is cuda:{device}")
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"a tensor is on {t.device}, expected cuda:{device}")
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _heads(t, name, like=None):
    """(pointer, token stride, heads) of a bf16 [T, heads, dim] tensor whose heads are contiguous; (None, 0, 0) for None."""
    if t is None:
        return None, 0, 0
    shape = t.shape
    if t.dtype is not torch.bfloat16 or len(shape) != 3:
        raise ValueError(f"{name}: expected a bf16 tensor [tokens, heads, dim]")
    if like is not None and shape != like:
        raise ValueError(f"{name}: shape {tuple(shape)}, expected {tuple(like)}")
    n, h, d = shape
    st, sh, sd = t.stride()
    if (sd != 1 and d > 1) or (sh != d and h > 1):
        raise ValueError(f"{name}: the heads of a token must be contiguous")
    return t.data_ptr(), (st if n > 1 else h * d), h


def _vec(t, dtype, name, shape=None):
    """Pointer of a contiguous tensor (None stays None)."""
    if t is None:
        return None
    if t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor of {dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {shape}")
    return t.data_ptr()


def _workspace(t):
    """(pointer, bytes) of a workspace; its bytes lie one after another."""
    if t is None:
        return None, 0
    if not t.is_contiguous():
        raise ValueError("workspace: expected a contiguous tensor")
    return t.data_ptr(), t.numel() * t.element_size()


def _table(cos_sin):
    """(pointer, rows, rotated elements) of a rotation table fp32 [rows, rot]."""
    if cos_sin is None:
        return None, 0, 0
    if cos_sin.dim() != 2:
        raise ValueError("cos_sin: expected [positions, rot_dim]")
    return _vec(cos_sin, torch.float32, "cos_sin"), cos_sin.shape[0], cos_sin.shape[1]


def rmsnorm_rope_fwd(q, k, q_gain, k_gain, cos_sin, positions, q_out, k_out, eps=1e-6, interleaved=False, normalise=True,
                     stream=None):
    """RMS norm of every head of q [T, Hq, D] and k [T, Hk, D] (k may be None) and rotation by cos_sin [P, rot] (may be None)
    at int32 positions [T] (None: row index).  q_out / k_out may be q / k themselves."""
    raw = _on_current_device(stream, q, k, q_gain, k_gain, cos_sin, positions, q_out, k_out)
    qp, qs, qh = _heads(q, "q")
    T, _, D = shape = q.shape
    qop, qos, _ = _heads(q_out, "q_out", shape)
    if k is None:
        kp = kop = None
        ks = kos = kh = 0
    else:
        kp, ks, kh = _heads(k, "k")
        if k_out is None or k.shape != (T, kh, D):
            raise ValueError("k: expected [tokens, heads, dim] with q's tokens and dim, and a k_out")
        kop, kos, _ = _heads(k_out, "k_out", (T, kh, D))
    tp, rows, rot = _table(cos_sin)
    _check(lib.rmsnorm_rope_fwd(qp, qs, qh, kp, ks, kh, T, D, 1 if normalise else 0, _vec(q_gain, torch.bfloat16, "q_gain", (D,)),
                                _vec(k_gain, torch.bfloat16, "k_gain", (D,)), eps, tp, rows, rot, 1 if interleaved else 0,
                                _vec(positions, torch.int32, "positions", (T,)), qop, qos, kop, kos, raw), "rmsnorm_rope_fwd")


def rmsnorm_rope_bwd_workspace_bytes(T: int, q_heads: int, k_heads: int, dim: int) -> int:
    return int(lib.rmsnorm_rope_bwd_workspace_bytes(T, q_heads, k_heads, dim))


def rmsnorm_rope_bwd(q, k, grad_q, grad_k, q_gain, k_gain, cos_sin, positions, dq, dk, q_dgain=None, k_dgain=None, workspace=None,
                     eps=1e-6, interleaved=False, normalise=True, stream=None):
    """Gradient of rmsnorm_rope_fwd: grad_q / grad_k -> dq / dk (and fp32 q_dgain / k_dgain [D]); q and k are the forward's inputs
    (None with normalise=False, which does not read them)."""
    raw = _on_current_device(stream, grad_q, q, k, grad_k, q_gain, k_gain, cos_sin, positions, dq, dk, q_dgain, k_dgain, workspace)
    gqp, gqs, qh = _heads(grad_q, "grad_q")
    T, _, D = shape = grad_q.shape
    if grad_k is not None and (grad_k.shape[0] != T or grad_k.shape[2] != D or dk is None):
        raise ValueError("grad_k: expected [tokens, heads, dim] with grad_q's tokens and dim, and a dk")
    if normalise and (q is None or (k is None) != (grad_k is None)):
        raise ValueError("q / k: the forward's inputs are needed")
    gkp, gks, kh = _heads(grad_k, "grad_k")
    k_shape = (T, kh, D)
    qp, qs, _ = _heads(q, "q", shape)
    kp, ks, _ = _heads(k if kh else None, "k", k_shape)
    dqp, dqs, _ = _heads(dq, "dq", shape)
    dkp, dks, _ = _heads(dk if kh else None, "dk", k_shape)
    tp, rows, rot = _table(cos_sin)
    ws, ws_bytes = _workspace(workspace)
    _check(lib.rmsnorm_rope_bwd(qp, qs, qh, kp, ks, kh, gqp, gqs, gkp, gks, T, D, 1 if normalise else 0,
                                _vec(q_gain, torch.bfloat16, "q_gain", (D,)), _vec(k_gain, torch.bfloat16, "k_gain", (D,)), eps, tp,
                                rows, rot, 1 if interleaved else 0, _vec(positions, torch.int32, "positions", (T,)), dqp, dqs, dkp, dks,
                                _vec(q_dgain, torch.float32, "q_dgain", (D,)), _vec(k_dgain, torch.float32, "k_dgain", (D,)),
                                ws, ws_bytes, raw), "rmsnorm_rope_bwd")


def alloc_kv_cache(num_pages: int, kv_heads: int, page_size: int, dim: int, block: int = 16, device="cuda"):
    """(k_codes, k_scales, v_codes, v_scales) of an empty paged cache: E4M3 codes [pages, heads, page, dim] and one E8M0 scale for
    each `block` tokens of a head."""
    def one():
        return (torch.zeros((num_pages, kv_heads, page_size, dim), dtype=torch.uint8, device=device),
                torch.zeros((num_pages, kv_heads, page_size // block), dtype=torch.uint8, device=device))
    return one() + one()


def _cache(k_codes, k_scales, v_codes, v_scales):
    """(pages, heads, page size, dim, block) of a cache's four tensors and their pointers."""
    cs, ss = k_codes.shape, k_scales.shape
    if len(cs) != 4 or len(ss) != 3 or ss[2] < 1 or ss[:2] != cs[:2]:
        raise ValueError("cache: expected codes [pages, heads, page, dim] and scales [pages, heads, page / block]")
    pages, heads, page, dim = cs
    return (pages, heads, page, dim, page // ss[2] if page % ss[2] == 0 else 0, _vec(k_codes, torch.uint8, "k_codes"),
            _vec(k_scales, torch.uint8, "k_scales"), _vec(v_codes, torch.uint8, "v_codes", cs), _vec(v_scales, torch.uint8, "v_scales", ss))


def _sequences(cu, lens, page_table):
    """(sequences, pages a sequence) and the pointers of the three lists."""
    shape = page_table.shape
    if len(shape) != 2:
        raise ValueError("page_table: expected int32 [sequences, pages]")
    s, width = shape
    return (s, width, _vec(cu, torch.int32, "cu", (s + 1,)), _vec(lens, torch.int32, "kv_lens", (s,)),
            _vec(page_table, torch.int32, "page_table"))


def mxkv_append(k, v, cu_tokens, kv_lens, page_table, k_codes, k_scales, v_codes, v_scales, cos_sin=None, interleaved=False, stream=None):
    """Writes new tokens' keys (rotated by their place when cos_sin is given) and values [n, H, D] into the paged cache.
    kv_lens counts the new tokens; rows cu_tokens[s] .. cu_tokens[s+1]-1 are the last ones of sequence s."""
    raw = _on_current_device(stream, k, v, cu_tokens, kv_lens, page_table, k_codes, k_scales, v_codes, v_scales, cos_sin)
    pages, heads, page, dim, block, kc, ks, vc, vs = _cache(k_codes, k_scales, v_codes, v_scales)
    s, width, cup, lp, pt = _sequences(cu_tokens, kv_lens, page_table)
    kp, kst, kh = _heads(k, "k")
    shape = k.shape
    vp, vst, _ = _heads(v, "v", shape)
    n = shape[0]
    if kh != heads or shape[2] != dim:
        raise ValueError("k, v: heads and dim differ from the cache's")
    tp, rows, rot = _table(cos_sin)
    _check(lib.mxkv_append(kp, kst, vp, vst, n, heads, dim, cup, s, lp, pt, width, pages, page, block, tp, rows, rot,
                           1 if interleaved else 0, kc, ks, vc, vs, raw), "mxkv_append")


def mxkv_attention_workspace_bytes(n_tokens: int, n_seqs: int, max_q_len: int, max_kv_len: int, q_heads: int, kv_heads: int, dim: int) -> int:
    return int(lib.mxkv_attention_workspace_bytes(n_tokens, n_seqs, max_q_len, max_kv_len, q_heads, kv_heads, dim))


def mxkv_attention(q, cu_q, kv_lens, page_table, k_codes, k_scales, v_codes, v_scales, out, max_q_len, max_kv_len, scale, causal=True,
                   window=0, lse=None, workspace=None, stream=None):
    """Attention of the queries [n, Hq, D] over the paged cache; see mxkv_attention in include/mxnorm.h."""
    raw = _on_current_device(stream, q, cu_q, kv_lens, page_table, k_codes, k_scales, v_codes, v_scales, out, lse, workspace)
    pages, heads, page, dim, block, kc, ks, vc, vs = _cache(k_codes, k_scales, v_codes, v_scales)
    s, width, cup, lp, pt = _sequences(cu_q, kv_lens, page_table)
    qp, qst, qh = _heads(q, "q")
    n, _, d = shape = q.shape
    op, ost, _ = _heads(out, "out", shape)
    if d != dim:
        raise ValueError("q: dim differs from the cache's")
    ws, ws_bytes = _workspace(workspace)
    _check(lib.mxkv_attention(qp, qst, n, qh, heads, dim, cup, s, max_q_len, lp, max_kv_len, pt, width, pages, page, block, kc, ks, vc, vs,
                              scale, 1 if causal else 0, window, op, ost, _vec(lse, torch.float32, "lse", (n, qh)), ws, ws_bytes,
                              raw), "mxkv_attention")
