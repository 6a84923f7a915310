"""Thin ctypes binding of the C-ABI library ``libw2a8.so`` (see include/w2a8.h).

Argument marshalling only: every step of the path runs in the CUDA kernels of
the library.  torch supplies device memory and the current stream, nothing
else.  There is no CPU fallback: if the library is missing, ``lib()`` raises.
Function names match the C entry points.
"""
from __future__ import annotations

import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libw2a8.so")

EXPORTS = [
    "w2a8_version", "w2a8_status_string", "w2_packed_bytes", "w2_pack", "a8_quantize",
    "w2a8_workspace_bytes", "w2a8_workspace_init", "w2a8_workspace_status", "w2a8_gemm", "w2a8_gemm_partials",
    "w2a8_kernel_for", "w2a8_tensor_core_channels", "w2a8_tensor_core_ksplit", "w2a8_tensor_core_tile_tokens", "w2a8_gemm_h16", "w2a16_gemm", "w2a8_linear", "w2a8_linear_host_workspace_bytes", "w2a8_linear_host", "w2a8_gemm_static",
    "w2a8_gemm_grouped", "w2a8_linear_grouped", "w2a8_grouped_workspace_bytes", "w2a8_grouped_plan",
    "w2a8_read_probe", "w2a8_tensor_core_kind",
    "w2a8_linear_grouped_host", "w2a8_linear_grouped_host_workspace_bytes",
    "w2a8_lora_grouped", "w2a8_rope_frequencies", "w2a8_rope", "w2a8_qk_norm_rope",
]

_lib = None


class W2A8Error(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def lib() -> ctypes.CDLL:
    """Load the library once; raise if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -m paper_2508_06753_b200.build` "
                "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        L.w2a8_version.restype = i
        L.w2a8_status_string.restype = ctypes.c_char_p
        L.w2a8_status_string.argtypes = [i]
        L.w2_packed_bytes.restype = sz
        L.w2_packed_bytes.argtypes = [i, i]
        L.w2_pack.argtypes = [vp, i, i, vp, vp]
        L.a8_quantize.argtypes = [vp, i, i, vp, vp, vp]
        L.w2a8_workspace_bytes.restype = sz
        L.w2a8_workspace_bytes.argtypes = [i, i, i, i]
        L.w2a8_workspace_init.argtypes = [vp, sz, vp]
        L.w2a8_workspace_status.argtypes = [vp, vp]
        L.w2a8_gemm.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, vp, sz, vp]
        L.w2a8_gemm_h16.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, vp, sz, vp]
        L.w2a8_kernel_for.argtypes = [i, i, i, i]
        L.w2a8_tensor_core_channels.argtypes = [i, i, i, i]
        L.w2a8_tensor_core_ksplit.argtypes = [i, i, i, i]
        L.w2a8_tensor_core_tile_tokens.argtypes = [i, i, i, i]
        L.w2a16_gemm.argtypes = [vp, vp, vp, vp, i, i, i, i, vp, sz, vp]
        L.w2a8_gemm_partials.argtypes = [vp, vp, vp, i, i, i, i, vp, sz, vp]
        L.w2a8_linear.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, vp, sz, vp]
        L.w2a8_linear_host_workspace_bytes.restype = sz
        L.w2a8_linear_host_workspace_bytes.argtypes = [i, i, i, i]
        L.w2a8_linear_host.argtypes = [vp, i, i, vp, vp, i, i, vp, vp, sz, vp]
        L.w2a8_gemm_static.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, vp]
        L.w2a8_gemm_grouped.argtypes = [vp, vp, i, vp, vp, vp, vp, i, i, i, vp, sz, vp]
        L.w2a8_linear_grouped.argtypes = [vp, vp, vp, i, vp, vp, vp, vp, i, i, i, i, vp, sz, vp]
        L.w2a8_grouped_workspace_bytes.restype = sz
        L.w2a8_grouped_workspace_bytes.argtypes = [i, vp, i, i, i]
        L.w2a8_grouped_plan.argtypes = [i, vp, i, i, i, i]
        L.w2a8_linear_grouped_host_workspace_bytes.restype = sz
        L.w2a8_linear_grouped_host_workspace_bytes.argtypes = [i, vp, i, i, i]
        L.w2a8_linear_grouped_host.argtypes = [vp, i, i, i, vp, vp, vp, i, vp, vp, sz, vp]
        L.w2a8_linear_grouped_host.restype = i
        L.w2a8_tensor_core_kind.argtypes = [i, i, i, i]
        L.w2a8_tensor_core_kind.restype = i
        L.w2a8_read_probe.argtypes = [vp, sz, vp, vp]
        L.w2a8_read_probe.restype = i
        f, d = ctypes.c_float, ctypes.c_double
        L.w2a8_lora_grouped.argtypes = [vp, vp, i, i, vp, vp, i, vp, vp, vp, vp, i, vp, i, i, vp]
        L.w2a8_rope_frequencies.argtypes = [i, d, i, d, d, d, i, vp, vp]
        L.w2a8_rope.argtypes = [i, vp, i, vp, i, vp, vp, vp, i, i, i, i, vp, vp, f, vp]
        L.w2a8_qk_norm_rope.argtypes = [i, vp, i, vp, i, vp, f, vp, vp, vp, i, i, i, i, vp, vp, f, vp]
        for name in ("w2a8_lora_grouped", "w2a8_rope_frequencies", "w2a8_rope", "w2a8_qk_norm_rope"):
            getattr(L, name).restype = i
        for name in ("w2_pack", "a8_quantize", "w2a8_workspace_init", "w2a8_workspace_status", "w2a8_gemm",
                     "w2a8_gemm_partials", "w2a8_linear", "w2a8_linear_host", "w2a8_gemm_static",
                     "w2a8_gemm_grouped", "w2a8_linear_grouped", "w2a8_grouped_plan"):
            getattr(L, name).restype = i
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().w2a8_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != 0:
        raise W2A8Error(status, where)


def _stream(stream=None) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    # raw handle of the current stream of the current device, without building a Stream object
    return int(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _new(shape, dtype, device, stream=None) -> torch.Tensor:
    """A result's memory for a launch on `stream`: of that stream, since what the current one frees may still be written
    by its earlier work, and kept for the current one, where the result is read."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    here = torch.cuda.current_stream(device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    if here != stream:
        t.record_stream(here)
    return t


def w2a8_version() -> int:
    return int(lib().w2a8_version())


def w2_packed_bytes(N: int, K: int) -> int:
    return int(lib().w2_packed_bytes(N, K))


def w2a8_workspace_bytes(M: int, N: int, K: int, group: int) -> int:
    return int(lib().w2a8_workspace_bytes(M, N, K, group))


def w2a8_linear_host_workspace_bytes(M: int, N: int, K: int, group: int) -> int:
    return int(lib().w2a8_linear_host_workspace_bytes(M, N, K, group))


def new_workspace(nbytes: int, device="cuda", stream=None) -> torch.Tensor:
    """Allocate and zero-fill a workspace of at least `nbytes` bytes."""
    ws = _new(max(int(nbytes), 256), torch.uint8, device, stream)
    w2a8_workspace_init(ws, stream)
    return ws


def w2a8_workspace_init(workspace: torch.Tensor, stream=None):
    _check(lib().w2a8_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(),
                                     _stream(stream)), "w2a8_workspace_init")


def w2a8_workspace_status(workspace: torch.Tensor, stream=None) -> int:
    """Device status word of a workspace (0 = ok); synchronises the stream."""
    return int(lib().w2a8_workspace_status(_ptr(workspace), _stream(stream)))


def w2_pack(codes: torch.Tensor, packed: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """codes uint8 [N][K] (device) -> packed int32 [N][K/16] (bit pattern of uint32)."""
    N, K = codes.shape
    if packed is None:
        packed = _new((N, max(K // 16, 1)), torch.int32, codes.device, stream)
    _check(lib().w2_pack(_ptr(codes), N, K, _ptr(packed), _stream(stream)), "w2_pack")
    return packed


def a8_quantize(x_bf16: torch.Tensor, a: torch.Tensor | None = None,
                a_scale: torch.Tensor | None = None, stream=None):
    """x bf16 [M][K] (device) -> (a int8 [M][K], a_scale fp32 [M])."""
    M, K = x_bf16.shape
    if a is None:
        a = _new((M, K), torch.int8, x_bf16.device, stream)
    if a_scale is None:
        a_scale = _new((M,), torch.float32, x_bf16.device, stream)
    _check(lib().a8_quantize(_ptr(x_bf16), M, K, _ptr(a), _ptr(a_scale), _stream(stream)),
           "a8_quantize")
    return a, a_scale


def w2a8_gemm(a: torch.Tensor, a_scale: torch.Tensor, packed: torch.Tensor, w_scale: torch.Tensor,
              group: int, workspace: torch.Tensor, y: torch.Tensor | None = None, stream=None):
    """y fp32 [M][N] = scaled W2A8 product; see w2a8_gemm in include/w2a8.h."""
    M, K = a.shape
    N = packed.shape[0]
    if y is None:
        y = _new((M, N), torch.float32, a.device, stream)
    _check(lib().w2a8_gemm(_ptr(a), _ptr(a_scale), _ptr(packed), _ptr(w_scale), _ptr(y), M, N, K,
                           group, _ptr(workspace), workspace.numel() * workspace.element_size(),
                           _stream(stream)), "w2a8_gemm")
    return y


def w2a8_kernel_for(M: int, N: int, K: int, group: int) -> str:
    """'streaming' or 'tensor_core': the kernel w2a8_gemm uses for this shape."""
    r = int(lib().w2a8_kernel_for(M, N, K, group))
    _check(r if r < 0 else 0, "w2a8_kernel_for")
    return "tensor_core" if r == 1 else "streaming"


def w2a8_tensor_core_kind(M: int, N: int, K: int, group: int) -> int:
    """8 (int8 kernel), 16 (16-bit kernel on a bf16 copy of the activations) or 0 (streaming)."""
    r = int(lib().w2a8_tensor_core_kind(M, N, K, group))
    _check(r if r < 0 else 0, "w2a8_tensor_core_kind")
    return r


def w2a8_tensor_core_channels(M: int, N: int, K: int, group: int) -> int:
    """Channels of the problem computed by the tensor-core kernel (0 .. N); the rest, if any, is
    computed by the streaming kernel."""
    r = int(lib().w2a8_tensor_core_channels(M, N, K, group))
    _check(r if r < 0 else 0, "w2a8_tensor_core_channels")
    return r


def w2a8_tensor_core_ksplit(M: int, N: int, K: int, group: int) -> int:
    """K splits of the tensor-core kernel for this shape (0: streaming kernel; host only)."""
    r = int(lib().w2a8_tensor_core_ksplit(M, N, K, group))
    _check(r if r < 0 else 0, "w2a8_tensor_core_ksplit")
    return r


def w2a8_tensor_core_tile_tokens(M: int, N: int, K: int, group: int) -> int:
    """Token rows per tile of the tensor-core kernel for this shape (0: streaming kernel; host only)."""
    r = int(lib().w2a8_tensor_core_tile_tokens(M, N, K, group))
    _check(r if r < 0 else 0, "w2a8_tensor_core_tile_tokens")
    return r


def w2a8_gemm_h16(a: torch.Tensor, a_scale: torch.Tensor, packed: torch.Tensor, w_scale_h: torch.Tensor,
                  group: int, workspace: torch.Tensor, y: torch.Tensor | None = None,
                  out_dtype: torch.dtype = torch.float32, stream=None):
    """w2a8_gemm with binary16 weight scales (w_scale_h: float16 [N][K/group]) and an fp32 or bf16
    result (the dtype of y, else out_dtype); see w2a8_gemm_h16 in include/w2a8.h."""
    M, K = a.shape
    N = packed.shape[0]
    if w_scale_h.dtype != torch.float16:
        raise TypeError("w_scale_h must be float16")
    if y is None:
        y = _new((M, N), out_dtype, a.device, stream)
    if y.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("y must be float32 or bfloat16")
    _check(lib().w2a8_gemm_h16(_ptr(a), _ptr(a_scale), _ptr(packed), _ptr(w_scale_h), _ptr(y),
                               1 if y.dtype == torch.bfloat16 else 0, M, N, K, group, _ptr(workspace),
                               workspace.numel() * workspace.element_size(), _stream(stream)),
           "w2a8_gemm_h16")
    return y


def w2a16_gemm(x: torch.Tensor, packed: torch.Tensor, w_scale: torch.Tensor, group: int,
               workspace: torch.Tensor, y: torch.Tensor | None = None, stream=None):
    """bf16 x [M][K] (device, not quantised) -> y fp32 [M][N]; see w2a16_gemm in include/w2a8.h."""
    M, K = x.shape
    N = packed.shape[0]
    if x.dtype != torch.bfloat16:
        raise TypeError("x must be bfloat16")
    if y is None:
        y = _new((M, N), torch.float32, x.device, stream)
    _check(lib().w2a16_gemm(_ptr(x), _ptr(packed), _ptr(w_scale), _ptr(y), M, N, K, group, _ptr(workspace),
                            workspace.numel() * workspace.element_size(), _stream(stream)), "w2a16_gemm")
    return y


def w2a8_linear(x: torch.Tensor, packed: torch.Tensor, w_scale: torch.Tensor, group: int,
                workspace: torch.Tensor, a: torch.Tensor | None = None, a_scale: torch.Tensor | None = None,
                y: torch.Tensor | None = None, stream=None):
    """bf16 x [M][K] (device) -> (y fp32 [M][N], a int8 [M][K], a_scale fp32 [M]) in one call; see
    w2a8_linear in include/w2a8.h.  a / a_scale receive what a8_quantize would write."""
    M, K = x.shape
    N = packed.shape[0]
    if a is None:
        a = _new((M, K), torch.int8, x.device, stream)
    if a_scale is None:
        a_scale = _new((M,), torch.float32, x.device, stream)
    if y is None:
        y = _new((M, N), torch.float32, x.device, stream)
    _check(lib().w2a8_linear(_ptr(x), _ptr(a), _ptr(a_scale), _ptr(packed), _ptr(w_scale), _ptr(y), M, N, K,
                             group, _ptr(workspace), workspace.numel() * workspace.element_size(),
                             _stream(stream)), "w2a8_linear")
    return y, a, a_scale


def w2a8_gemm_partials(a: torch.Tensor, packed: torch.Tensor, group: int, workspace: torch.Tensor,
                       partials: torch.Tensor | None = None, stream=None):
    """Exact int32 per-group sums P[M][N][K/group] (parity/debug export)."""
    M, K = a.shape
    N = packed.shape[0]
    if partials is None:
        partials = _new((M, N, K // group), torch.int32, a.device, stream)
    _check(lib().w2a8_gemm_partials(_ptr(a), _ptr(packed), _ptr(partials), M, N, K, group,
                                    _ptr(workspace), workspace.numel() * workspace.element_size(),
                                    _stream(stream)), "w2a8_gemm_partials")
    return partials


def w2a8_linear_host(x_host: torch.Tensor, packed: torch.Tensor, w_scale: torch.Tensor, group: int,
                     y_host: torch.Tensor, workspace: torch.Tensor, stream=None):
    """Host bf16 x [M][K] -> host fp32 y [M][N]; copies, quantiser and GEMM enqueued on the stream."""
    M, K = x_host.shape
    N = packed.shape[0]
    _check(lib().w2a8_linear_host(_ptr(x_host), M, K, _ptr(packed), _ptr(w_scale), N, group,
                                  _ptr(y_host), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream(stream)),
           "w2a8_linear_host")
    return y_host


FUSE_AUTO, FUSE_OFF, FUSE_ON = -1, 0, 1


class Group:
    """Host-side argument block of the grouped entry points: the arrays of device pointers and of
    N, built once for a set of weight matrices (and, optionally, outputs) and reused every call."""

    def __init__(self, packed, w_scale, y=None):
        self.packed, self.w_scale = list(packed), list(w_scale)
        self.count = len(self.packed)
        self.N = [int(p.shape[0]) for p in self.packed]
        self.K = int(self.packed[0].shape[1]) * 16
        self._pk = (ctypes.c_void_p * self.count)(*[_ptr(p) for p in self.packed])
        self._sc = (ctypes.c_void_p * self.count)(*[_ptr(s) for s in self.w_scale])
        self._n = (ctypes.c_int * self.count)(*self.N)
        self.y = None
        self._y = None
        if y is not None:
            self.bind_outputs(y)

    def bind_outputs(self, y):
        self.y = list(y)
        self._y = (ctypes.c_void_p * self.count)(*[_ptr(t) for t in self.y])


def w2a8_grouped_workspace_bytes(N, M: int, K: int, group: int) -> int:
    arr = (ctypes.c_int * len(N))(*[int(n) for n in N])
    return int(lib().w2a8_grouped_workspace_bytes(len(N), arr, M, K, group))


def w2a8_grouped_plan(N, M: int, K: int, group: int, fuse: int = FUSE_AUTO) -> dict:
    """What a grouped call will do: {'one_launch': bool (whichever kernel), 'fused': bool (quantiser inside it)}."""
    arr = (ctypes.c_int * len(N))(*[int(n) for n in N])
    r = int(lib().w2a8_grouped_plan(len(N), arr, M, K, group, fuse))
    _check(r if r < 0 else 0, "w2a8_grouped_plan")
    return {"one_launch": bool(r & 1), "fused": bool(r & 2)}


def w2a8_gemm_grouped(a: torch.Tensor, a_scale: torch.Tensor, grp: Group, group: int,
                      workspace: torch.Tensor, y=None, stream=None):
    """y[i] = W2A8(a; matrix i) for the matrices of `grp`; see w2a8_gemm_grouped in include/w2a8.h."""
    M, K = a.shape
    if y is not None:
        grp.bind_outputs(y)
    elif grp.y is None or grp.y[0].shape[0] != M:
        grp.bind_outputs([_new((M, n), torch.float32, a.device, stream) for n in grp.N])
    _check(lib().w2a8_gemm_grouped(_ptr(a), _ptr(a_scale), grp.count, grp._pk, grp._sc, grp._y, grp._n, M, K,
                                   group, _ptr(workspace), workspace.numel() * workspace.element_size(),
                                   _stream(stream)), "w2a8_gemm_grouped")
    return grp.y


def w2a8_linear_grouped(x: torch.Tensor, grp: Group, group: int, workspace: torch.Tensor, fuse: int = FUSE_AUTO,
                        a: torch.Tensor | None = None, a_scale: torch.Tensor | None = None, y=None, stream=None):
    """bf16 x [M][K] (device) -> y[i] fp32 [M][N_i] for the matrices of `grp`; a / a_scale (optional when the
    call fuses) receive what a8_quantize would write.  See w2a8_linear_grouped in include/w2a8.h."""
    M, K = x.shape
    if y is not None:
        grp.bind_outputs(y)
    elif grp.y is None or grp.y[0].shape[0] != M:
        grp.bind_outputs([_new((M, n), torch.float32, x.device, stream) for n in grp.N])
    _check(lib().w2a8_linear_grouped(_ptr(x), _ptr(a), _ptr(a_scale), grp.count, grp._pk, grp._sc, grp._y,
                                     grp._n, M, K, group, fuse, _ptr(workspace),
                                     workspace.numel() * workspace.element_size(), _stream(stream)),
           "w2a8_linear_grouped")
    return grp.y


def w2a8_linear_grouped_host_workspace_bytes(N, M: int, K: int, group: int) -> int:
    arr = (ctypes.c_int * len(N))(*[int(n) for n in N])
    return int(lib().w2a8_linear_grouped_host_workspace_bytes(len(N), arr, M, K, group))


def w2a8_linear_grouped_host(x_host: torch.Tensor, grp: Group, group: int, y_host, workspace: torch.Tensor,
                             stream=None):
    """Host bf16 x [M][K] -> host fp32 y_host[i] [M][N_i] for the matrices of `grp` (device); x is
    brought over and quantised once.  See w2a8_linear_grouped_host in include/w2a8.h."""
    M, K = x_host.shape
    ys = (ctypes.c_void_p * grp.count)(*[_ptr(t) for t in y_host])
    _check(lib().w2a8_linear_grouped_host(_ptr(x_host), M, K, grp.count, grp._pk, grp._sc, grp._n, group, ys,
                                          _ptr(workspace), workspace.numel() * workspace.element_size(),
                                          _stream(stream)), "w2a8_linear_grouped_host")
    return y_host


def _want(t: torch.Tensor, name: str, dtype, shape, device):
    """The tensor as the C entry points expect it: type, shape, device, rows without gaps."""
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}".replace("torch.", ""))
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _c_ints(**sizes):
    """Refuses sizes that the library's ints would not hold: ctypes hands on their lower 32 bits."""
    for name, n in sizes.items():
        if not -2 ** 31 <= n < 2 ** 31:
            raise ValueError(f"{name} is {n}: more than 32 bits")


def _launch_stream(device, index, stream) -> int:
    """Raw handle of the stream to launch on.  The launch goes to the current device: tensors of another one (`index`;
    -1: not on a GPU) are refused, and so is a stream of another."""
    if index < 0:
        raise ValueError(f"tensors are on {device}: a CUDA device is needed")
    here = torch._C._cuda_getDevice()
    if index != here or (stream is not None and stream.device.index != here):
        raise ValueError(f"tensors or stream are on another device than the current one (cuda:{here})")
    return torch._C._cuda_getCurrentRawStream(here) if stream is None else int(stream.cuda_stream)


_BF16, _F32, _F64, _I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32


class LoraGroup:
    """Host-side argument block of w2a8_lora_grouped: the adapters of the matrices that share their activations,
    A[i] bf16 [adapters][rank_max][K] and B[i] bf16 [adapters][N_i][rank_max], with `rank` (int32 [adapters], None:
    rank_max) and `scale` (fp32 [adapters], None: 1).  Built once and reused every call; the tensors are held, so
    their values may change between calls."""

    def __init__(self, A, B, rank=None, scale=None):
        self.A, self.B, self.rank, self.scale = list(A), list(B), rank, scale
        self.count = len(self.A)
        if self.count < 1 or len(self.B) != self.count:
            raise ValueError("A and B must be lists of one tensor per matrix")
        self.adapters, self.rank_max, self.K = (int(n) for n in self.A[0].shape)
        self.N = [int(b.shape[1]) for b in self.B]
        _c_ints(adapters=self.adapters, rank_max=self.rank_max, K=self.K, N=max(self.N))
        self.device, self.index = self.A[0].device, self.A[0].get_device()
        for a, b, n in zip(self.A, self.B, self.N):
            _want(a, "A", torch.bfloat16, (self.adapters, self.rank_max, self.K), self.device)
            _want(b, "B", torch.bfloat16, (self.adapters, n, self.rank_max), self.device)
        if rank is not None:
            _want(rank, "rank", torch.int32, (self.adapters,), self.device)
        if scale is not None:
            _want(scale, "scale", torch.float32, (self.adapters,), self.device)
        ptrs = ctypes.c_void_p * self.count
        self._a, self._b = ptrs(*[_ptr(t) for t in self.A]), ptrs(*[_ptr(t) for t in self.B])
        self._n = (ctypes.c_int * self.count)(*self.N)
        self._rank, self._scale = _ptr(rank), _ptr(scale)
        self._ptrs = ptrs

    def _outputs(self, name, tensors, M, dtype, index):
        if len(tensors) != self.count:
            raise ValueError(f"{name} must have one tensor per matrix")
        ptrs = []
        for t, n in zip(tensors, self.N):
            if t.dtype is not dtype or t.shape != (M, n) or t.get_device() != index or not t.is_contiguous():
                _want(t, name, dtype, (M, n), self.device)
            ptrs.append(t.data_ptr())
        return self._ptrs(*ptrs)


def w2a8_lora_grouped(x: torch.Tensor, adapter: torch.Tensor, lora: LoraGroup, base=None, y=None,
                      out_dtype: torch.dtype = torch.float32, stream=None):
    """y[i] = base[i] + the adapters of x's tokens on matrix i (adapter int32 [M]; outside [0, adapters): none), e.g.
    on the results of w2a8_linear_grouped.  base: list of [M][N_i] (fp32, or all bf16) or None = 0; y: list of outputs,
    may be `base` itself (in place), None: new ones.  See w2a8_lora_grouped in include/w2a8.h."""
    device, index = lora.device, lora.index
    M = x.shape[0]
    raw = _launch_stream(device, index, stream)
    if x.dtype is not _BF16 or x.shape != (M, lora.K) or x.get_device() != index or not x.is_contiguous():
        _want(x, "x", _BF16, (M, lora.K), device)
    if adapter.dtype is not _I32 or adapter.shape != (M,) or adapter.get_device() != index or not adapter.is_contiguous():
        _want(adapter, "adapter", _I32, (M,), device)
    dtype = base[0].dtype if base is not None else y[0].dtype if y is not None else out_dtype
    if dtype is not _F32 and dtype is not _BF16:
        raise TypeError("base and y must be float32 or bfloat16")
    if y is None:
        y = [_new((M, n), dtype, device, stream) for n in lora.N]
    py = lora._outputs("y", y, M, dtype, index)
    pb = None if base is None else py if base is y else lora._outputs("base", base, M, dtype, index)
    status = lib().w2a8_lora_grouped(x.data_ptr(), adapter.data_ptr(), lora.adapters, lora.rank_max, lora._rank,
                                     lora._scale, lora.count, lora._a, lora._b, pb, py,
                                     1 if dtype is _BF16 else 0, lora._n, M, lora.K, raw)
    if status:
        _check(status, "w2a8_lora_grouped")
    return y


ROPE_SCALINGS = {"plain": 0, "linear": 1, "ntk": 2, "llama3": 3, "yarn": 4}


def w2a8_rope_frequencies(rot_dim: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
                          low: float = 1.0, high: float = 32.0, original_length: int = 0, device="cuda"):
    """(inv_freq float64 [rot_dim / 2] on `device`, amplitude) for the rope entry points; scaling: a key of
    ROPE_SCALINGS.  low / high: the full turns within original_length between which "llama3" and "yarn" mix.  See
    w2a8_rope_frequencies in include/w2a8.h."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(ROPE_SCALINGS)}")
    _c_ints(rot_dim=rot_dim, original_length=original_length)
    freq = torch.empty(max(int(rot_dim) // 2, 1), dtype=torch.float64)
    amplitude = ctypes.c_float()
    _check(lib().w2a8_rope_frequencies(rot_dim, base, ROPE_SCALINGS[scaling], factor, low, high, original_length,
                                       _ptr(freq), ctypes.addressof(amplitude)), "w2a8_rope_frequencies")
    return freq.to(device), float(amplitude.value)


class Heads:
    """Host-side argument block of the rope entry points: results x[i] [M][heads_i][head_dim] (fp32, or all bf16;
    views with strides are fine as long as the values of a head are consecutive), the outputs, and the norms' weights
    (fp32 [head_dim] or None, one per result).  out: a list of the same shapes (fp32 or bf16), `x` itself for in
    place, or None: new ones of out_dtype (None: x's), memory of the current stream.  Built once and reused every
    call."""

    def __init__(self, x, out=None, weight=None, out_dtype=None):
        self.x = list(x)
        self.count = len(self.x)
        if not 1 <= self.count <= 4:
            raise ValueError("1 to 4 results")
        self.M, _, self.head_dim = (int(n) for n in self.x[0].shape)
        _c_ints(**{"a size of x": max(int(n) for t in self.x for n in t.shape)})
        self.device, self.index, self.dtype = self.x[0].device, self.x[0].get_device(), self.x[0].dtype
        if out is None:
            out = [torch.empty(t.shape, dtype=out_dtype or self.dtype, device=self.device) for t in self.x]
        self.out = list(out)
        self.weight = [None] * self.count if weight is None else list(weight)
        if len(self.out) != self.count or len(self.weight) != self.count:
            raise ValueError("x, out and weight must have one entry per result")
        self.out_dtype = self.out[0].dtype
        for what, tensors, dtype in (("x", self.x, self.dtype), ("out", self.out, self.out_dtype)):
            if dtype not in (torch.float32, torch.bfloat16):
                raise TypeError(f"{what} must be float32 or bfloat16")
            for t, like in zip(tensors, self.x):
                if t.dtype != dtype:
                    raise TypeError(f"{what}: tensors of one type")
                if t.dim() != 3 or t.shape != like.shape or t.shape[0] != self.M or t.shape[2] != self.head_dim:
                    raise ValueError(f"{what} must be [tokens][heads][head_dim]")
                if t.device != self.device:
                    raise ValueError(f"{what} is on {t.device}, not on {self.device}")
                if t.stride(2) != 1:
                    raise ValueError(f"{what}: the values of a head must be consecutive")
        for w in self.weight:
            if w is not None:
                _want(w, "weight", torch.float32, (self.head_dim,), self.device)
        ptrs, strides = ctypes.c_void_p * self.count, ctypes.c_int64 * (2 * self.count)
        self._x, self._out = ptrs(*[_ptr(t) for t in self.x]), ptrs(*[_ptr(t) for t in self.out])
        self._w = ptrs(*[_ptr(w) for w in self.weight])
        self._xs = strides(*[t.stride(d) for t in self.x for d in (0, 1)])
        self._os = strides(*[t.stride(d) for t in self.out for d in (0, 1)])
        self._heads = (ctypes.c_int * self.count)(*[int(t.shape[1]) for t in self.x])
        self._x16, self._o16 = int(self.dtype is torch.bfloat16), int(self.out_dtype is torch.bfloat16)


def _rope_angles(heads: Heads, positions, inv_freq) -> int:
    """Checks positions and inv_freq; the number of values of a head that turn."""
    if positions is None:
        raise ValueError("positions are needed for the rotation")
    half, index = inv_freq.shape[0], heads.index
    if inv_freq.dtype is not _F64 or inv_freq.dim() != 1 or inv_freq.get_device() != index or not inv_freq.is_contiguous():
        _want(inv_freq, "inv_freq", _F64, (half,), heads.device)
    if (positions.dtype is not _I32 or positions.shape != (heads.M,) or positions.get_device() != index
            or not positions.is_contiguous()):
        _want(positions, "positions", _I32, (heads.M,), heads.device)
    return 2 * half


def w2a8_rope(heads: Heads, positions: torch.Tensor, inv_freq: torch.Tensor, amplitude: float = 1.0,
              interleaved: bool = False, stream=None):
    """Rotary positions (int32 [M]) on the results of `heads`; the first 2 * len(inv_freq) values of a head turn.
    inv_freq (float64) and amplitude: from w2a8_rope_frequencies.  Returns heads.out.  See w2a8_rope in
    include/w2a8.h."""
    raw = _launch_stream(heads.device, heads.index, stream)
    rot = _rope_angles(heads, positions, inv_freq)
    status = lib().w2a8_rope(heads.count, heads._x, heads._x16, heads._out, heads._o16, heads._heads, heads._xs,
                             heads._os, heads.M, heads.head_dim, rot, 1 if interleaved else 0, positions.data_ptr(),
                             inv_freq.data_ptr(), amplitude, raw)
    if status:
        _check(status, "w2a8_rope")
    return heads.out


def w2a8_qk_norm_rope(heads: Heads, eps: float, positions: torch.Tensor | None = None,
                      inv_freq: torch.Tensor | None = None, amplitude: float = 1.0, interleaved: bool = False,
                      stream=None):
    """The norm of every head (times heads.weight) and the rotation in one pass; without inv_freq the norm alone.
    Returns heads.out.  See w2a8_qk_norm_rope in include/w2a8.h."""
    raw = _launch_stream(heads.device, heads.index, stream)
    rot = 0 if inv_freq is None else _rope_angles(heads, positions, inv_freq)
    status = lib().w2a8_qk_norm_rope(heads.count, heads._x, heads._x16, heads._out, heads._o16, heads._w, eps,
                                     heads._heads, heads._xs, heads._os, heads.M, heads.head_dim, rot,
                                     1 if interleaved else 0, positions.data_ptr() if rot else None,
                                     inv_freq.data_ptr() if rot else None, amplitude, raw)
    if status:
        _check(status, "w2a8_qk_norm_rope")
    return heads.out


def w2a8_read_probe(buffer: torch.Tensor, sink: torch.Tensor, stream=None):
    """Enqueue one read-only pass over `buffer` (see w2a8_read_probe in include/w2a8.h)."""
    _check(lib().w2a8_read_probe(_ptr(buffer), buffer.numel() * buffer.element_size(), _ptr(sink),
                                 _stream(stream)), "w2a8_read_probe")


STATIC_SCRATCH_BYTES = 8 << 20


def w2a8_gemm_static(a: torch.Tensor, a_scale: torch.Tensor, packed: torch.Tensor,
                     w_scale: torch.Tensor, group: int, y: torch.Tensor | None = None, stream=None):
    """w2a8_gemm for callers with no workspace to give: the kernel's scratch is a fixed
    array inside the library (at most STATIC_SCRATCH_BYTES; larger problems raise), so
    nothing is allocated on the library side.  Calls share that array: keep them on one
    stream.  See w2a8_gemm_static in include/w2a8.h."""
    M, K = a.shape
    N = packed.shape[0]
    if y is None:
        y = _new((M, N), torch.float32, a.device, stream)
    _check(lib().w2a8_gemm_static(_ptr(a), _ptr(a_scale), _ptr(packed), _ptr(w_scale), _ptr(y), M, N, K,
                                  group, _stream(stream)), "w2a8_gemm_static")
    return y
