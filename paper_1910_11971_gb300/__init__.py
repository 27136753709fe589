"""Python binding of libcci.so: CCI-sparse layers (arXiv 1910.11971) on GB300.

Argument marshalling only.  Every step of the computation runs in the CUDA
kernels of ``libcci.so`` (built from ``csrc/`` by ``build.py``); PyTorch is used
for device memory and the current stream.  There is no CPU path: if the
library is missing or a call fails, an exception is raised.

    values, idx = pack(W, G, K)                         # Sec. 3.1 / 5.1
    Y = linear(X, values, idx, Cout, G, K)              # Alg. 2, Y[N][Cout] fp32
    Y = conv2d(X, values, idx, Cout, G, K, KH, KW, stride, pad)  # NHWC

Layouts are those of ``include/cci.h``: W [Cout][R], values/idx [Cout/G][R][K],
X [N][Cin] (product) or NHWC [B][H][W][Cin] (convolution), Y fp32.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libcci.so")

F32, BF16 = 0, 1
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3, "sigmoid": 4}
GATED_FORWARD, GATED_PACKED, GATED_BACKWARD = 0, 1, 2
HEAD_FORWARD, HEAD_BACKWARD = 0, 1
ALGO_AUTO, ALGO_GENERIC, ALGO_REGTILE, ALGO_DENSE_TC, ALGO_EXPAND, ALGO_DENSE_TC_WS = 0, 1, 2, 3, 4, 5

STATUS_NAMES = {
    0: "CCI_OK", 1: "CCI_ERR_NULL", 2: "CCI_ERR_SHAPE", 3: "CCI_ERR_GROUP", 4: "CCI_ERR_DTYPE",
    5: "CCI_ERR_ALIGN", 6: "CCI_ERR_VALUE", 7: "CCI_ERR_CUDA", 8: "CCI_ERR_TIMEOUT",
    9: "CCI_ERR_UNSUPPORTED", 10: "CCI_ERR_INDEX", 11: "CCI_ERR_WORKSPACE",
}

# exported symbols with their ctypes signatures (the declarations of cci.h)
_P, _I64, _I32, _U32P = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p
SIGNATURES = {
    "cci_pack": (_I32, [_P, _I32, _I64, _I64, _I32, _I32, _P, _P, _U32P, _P]),
    "cci_linear": (_I32, [_P, _I32, _I64, _I64, _P, _P, _I64, _I32, _I32, _P, _U32P, _P]),
    "cci_linear_ex": (_I32, [_P, _I32, _I64, _I64, _P, _P, _I64, _I32, _I32, _P, _U32P, _I32, _P]),
    "cci_conv2d": (_I32, [_P, _I32, _I64, _I64, _I64, _I64, _P, _P, _I64, _I32, _I32, _I32, _I32,
                          _I32, _I32, _I32, _I32, _P, _U32P, _P]),
    "cci_conv2d_ex": (_I32, [_P, _I32, _I64, _I64, _I64, _I64, _P, _P, _I64, _I32, _I32, _I32, _I32,
                             _I32, _I32, _I32, _I32, _P, _U32P, _I32, _P]),
    "cci_linear_ws": (_I32, [_P, _I32, _I64, _I64, _P, _P, _I64, _I32, _I32, _P, _U32P, _I32, _P,
                             ctypes.c_size_t, _P]),
    "cci_conv2d_ws": (_I32, [_P, _I32, _I64, _I64, _I64, _I64, _P, _P, _I64, _I32, _I32, _I32, _I32,
                             _I32, _I32, _I32, _I32, _P, _U32P, _I32, _P, ctypes.c_size_t, _P]),
    "cci_linear_fused": (_I32, [_P, _I32, _I64, _I64, _P, _P, _I64, _I32, _I32, _P, _I32, _I32, _P,
                                _U32P, _P, ctypes.c_size_t, _P]),
    "cci_conv2d_fused": (_I32, [_P, _I32, _I64, _I64, _I64, _I64, _P, _P, _I64, _I32, _I32, _I32,
                                _I32, _I32, _I32, _I32, _I32, _P, _I32, _I32, _P, _U32P, _P,
                                ctypes.c_size_t, _P]),
    "cci_pack_stats": (_I32, [_P, _I32, _I64, _I64, _I32, _I32, _P, _P]),
    "cci_bbs_pack": (_I32, [_P, _I32, _I64, _I64, _I32, _I32, _P, _P, _U32P, _P]),
    "cci_bbs_linear": (_I32, [_P, _I32, _I64, _I64, _P, _P, _I64, _I32, _I32, _P, _U32P, _I32, _P,
                              ctypes.c_size_t, _P]),
    "cci_td_mask": (_I32, [_P, _I32, _I64, _I64, _I32, _I32, ctypes.c_float, _P, _P, _P, _U32P, _P]),
    "cci_td_drop_rate": (ctypes.c_float, [_I64, _I64, ctypes.c_float, ctypes.c_float]),
    "cci_workspace_size": (ctypes.c_size_t, [_I32, _I32, _I64, _I64]),
    "cci_linear_host_buffer_size": (ctypes.c_size_t, [_I32, _I64, _I64, _I64]),
    "cci_linear_host": (_I32, [_P, _I32, _I64, _I64, _P, _P, _I64, _I32, _I32, _P, _I64, _P,
                               ctypes.c_size_t, _U32P, _P, _P, _P]),
    "cci_linear_dense_tc_static": (_I32, [_P, _I32, _I64, _I64, _P, _P, _I64, _I32, _I32, _P, _U32P,
                                          _P]),
    "cci_dense_linear_tc": (_I32, [_P, _I32, _I64, _I64, _P, _I64, _P, _U32P, _P]),
    "cci_dense_planes": (_I32, [_P, _I32, _I64, _I64, _P, ctypes.c_size_t, _P]),
    "cci_dense_conv2d_tc": (_I32, [_P, _I32, _I64, _I64, _I64, _I64, _P, _I64, _I32, _I32, _I32, _I32,
                                   _I32, _I32, _P, _U32P, _P]),
    "cci_layer_norm": (_I32, [_P, _I32, _I64, _I64, _I64, _P, _P, ctypes.c_float, _P, _P, _P, _P]),
    "cci_layer_norm_workspace_size": (ctypes.c_size_t, [_I64, _I64]),
    "cci_layer_norm_backward": (_I32, [_P, _I64, _P, _I64, _I32, _I64, _I64, _P, _P, _P, _P, _P, _P, _P,
                                       ctypes.c_size_t, _P]),
    "cci_layer_norm_backward_ex": (_I32, [_P, _I64, _P, _I64, _I32, _I64, _I64, _P, _P, _P, _P, _P, _P, _U32P, _P,
                                          ctypes.c_size_t, _P]),
    "cci_token_logprobs": (_I32, [_P, _I32, _I64, _I64, _I64, _P, _I64, _I32, _P, _P, _P, _P, _P, _U32P, _P]),
    "cci_token_logprobs_backward": (_I32, [_P, _I32, _I64, _I64, _I64, _P, _P, _I64, _P, _P, _P, _P, _I64, _U32P,
                                           _P]),
    "cci_gated_workspace_size": (ctypes.c_size_t, [_I32, _I32, _I64, _I64, _I64]),
    "cci_gated_linear": (_I32, [_P, _I32, _I64, _I64, _P, _P, _I64, _I32, _P, _P, _P, _U32P, _P, ctypes.c_size_t,
                                _P]),
    "cci_gated_linear_packed": (_I32, [_P, _I32, _I64, _I64, _P, _P, _P, _P, _I64, _I32, _I32, _I32, _P, _U32P, _P,
                                       ctypes.c_size_t, _P]),
    "cci_gated_linear_backward": (_I32, [_P, _P, _I32, _I64, _I64, _P, _P, _I64, _I32, _P, _P, _P, _P, _P, _U32P, _P,
                                         ctypes.c_size_t, _P]),
    "cci_distillation_workspace_size": (ctypes.c_size_t, [_I64, _I64]),
    "cci_distillation_loss": (_I32, [_P, _I32, _I64, _I64, _I64, _P, _P, _I32, ctypes.c_float, _I32, _P, _P, _U32P, _P,
                                     ctypes.c_size_t, _P]),
    "cci_distillation_loss_backward": (_I32, [_P, _P, _I32, _I64, _I64, _I64, _P, _P, _I32, ctypes.c_float, _I32, _P, _P,
                                              _I64, _P]),
    "cci_rms_norm": (_I32, [_P, _I32, _I64, _I64, _I64, _P, _I64, _P, ctypes.c_float, _P, _P, _P, _P]),
    "cci_rms_norm_fp8": (_I32, [_P, _I32, _I64, _I64, _I64, _P, _I64, _P, ctypes.c_float, _I32, _P, _P, _P, _P, _P]),
    "cci_rms_norm_workspace_size": (ctypes.c_size_t, [_I64, _I64]),
    "cci_rms_norm_backward": (_I32, [_P, _I64, _P, _I64, _P, _I64, _I32, _I64, _I64, _P, _P, _P, _P, _P,
                                     ctypes.c_size_t, _P]),
    "cci_head_workspace_size": (ctypes.c_size_t, [_I32, _I32, _I64, _I64, _I64]),
    "cci_linear_cross_entropy": (_I32, [_P, _I32, _I64, _I64, _P, _I64, _P, _I64, _P, _P, _U32P, _P, ctypes.c_size_t,
                                        _P]),
    "cci_linear_cross_entropy_backward": (_I32, [_P, _P, _I32, _I64, _I64, _P, _I64, _P, _I64, _P, _P, _P, _U32P, _P,
                                                 ctypes.c_size_t, _P]),
    "cci_kernel_name": (ctypes.c_char_p, [_I32, _I64, _I64, _I64, _I32, _I32, _I32]),
    "cci_status_string": (ctypes.c_char_p, [_I32]),
    "cci_decode_device_status": (_I32, [ctypes.c_uint32]),
    "cci_version": (_I32, []),
    "cci_fma_probe": (_I32, [_P, _I32, _I32, _I32, _P]),
    "cci_wait_probe": (_I32, [_U32P, _I32, _P]),
}

_lib = None


class CCIError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        text = lib().cci_status_string(self.status).decode() if _lib is not None else ""
        super().__init__(f"{where}: {STATUS_NAMES.get(self.status, self.status)} ({text})")


def lib() -> ctypes.CDLL:
    """The loaded libcci.so.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libcci.so is not built ({LIB_PATH}); run "
                               "`python -m paper_1910_11971_gb300.build` (needs nvcc)")
        h = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(h, name)
            fn.restype = res
            fn.argtypes = args
        _lib = h
    return _lib


def status_string(code: int) -> str:
    return lib().cci_status_string(int(code)).decode()


def decode_status(word: int) -> int:
    return int(lib().cci_decode_device_status(ctypes.c_uint32(int(word) & 0xffffffff)))


_DTYPE_CODES = {torch.float32: F32, torch.bfloat16: BF16}


def _dtype_code(t: torch.Tensor) -> int:
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}: float32 or bfloat16")
    return code


def _stream(device: torch.device) -> int:
    # the handle alone: a Stream object for it costs 2 us a call
    index = device.index
    if index is None:
        # a GPU tensor's device always has an index.  A host tensor's has none and is
        # refused here: its address must not reach a kernel (asking every device for
        # its type costs 0.3 us a call)
        if device.type != "cuda":
            raise ValueError(f"Expected a cuda device, but got: {device}")
        index = torch.cuda.current_device()
    return torch._C._cuda_getCurrentRawStream(index)


def _cuda_contig(t: torch.Tensor, name: str) -> None:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _check(code: int, where: str) -> None:
    if code != 0:
        raise CCIError(code, where)


def new_status(device) -> torch.Tensor:
    """A zeroed device status word for the ``status=`` argument of the calls."""
    return torch.zeros(1, dtype=torch.int32, device=device)


def read_status(status: torch.Tensor) -> int:
    """Synchronise and return the first error recorded in a status word (0 = none)."""
    return decode_status(int(status.item()))


def pack(W: torch.Tensor, G: int, K: int, *, status: Optional[torch.Tensor] = None,
         check: bool = True, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None):
    """Per-group top-K by |w| (ties to the lower index) -> (values, idx).

    W: CUDA [Cout][R] float32 or bfloat16.  With ``check`` (the default) the call
    synchronises and raises on NaN weights; with ``check=False`` it stays
    asynchronous and records errors only in ``status`` (if given)."""
    _cuda_contig(W, "W")
    Cout, R = W.shape
    if G < 1 or Cout % G:
        raise CCIError(3, "pack")
    if out is None:
        values = torch.empty((Cout // G, R, K), dtype=W.dtype, device=W.device)
        idx = torch.empty((Cout // G, R, K), dtype=torch.uint8, device=W.device)
    else:
        values, idx = out
    own_status = status is None and check
    if own_status:
        status = new_status(W.device)
    code = lib().cci_pack(W.data_ptr(), _dtype_code(W), Cout, R, G, K, values.data_ptr(),
                          idx.data_ptr(), status.data_ptr() if status is not None else None,
                          _stream(W.device))
    _check(code, "cci_pack")
    if check:
        dev = read_status(status)
        if dev:
            raise CCIError(dev, "cci_pack (device)")
    return values, idx


def workspace_size(algo: int, dtype: torch.dtype, Cout: int, R: int) -> int:
    """Bytes of workspace the kernel family needs for a layer (0: none)."""
    return int(lib().cci_workspace_size(algo, F32 if dtype == torch.float32 else BF16, Cout, R))


def new_workspace(algo: int, dtype: torch.dtype, Cout: int, R: int, device) -> Optional[torch.Tensor]:
    return _workspace(workspace_size(algo, dtype, Cout, R), device)


def _ws(workspace: Optional[torch.Tensor]):
    if workspace is None:
        return None, 0
    return workspace.data_ptr(), workspace.nbytes


def linear(X: torch.Tensor, values: torch.Tensor, idx: torch.Tensor, Cout: int, G: int, K: int, *,
           out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
           algo: int = ALGO_AUTO, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y[N][Cout] (fp32) = the CCI-sparse product of X[N][Cin] (Alg. 2).

    ``workspace``: device buffer for the families that need one (see
    ``workspace_size``); with ``algo`` AUTO or ``ALGO_DENSE_TC_WS`` and none given,
    the one that family asks for is allocated here from PyTorch memory (the
    library allocates nothing), so AUTO can reach its fastest family."""
    _cuda_contig(X, "X")
    N, Cin = X.shape
    if workspace is None and algo == ALGO_AUTO:
        workspace = _workspace(_auto_bytes(X.dtype, Cin, Cin, Cout, G, K, False), X.device)
    elif workspace is None and algo == ALGO_DENSE_TC_WS:
        workspace = new_workspace(algo, X.dtype, Cout, Cin, X.device)
    Y = out if out is not None else torch.empty((N, Cout), dtype=torch.float32, device=X.device)
    wp, wb = _ws(workspace)
    code = lib().cci_linear_ws(X.data_ptr(), _dtype_code(X), N, Cin, values.data_ptr(),
                               idx.data_ptr(), Cout, G, K, Y.data_ptr(),
                               status.data_ptr() if status is not None else None, algo, wp, wb,
                               _stream(X.device))
    _check(code, "cci_linear")
    return Y


_copy_streams = {}


def host_chunk(N: int) -> int:
    """Default columns per chunk of ``linear_host``: about an eighth of N, in
    whole 128-column tiles."""
    eighth = (N + 7) // 8
    return max(128, (eighth + 127) // 128 * 128)


def host_buffer(dtype: torch.dtype, Cin: int, Cout: int, chunk: int, device) -> torch.Tensor:
    """A device buffer for ``linear_host`` (the library allocates nothing)."""
    n = lib().cci_linear_host_buffer_size(F32 if dtype == torch.float32 else BF16, Cin, Cout, chunk)
    if not n:
        raise ValueError("cci_linear_host_buffer_size: invalid shape")
    return torch.empty(n, dtype=torch.uint8, device=device)


def linear_host(X_host: torch.Tensor, values: torch.Tensor, idx: torch.Tensor, Cout: int, G: int, K: int, *,
                out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                chunk: Optional[int] = None, buffer: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``linear`` with X and Y in host memory (``cci_linear_host``): column chunks
    are copied in, multiplied and copied out on three streams, overlapping.
    X_host should be pinned; the result ``out`` (pinned fp32 [N][Cout], allocated
    when not given) is complete once the device's current stream has been
    synchronised."""
    if X_host.is_cuda or not X_host.is_contiguous():
        raise ValueError("X_host must be a contiguous host tensor")
    dev = values.device
    N, Cin = X_host.shape
    chunk = chunk or host_chunk(N)
    if buffer is None:
        buffer = host_buffer(X_host.dtype, Cin, Cout, chunk, dev)
    Y = out if out is not None else torch.empty((N, Cout), dtype=torch.float32).pin_memory()
    if Y.is_cuda or not Y.is_contiguous() or Y.dtype != torch.float32:
        raise ValueError("out must be a contiguous fp32 host tensor")
    key = (dev.index if dev.index is not None else torch.cuda.current_device())
    if key not in _copy_streams:
        _copy_streams[key] = (torch.cuda.Stream(dev), torch.cuda.Stream(dev))
    s_in, s_out = _copy_streams[key]
    code = lib().cci_linear_host(X_host.data_ptr(), _dtype_code(X_host), N, Cin, values.data_ptr(),
                                 idx.data_ptr(), Cout, G, K, Y.data_ptr(), chunk, buffer.data_ptr(),
                                 buffer.numel(), status.data_ptr() if status is not None else None,
                                 _stream(dev), s_in.cuda_stream, s_out.cuda_stream)
    _check(code, "cci_linear_host")
    return Y


def conv_out_hw(H: int, W: int, KH: int, KW: int, stride: Sequence[int], pad: Sequence[int]):
    return (H + 2 * pad[0] - KH) // stride[0] + 1, (W + 2 * pad[1] - KW) // stride[1] + 1


def conv2d(X: torch.Tensor, values: torch.Tensor, idx: torch.Tensor, Cout: int, G: int, K: int,
           KH: int, KW: int, stride=(1, 1), pad=(0, 0), *, out: Optional[torch.Tensor] = None,
           status: Optional[torch.Tensor] = None, algo: int = ALGO_AUTO,
           workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y NHWC [B][P][Q][Cout] (fp32) = CCI-sparse convolution of X NHWC [B][H][W][Cin]."""
    _cuda_contig(X, "X")
    B, H, W, Cin = X.shape
    P, Q = conv_out_hw(H, W, KH, KW, stride, pad)
    Y = out if out is not None else torch.empty((B, max(P, 0), max(Q, 0), Cout), dtype=torch.float32,
                                                device=X.device)
    if workspace is None and algo == ALGO_AUTO:
        workspace = _workspace(_auto_bytes(X.dtype, Cin, KH * KW * Cin, Cout, G, K, max(stride) > 2), X.device)
    elif workspace is None and algo == ALGO_DENSE_TC_WS:
        workspace = new_workspace(algo, X.dtype, Cout, KH * KW * Cin, X.device)
    wp, wb = _ws(workspace)
    code = lib().cci_conv2d_ws(X.data_ptr(), _dtype_code(X), B, H, W, Cin, values.data_ptr(),
                               idx.data_ptr(), Cout, KH, KW, stride[0], stride[1], pad[0], pad[1],
                               G, K, Y.data_ptr(), status.data_ptr() if status is not None else None,
                               algo, wp, wb, _stream(X.device))
    _check(code, "cci_conv2d")
    return Y


def bbs_pack(W: torch.Tensor, G: int, K: int, *, status: Optional[torch.Tensor] = None):
    """(values[Cout][R/G][K], idx[Cout][R/G][K]) of the balanced-sparse form of W
    (groups of G consecutive inputs; ``cci_bbs_pack``)."""
    _cuda_contig(W, "W")
    Cout, R = W.shape
    values = torch.empty((Cout, R // G, K), dtype=W.dtype, device=W.device)
    idx = torch.empty((Cout, R // G, K), dtype=torch.uint8, device=W.device)
    _check(lib().cci_bbs_pack(W.data_ptr(), _dtype_code(W), Cout, R, G, K, values.data_ptr(), idx.data_ptr(),
                              status.data_ptr() if status is not None else None, _stream(W.device)),
           "cci_bbs_pack")
    return values, idx


def bbs_linear(X: torch.Tensor, values: torch.Tensor, idx: torch.Tensor, Cout: int, G: int, K: int, *,
               out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
               algo: int = ALGO_AUTO, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y[N][Cout] (fp32) = the balanced-sparse product (``cci_bbs_linear``); with AUTO
    or ALGO_DENSE_TC_WS and no workspace, one is allocated here."""
    _cuda_contig(X, "X")
    N, Cin = X.shape
    if workspace is None and algo in (ALGO_AUTO, ALGO_DENSE_TC_WS):
        workspace = new_workspace(ALGO_DENSE_TC_WS, X.dtype, Cout, Cin, X.device)
    Y = out if out is not None else torch.empty((N, Cout), dtype=torch.float32, device=X.device)
    wp, wb = _ws(workspace)
    _check(lib().cci_bbs_linear(X.data_ptr(), _dtype_code(X), N, Cin, values.data_ptr(), idx.data_ptr(), Cout,
                                G, K, Y.data_ptr(), status.data_ptr() if status is not None else None, algo, wp,
                                wb, _stream(X.device)), "cci_bbs_linear")
    return Y


def td_mask(W: torch.Tensor, G: int, K: int, rate: float, uniforms: torch.Tensor, *,
            out: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
            status: Optional[torch.Tensor] = None):
    """(W_out, mask) of one targeted-dropout step (``cci_td_mask``): candidates (the
    weights packing would drop) zeroed where ``uniforms < rate``."""
    _cuda_contig(W, "W")
    _cuda_contig(uniforms, "uniforms")
    Cout, R = W.shape
    Wo = out if out is not None else torch.empty_like(W)
    m = mask if mask is not None else torch.empty((Cout, R), dtype=torch.uint8, device=W.device)
    _check(lib().cci_td_mask(W.data_ptr(), _dtype_code(W), Cout, R, G, K, float(rate), uniforms.data_ptr(),
                             Wo.data_ptr(), m.data_ptr(), status.data_ptr() if status is not None else None,
                             _stream(W.device)), "cci_td_mask")
    return Wo, m


def td_drop_rate(step: int, ramp_steps: int, start: float = 0.5, end: float = 1.0) -> float:
    """The candidate drop rate of Sec. 5.1 at ``step`` (``cci_td_drop_rate``): from
    ``start`` (50 %) toward ``end`` (100 %), linear over ``ramp_steps`` steps and then
    constant (the paper fixes the end points only)."""
    return float(lib().cci_td_drop_rate(int(step), int(ramp_steps), float(start), float(end)))


def pack_stats(W: torch.Tensor, G: int, K: int, counts: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Adds (nonzero weights of W, nonzero weights packing with (G, K) drops) into
    ``counts`` (int64 device tensor of 2, zeroed here when not given) and returns it
    (``cci_pack_stats``; read it after a sync)."""
    _cuda_contig(W, "W")
    Cout, R = W.shape
    if counts is None:
        counts = torch.zeros(2, dtype=torch.int64, device=W.device)
    _check(lib().cci_pack_stats(W.data_ptr(), _dtype_code(W), Cout, R, G, K, counts.data_ptr(),
                                _stream(W.device)), "cci_pack_stats")
    return counts


def _out_code(dtype: torch.dtype) -> int:
    if dtype == torch.float32:
        return F32
    if dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported output dtype {dtype}: float32 or bfloat16")


def linear_fused(X: torch.Tensor, values: torch.Tensor, idx: torch.Tensor, Cout: int, G: int, K: int, *,
                 bias: Optional[torch.Tensor] = None, relu: bool = False,
                 out_dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y[N][Cout] = relu?(product + bias) in ``out_dtype`` (fp32 or bf16), on a
    tensor-core family (``cci_linear_fused``: the fused one where AUTO takes it,
    else the workspace one, whose workspace is allocated here when not given)."""
    _cuda_contig(X, "X")
    N, Cin = X.shape
    if workspace is None:
        workspace = _workspace(_epilogue_bytes(X.dtype, Cin, Cin, Cout, G, K, False), X.device)
    Y = out if out is not None else torch.empty((N, Cout), dtype=out_dtype, device=X.device)
    if bias is not None:
        _cuda_contig(bias, "bias")
    wp, wb = _ws(workspace)
    code = lib().cci_linear_fused(X.data_ptr(), _dtype_code(X), N, Cin, values.data_ptr(), idx.data_ptr(),
                                  Cout, G, K, bias.data_ptr() if bias is not None else None, int(relu),
                                  _out_code(Y.dtype), Y.data_ptr(),
                                  status.data_ptr() if status is not None else None, wp, wb,
                                  _stream(X.device))
    _check(code, "cci_linear_fused")
    return Y


def conv2d_fused(X: torch.Tensor, values: torch.Tensor, idx: torch.Tensor, Cout: int, G: int, K: int,
                 KH: int, KW: int, stride=(1, 1), pad=(0, 0), *, bias: Optional[torch.Tensor] = None,
                 relu: bool = False, out_dtype: torch.dtype = torch.float32,
                 out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y NHWC [B][P][Q][Cout] = relu?(convolution + bias) in ``out_dtype`` (fp32 or
    bf16), on a tensor-core family (``cci_conv2d_fused``, as ``linear_fused``)."""
    _cuda_contig(X, "X")
    B, H, W, Cin = X.shape
    P, Q = conv_out_hw(H, W, KH, KW, stride, pad)
    Y = out if out is not None else torch.empty((B, max(P, 0), max(Q, 0), Cout), dtype=out_dtype,
                                                device=X.device)
    if workspace is None:
        workspace = _workspace(_epilogue_bytes(X.dtype, Cin, KH * KW * Cin, Cout, G, K, max(stride) > 2), X.device)
    if bias is not None:
        _cuda_contig(bias, "bias")
    wp, wb = _ws(workspace)
    code = lib().cci_conv2d_fused(X.data_ptr(), _dtype_code(X), B, H, W, Cin, values.data_ptr(),
                                  idx.data_ptr(), Cout, KH, KW, stride[0], stride[1], pad[0], pad[1], G, K,
                                  bias.data_ptr() if bias is not None else None, int(relu),
                                  _out_code(Y.dtype), Y.data_ptr(),
                                  status.data_ptr() if status is not None else None, wp, wb,
                                  _stream(X.device))
    _check(code, "cci_conv2d_fused")
    return Y


def dense_planes(W: torch.Tensor) -> torch.Tensor:
    """Dense weights W[Cout][R] (OHWI rows for a convolution) in the workspace
    layout of the dense tensor-core family (``cci_dense_planes``), for
    ``dense_linear_tc`` / ``dense_conv2d_tc``: bf16 as is, fp32 as its two
    operand planes (a byte tensor)."""
    _cuda_contig(W, "W")
    Cout = W.shape[0]
    R = W.numel() // Cout
    Wd = new_workspace(ALGO_DENSE_TC_WS, W.dtype, Cout, R, W.device)
    _check(lib().cci_dense_planes(W.data_ptr(), _dtype_code(W), Cout, R, Wd.data_ptr(), Wd.numel(),
                                  _stream(W.device)), "cci_dense_planes")
    return Wd


def dense_linear_tc(X: torch.Tensor, Wd: torch.Tensor, Cout: int, *, out: Optional[torch.Tensor] = None,
                    status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y[N][Cout] = X Wd^T on the library's tensor-core GEMM with dense weights and
    no decompression (``cci_dense_linear_tc``).  Wd is the dense family's workspace
    layout, as ``dense_planes`` writes it."""
    _cuda_contig(X, "X")
    _cuda_contig(Wd, "Wd")
    N, Cin = X.shape
    Y = out if out is not None else torch.empty((N, Cout), dtype=torch.float32, device=X.device)
    _check(lib().cci_dense_linear_tc(X.data_ptr(), _dtype_code(X), N, Cin, Wd.data_ptr(), Cout, Y.data_ptr(),
                                     status.data_ptr() if status is not None else None, _stream(X.device)),
           "cci_dense_linear_tc")
    return Y


def dense_conv2d_tc(X: torch.Tensor, Wd: torch.Tensor, Cout: int, KH: int, KW: int, stride=(1, 1), pad=(0, 0), *,
                    out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """NHWC convolution on the library's tensor-core GEMM with dense OHWI weights in
    the dense family's workspace layout and no decompression (``cci_dense_conv2d_tc``)."""
    _cuda_contig(X, "X")
    _cuda_contig(Wd, "Wd")
    B, H, W, Cin = X.shape
    P, Q = conv_out_hw(H, W, KH, KW, stride, pad)
    Y = out if out is not None else torch.empty((B, max(P, 0), max(Q, 0), Cout), dtype=torch.float32,
                                                device=X.device)
    _check(lib().cci_dense_conv2d_tc(X.data_ptr(), _dtype_code(X), B, H, W, Cin, Wd.data_ptr(), Cout, KH, KW,
                                     stride[0], stride[1], pad[0], pad[1], Y.data_ptr(),
                                     status.data_ptr() if status is not None else None, _stream(X.device)),
           "cci_dense_conv2d_tc")
    return Y


# ---------------------------------------------------------------------------
# the layers around a pruned projection.  Plain functions, as all of this binding: no graph is recorded for
# tensors that require gradients; a training step makes the *_backward calls itself
# ---------------------------------------------------------------------------

def _device(t: torch.Tensor, name: str) -> int:
    """Index of the GPU that holds t, which must be the current one: a call's kernels run there."""
    index = t.get_device()
    if index < 0:
        raise ValueError(f"{name} must be a CUDA tensor")
    if index != torch._C._cuda_getDevice():
        raise ValueError(f"{name} must be on the current CUDA device")
    return index


def _rows(t: torch.Tensor, name: str, index: Optional[int] = None) -> int:
    """Row stride of a matrix (on GPU `index`, where that is not known yet) whose rows are contiguous."""
    if index is not None and t.get_device() != index:
        raise ValueError(f"{name} must be a CUDA tensor on the call's device")
    if t.dim() != 2:
        raise ValueError(f"{name} must be a matrix")
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have contiguous rows")
    ld = t.stride(0) if rows > 1 else cols
    if ld < cols:
        raise ValueError(f"{name} must not have overlapping rows")
    return ld


def _vec(t: Optional[torch.Tensor], n: int, name: str, index: int, dtype: torch.dtype = torch.float32) -> Optional[int]:
    """Address of a contiguous vector of n elements on GPU `index` (None: NULL)."""
    if t is None:
        return None
    if t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor on the call's device")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.numel() != n:
        raise ValueError(f"{name} must have {n} elements")
    return t.data_ptr()


def _status_word(status: torch.Tensor, index: int) -> int:
    """Address of a status word (``new_status``) on GPU `index`."""
    if status.get_device() != index or status.dtype not in (torch.int32, torch.uint32) or status.numel() < 1:
        raise ValueError("status must be a 32-bit integer CUDA tensor on the call's device")
    return status.data_ptr()


def _space(workspace: torch.Tensor, index: int):
    """Address and bytes of a workspace on GPU `index`."""
    if workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA tensor on the call's device")
    return workspace.data_ptr(), workspace.nbytes


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *,
               eps: float = 1e-5, out: Optional[torch.Tensor] = None):
    """(y, mean, rstd) of the rows of x[N][D] (``cci_layer_norm``): y in x's dtype, the
    fp32 mean and 1 / sqrt(var + eps) of each row for the backward pass.  ``weight`` and ``bias``
    are fp32 [D]; x may have a row stride."""
    index = _device(x, "x")
    ld = _rows(x, "x")
    N, D = x.shape
    if out is not None:
        _like(out, (N, D), x.dtype, "out", index)
    y = out if out is not None else torch.empty((N, D), dtype=x.dtype, device=x.device)
    # small outputs are allocated one by one: views of one allocation cost the host more
    mean = torch.empty(N, dtype=torch.float32, device=x.device)
    rstd = torch.empty(N, dtype=torch.float32, device=x.device)
    _check(lib().cci_layer_norm(x.data_ptr(), _dtype_code(x), N, D, ld, _vec(weight, D, "weight", index),
                                _vec(bias, D, "bias", index), eps, y.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                torch._C._cuda_getCurrentRawStream(index)), "cci_layer_norm")
    return y, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        weight: Optional[torch.Tensor] = None, *, out: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """(dx, dweight, dbias) of ``layer_norm`` (``cci_layer_norm_backward_ex``): dx in x's dtype,
    the parameters' gradients fp32 [D], whether or not the forward call had them."""
    index = _device(x, "x")
    ldx, lddy = _rows(x, "x"), _rows(dy, "dy", index)
    N, D = x.shape
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must have x's shape and dtype")
    if out is not None:
        _like(out, (N, D), x.dtype, "out", index)
    dx = out if out is not None else torch.empty((N, D), dtype=x.dtype, device=x.device)
    dw = torch.empty(D, dtype=torch.float32, device=x.device)
    db = torch.empty(D, dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = _workspace(_norm_bytes(N, D, index), x.device)
    wp, wb = (None, 0) if workspace is None else _space(workspace, index)
    _check(lib().cci_layer_norm_backward_ex(dy.data_ptr(), lddy, x.data_ptr(), ldx, _dtype_code(x), N, D,
                                            _vec(mean, N, "mean", index), _vec(rstd, N, "rstd", index),
                                            _vec(weight, D, "weight", index), dx.data_ptr(), dw.data_ptr(),
                                            db.data_ptr(),
                                            None if status is None else _status_word(status, index),
                                            wp, wb,
                                            torch._C._cuda_getCurrentRawStream(index)), "cci_layer_norm_backward")
    return dx, dw, db


def _summed(x: torch.Tensor, residual: Optional[torch.Tensor], h: Optional[torch.Tensor]):
    """(device, N, D, ldx, residual's address and stride, h) of a root-mean-square norm's rows."""
    index = _device(x, "x")
    ld = _rows(x, "x")
    N, D = x.shape
    if residual is None:
        if h is not None:
            raise ValueError("h is written only where there is a residual")
        return index, N, D, ld, None, D, None
    ldr = _rows(residual, "residual", index)
    if residual.shape != x.shape or residual.dtype != x.dtype:
        raise ValueError("residual must have x's shape and dtype")
    if h is None:
        h = torch.empty((N, D), dtype=x.dtype, device=x.device)
    else:
        _like(h, (N, D), x.dtype, "h", index)
    return index, N, D, ld, residual.data_ptr(), ldr, h


def rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, *, residual: Optional[torch.Tensor] = None,
             eps: float = 1e-5, out: Optional[torch.Tensor] = None, h: Optional[torch.Tensor] = None):
    """(y, h, rstd) of the rows of x[N][D] (``cci_rms_norm``): h = x + residual and y = (x + residual) rstd weight in
    x's dtype, rstd the fp32 1 / sqrt(mean square + eps) of each row; without a residual h is x itself.  ``weight`` is
    fp32 [D]; x and residual may have row strides.  ``out`` takes y and ``h`` takes h, which may be the
    residual (the residual stream updated in place)."""
    index, N, D, ld, rp, ldr, h = _summed(x, residual, h)
    if out is not None:
        _like(out, (N, D), x.dtype, "out", index)
    y = out if out is not None else torch.empty((N, D), dtype=x.dtype, device=x.device)
    rstd = torch.empty(N, dtype=torch.float32, device=x.device)
    _check(lib().cci_rms_norm(x.data_ptr(), _dtype_code(x), N, D, ld, rp, ldr, _vec(weight, D, "weight", index), eps,
                              y.data_ptr(), None if h is None else h.data_ptr(), rstd.data_ptr(),
                              torch._C._cuda_getCurrentRawStream(index)), "cci_rms_norm")
    return y, x if h is None else h, rstd


def rms_norm_fp8(x: torch.Tensor, weight: Optional[torch.Tensor] = None, *, residual: Optional[torch.Tensor] = None,
                 group: int = 0, eps: float = 1e-5, h: Optional[torch.Tensor] = None):
    """(q, scales, h, rstd): ``rms_norm`` with y in 8 bits (``cci_rms_norm_fp8``), y = q * scale: q [N][D] of
    ``torch.float8_e4m3fn``, fp32 scales [N][1] (``group`` 0) or one per 128 columns, [N][ceil(D / 128)] (``group``
    128).  D a multiple of 8."""
    index, N, D, ld, rp, ldr, h = _summed(x, residual, h)
    q = torch.empty((N, D), dtype=torch.float8_e4m3fn, device=x.device)
    scales = torch.empty((N, -(-D // 128) if group else 1), dtype=torch.float32, device=x.device)
    rstd = torch.empty(N, dtype=torch.float32, device=x.device)
    _check(lib().cci_rms_norm_fp8(x.data_ptr(), _dtype_code(x), N, D, ld, rp, ldr, _vec(weight, D, "weight", index), eps,
                                  group, q.data_ptr(), scales.data_ptr(), None if h is None else h.data_ptr(),
                                  rstd.data_ptr(), torch._C._cuda_getCurrentRawStream(index)), "cci_rms_norm_fp8")
    return q, scales, x if h is None else h, rstd


def rms_norm_backward(dy: torch.Tensor, h: torch.Tensor, rstd: torch.Tensor, weight: Optional[torch.Tensor] = None, *,
                      dh: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None):
    """(dx, dweight) of ``rms_norm`` (``cci_rms_norm_backward``) from the gradient of y and, with ``dh``, the one that
    h has besides: dx, of x and of the residual alike, in h's dtype, the weight's gradient fp32 [D], whether or not the
    forward call had one."""
    index = _device(h, "h")
    ldh, lddy = _rows(h, "h"), _rows(dy, "dy", index)
    N, D = h.shape
    if dy.shape != h.shape or dy.dtype != h.dtype:
        raise ValueError("dy must have h's shape and dtype")
    lddh = D
    if dh is not None:
        lddh = _rows(dh, "dh", index)
        if dh.shape != h.shape or dh.dtype != h.dtype:
            raise ValueError("dh must have h's shape and dtype")
    if out is not None:
        _like(out, (N, D), h.dtype, "out", index)
    dx = out if out is not None else torch.empty((N, D), dtype=h.dtype, device=h.device)
    dw = torch.empty(D, dtype=torch.float32, device=h.device)
    if workspace is None:
        workspace = _workspace(_rms_bytes(N, D, index), h.device)
    wp, wb = (None, 0) if workspace is None else _space(workspace, index)
    _check(lib().cci_rms_norm_backward(dy.data_ptr(), lddy, h.data_ptr(), ldh, None if dh is None else dh.data_ptr(),
                                       lddh, _dtype_code(h), N, D, _vec(rstd, N, "rstd", index),
                                       _vec(weight, D, "weight", index), dx.data_ptr(), dw.data_ptr(), wp, wb,
                                       torch._C._cuda_getCurrentRawStream(index)), "cci_rms_norm_backward")
    return dx, dw


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, *, top: int = 0, ignore_index: int = -100,
                   status: Optional[torch.Tensor] = None):
    """(logp, entropy, stats, top_logp, top_idx) of the rows of logits[N][V] and one token (int64) each
    (``cci_token_logprobs``): the token's log probability (0 for ``ignore_index``), the row's entropy,
    (maximum, log of the sum of exp(x - maximum)) for the backward pass, and the ``top`` (at most 32)
    most probable tokens' log probabilities and indices, ties to the lower index (None for top = 0).
    The logits may have a row stride."""
    index = _device(logits, "logits")
    ld = _rows(logits, "logits")
    N, V = logits.shape
    logp = torch.empty(N, dtype=torch.float32, device=logits.device)
    entropy = torch.empty(N, dtype=torch.float32, device=logits.device)
    stats = torch.empty((N, 2), dtype=torch.float32, device=logits.device)
    top_logp = torch.empty((N, top), dtype=torch.float32, device=logits.device) if top else None
    top_idx = torch.empty((N, top), dtype=torch.int32, device=logits.device) if top else None
    _check(lib().cci_token_logprobs(logits.data_ptr(), _dtype_code(logits), N, V, ld,
                                    _vec(tokens, N, "tokens", index, torch.int64), ignore_index, top, logp.data_ptr(),
                                    entropy.data_ptr(), stats.data_ptr(), top_logp.data_ptr() if top else None,
                                    top_idx.data_ptr() if top else None,
                                    None if status is None else _status_word(status, index),
                                    torch._C._cuda_getCurrentRawStream(index)),
           "cci_token_logprobs")
    return logp, entropy, stats, top_logp, top_idx


def token_logprobs_backward(logits: torch.Tensor, tokens: Optional[torch.Tensor], stats: torch.Tensor, *,
                            dlogp: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                            dentropy: Optional[torch.Tensor] = None, ignore_index: int = -100,
                            out: Optional[torch.Tensor] = None,
                            status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of ``token_logprobs`` to the logits, in their dtype (``cci_token_logprobs_backward``):
    of logp weighted by ``dlogp`` and of the entropy weighted by ``dentropy`` (which needs ``entropy``, as
    the forward call returned it).  Rows padded by up to 64 logits keep their stride in the result, unless
    ``out`` is given; ``out`` may be the logits."""
    index = _device(logits, "logits")
    ld = _rows(logits, "logits")
    N, V = logits.shape
    if out is None:
        # a padded row's stride (rows then start on the same 16-byte words), not that of a wide matrix' slice
        ldd = ld if ld <= V + 64 else V
        out = torch.empty((N, ldd), dtype=logits.dtype, device=logits.device)
        if ldd != V:
            out = out[:, :V]
    else:
        ldd = _rows(out, "out", index)
        if out.shape != logits.shape or out.dtype != logits.dtype:
            raise ValueError("out must have the logits' shape and dtype")
    _check(lib().cci_token_logprobs_backward(logits.data_ptr(), _dtype_code(logits), N, V, ld,
                                             _vec(stats, 2 * N, "stats", index),
                                             _vec(tokens, N, "tokens", index, torch.int64), ignore_index,
                                             _vec(dlogp, N, "dlogp", index), _vec(entropy, N, "entropy", index),
                                             _vec(dentropy, N, "dentropy", index), out.data_ptr(), ldd,
                                             None if status is None else _status_word(status, index),
                                             torch._C._cuda_getCurrentRawStream(index)), "cci_token_logprobs_backward")
    return out


def distillation_loss(logits: torch.Tensor, top_idx: torch.Tensor, top_logp: torch.Tensor, *, temperature: float = 1.0,
                      tail: bool = False, status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """(loss, stats) of a student's logits[N][V] against a teacher's top_idx (int32) and top_logp (fp32) [N][k]
    (``cci_distillation_loss``; the lists of ``token_logprobs(..., top=k)`` on the teacher's logits, k at most 128): the
    cross entropy of the teacher's listed probabilities, renormalised at the temperature or, with ``tail``, as they are
    with all that is not listed as one more outcome; index -1 lists nothing.  ``stats`` [N][4] is for the backward
    pass.  The logits may have a row stride."""
    index = _device(logits, "logits")
    ld = _rows(logits, "logits")
    N, V = logits.shape
    ip, vp, k = _lists(top_idx, top_logp, N, index)
    loss = torch.empty(N, dtype=torch.float32, device=logits.device)
    stats = torch.empty((N, 4), dtype=torch.float32, device=logits.device)
    if workspace is None:
        workspace = _workspace(_distillation_bytes(N, V, index), logits.device)
    wp, wb = (None, 0) if workspace is None else _space(workspace, index)
    _check(lib().cci_distillation_loss(logits.data_ptr(), _dtype_code(logits), N, V, ld, ip, vp, k, temperature, int(tail),
                                       loss.data_ptr(), stats.data_ptr(),
                                       None if status is None else _status_word(status, index), wp, wb,
                                       torch._C._cuda_getCurrentRawStream(index)), "cci_distillation_loss")
    return loss, stats


def distillation_loss_backward(dloss: torch.Tensor, logits: torch.Tensor, top_idx: torch.Tensor, top_logp: torch.Tensor,
                               stats: torch.Tensor, *, temperature: float = 1.0, tail: bool = False,
                               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of ``distillation_loss`` to the logits, in their dtype (``cci_distillation_loss_backward``), from the
    fp32 gradient of each row's loss and the forward call's stats.  Rows padded by up to 64 logits keep their stride in
    the result, unless ``out`` is given; ``out`` may be the logits."""
    index = _device(logits, "logits")
    ld = _rows(logits, "logits")
    N, V = logits.shape
    ip, vp, k = _lists(top_idx, top_logp, N, index)
    out, ldd = _like_logits(logits, ld, out, index)
    _check(lib().cci_distillation_loss_backward(_vec(dloss, N, "dloss", index), logits.data_ptr(), _dtype_code(logits), N,
                                                V, ld, ip, vp, k, temperature, int(tail),
                                                _vec(stats, 4 * N, "stats", index), out.data_ptr(), ldd,
                                                torch._C._cuda_getCurrentRawStream(index)),
           "cci_distillation_loss_backward")
    return out


@functools.lru_cache(maxsize=4096)
def _distillation_bytes(N: int, V: int, device_index: int) -> int:
    with torch.cuda.device(device_index):
        return int(lib().cci_distillation_workspace_size(N, V))


def _lists(top_idx: torch.Tensor, top_logp: torch.Tensor, N: int, index: int):
    """Addresses and width of a teacher's lists [N][k]."""
    if top_idx.dim() != 2 or top_idx.shape[0] != N or top_logp.shape != top_idx.shape:
        raise ValueError(f"top_idx and top_logp must be ({N}, k)")
    k = top_idx.shape[1]
    return _vec(top_idx, N * k, "top_idx", index, torch.int32), _vec(top_logp, N * k, "top_logp", index), k


def _like_logits(logits: torch.Tensor, ld: int, out: Optional[torch.Tensor], index: int):
    """A gradient's rows for logits of row stride ld, and their stride."""
    N, V = logits.shape
    if out is None:
        # a padded row's stride (rows then start on the same 16-byte words), not that of a wide matrix' slice
        ldd = ld if ld <= V + 64 else V
        out = torch.empty((N, ldd), dtype=logits.dtype, device=logits.device)
        return (out[:, :V] if ldd != V else out), ldd
    ldd = _rows(out, "out", index)
    if out.shape != logits.shape or out.dtype != logits.dtype:
        raise ValueError("out must have the logits' shape and dtype")
    return out, ldd


def _act_code(act: str) -> int:
    code = ACTIVATIONS.get(act)
    if code is None:
        raise ValueError(f"unknown activation {act!r}: one of {', '.join(ACTIVATIONS)}")
    return code


def gated_workspace(call: int, dtype: torch.dtype, N: int, D: int, F: int, device) -> Optional[torch.Tensor]:
    """The workspace of a gated block's call (``GATED_FORWARD``, ``GATED_PACKED`` or ``GATED_BACKWARD``), from
    PyTorch memory: None when it needs none."""
    device = torch.device(device)
    index = device.index if device.index is not None else torch.cuda.current_device()
    return _workspace(_gated_bytes(call, F32 if dtype == torch.float32 else BF16, N, D, F, index), device)


@functools.lru_cache(maxsize=4096)
def _gated_bytes(call: int, dtype: int, N: int, D: int, F: int, device_index: int) -> int:
    with torch.cuda.device(device_index):  # some sizes depend on the device's SMs
        return int(lib().cci_gated_workspace_size(call, dtype, N, D, F))


def gated_linear(X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, *, act: str = "silu", save: bool = False,
                 out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None):
    """H[N][F] = act(X Wg^T) * (X Wu^T) in X's dtype (``cci_gated_linear``): both projections of a gated
    feed-forward block, the activation (a key of ``ACTIVATIONS``) and the product in one kernel.
    X [N][D], Wg and Wu dense [F][D]; D and F multiples of 8.  ``save``: returns (H, g, u) with the fp32
    pre-activations for ``gated_linear_backward``."""
    index = _device(X, "X")
    if not X.is_contiguous():
        raise ValueError("X must be contiguous")
    N, D = X.shape
    F = Wg.shape[0]
    _like(Wg, (F, D), X.dtype, "Wg", index)
    _like(Wu, (F, D), X.dtype, "Wu", index)
    code = _dtype_code(X)
    if out is not None:
        _like(out, (N, F), X.dtype, "out", index)
    H = out if out is not None else torch.empty((N, F), dtype=X.dtype, device=X.device)
    g = torch.empty((N, F), dtype=torch.float32, device=X.device) if save else None
    u = torch.empty((N, F), dtype=torch.float32, device=X.device) if save else None
    if workspace is None:
        workspace = _workspace(_gated_bytes(GATED_FORWARD, code, N, D, F, index), X.device)
    wp, wb = (None, 0) if workspace is None else _space(workspace, index)
    _check(lib().cci_gated_linear(X.data_ptr(), code, N, D, Wg.data_ptr(), Wu.data_ptr(), F, _act_code(act),
                                  H.data_ptr(), g.data_ptr() if save else None, u.data_ptr() if save else None,
                                  None if status is None else _status_word(status, index),
                                  wp, wb, torch._C._cuda_getCurrentRawStream(index)),
           "cci_gated_linear")
    return (H, g, u) if save else H


def gated_linear_packed(X: torch.Tensor, gate: Tuple[torch.Tensor, torch.Tensor],
                        up: Tuple[torch.Tensor, torch.Tensor], F: int, G: int, K: int, *, act: str = "silu",
                        out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``gated_linear`` with packed weights: ``gate`` and ``up`` are the (values, idx) pairs of ``pack``
    for [F][D] weights, both with (G, K) (``cci_gated_linear_packed``)."""
    index = _device(X, "X")
    if not X.is_contiguous():
        raise ValueError("X must be contiguous")
    N, D = X.shape
    if G < 1 or F % G:
        raise CCIError(3, "gated_linear_packed")
    for (v, i), name in ((gate, "gate"), (up, "up")):
        _like(v, (F // G, D, K), X.dtype, name + " values", index)
        _like(i, (F // G, D, K), torch.uint8, name + " idx", index)
    code = _dtype_code(X)
    if out is not None:
        _like(out, (N, F), X.dtype, "out", index)
    H = out if out is not None else torch.empty((N, F), dtype=X.dtype, device=X.device)
    if workspace is None:
        workspace = _workspace(_gated_bytes(GATED_PACKED, code, N, D, F, index), X.device)
    wp, wb = (None, 0) if workspace is None else _space(workspace, index)
    _check(lib().cci_gated_linear_packed(X.data_ptr(), code, N, D, gate[0].data_ptr(), gate[1].data_ptr(),
                                         up[0].data_ptr(), up[1].data_ptr(), F, G, K, _act_code(act), H.data_ptr(),
                                         None if status is None else _status_word(status, index), wp, wb,
                                         torch._C._cuda_getCurrentRawStream(index)), "cci_gated_linear_packed")
    return H


def gated_linear_backward(dH: torch.Tensor, X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, g: torch.Tensor,
                          u: torch.Tensor, *, act: str = "silu", need_dx: bool = True, need_dw: bool = True,
                          status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """(dX, dWg, dWu) of ``gated_linear`` (``cci_gated_linear_backward``) from the gradient of H and the saved
    g and u, each in X's dtype; None for those not asked for (``need_dx``, ``need_dw``)."""
    index = _device(X, "X")
    if not X.is_contiguous():
        raise ValueError("X must be contiguous")
    N, D = X.shape
    F = Wg.shape[0]
    _like(dH, (N, F), X.dtype, "dH", index)
    _like(Wg, (F, D), X.dtype, "Wg", index)
    _like(Wu, (F, D), X.dtype, "Wu", index)
    _like(g, (N, F), torch.float32, "g", index)
    _like(u, (N, F), torch.float32, "u", index)
    code = _dtype_code(X)
    dX = torch.empty_like(X) if need_dx else None
    dWg, dWu = (torch.empty_like(Wg), torch.empty_like(Wu)) if need_dw else (None, None)
    if workspace is None:
        workspace = _workspace(_gated_bytes(GATED_BACKWARD, code, N, D, F, index), X.device)
    wp, wb = (None, 0) if workspace is None else _space(workspace, index)
    _check(lib().cci_gated_linear_backward(dH.data_ptr(), X.data_ptr(), code, N, D, Wg.data_ptr(), Wu.data_ptr(), F,
                                           _act_code(act), g.data_ptr(), u.data_ptr(),
                                           dX.data_ptr() if need_dx else None, dWg.data_ptr() if need_dw else None,
                                           dWu.data_ptr() if need_dw else None,
                                           None if status is None else _status_word(status, index), wp, wb,
                                           torch._C._cuda_getCurrentRawStream(index)), "cci_gated_linear_backward")
    return dX, dWg, dWu


def head_workspace(call: int, dtype: torch.dtype, N: int, D: int, V: int, device) -> Optional[torch.Tensor]:
    """The workspace of a head's cross entropy (``HEAD_FORWARD`` or ``HEAD_BACKWARD``), from PyTorch memory: None
    when it needs none."""
    device = torch.device(device)
    index = device.index if device.index is not None else torch.cuda.current_device()
    return _workspace(_head_bytes(call, F32 if dtype == torch.float32 else BF16, N, D, V, index), device)


@functools.lru_cache(maxsize=4096)
def _head_bytes(call: int, dtype: int, N: int, D: int, V: int, device_index: int) -> int:
    with torch.cuda.device(device_index):  # depends on the device's SMs
        return int(lib().cci_head_workspace_size(call, dtype, N, D, V))


def _head_operands(X: torch.Tensor, W: torch.Tensor):
    """(device, N, D, V, type's code) of a head's inputs and weights."""
    index = _device(X, "X")
    if X.dim() != 2 or not X.is_contiguous():
        raise ValueError("X must be a contiguous matrix")
    if W.dim() != 2:
        raise ValueError("W must be a matrix")
    N, D = X.shape
    V = W.shape[0]
    _like(W, (V, D), X.dtype, "W", index)
    return index, N, D, V, _dtype_code(X)


def linear_cross_entropy(X: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, *, ignore_index: int = -100,
                         status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """(loss, stats) of the logits X W^T and one target (int64) a row, without keeping the logits
    (``cci_linear_cross_entropy``): the fp32 loss of each row (0 for ``ignore_index``) and (maximum, log of the sum
    of exp(logit - maximum)) for the backward pass.  X [N][D], W [V][D]; D a multiple of 8, V of any size."""
    index, N, D, V, code = _head_operands(X, W)
    loss = torch.empty(N, dtype=torch.float32, device=X.device)
    stats = torch.empty((N, 2), dtype=torch.float32, device=X.device)
    if workspace is None:
        workspace = _workspace(_head_bytes(HEAD_FORWARD, code, N, D, V, index), X.device)
    wp, wb = (None, 0) if workspace is None else _space(workspace, index)
    _check(lib().cci_linear_cross_entropy(X.data_ptr(), code, N, D, W.data_ptr(), V,
                                          _vec(targets, N, "targets", index, torch.int64), ignore_index,
                                          loss.data_ptr(), stats.data_ptr(),
                                          None if status is None else _status_word(status, index), wp, wb,
                                          torch._C._cuda_getCurrentRawStream(index)), "cci_linear_cross_entropy")
    return loss, stats


def linear_cross_entropy_backward(dloss: torch.Tensor, X: torch.Tensor, W: torch.Tensor, targets: torch.Tensor,
                                  stats: torch.Tensor, *, ignore_index: int = -100, need_dx: bool = True,
                                  need_dw: bool = True, status: Optional[torch.Tensor] = None,
                                  workspace: Optional[torch.Tensor] = None):
    """(dX, dW) of ``linear_cross_entropy`` (``cci_linear_cross_entropy_backward``) from the fp32 gradient of each
    row's loss and the forward call's stats, each in X's dtype; None for those not asked for (``need_dx``,
    ``need_dw``)."""
    index, N, D, V, code = _head_operands(X, W)
    dX = torch.empty_like(X) if need_dx else None
    dW = torch.empty_like(W) if need_dw else None
    if workspace is None:
        workspace = _workspace(_head_bytes(HEAD_BACKWARD, code, N, D, V, index), X.device)
    wp, wb = (None, 0) if workspace is None else _space(workspace, index)
    _check(lib().cci_linear_cross_entropy_backward(_vec(dloss, N, "dloss", index), X.data_ptr(), code, N, D,
                                                   W.data_ptr(), V, _vec(targets, N, "targets", index, torch.int64),
                                                   ignore_index, _vec(stats, 2 * N, "stats", index),
                                                   dX.data_ptr() if need_dx else None,
                                                   dW.data_ptr() if need_dw else None,
                                                   None if status is None else _status_word(status, index), wp, wb,
                                                   torch._C._cuda_getCurrentRawStream(index)),
           "cci_linear_cross_entropy_backward")
    return dX, dW


def _like(t: torch.Tensor, shape, dtype: torch.dtype, name: str, index: int) -> None:
    if t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor on the call's device")
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError(f"{name} must be {tuple(shape)} of {dtype}")


@functools.lru_cache(maxsize=4096)
def _norm_bytes(N: int, D: int, device_index: int) -> int:
    with torch.cuda.device(device_index):
        return int(lib().cci_layer_norm_workspace_size(N, D))


@functools.lru_cache(maxsize=4096)
def _rms_bytes(N: int, D: int, device_index: int) -> int:
    with torch.cuda.device(device_index):
        return int(lib().cci_rms_norm_workspace_size(N, D))


def kernel_name(dtype: torch.dtype, Cin: int, R: int, Cout: int, G: int, K: int,
                algo: int = ALGO_AUTO) -> str:
    """The kernel family a call would run (``cci_kernel_name``; for AUTO: given the
    workspace ``auto_workspace`` provides)."""
    code = F32 if dtype == torch.float32 else BF16
    return lib().cci_kernel_name(code, Cin, R, Cout, G, K, algo).decode()


def auto_workspace(dtype: torch.dtype, Cin: int, R: int, Cout: int, G: int, K: int,
                   device, stride: int = 1) -> Optional[torch.Tensor]:
    """The workspace AUTO needs to reach its fastest family for a layer (R = Cin
    for a product, KH*KW*Cin for a convolution of the given largest stride), from
    PyTorch memory: None when that family needs none (the library allocates
    nothing itself)."""
    return _workspace(_auto_bytes(dtype, Cin, R, Cout, G, K, stride > 2), device)


# What a layer's sizes alone settle, looked up once per layer shape: these
# questions to the library took 5 of the 17 us that a call spent in Python.
@functools.lru_cache(maxsize=4096)
def _auto_bytes(dtype: torch.dtype, Cin: int, R: int, Cout: int, G: int, K: int, wide_stride: bool) -> int:
    """Workspace bytes with which AUTO reaches its fastest family (0: none needed)."""
    if _fused_first(dtype, Cin, R, Cout, G, K, wide_stride):
        return 0
    if not kernel_name(dtype, Cin, R, Cout, G, K, ALGO_DENSE_TC_WS):
        return 0
    return workspace_size(ALGO_DENSE_TC_WS, dtype, Cout, R)


@functools.lru_cache(maxsize=4096)
def _epilogue_bytes(dtype: torch.dtype, Cin: int, R: int, Cout: int, G: int, K: int, wide_stride: bool) -> int:
    """Workspace bytes of the entry points with an output stage (0: none needed)."""
    if _fused_first(dtype, Cin, R, Cout, G, K, wide_stride):
        return 0
    return workspace_size(ALGO_DENSE_TC_WS, dtype, Cout, R)


def _fused_first(dtype, Cin, R, Cout, G, K, wide_stride) -> bool:
    return kernel_name(dtype, Cin, R, Cout, G, K, ALGO_AUTO).startswith("dense_tc_fused") and not wide_stride


def _workspace(nbytes: int, device) -> Optional[torch.Tensor]:
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def fma_probe(out: torch.Tensor, blocks: int, threads: int, iters: int) -> None:
    _check(lib().cci_fma_probe(out.data_ptr(), blocks, threads, iters, _stream(out.device)),
           "cci_fma_probe")
