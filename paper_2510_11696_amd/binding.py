"""ctypes binding of libqerl_nvfp4.so: argument marshalling only.

Every function takes torch tensors living on the GPU, checks dtypes/devices,
and passes raw device pointers, sizes and the current HIP stream to the C ABI
declared in include/qerl_nvfp4.h.  No arithmetic of the method happens here and
there is no fallback: if the library is missing or a tensor is not on the GPU
the call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqerl_nvfp4.so")

_c_i64 = ctypes.c_int64
_c_sz = ctypes.c_size_t
_c_p = ctypes.c_void_p

_SIGNATURES = {
    "qerl_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "qerl_last_hip_error": (ctypes.c_int, []),
    "nvfp4_quantize": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p, _c_sz, _c_p]),
    "nvfp4_quantize_workspace_bytes": (_c_sz, [_c_i64, _c_i64]),
    "nvfp4_dequantize": (ctypes.c_int, [_c_p, _c_p, _c_p, _c_i64, _c_i64, _c_p, _c_p]),
    "nvfp4_lora_linear": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_i64,
                                         _c_p, _c_p, _c_i64, ctypes.c_float, _c_p, _c_i64,
                                         _c_p, _c_sz, _c_p]),
    "nvfp4_lora_linear_workspace_bytes": (_c_sz, [_c_i64, _c_i64, _c_i64, _c_i64]),
    "nvfp4_prepack_bytes": (_c_sz, [_c_i64, _c_i64]),
    "nvfp4_prepack": (ctypes.c_int, [_c_p, _c_p, _c_i64, _c_i64, _c_p, _c_p]),
    "nvfp4_lora_linear_packed": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_i64,
                                                _c_p, _c_p, _c_i64, ctypes.c_float, _c_p, _c_i64,
                                                _c_p, _c_sz, _c_p]),
    "nvfp4_lora_linear_packed_noalloc_max_bytes": (_c_sz, []),
    "nvfp4_lora_linear_packed_noalloc": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_i64,
                                                        _c_p, _c_p, _c_i64, ctypes.c_float, _c_p, _c_i64, _c_p]),
    "nvfp4_lora_linear_swiglu_workspace_bytes": (_c_sz, [_c_i64, _c_i64, _c_i64, _c_i64]),
    "nvfp4_lora_linear_packed_swiglu": (ctypes.c_int, [_c_p, _c_p, _c_i64, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_i64,
                                                       _c_p, _c_p, _c_i64, ctypes.c_float, _c_p, _c_i64,
                                                       _c_p, _c_sz, _c_p]),
    "nvfp4_prepack_t_bytes": (_c_sz, [_c_i64, _c_i64]),
    "nvfp4_prepack_t": (ctypes.c_int, [_c_p, _c_p, _c_i64, _c_i64, _c_p, _c_p]),
    "nvfp4_lora_linear_backward_workspace_bytes": (_c_sz, [_c_i64, _c_i64, _c_i64, _c_i64]),
    "nvfp4_lora_linear_backward_group_workspace_bytes": (_c_sz, [_c_i64, _c_i64, _c_p, ctypes.c_int]),
    "nvfp4_lora_linear_backward_group": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, ctypes.c_int, _c_p, _c_i64, _c_p, _c_sz, _c_p]),
    "nvfp4_lora_linear_backward": (ctypes.c_int, [_c_p, _c_p, _c_i64, _c_i64, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p,
                                                  _c_i64, ctypes.c_float, _c_p, _c_i64, _c_p, _c_p, _c_p, _c_sz, _c_p]),
    "nvfp4_lora_linear_packed_group": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, ctypes.c_int,
                                                      _c_p, _c_sz, _c_p]),
    "qerl_workspace_init": (ctypes.c_int, [_c_p, _c_sz, _c_p]),
    "aqn_rmsnorm": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, ctypes.c_float,
                                   _c_p, _c_i64, _c_p]),
    "aqn_rmsnorm_lora_down": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, ctypes.c_float,
                                             _c_p, _c_i64, _c_p, _c_p, _c_p, ctypes.c_int, _c_p]),
    "aqn_sigma": (ctypes.c_double, [ctypes.c_int, ctypes.c_int, ctypes.c_double, ctypes.c_double]),
    "aqn_sigma_schedule": (ctypes.c_double, [ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_double, ctypes.c_double]),
    "aqn_noise_fill": (ctypes.c_int, [_c_p, _c_i64, ctypes.c_float, ctypes.c_uint64, ctypes.c_uint64, _c_p]),
    "mxfp4_quantize": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p]),
    "mxfp4_dequantize": (ctypes.c_int, [_c_p, _c_p, _c_i64, _c_i64, _c_p, _c_p]),
    "mxfp8_quantize": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p]),
    "mxfp4_prepack_bytes": (_c_sz, [_c_i64, _c_i64]),
    "mxfp4_prepack": (ctypes.c_int, [_c_p, _c_p, _c_i64, _c_i64, _c_p, _c_p]),
    "mxfp4_linear_native_workspace_bytes": (_c_sz, [_c_i64, _c_i64, _c_i64]),
    "mxfp4_linear_native": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_i64, _c_p, _c_i64, _c_p, _c_sz, _c_p]),
    "mxfp4_lora_linear_native_workspace_bytes": (_c_sz, [_c_i64, _c_i64, _c_i64, _c_i64]),
    "mxfp4_lora_linear_native": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_i64, _c_p, _c_p, _c_i64, ctypes.c_float, _c_p,
                                                _c_p, _c_i64, _c_p, _c_sz, _c_p]),
    "aqn_rmsnorm_nvfp4_lora_linear_group_workspace_bytes": (_c_sz, [_c_i64, _c_i64, _c_p, _c_p, ctypes.c_int]),
    "aqn_rmsnorm_nvfp4_lora_linear_group": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, ctypes.c_float,
                                                           _c_p, ctypes.c_int, _c_p, _c_sz, _c_p]),
    "aqn_rmsnorm_nvfp4_lora_mlp_workspace_bytes": (_c_sz, [_c_i64] * 7),
    "aqn_rmsnorm_nvfp4_lora_mlp": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, ctypes.c_float,
                                                  _c_p, _c_p, _c_p, _c_p, _c_sz, _c_p]),
    "lm_head_prepack_t_bytes": (_c_sz, [_c_i64, _c_i64]),
    "lm_head_prepack_t": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p]),
    "lm_head_logprob_workspace_bytes": (_c_sz, [_c_i64, _c_i64, _c_i64, ctypes.c_int]),
    "lm_head_logprob": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_i64, _c_i64, _c_p, ctypes.c_float, _c_p, _c_p, _c_p,
                                       _c_p, _c_sz, _c_p]),
    "lm_head_logprob_grad": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_i64, _c_i64, _c_p, _c_p, ctypes.c_float, _c_p, _c_p,
                                            _c_p, _c_p, _c_i64, _c_p, _c_sz, _c_p]),
    "lm_head_logprob_backward": (ctypes.c_int, [_c_p, _c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_i64, _c_p]),
    "lora_adamw_plan_bytes": (_c_sz, [_c_p, ctypes.c_int]),
    "lora_adamw_state_elements": (_c_i64, [_c_p, ctypes.c_int]),
    "lora_adamw_make_plan": (ctypes.c_int, [_c_p, ctypes.c_int, _c_p, _c_sz, _c_p, _c_p]),
    "lora_adamw_check_state": (ctypes.c_int, [_c_p, ctypes.c_int, _c_p, _c_p]),
    "lora_adamw_step": (ctypes.c_int, [_c_p, _c_p, _c_p, _c_p]),
    "lora_adamw_grad_norm": (ctypes.c_int, [_c_p, ctypes.c_double, _c_p, _c_p, _c_p]),
    "lora_adamw_moments": (ctypes.c_int, [_c_p, _c_p, _c_p, _c_p, _c_p]),
    "qerl_workspace_status": (ctypes.c_int, [_c_p, _c_p]),
    "qerl_status_from_error_word": (ctypes.c_int, [ctypes.c_uint32]),
    "qerl_selftest_wait_gives_up": (ctypes.c_int, [_c_p, ctypes.c_size_t, ctypes.c_uint32, _c_p]),
    "qerl_peak_stream_read": (ctypes.c_int, [_c_p, _c_sz, ctypes.c_int, ctypes.c_int, _c_p, _c_p]),
    "qerl_peak_mfma_bf16": (ctypes.c_int, [_c_p, ctypes.c_int, ctypes.c_int, _c_p, _c_p]),
}

EXPORTED_SYMBOLS = tuple(_SIGNATURES)

_lib = None


class QerlError(RuntimeError):
    def __init__(self, fn: str, status: int, detail: str):
        super().__init__(f"{fn} failed with status {status}: {detail}")
        self.status = status


def load_library() -> ctypes.CDLL:
    """Load the HIP library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -m paper_2510_11696_amd.build`")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def _check(fn: str, status: int) -> None:
    if status != 0:
        lib = load_library()
        detail = lib.qerl_status_string(status).decode()
        if status == -5:
            detail += f" (hipError_t {lib.qerl_last_hip_error()})"
        raise QerlError(fn, status, detail)


def _dev(t: torch.Tensor, dtype, name: str) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str):
    """(rows, cols, leading dimension) of a 2-D tensor with unit inner stride."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be 2-D with contiguous rows")
    ld = t.stride(0) if t.shape[0] > 1 else max(t.shape[1], t.stride(0))
    return t.shape[0], t.shape[1], ld


def _stream() -> int:
    """The current device's current stream (torch.cuda.current_stream().cuda_stream, without the objects in between: two microseconds a call)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _here(device, name: str) -> None:
    """Launches go to the current device's current stream: tensors of another device are refused."""
    if device.index != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on {device}, the current device is cuda:{torch._C._cuda_getDevice()}")


def _flat(t: torch.Tensor, dtype, n: int, device, name: str) -> int:
    p = _dev(t, dtype, name)
    if not t.is_contiguous() or t.numel() != n or t.device != device:
        raise ValueError(f"{name} must be contiguous, of {n} elements, on {device}")
    return p


class Workspace:
    """Device scratch for nvfp4_lora_linear, initialised once."""

    def __init__(self, nbytes: int, device="cuda"):
        self.buf = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
        assert self.buf.data_ptr() % 256 == 0
        _check("qerl_workspace_init",
               load_library().qerl_workspace_init(self.buf.data_ptr(), self.buf.numel(), _stream()))

    @property
    def ptr(self) -> int:
        return self.buf.data_ptr()

    @property
    def nbytes(self) -> int:
        return self.buf.numel()


def aqn_rmsnorm_lora_down(x, gain, noise, eps, As, out: Optional[torch.Tensor] = None, ts=None):
    """RMSNorm as aqn_rmsnorm plus t_i = y A_i^T of the adapters As that read y, one launch (M <= 16).
    Each t_i comes as T_PARTS partial sums over slices of H, fp32 [T_PARTS, M, r_i] (t_i.sum(0) is the
    product).  Returns (y, [t_i]); pass the t_i as `ts` to nvfp4_lora_linear_packed_group."""
    lib = load_library()
    M, H, ldx = _rows(x, "x")
    if gain.numel() != H or not gain.is_contiguous():
        raise ValueError("gain must be contiguous [H]")
    n_ptr = None
    if noise is not None:
        if noise.numel() != H or not noise.is_contiguous():
            raise ValueError("noise must be contiguous [H]")
        n_ptr = _dev(noise, torch.float32, "noise")
    if out is None:
        out = torch.empty((M, H), dtype=torch.bfloat16, device=x.device)
    _, _, ldy = _rows(out, "out")
    n = len(As)
    for A in As:
        if A.dim() != 2 or A.shape[1] != H or not A.is_contiguous():
            raise ValueError("every A must be contiguous [r, H]")
    if ts is None:
        ts = [torch.empty((T_PARTS, M, A.shape[0]), dtype=torch.float32, device=x.device) for A in As]
    a_arr = (ctypes.c_void_p * n)(*[_dev(A, torch.bfloat16, "A") for A in As])
    r_arr = (ctypes.c_int64 * n)(*[A.shape[0] for A in As])
    t_arr = (ctypes.c_void_p * n)(*[_dev(t, torch.float32, "t") for t in ts])
    _check("aqn_rmsnorm_lora_down", lib.aqn_rmsnorm_lora_down(
        _dev(x, torch.bfloat16, "x"), M, H, ldx, _dev(gain, torch.bfloat16, "gain"), n_ptr, float(eps),
        _dev(out, torch.bfloat16, "out"), ldy, ctypes.cast(a_arr, _c_p), ctypes.cast(r_arr, _c_p),
        ctypes.cast(t_arr, _c_p), n, _stream()))
    return out, ts


def aqn_sigma(stage: int, num_stages: int, sigma_start: float, sigma_end: float) -> float:
    return float(load_library().aqn_sigma(stage, num_stages, sigma_start, sigma_end))


SCHEDULE_KINDS = {"exponential": 0, "linear": 1, "cosine": 2, "logarithmic": 3}


def aqn_sigma_schedule(kind: str, stage: int, num_stages: int, sigma_start: float, sigma_end: float) -> float:
    return float(load_library().aqn_sigma_schedule(SCHEDULE_KINDS[kind], stage, num_stages, sigma_start, sigma_end))


def aqn_noise_fill(n: int, sigma: float, seed: int, subsequence: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """fp32 [n] on the GPU: N(0, sigma^2) noise, a pure function of (seed, subsequence, n, sigma)."""
    if out is None:
        out = torch.empty((n,), dtype=torch.float32, device="cuda")
    if out.numel() < n:
        raise ValueError("out is too small")
    _check("aqn_noise_fill", load_library().aqn_noise_fill(
        _dev(out, torch.float32, "out"), n, float(sigma), seed & (2 ** 64 - 1), subsequence & (2 ** 64 - 1), _stream()))
    return out


def nvfp4_quantize_workspace_bytes(N: int, K: int) -> int:
    return int(load_library().nvfp4_quantize_workspace_bytes(N, K))


def nvfp4_lora_linear_workspace_bytes(M: int, N: int, K: int, r: int) -> int:
    return int(load_library().nvfp4_lora_linear_workspace_bytes(M, N, K, r))


def nvfp4_quantize(W: torch.Tensor):
    """W[N,K] bf16 -> (codes[N,K/2] u8, scales[N,K/16] u8, tensor_scale[1] f32)."""
    lib = load_library()
    N, K, ldw = _rows(W, "W")
    dev = W.device
    codes = torch.empty((N, K // 2), dtype=torch.uint8, device=dev)
    scales = torch.empty((N, K // 16), dtype=torch.uint8, device=dev)
    ts = torch.empty(1, dtype=torch.float32, device=dev)
    ws = torch.empty(lib.nvfp4_quantize_workspace_bytes(N, K), dtype=torch.uint8, device=dev)
    _check("nvfp4_quantize", lib.nvfp4_quantize(
        _dev(W, torch.bfloat16, "W"), N, K, ldw, codes.data_ptr(), scales.data_ptr(), ts.data_ptr(),
        ws.data_ptr(), ws.numel(), _stream()))
    return codes, scales, ts


def nvfp4_dequantize(codes: torch.Tensor, scales: torch.Tensor, tensor_scale: torch.Tensor):
    lib = load_library()
    N, K2 = codes.shape
    K = 2 * K2
    out = torch.empty((N, K), dtype=torch.float32, device=codes.device)
    _check("nvfp4_dequantize", lib.nvfp4_dequantize(
        _dev(codes, torch.uint8, "codes"), _dev(scales, torch.uint8, "scales"),
        _dev(tensor_scale, torch.float32, "tensor_scale"), N, K, out.data_ptr(), _stream()))
    return out


def nvfp4_lora_linear(x, codes, scales, tensor_scale, A: Optional[torch.Tensor] = None,
                      B: Optional[torch.Tensor] = None, lora_scale: float = 0.0,
                      workspace: Optional[Workspace] = None, out: Optional[torch.Tensor] = None):
    """y[M,N] = tensor_scale * x . dequant(codes, scales)^T + lora_scale * (x A^T) B^T, bf16."""
    lib = load_library()
    M, K, ldx = _rows(x, "x")
    N = codes.shape[0]
    if codes.shape[1] * 2 != K or tuple(scales.shape) != (N, K // 16):
        raise ValueError("codes must be [N, K/2] and scales [N, K/16]")
    if not codes.is_contiguous() or not scales.is_contiguous():
        raise ValueError("codes and scales must be contiguous")
    r = 0
    a_ptr = b_ptr = None
    if A is not None and B is not None and A.shape[0] > 0:
        r = A.shape[0]
        if tuple(A.shape) != (r, K) or tuple(B.shape) != (N, r) or not A.is_contiguous() or not B.is_contiguous():
            raise ValueError("A must be contiguous [r, K] and B contiguous [N, r]")
        a_ptr, b_ptr = _dev(A, torch.bfloat16, "A"), _dev(B, torch.bfloat16, "B")
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=x.device)
    _, n_out, ldy = _rows(out, "out")
    if out.shape[0] != M or n_out != N:
        raise ValueError("out must be [M, N]")
    need = lib.nvfp4_lora_linear_workspace_bytes(M, N, K, r)
    if workspace is None:
        workspace = Workspace(need, x.device)
    _check("nvfp4_lora_linear", lib.nvfp4_lora_linear(
        _dev(x, torch.bfloat16, "x"), M, K, ldx, _dev(codes, torch.uint8, "codes"),
        _dev(scales, torch.uint8, "scales"), _dev(tensor_scale, torch.float32, "tensor_scale"), N,
        a_ptr, b_ptr, r, float(lora_scale), _dev(out, torch.bfloat16, "out"), ldy,
        workspace.ptr, workspace.nbytes, _stream()))
    return out


class PackedWeight:
    """Tile-packed NVFP4 weight (see nvfp4_prepack in the header) plus its shape."""

    def __init__(self, packed: torch.Tensor, tensor_scale: torch.Tensor, N: int, K: int):
        self.packed, self.tensor_scale, self.N, self.K = packed, tensor_scale, int(N), int(K)


def nvfp4_prepack(codes: torch.Tensor, scales: torch.Tensor, tensor_scale: torch.Tensor) -> PackedWeight:
    lib = load_library()
    N, K2 = codes.shape
    K = 2 * K2
    if tuple(scales.shape) != (N, K // 16) or not codes.is_contiguous() or not scales.is_contiguous():
        raise ValueError("codes must be contiguous [N, K/2] and scales contiguous [N, K/16]")
    packed = torch.empty(max(lib.nvfp4_prepack_bytes(N, K), 16), dtype=torch.uint8, device=codes.device)
    _check("nvfp4_prepack", lib.nvfp4_prepack(
        _dev(codes, torch.uint8, "codes"), _dev(scales, torch.uint8, "scales"), N, K,
        packed.data_ptr(), _stream()))
    return PackedWeight(packed, tensor_scale, N, K)


def nvfp4_lora_linear_packed(x, w: PackedWeight, A: Optional[torch.Tensor] = None,
                             B: Optional[torch.Tensor] = None, lora_scale: float = 0.0,
                             workspace: Optional[Workspace] = None, out: Optional[torch.Tensor] = None):
    """Same result as nvfp4_lora_linear, from tile-packed weights."""
    lib = load_library()
    M, K, ldx = _rows(x, "x")
    N = w.N
    if K != w.K:
        raise ValueError("x has the wrong number of columns")
    r = 0
    a_ptr = b_ptr = None
    if A is not None and B is not None and A.shape[0] > 0:
        r = A.shape[0]
        if tuple(A.shape) != (r, K) or tuple(B.shape) != (N, r) or not A.is_contiguous() or not B.is_contiguous():
            raise ValueError("A must be contiguous [r, K] and B contiguous [N, r]")
        a_ptr, b_ptr = _dev(A, torch.bfloat16, "A"), _dev(B, torch.bfloat16, "B")
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=x.device)
    _, n_out, ldy = _rows(out, "out")
    if out.shape[0] != M or n_out != N:
        raise ValueError("out must be [M, N]")
    if workspace is None:
        workspace = Workspace(lib.nvfp4_lora_linear_workspace_bytes(M, N, K, r), x.device)
    _check("nvfp4_lora_linear_packed", lib.nvfp4_lora_linear_packed(
        _dev(x, torch.bfloat16, "x"), M, K, ldx, _dev(w.packed, torch.uint8, "packed"),
        _dev(w.tensor_scale, torch.float32, "tensor_scale"), N, a_ptr, b_ptr, r, float(lora_scale),
        _dev(out, torch.bfloat16, "out"), ldy, workspace.ptr, workspace.nbytes, _stream()))
    return out


def nvfp4_lora_linear_packed_noalloc(x, w: PackedWeight, A: Optional[torch.Tensor], B: Optional[torch.Tensor],
                                     lora_scale: float, out: torch.Tensor):
    """nvfp4_lora_linear_packed on the library's own per-GPU scratch array: no workspace, nothing allocated
    (the caller brings `out`).  Calls on one GPU share that array and must not overlap."""
    lib = load_library()
    M, K, ldx = _rows(x, "x")
    if K != w.K:
        raise ValueError("x has the wrong number of columns")
    r = 0
    a_ptr = b_ptr = None
    if A is not None and B is not None and A.shape[0] > 0:
        r = A.shape[0]
        if tuple(A.shape) != (r, K) or tuple(B.shape) != (w.N, r) or not A.is_contiguous() or not B.is_contiguous():
            raise ValueError("A must be contiguous [r, K] and B contiguous [N, r]")
        a_ptr, b_ptr = _dev(A, torch.bfloat16, "A"), _dev(B, torch.bfloat16, "B")
    _, n_out, ldy = _rows(out, "out")
    if out.shape[0] != M or n_out != w.N:
        raise ValueError("out must be [M, N]")
    _check("nvfp4_lora_linear_packed_noalloc", lib.nvfp4_lora_linear_packed_noalloc(
        _dev(x, torch.bfloat16, "x"), M, K, ldx, _dev(w.packed, torch.uint8, "packed"),
        _dev(w.tensor_scale, torch.float32, "tensor_scale"), w.N, a_ptr, b_ptr, r, float(lora_scale),
        _dev(out, torch.bfloat16, "out"), ldy, _stream()))
    return out


def nvfp4_lora_linear_packed_swiglu(gate, up, w: PackedWeight, A: Optional[torch.Tensor] = None,
                                    B: Optional[torch.Tensor] = None, lora_scale: float = 0.0,
                                    workspace: Optional[Workspace] = None, out: Optional[torch.Tensor] = None):
    """The down projection applied to bf16(bf16(SiLU(gate)) * up)."""
    lib = load_library()
    M, K, ldg = _rows(gate, "gate")
    M2, K2, ldu = _rows(up, "up")
    N = w.N
    if K != w.K or (M2, K2) != (M, K):
        raise ValueError("gate and up must both be [M, K]")
    r = 0
    a_ptr = b_ptr = None
    if A is not None and B is not None and A.shape[0] > 0:
        r = A.shape[0]
        if tuple(A.shape) != (r, K) or tuple(B.shape) != (N, r) or not A.is_contiguous() or not B.is_contiguous():
            raise ValueError("A must be contiguous [r, K] and B contiguous [N, r]")
        a_ptr, b_ptr = _dev(A, torch.bfloat16, "A"), _dev(B, torch.bfloat16, "B")
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=gate.device)
    _, n_out, ldy = _rows(out, "out")
    if out.shape[0] != M or n_out != N:
        raise ValueError("out must be [M, N]")
    if workspace is None:
        workspace = Workspace(lib.nvfp4_lora_linear_swiglu_workspace_bytes(M, N, K, r), gate.device)
    _check("nvfp4_lora_linear_packed_swiglu", lib.nvfp4_lora_linear_packed_swiglu(
        _dev(gate, torch.bfloat16, "gate"), _dev(up, torch.bfloat16, "up"), M, K, ldg, ldu,
        _dev(w.packed, torch.uint8, "packed"), _dev(w.tensor_scale, torch.float32, "tensor_scale"), N, a_ptr, b_ptr, r,
        float(lora_scale), _dev(out, torch.bfloat16, "out"), ldy, workspace.ptr, workspace.nbytes, _stream()))
    return out


class PackedWeightT:
    """The transposed tile order of one NVFP4 weight (nvfp4_prepack_t), for the backward pass."""

    def __init__(self, packed, tensor_scale, N, K):
        self.packed, self.tensor_scale, self.N, self.K = packed, tensor_scale, N, K


def nvfp4_prepack_t(codes: torch.Tensor, scales: torch.Tensor, tensor_scale: torch.Tensor) -> PackedWeightT:
    lib = load_library()
    N, K = codes.shape[0], codes.shape[1] * 2
    if tuple(scales.shape) != (N, K // 16) or not codes.is_contiguous() or not scales.is_contiguous():
        raise ValueError("codes must be contiguous [N, K/2] and scales contiguous [N, K/16]")
    packed = torch.empty((lib.nvfp4_prepack_t_bytes(N, K),), dtype=torch.uint8, device=codes.device)
    _check("nvfp4_prepack_t", lib.nvfp4_prepack_t(_dev(codes, torch.uint8, "codes"), _dev(scales, torch.uint8, "scales"),
                                                  N, K, _dev(packed, torch.uint8, "packed"), _stream()))
    return PackedWeightT(packed, tensor_scale, N, K)


def _grad_buffer(t: Optional[torch.Tensor], shape, device, name: str) -> torch.Tensor:
    if t is None:
        return torch.empty(shape, dtype=torch.float32, device=device)
    if tuple(t.shape) != shape or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be contiguous {list(shape)} on {device}")
    return t


def nvfp4_lora_linear_backward(x, dy, w: PackedWeightT, A: Optional[torch.Tensor] = None,
                               B: Optional[torch.Tensor] = None, lora_scale: float = 0.0,
                               workspace: Optional[torch.Tensor] = None, dA: Optional[torch.Tensor] = None,
                               dB: Optional[torch.Tensor] = None):
    """(dx bf16 [M, K], dA fp32 [r, K] or None, dB fp32 [N, r] or None).  dA, dB: where to write the gradients (an optimizer's
    buffers), or None for new tensors; without rows they are zero."""
    lib = load_library()
    M, N, lddy = _rows(dy, "dy")
    K = w.K
    if N != w.N:
        raise ValueError("dy has the wrong number of columns")
    r = 0
    x_ptr = a_ptr = b_ptr = da_ptr = db_ptr = None
    ldx = K
    if A is not None and B is not None and A.shape[0] > 0:
        r = A.shape[0]
        if tuple(A.shape) != (r, K) or tuple(B.shape) != (N, r) or not A.is_contiguous() or not B.is_contiguous():
            raise ValueError("A must be contiguous [r, K] and B contiguous [N, r]")
        Mx, Kx, ldx = _rows(x, "x")
        if (Mx, Kx) != (M, K):
            raise ValueError("x must be [M, K]")
        x_ptr = _dev(x, torch.bfloat16, "x")
        a_ptr, b_ptr = _dev(A, torch.bfloat16, "A"), _dev(B, torch.bfloat16, "B")
        dA, dB = _grad_buffer(dA, (r, K), dy.device, "dA"), _grad_buffer(dB, (N, r), dy.device, "dB")
        da_ptr, db_ptr = _dev(dA, torch.float32, "dA"), _dev(dB, torch.float32, "dB")
        if M == 0:
            dA.zero_()
            dB.zero_()
    elif dA is not None or dB is not None:
        raise ValueError("dA and dB belong to an adapter")
    dx = torch.empty((M, K), dtype=torch.bfloat16, device=dy.device)
    need = lib.nvfp4_lora_linear_backward_workspace_bytes(M, N, K, r)
    if workspace is None:
        workspace = torch.empty((need + 256,), dtype=torch.uint8, device=dy.device)
    base = workspace.data_ptr()
    ws_ptr = (base + 255) & ~255
    _check("nvfp4_lora_linear_backward", lib.nvfp4_lora_linear_backward(
        x_ptr, _dev(dy, torch.bfloat16, "dy"), M, K, N, ldx, lddy, _dev(w.packed, torch.uint8, "packed_t"),
        _dev(w.tensor_scale, torch.float32, "tensor_scale"), a_ptr, b_ptr, r, float(lora_scale),
        _dev(dx, torch.bfloat16, "dx"), K, da_ptr, db_ptr, ws_ptr, workspace.numel() - (ws_ptr - base), _stream()))
    return dx, dA, dB


class _BackwardDesc(ctypes.Structure):
    """Mirror of qerl_backward_desc in the header."""
    _fields_ = [("dy", _c_p), ("lddy", _c_i64), ("N", _c_i64), ("packed_t", _c_p), ("tensor_scale", _c_p), ("A", _c_p), ("B", _c_p),
                ("r", _c_i64), ("lora_scale", ctypes.c_float), ("dA", _c_p), ("dB", _c_p)]


def nvfp4_lora_linear_backward_group(x, dys, weights, As=None, Bs=None, lora_scales=None, workspace: Optional[torch.Tensor] = None,
                                     dAs=None, dBs=None):
    """Backward of several linears that read the same x: (dx bf16 [M, K] summed over the members, [(dA_i, dB_i)]).  dAs, dBs: lists of
    tensors (or None) to write the gradients to; without rows they are zero."""
    lib = load_library()
    n = len(weights)
    As = As if As is not None else [None] * n
    Bs = Bs if Bs is not None else [None] * n
    lora_scales = lora_scales if lora_scales is not None else [0.0] * n
    M, K, ldx = _rows(x, "x")
    if any(v is not None and len(v) != n for v in (dAs, dBs)):
        raise ValueError("dAs and dBs must have a place for every member")
    descs = (_BackwardDesc * n)()
    grads, keep = [], []
    for i, (dy, w) in enumerate(zip(dys, weights)):
        Mi, N, lddy = _rows(dy, "dy")
        if Mi != M or N != w.N or w.K != K:
            raise ValueError("every dy must be [M, N_i] and every member must have K columns")
        d = descs[i]
        d.dy, d.lddy, d.N = _dev(dy, torch.bfloat16, "dy"), lddy, N
        d.packed_t, d.tensor_scale = _dev(w.packed, torch.uint8, "packed_t"), _dev(w.tensor_scale, torch.float32, "tensor_scale")
        A, B = As[i], Bs[i]
        dA = dB = None
        if A is not None and B is not None and A.shape[0] > 0:
            r = A.shape[0]
            if tuple(A.shape) != (r, K) or tuple(B.shape) != (N, r) or not A.is_contiguous() or not B.is_contiguous():
                raise ValueError("A must be contiguous [r, K] and B contiguous [N, r]")
            dA = _grad_buffer(dAs[i] if dAs is not None else None, (r, K), x.device, "dA")
            dB = _grad_buffer(dBs[i] if dBs is not None else None, (N, r), x.device, "dB")
            d.A, d.B, d.r, d.lora_scale = _dev(A, torch.bfloat16, "A"), _dev(B, torch.bfloat16, "B"), r, float(lora_scales[i])
            d.dA, d.dB = _dev(dA, torch.float32, "dA"), _dev(dB, torch.float32, "dB")
            if M == 0:
                dA.zero_()
                dB.zero_()
        elif any(v is not None and v[i] is not None for v in (dAs, dBs)):
            raise ValueError("dA and dB belong to an adapter")
        grads.append((dA, dB))
        keep.append((dy, A, B))
    dx = torch.empty((M, K), dtype=torch.bfloat16, device=x.device)
    need = lib.nvfp4_lora_linear_backward_group_workspace_bytes(M, K, ctypes.cast(descs, _c_p), n)
    if need == 0:
        raise ValueError("a backward group has 1..4 members")
    if workspace is None:
        workspace = torch.empty((need + 256,), dtype=torch.uint8, device=x.device)
    base = workspace.data_ptr()
    ws_ptr = (base + 255) & ~255
    _check("nvfp4_lora_linear_backward_group", lib.nvfp4_lora_linear_backward_group(
        _dev(x, torch.bfloat16, "x"), M, K, ldx, ctypes.cast(descs, _c_p), n, _dev(dx, torch.bfloat16, "dx"), K,
        ws_ptr, workspace.numel() - (ws_ptr - base), _stream()))
    return dx, grads


T_PARTS = 8   # QERL_T_PARTS in the header


class _LinearDesc(ctypes.Structure):
    """Mirror of qerl_linear_desc in the header."""
    _fields_ = [("packed", _c_p), ("tensor_scale", _c_p), ("N", _c_i64), ("A", _c_p), ("B", _c_p),
                ("r", _c_i64), ("lora_scale", ctypes.c_float), ("y", _c_p), ("ldy", _c_i64), ("t", _c_p),
                ("bias", _c_p)]


def nvfp4_lora_linear_packed_group(x, weights, As=None, Bs=None, lora_scales=None,
                                   workspace: Optional[Workspace] = None, outs=None, ts=None, biases=None):
    """Several packed linears that read the same x (q/k/v, gate/up) in one launch.
    weights: list of PackedWeight; As/Bs: lists of LoRA matrices (or None); ts: optional list of
    precomputed x A^T (fp32 [M, r], from aqn_rmsnorm_lora_down); biases: optional list of bf16 [N]
    vectors (or None); returns the list of outputs."""
    lib = load_library()
    M, K, ldx = _rows(x, "x")
    n = len(weights)
    As = As if As is not None else [None] * n
    Bs = Bs if Bs is not None else [None] * n
    lora_scales = lora_scales if lora_scales is not None else [0.0] * n
    if outs is None:
        outs = [torch.empty((M, w.N), dtype=torch.bfloat16, device=x.device) for w in weights]
    descs = (_LinearDesc * n)()
    n_sum = r_sum = 0
    for i, w in enumerate(weights):
        if w.K != K:
            raise ValueError("every member must have K columns")
        r = 0
        a_ptr = b_ptr = None
        if As[i] is not None and Bs[i] is not None and As[i].shape[0] > 0:
            r = As[i].shape[0]
            if tuple(As[i].shape) != (r, K) or tuple(Bs[i].shape) != (w.N, r) or not As[i].is_contiguous() \
                    or not Bs[i].is_contiguous():
                raise ValueError("A must be contiguous [r, K] and B contiguous [N, r]")
            a_ptr, b_ptr = _dev(As[i], torch.bfloat16, "A"), _dev(Bs[i], torch.bfloat16, "B")
        _, n_out, ldy = _rows(outs[i], "out")
        if outs[i].shape[0] != M or n_out != w.N:
            raise ValueError("out must be [M, N]")
        t_ptr = None
        if ts is not None and ts[i] is not None and r > 0:
            if tuple(ts[i].shape) != (T_PARTS, M, r) or not ts[i].is_contiguous():
                raise ValueError("t must be contiguous [T_PARTS, M, r] as aqn_rmsnorm_lora_down writes it")
            t_ptr = _dev(ts[i], torch.float32, "t")
        bias_ptr = None
        if biases is not None and biases[i] is not None:
            if tuple(biases[i].shape) != (w.N,) or not biases[i].is_contiguous():
                raise ValueError("bias must be contiguous [N]")
            bias_ptr = _dev(biases[i], torch.bfloat16, "bias")
        descs[i] = _LinearDesc(_dev(w.packed, torch.uint8, "packed"),
                               _dev(w.tensor_scale, torch.float32, "tensor_scale"), w.N, a_ptr, b_ptr, r,
                               float(lora_scales[i]), _dev(outs[i], torch.bfloat16, "out"), ldy, t_ptr, bias_ptr)
        n_sum += w.N
        r_sum += r
    if workspace is None:
        workspace = Workspace(lib.nvfp4_lora_linear_workspace_bytes(M, n_sum, K, r_sum), x.device)
    _check("nvfp4_lora_linear_packed_group", lib.nvfp4_lora_linear_packed_group(
        _dev(x, torch.bfloat16, "x"), M, K, ldx, ctypes.cast(descs, _c_p), n,
        workspace.ptr, workspace.nbytes, _stream()))
    return outs


def _make_desc(w: PackedWeight, A, B, lora_scale, out, bias, K):
    """One qerl_linear_desc from torch tensors (out may be None: y = NULL); returns (desc, r)."""
    if w.K != K:
        raise ValueError("every member must have K columns")
    r = 0
    a_ptr = b_ptr = None
    if A is not None and B is not None and A.shape[0] > 0:
        r = A.shape[0]
        if tuple(A.shape) != (r, K) or tuple(B.shape) != (w.N, r) or not A.is_contiguous() or not B.is_contiguous():
            raise ValueError("A must be contiguous [r, K] and B contiguous [N, r]")
        a_ptr, b_ptr = _dev(A, torch.bfloat16, "A"), _dev(B, torch.bfloat16, "B")
    y_ptr, ldy = None, 0
    if out is not None:
        _, n_out, ldy = _rows(out, "out")
        if n_out != w.N:
            raise ValueError("out must be [M, N]")
        y_ptr = _dev(out, torch.bfloat16, "out")
    bias_ptr = None
    if bias is not None:
        if tuple(bias.shape) != (w.N,) or not bias.is_contiguous():
            raise ValueError("bias must be contiguous [N]")
        bias_ptr = _dev(bias, torch.bfloat16, "bias")
    return _LinearDesc(_dev(w.packed, torch.uint8, "packed"), _dev(w.tensor_scale, torch.float32, "tensor_scale"),
                       w.N, a_ptr, b_ptr, r, float(lora_scale), y_ptr, ldy, None, bias_ptr), r


def _norm_args(x, gain, noise):
    M, H, ldx = _rows(x, "x")
    g_ptr = n_ptr = None
    if gain is not None:
        if gain.numel() != H or not gain.is_contiguous():
            raise ValueError("gain must be contiguous [H]")
        g_ptr = _dev(gain, torch.bfloat16, "gain")
        if noise is not None:
            if noise.numel() != H or not noise.is_contiguous():
                raise ValueError("noise must be contiguous [H]")
            n_ptr = _dev(noise, torch.float32, "noise")
    return M, H, ldx, g_ptr, n_ptr


def aqn_rmsnorm_nvfp4_lora_linear_group(x, gain, noise, eps, weights, As=None, Bs=None, lora_scales=None,
                                        workspace: Optional[Workspace] = None, outs=None, biases=None):
    """AQN RMSNorm of x (gain None: x as it is), then the packed linears `weights` on it, in one call.
    Returns the list of outputs."""
    lib = load_library()
    M, K, ldx, g_ptr, n_ptr = _norm_args(x, gain, noise)
    n = len(weights)
    As = As if As is not None else [None] * n
    Bs = Bs if Bs is not None else [None] * n
    lora_scales = lora_scales if lora_scales is not None else [0.0] * n
    biases = biases if biases is not None else [None] * n
    if outs is None:
        outs = [torch.empty((M, w.N), dtype=torch.bfloat16, device=x.device) for w in weights]
    descs = (_LinearDesc * n)()
    rs = []
    for i, w in enumerate(weights):
        if outs[i].shape[0] != M:
            raise ValueError("out must be [M, N]")
        descs[i], r = _make_desc(w, As[i], Bs[i], lora_scales[i], outs[i], biases[i], K)
        rs.append(r)
    if workspace is None:
        workspace = Workspace(aqn_rmsnorm_nvfp4_lora_linear_group_workspace_bytes(M, K, [w.N for w in weights], rs), x.device)
    _check("aqn_rmsnorm_nvfp4_lora_linear_group", lib.aqn_rmsnorm_nvfp4_lora_linear_group(
        _dev(x, torch.bfloat16, "x"), M, K, ldx, g_ptr, n_ptr, float(eps), ctypes.cast(descs, _c_p), n,
        workspace.ptr, workspace.nbytes, _stream()))
    return outs


def aqn_rmsnorm_nvfp4_lora_linear_group_workspace_bytes(M: int, K: int, Ns, rs) -> int:
    n = len(Ns)
    return int(load_library().aqn_rmsnorm_nvfp4_lora_linear_group_workspace_bytes(
        M, K, ctypes.cast((ctypes.c_int64 * n)(*Ns), _c_p), ctypes.cast((ctypes.c_int64 * n)(*rs), _c_p), n))


def aqn_rmsnorm_nvfp4_lora_mlp(x, gain, noise, eps, gate: PackedWeight, up: PackedWeight, down: PackedWeight,
                               As=(None, None, None), Bs=(None, None, None), lora_scales=(0.0, 0.0, 0.0),
                               workspace: Optional[Workspace] = None, out: Optional[torch.Tensor] = None):
    """Feed-forward block: AQN RMSNorm -> gate, up -> SiLU(gate) * up -> down, in one call.
    As / Bs / lora_scales are (gate, up, down) triples.  Returns down's output [M, down.N]."""
    lib = load_library()
    M, H, ldx, g_ptr, n_ptr = _norm_args(x, gain, noise)
    if gate.N != up.N or down.K != gate.N:
        raise ValueError("gate and up must have the same N, which is down's K")
    if out is None:
        out = torch.empty((M, down.N), dtype=torch.bfloat16, device=x.device)
    if out.shape[0] != M:
        raise ValueError("out must be [M, N]")
    dg, rg = _make_desc(gate, As[0], Bs[0], lora_scales[0], None, None, H)
    du, ru = _make_desc(up, As[1], Bs[1], lora_scales[1], None, None, H)
    dd, rd = _make_desc(down, As[2], Bs[2], lora_scales[2], out, None, gate.N)
    if workspace is None:
        workspace = Workspace(lib.aqn_rmsnorm_nvfp4_lora_mlp_workspace_bytes(M, H, gate.N, down.N, rg, ru, rd), x.device)
    _check("aqn_rmsnorm_nvfp4_lora_mlp", lib.aqn_rmsnorm_nvfp4_lora_mlp(
        _dev(x, torch.bfloat16, "x"), M, H, ldx, g_ptr, n_ptr, float(eps), ctypes.byref(dg), ctypes.byref(du),
        ctypes.byref(dd), workspace.ptr, workspace.nbytes, _stream()))
    return out


def workspace_status(workspace: Workspace) -> int:
    """0, or the negative status a kernel's abandoned wait left in the workspace (synchronises)."""
    return int(load_library().qerl_workspace_status(workspace.ptr, _stream()))


def aqn_rmsnorm(x, gain, noise: Optional[torch.Tensor] = None, eps: float = 1e-6,
                out: Optional[torch.Tensor] = None):
    """y = (gain + noise) * x / sqrt(mean(x^2) + eps), bf16; noise=None is the noise-free stage."""
    lib = load_library()
    M, H, ldx = _rows(x, "x")
    if gain.numel() != H or not gain.is_contiguous():
        raise ValueError("gain must be contiguous [H]")
    n_ptr = None
    if noise is not None:
        if noise.numel() != H or not noise.is_contiguous():
            raise ValueError("noise must be contiguous [H]")
        n_ptr = _dev(noise, torch.float32, "noise")
    if out is None:
        out = torch.empty((M, H), dtype=torch.bfloat16, device=x.device)
    _, _, ldy = _rows(out, "out")
    _check("aqn_rmsnorm", lib.aqn_rmsnorm(
        _dev(x, torch.bfloat16, "x"), M, H, ldx, _dev(gain, torch.bfloat16, "gain"), n_ptr,
        float(eps), _dev(out, torch.bfloat16, "out"), ldy, _stream()))
    return out


# ---- MXFP4 variant ---------------------------------------------------------------------------------
def mxfp4_quantize(W: torch.Tensor):
    """W [N, K] bf16 (rows may be strided) -> (codes [N, K/2] u8, scales [N, K/32] u8 E8M0)."""
    N, K, ldw = _rows(W, "W")
    codes = torch.empty((N, K // 2), dtype=torch.uint8, device=W.device)
    scales = torch.empty((N, K // 32), dtype=torch.uint8, device=W.device)
    _check("mxfp4_quantize", load_library().mxfp4_quantize(
        _dev(W, torch.bfloat16, "W"), N, K, ldw, _dev(codes, torch.uint8, "codes"), _dev(scales, torch.uint8, "scales"), _stream()))
    return codes, scales


def mxfp4_dequantize(codes: torch.Tensor, scales: torch.Tensor) -> torch.Tensor:
    N, K = codes.shape[0], codes.shape[1] * 2
    W = torch.empty((N, K), dtype=torch.float32, device=codes.device)
    _check("mxfp4_dequantize", load_library().mxfp4_dequantize(
        _dev(codes, torch.uint8, "codes"), _dev(scales, torch.uint8, "scales"), N, K, _dev(W, torch.float32, "W"), _stream()))
    return W


def mxfp8_quantize(x: torch.Tensor):
    """x [M, K] bf16 -> (codes [M, K] u8 E4M3, scales [M, K/32] u8 E8M0)."""
    M, K, ldx = _rows(x, "x")
    codes = torch.empty((M, K), dtype=torch.uint8, device=x.device)
    scales = torch.empty((M, K // 32), dtype=torch.uint8, device=x.device)
    _check("mxfp8_quantize", load_library().mxfp8_quantize(
        _dev(x, torch.bfloat16, "x"), M, K, ldx, _dev(codes, torch.uint8, "codes"), _dev(scales, torch.uint8, "scales"), _stream()))
    return codes, scales


class MxPackedWeight:
    """MXFP4 weights in the tile order of the scaled matrix instruction."""

    def __init__(self, packed: torch.Tensor, N: int, K: int):
        self.packed, self.N, self.K = packed, N, K


def mxfp4_prepack(codes: torch.Tensor, scales: torch.Tensor) -> MxPackedWeight:
    lib = load_library()
    N, K = codes.shape[0], codes.shape[1] * 2
    if not codes.is_contiguous() or not scales.is_contiguous() or tuple(scales.shape) != (N, K // 32):
        raise ValueError("codes [N, K/2] and scales [N, K/32] must be contiguous")
    packed = torch.empty((lib.mxfp4_prepack_bytes(N, K),), dtype=torch.uint8, device=codes.device)
    _check("mxfp4_prepack", lib.mxfp4_prepack(_dev(codes, torch.uint8, "codes"), _dev(scales, torch.uint8, "scales"), N, K,
                                              _dev(packed, torch.uint8, "packed"), _stream()))
    return MxPackedWeight(packed, N, K)


def mxfp4_linear_native(x: torch.Tensor, w: MxPackedWeight, workspace: Optional[torch.Tensor] = None,
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y = MXFP8(x) . MXFP4(W)^T on the block-scaled matrix instruction (any number of tokens)."""
    lib = load_library()
    M, K, ldx = _rows(x, "x")
    if K != w.K:
        raise ValueError("x must have K columns")
    if out is None:
        out = torch.empty((M, w.N), dtype=torch.bfloat16, device=x.device)
    _, n_out, ldy = _rows(out, "out")
    if out.shape[0] != M or n_out != w.N:
        raise ValueError("out must be [M, N]")
    need = lib.mxfp4_linear_native_workspace_bytes(M, w.N, K)
    if workspace is None:
        workspace = torch.empty((need + 256,), dtype=torch.uint8, device=x.device)
    base = workspace.data_ptr()
    ptr = (base + 255) & ~255
    _check("mxfp4_linear_native", lib.mxfp4_linear_native(
        _dev(x, torch.bfloat16, "x"), M, K, ldx, _dev(w.packed, torch.uint8, "packed"), w.N,
        _dev(out, torch.bfloat16, "out"), ldy, ptr, workspace.numel() - (ptr - base), _stream()))
    return out


def mxfp4_lora_linear_native(x: torch.Tensor, w: MxPackedWeight, A: Optional[torch.Tensor] = None,
                             B: Optional[torch.Tensor] = None, lora_scale: float = 0.0,
                             bias: Optional[torch.Tensor] = None, workspace: Optional[Workspace] = None,
                             out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y = MXFP8(x) . MXFP4(W)^T + lora_scale * (x A^T) B^T + bias (Eq. 2 on the native product)."""
    lib = load_library()
    M, K, ldx = _rows(x, "x")
    if K != w.K:
        raise ValueError("x must have K columns")
    r = 0
    a_ptr = b_ptr = None
    if A is not None and B is not None and A.shape[0] > 0:
        r = A.shape[0]
        if tuple(A.shape) != (r, K) or tuple(B.shape) != (w.N, r) or not A.is_contiguous() or not B.is_contiguous():
            raise ValueError("A must be contiguous [r, K] and B contiguous [N, r]")
        a_ptr, b_ptr = _dev(A, torch.bfloat16, "A"), _dev(B, torch.bfloat16, "B")
    bias_ptr = None
    if bias is not None:
        if tuple(bias.shape) != (w.N,) or not bias.is_contiguous():
            raise ValueError("bias must be contiguous [N]")
        bias_ptr = _dev(bias, torch.bfloat16, "bias")
    if out is None:
        out = torch.empty((M, w.N), dtype=torch.bfloat16, device=x.device)
    _, n_out, ldy = _rows(out, "out")
    if out.shape[0] != M or n_out != w.N:
        raise ValueError("out must be [M, N]")
    if workspace is None:
        need = lib.mxfp4_lora_linear_native_workspace_bytes(M, w.N, K, r)
        if need == 0:
            raise ValueError("rank not supported by mxfp4_lora_linear_native")
        workspace = Workspace(need, x.device)
    _check("mxfp4_lora_linear_native", lib.mxfp4_lora_linear_native(
        _dev(x, torch.bfloat16, "x"), M, K, ldx, _dev(w.packed, torch.uint8, "packed"), w.N, a_ptr, b_ptr, r,
        float(lora_scale), bias_ptr, _dev(out, torch.bfloat16, "out"), ldy, workspace.ptr, workspace.nbytes, _stream()))
    return out


# ---- log-probabilities under the language-model head ----------------------------------------------------
class LmHead:
    """The frozen head W [V, H] and, for the gradient, its transposed order (lm_head_prepack_t in the header)."""

    def __init__(self, weight: torch.Tensor, weight_t: Optional[torch.Tensor]):
        self.weight, self.weight_t = weight, weight_t
        self.V, self.H, self._ldw = _rows(weight, "W")
        self.device = weight.device


def lm_head_prepack(W: torch.Tensor, gradient: bool = True) -> LmHead:
    """W [V, H] bf16 (rows may be strided) as the log-probability functions take it; gradient=False leaves out the transposed order that
    lm_head_logprob_grad reads."""
    lib = load_library()
    V, H, ldw = _rows(W, "W")
    w_ptr = _dev(W, torch.bfloat16, "W")
    _here(W.device, "W")
    wt = None
    if gradient:
        wt = torch.empty((H, -(-V // 64) * 64), dtype=torch.bfloat16, device=W.device)
        _check("lm_head_prepack_t", lib.lm_head_prepack_t(w_ptr, V, H, ldw, wt.data_ptr(), _stream()))
    return LmHead(W, wt)


def lm_head_workspace(M: int, V: int, H: int, gradient: bool = True, device="cuda") -> torch.Tensor:
    """Scratch for calls of up to M rows; needs no initialisation."""
    need = int(load_library().lm_head_logprob_workspace_bytes(M, V, H, int(gradient)))
    if need == 0:
        raise ValueError("sizes not supported by lm_head_logprob")
    return torch.empty((need + 256,), dtype=torch.uint8, device=device)


def _head_call(name, x, head, targets, inv_temperature, entropy, workspace, out):
    lib = load_library()
    gradient = name == "lm_head_logprob_grad"
    M, H, ldx = _rows(x, "x")
    x_ptr = _dev(x, torch.bfloat16, "x")
    device = x.device
    _here(device, "x")
    if H != head.H:
        raise ValueError("x must have as many columns as the head")
    if head.device != device:
        raise ValueError("x and the head must be on one device")
    if gradient and head.weight_t is None:
        raise ValueError("the head was packed without its transposed order: lm_head_prepack(W, gradient=True)")
    if out is None:
        new = lambda *shape: torch.empty(shape, dtype=torch.float32, device=device)
        out = (new(M), new(M), new(M) if entropy else None) + ((new(M, H),) if gradient else ())
        rows = [out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr() if entropy else None]
        slope = (out[3].data_ptr(), H) if gradient else ()
    else:
        if len(out) != (4 if gradient else 3):
            raise ValueError("out must be (logprob, lse, entropy or None%s)" % (", slope" if gradient else ""))
        if (out[2] is not None) != bool(entropy):
            raise ValueError("entropy=True and its place in out go together")
        rows = [_flat(t, torch.float32, M, device, n) if t is not None else None for t, n in zip(out, ("logprob", "lse", "entropy"))]
        slope = ()
        if gradient:
            Ms, Hs, lds = _rows(out[3], "slope")
            if (Ms, Hs) != (M, H) or out[3].device != device:
                raise ValueError("slope must be [M, H] beside x")
            slope = _dev(out[3], torch.float32, "slope"), lds
    if workspace is None:
        workspace = lm_head_workspace(M, head.V, H, gradient, device)
    base = _dev(workspace, torch.uint8, "workspace")
    if not workspace.is_contiguous() or workspace.device != device:
        raise ValueError("workspace must be contiguous and beside x")
    ptr = (base + 255) & ~255
    _check(name, getattr(lib, name)(
        x_ptr, M, H, ldx, _dev(head.weight, torch.bfloat16, "W"), head.V, head._ldw, *((head.weight_t.data_ptr(),) if gradient else ()),
        _flat(targets, torch.int64, M, device, "targets"), float(inv_temperature), *rows, *slope, ptr, workspace.numel() - (ptr - base), _stream()))
    return tuple(out)


def lm_head_logprob(x, head: LmHead, targets: torch.Tensor, inv_temperature: float = 1.0, entropy: bool = False,
                    workspace: Optional[torch.Tensor] = None, out=None):
    """(logprob, lse, entropy or None), fp32 [M], of the tokens `targets` (int64 [M]) under softmax(inv_temperature * x W^T).  A target
    below 0 marks a row without a loss (zeros), one beyond the vocabulary gives NaN."""
    return _head_call("lm_head_logprob", x, head, targets, inv_temperature, entropy, workspace, out)


def lm_head_logprob_grad(x, head: LmHead, targets: torch.Tensor, inv_temperature: float = 1.0, entropy: bool = False,
                         workspace: Optional[torch.Tensor] = None, out=None):
    """(logprob, lse, entropy or None, slope): lm_head_logprob and slope = d logprob / dx, fp32 [M, H], for
    lm_head_logprob_backward."""
    return _head_call("lm_head_logprob_grad", x, head, targets, inv_temperature, entropy, workspace, out)


def lm_head_logprob_backward(grad_logprob: torch.Tensor, slope: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dx [M, H] bf16 = grad_logprob[m] * slope[m]."""
    M, H, lds = _rows(slope, "slope")
    s_ptr = _dev(slope, torch.float32, "slope")
    _here(slope.device, "slope")
    if out is None:
        out = torch.empty((M, H), dtype=torch.bfloat16, device=slope.device)
    Mo, Ho, lddx = _rows(out, "out")
    if (Mo, Ho) != (M, H) or out.device != slope.device:
        raise ValueError("out must be [M, H] beside slope")
    _check("lm_head_logprob_backward", load_library().lm_head_logprob_backward(
        _flat(grad_logprob, torch.float32, M, slope.device, "grad_logprob"), s_ptr, lds, M, H, _dev(out, torch.bfloat16, "out"), lddx, _stream()))
    return out


# ---- AdamW on the adapters ---------------------------------------------------------------------------
class _AdamWTensor(ctypes.Structure):
    """Mirror of qerl_adamw_tensor in the header."""
    _fields_ = [("param", _c_p), ("copy", _c_p), ("grad", _c_p), ("n", _c_i64)]


class _AdamWPlanStruct(ctypes.Structure):
    """Mirror of qerl_adamw_plan in the header."""
    _fields_ = [("table", _c_p), ("elements", _c_i64), ("chunks", _c_i64), ("n_tensors", ctypes.c_int32)]


class _AdamWState(ctypes.Structure):
    """Mirror of qerl_adamw_state in the header."""
    _fields_ = [("bits", ctypes.c_int32), ("m", _c_p), ("v", _c_p), ("m_scale", _c_p), ("v_scale", _c_p)]


class _AdamWHyper(ctypes.Structure):
    """Mirror of qerl_adamw_hyper in the header."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("step", _c_i64), ("seed", ctypes.c_uint64), ("lr_device", _c_p),
                ("step_device", _c_p), ("grad_scale", _c_p)]


class AdamWPlan:
    """The tensors of an optimizer step (see lora_adamw_make_plan in the header) and its moments.  Holds references to all of
    them; every step reads the gradients from the tensors given here, so the backward pass has to write those (its `dA` and `dB`
    arguments, or a copy)."""

    def __init__(self, struct, table, tensors, moments, m, v, m_scale, v_scale):
        self.struct, self.table, self.tensors, self.bits = struct, table, tensors, moments.bits
        self.m, self.v, self.m_scale, self.v_scale = m, v, m_scale, v_scale
        self.elements, self.device = int(struct.elements), table.device
        self._refs = ctypes.byref(struct), ctypes.byref(moments)


def lora_adamw_plan(params, grads, copies=None, state_bits: int = 8, state=None) -> AdamWPlan:
    """params, grads: lists of contiguous fp32 tensors; copies: None or a list of bf16 tensors (or None) that each step writes
    from the updated parameters; state: None (zeros) or the moments to go on from, (m, v, m_scale, v_scale) as uint8 for 8 bits,
    (m, v) as fp32 for 32, laid out as the header says.  Memory that a step writes (parameters, copies, moments) must not be given twice."""
    lib = load_library()
    n = len(params)
    copies = copies if copies is not None else [None] * n
    if n == 0 or len(grads) != n or len(copies) != n:
        raise ValueError("params, grads and copies must be lists of one length, not empty")
    if state_bits not in (8, 32):
        raise ValueError("state_bits must be 8 or 32")
    if not params[0].is_cuda:
        raise TypeError("param must be a GPU tensor")
    device = params[0].device
    _here(device, "param")
    tensors = (_AdamWTensor * n)()
    for i, (p, g, c) in enumerate(zip(params, grads, copies)):
        tensors[i] = _AdamWTensor(_flat(p, torch.float32, p.numel(), device, "param"),
                                  _flat(c, torch.bfloat16, p.numel(), device, "copy") if c is not None else None,
                                  _flat(g, torch.float32, p.numel(), device, "grad"), p.numel())
    arr = ctypes.cast(tensors, _c_p)
    total, need = int(lib.lora_adamw_state_elements(arr, n)), int(lib.lora_adamw_plan_bytes(arr, n))
    if total < 0 or need == 0:
        raise ValueError("too many elements")
    if state is None:
        dt = torch.uint8 if state_bits == 8 else torch.float32
        state = [torch.zeros((k,), dtype=dt, device=device) for k in ([total, total] + ([total // 32] * 2 if state_bits == 8 else []))]
    if len(state) != (4 if state_bits == 8 else 2):
        raise ValueError("state must be (m, v, m_scale, v_scale) for 8 bits, (m, v) for 32")
    for t, k, name in zip(state, (total, total, total // 32, total // 32), ("m", "v", "m_scale", "v_scale")):
        _flat(t, torch.uint8 if state_bits == 8 else torch.float32, k, device, name)
    m, v, ms, vs = (*state, None, None)[:4]
    table = torch.empty((need,), dtype=torch.uint8, device=device)
    struct = _AdamWPlanStruct()
    moments = _AdamWState(state_bits, *(t.data_ptr() for t in state))
    _check("lora_adamw_check_state", lib.lora_adamw_check_state(arr, n, table.data_ptr(), ctypes.byref(moments)))
    _check("lora_adamw_make_plan", lib.lora_adamw_make_plan(arr, n, table.data_ptr(), table.numel(), ctypes.byref(struct), _stream()))
    return AdamWPlan(struct, table, (list(params), list(grads), list(copies)), moments, m, v, ms, vs)


def lora_adamw_step(plan: AdamWPlan, lr: Optional[float] = None, step: Optional[int] = None, beta1: float = 0.9, beta2: float = 0.999,
                    eps: float = 1e-8, weight_decay: float = 0.0, seed: int = 0, grad_scale: Optional[torch.Tensor] = None,
                    lr_device: Optional[torch.Tensor] = None, step_device: Optional[torch.Tensor] = None) -> None:
    """One AdamW step on everything in `plan`, in place.  step counts from 1.  grad_scale: fp32 tensor of one element (from
    lora_adamw_grad_norm).  lr_device (fp32) and step_device (int64), tensors of one element, take the place of lr and step in steps
    that are captured and replayed."""
    if (lr is None) == (lr_device is None) or (step is None) == (step_device is None):
        raise ValueError("give lr or lr_device, and step or step_device")
    _here(plan.device, "the plan")
    one = lambda t, dt, name: _flat(t, dt, 1, plan.device, name) if t is not None else None
    h = _AdamWHyper(0.0 if lr is None else float(lr), float(beta1), float(beta2), float(eps), float(weight_decay), 1 if step is None else int(step),
                    int(seed) & (2 ** 64 - 1), one(lr_device, torch.float32, "lr_device"), one(step_device, torch.int64, "step_device"), one(grad_scale, torch.float32, "grad_scale"))
    _check("lora_adamw_step", load_library().lora_adamw_step(*plan._refs, ctypes.byref(h), _stream()))


def lora_adamw_grad_norm(plan: AdamWPlan, max_norm: float, out=None):
    """(norm, scale), fp32 tensors of one element: the 2-norm of all gradients of `plan` and the factor that clips it to max_norm
    (NaN if the norm is not finite), for lora_adamw_step's grad_scale."""
    _here(plan.device, "the plan")
    norm, scale = out if out is not None else (torch.empty((1,), dtype=torch.float32, device=plan.device) for _ in range(2))
    _check("lora_adamw_grad_norm", load_library().lora_adamw_grad_norm(
        plan._refs[0], float(max_norm), _flat(norm, torch.float32, 1, plan.device, "norm"), _flat(scale, torch.float32, 1, plan.device, "scale"), _stream()))
    return norm, scale


def lora_adamw_moments(plan: AdamWPlan):
    """(m, v) of an 8-bit plan as fp32 [plan.elements]."""
    _here(plan.device, "the plan")
    m, v = (torch.empty((plan.elements,), dtype=torch.float32, device=plan.device) for _ in range(2))
    _check("lora_adamw_moments", load_library().lora_adamw_moments(
        *plan._refs, m.data_ptr(), v.data_ptr(), _stream()))
    return m, v
