"""ctypes binding of libbitlinear_b200.so: argument marshalling only.

Function names match the C ABI (include/bitlinear.h).  Tensors are torch CUDA
tensors used purely as device memory; `stream` defaults to torch's current
stream.  There is no fallback: if the shared library is missing or a call
returns an error status, an exception is raised.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

import torch

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libbitlinear_b200.so"

OK = 0
ERR_ARG, ERR_SHAPE, ERR_ALIGN, ERR_WORKSPACE, ERR_ARCH, ERR_CUDA, ERR_TIMEOUT, ERR_RANGE, ERR_BADCODE = range(-1, -10, -1)
ERR_PAGE = -10
PATH_AUTO, PATH_DP4A, PATH_MMA, PATH_TCGEN05 = 0, 1, 2, 3

EXPORTS = [
    "bitlinear_status_string",
    "bitlinear_packed_bytes",
    "bitlinear_workspace_bytes",
    "bitlinear_quantize_weights",
    "bitlinear_quantize_acts",
    "bitlinear_rmsnorm_quantize_acts",
    "bitlinear_swiglu_quantize_acts",
    "bitlinear_quantize_acts_bits",
    "bitlinear_forward",
    "bitlinear_forward_act_bits",
    "bitlinear_forward_rmsnorm",
    "bitlinear_forward_swiglu",
    "bitlinear_forward_static",
    "bitlinear_sequence_workspace_bytes",
    "bitlinear_sequence_create",
    "bitlinear_sequence_create_rmsnorm",
    "bitlinear_sequence_create_swiglu",
    "bitlinear_forward_sequence",
    "bitlinear_forward_sequence_stage",
    "bitlinear_sequence_destroy",
    "bitlinear_matmul_i32",
    "bitlinear_unpack_weights",
    "bitlinear_validate_packed",
    "bitlinear_packed_bytes_trits",
    "bitlinear_quantize_weights_trits",
    "bitlinear_forward_trits",
    "bitlinear_sequence_create_trits",
    "bitlinear_matmul_i32_trits",
    "bitlinear_unpack_weights_trits",
    "bitlinear_kv_cache_bytes",
    "bitlinear_rope_table",
    "bitlinear_kv_append",
    "bitlinear_attend_workspace_bytes",
    "bitlinear_attend_decode",
    "bitlinear_attend_prompt",
    "bitlinear_kv_append_rmsnorm",
    "bitlinear_attend_weigh_workspace_bytes",
    "bitlinear_attend_decode_weigh",
    "bitlinear_kv_select",
    "bitlinear_kv_select_any_order",
    "bitlinear_kv_compact",
    "bitlinear_attend_shared_workspace_bytes",
    "bitlinear_attend_decode_shared",
    "bitlinear_probe_int8_peak",
    "bitlinear_test_expire_next_wait",
    "bitlinear_poll_status",
]


class BitLinearError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class LayerDesc(ctypes.Structure):
    _fields_ = [
        ("packed", ctypes.c_void_p),
        ("gamma", ctypes.c_void_p),
        ("X", ctypes.c_void_p),
        ("Y", ctypes.c_void_p),
        ("M", ctypes.c_int64),
        ("K", ctypes.c_int64),
        ("N", ctypes.c_int64),
    ]


class KVCacheDesc(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p),
        ("status", ctypes.c_void_p),
        ("n_pages", ctypes.c_int64),
        ("kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("bits", ctypes.c_int32),
    ]


class KVMarksDesc(ctypes.Structure):
    _fields_ = [("mass", ctypes.c_void_p), ("pos", ctypes.c_void_p)]


class KVBatchDesc(ctypes.Structure):
    _fields_ = [
        ("page_table", ctypes.c_void_p),
        ("kv_lens", ctypes.c_void_p),
        ("cu_tokens", ctypes.c_void_p),
        ("n_seqs", ctypes.c_int64),
        ("table_stride", ctypes.c_int64),
        ("table_pages", ctypes.c_int64),
    ]


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads the CUDA library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not LIB_PATH.exists():
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2402_17764_b200.build` "
            "(the BitLinear path has no CPU or PyTorch fallback)")
    L = ctypes.CDLL(str(LIB_PATH))
    i64, vp, sz, ci, cf = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float
    L.bitlinear_status_string.argtypes = [ci]
    L.bitlinear_status_string.restype = ctypes.c_char_p
    L.bitlinear_packed_bytes.argtypes = [i64, i64]
    L.bitlinear_packed_bytes.restype = sz
    L.bitlinear_workspace_bytes.argtypes = [i64, i64, i64]
    L.bitlinear_workspace_bytes.restype = sz
    L.bitlinear_quantize_weights.argtypes = [vp, i64, i64, cf, vp, vp, vp]
    L.bitlinear_quantize_acts.argtypes = [vp, i64, i64, vp, vp, vp, vp]
    L.bitlinear_forward.argtypes = [vp, vp, vp, i64, i64, i64, vp, vp, sz, vp]
    L.bitlinear_rmsnorm_quantize_acts.argtypes = [vp, vp, cf, i64, i64, vp, vp, vp, vp]
    L.bitlinear_forward_rmsnorm.argtypes = [vp, vp, vp, vp, cf, i64, i64, i64, vp, vp, sz, vp]
    L.bitlinear_swiglu_quantize_acts.argtypes = [vp, vp, i64, i64, vp, vp, vp, vp]
    L.bitlinear_forward_swiglu.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, vp, sz, vp]
    L.bitlinear_quantize_acts_bits.argtypes = [vp, i64, i64, ci, vp, vp, vp, vp]
    L.bitlinear_forward_act_bits.argtypes = [vp, vp, vp, i64, i64, i64, ci, vp, vp, sz, vp]
    L.bitlinear_forward_static.argtypes = [vp, vp, vp, i64, i64, i64, vp, vp]
    L.bitlinear_sequence_workspace_bytes.argtypes = [ctypes.POINTER(LayerDesc), ci]
    L.bitlinear_sequence_workspace_bytes.restype = sz
    L.bitlinear_sequence_create.argtypes = [ctypes.POINTER(LayerDesc), ci, vp, sz, ctypes.POINTER(vp)]
    L.bitlinear_sequence_create_rmsnorm.argtypes = [ctypes.POINTER(LayerDesc), ctypes.POINTER(vp), cf, ci, vp, sz,
                                                    ctypes.POINTER(vp)]
    L.bitlinear_sequence_create_swiglu.argtypes = [ctypes.POINTER(LayerDesc), ctypes.POINTER(vp), ctypes.POINTER(vp), cf,
                                                   ci, vp, sz, ctypes.POINTER(vp)]
    L.bitlinear_forward_sequence.argtypes = [vp, vp]
    L.bitlinear_forward_sequence_stage.argtypes = [vp, ci, vp]
    L.bitlinear_sequence_destroy.argtypes = [vp]
    L.bitlinear_sequence_destroy.restype = None
    L.bitlinear_matmul_i32.argtypes = [vp, vp, i64, i64, i64, vp, ci, vp, sz, vp]
    L.bitlinear_unpack_weights.argtypes = [vp, i64, i64, vp, vp]
    L.bitlinear_poll_status.argtypes = [vp, vp, ctypes.POINTER(ci)]
    L.bitlinear_validate_packed.argtypes = [vp, i64, i64, vp, vp]
    L.bitlinear_packed_bytes_trits.argtypes = [i64, i64]
    L.bitlinear_packed_bytes_trits.restype = sz
    L.bitlinear_quantize_weights_trits.argtypes = [vp, i64, i64, cf, vp, vp, vp]
    L.bitlinear_forward_trits.argtypes = [vp, vp, vp, i64, i64, i64, vp, vp, sz, vp]
    L.bitlinear_sequence_create_trits.argtypes = [ctypes.POINTER(LayerDesc), ci, vp, sz, ctypes.POINTER(vp)]
    L.bitlinear_matmul_i32_trits.argtypes = [vp, vp, i64, i64, i64, vp, vp, sz, vp]
    L.bitlinear_unpack_weights_trits.argtypes = [vp, i64, i64, vp, vp]
    L.bitlinear_probe_int8_peak.argtypes = [ci, vp, ctypes.POINTER(i64), vp]
    L.bitlinear_test_expire_next_wait.argtypes = [ctypes.c_uint32, ci]
    L.bitlinear_test_expire_next_wait.restype = None
    # (the two descriptors travel as addresses: KVCache and KVBatch keep them)
    L.bitlinear_kv_cache_bytes.argtypes = [i64, ci, ci, ci, ci]
    L.bitlinear_kv_cache_bytes.restype = sz
    L.bitlinear_rope_table.argtypes = [vp, i64, ci, ctypes.c_double, vp]
    L.bitlinear_kv_append.argtypes = [vp, vp, vp, i64, vp, i64, vp, i64, i64, ci, vp, i64, ci, vp, i64, vp]
    L.bitlinear_attend_workspace_bytes.argtypes = [ci, ci, ci, ci]
    L.bitlinear_attend_workspace_bytes.restype = sz
    L.bitlinear_attend_decode.argtypes = [vp, vp, vp, i64, ci, cf, vp, i64, vp, sz, vp]
    L.bitlinear_attend_prompt.argtypes = [vp, vp, vp, i64, i64, ci, cf, vp, i64, vp, sz, vp]
    L.bitlinear_kv_append_rmsnorm.argtypes = [vp, vp, vp, i64, vp, i64, vp, i64, i64, ci, vp, vp, cf, vp, i64, ci, vp, vp, vp, i64, vp]
    L.bitlinear_attend_weigh_workspace_bytes.argtypes = [ci, ci, ci, ci, i64, i64]
    L.bitlinear_attend_weigh_workspace_bytes.restype = sz
    L.bitlinear_attend_decode_weigh.argtypes = [vp, vp, vp, vp, i64, ci, cf, vp, i64, vp, sz, vp]
    L.bitlinear_kv_select.argtypes = [vp, vp, vp, i64, i64, vp, vp, vp]
    L.bitlinear_kv_select_any_order.argtypes = [vp, vp, vp, i64, i64, vp, vp, vp]
    L.bitlinear_kv_compact.argtypes = [vp, vp, vp, i64, vp, vp]
    L.bitlinear_attend_shared_workspace_bytes.argtypes = [ci, ci, ci, i64]
    L.bitlinear_attend_shared_workspace_bytes.restype = sz
    L.bitlinear_attend_decode_shared.argtypes = [vp, vp, vp, vp, i64, ci, cf, i64, vp, i64, vp, sz, vp]
    _lib = L
    return L


def status_string(status: int) -> str:
    return load_library().bitlinear_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != OK:
        raise BitLinearError(status, where)


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def packed_bytes(N: int, K: int) -> int:
    return int(load_library().bitlinear_packed_bytes(N, K))


def workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load_library().bitlinear_workspace_bytes(M, N, K))


def alloc_workspace(M: int, N: int, K: int, device="cuda") -> torch.Tensor:
    n = workspace_bytes(M, N, K)
    if n == 0:
        raise BitLinearError(ERR_SHAPE, "bitlinear_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def quantize_weights(W: torch.Tensor, eps: float = 1e-5, packed: torch.Tensor | None = None,
                     gamma: torch.Tensor | None = None, stream=None):
    """bitlinear_quantize_weights: fp32 [N, K] -> (packed uint8 buffer, gamma fp32[1])."""
    N, K = W.shape
    if packed is None:
        packed = torch.empty(max(packed_bytes(N, K), 16), dtype=torch.uint8, device=W.device)
    if gamma is None:
        gamma = torch.empty(1, dtype=torch.float32, device=W.device)
    st = load_library().bitlinear_quantize_weights(_ptr(W), N, K, float(eps), _ptr(packed), _ptr(gamma), _stream(stream))
    _check(st, "bitlinear_quantize_weights")
    return packed, gamma


def packed_bytes_trits(N: int, K: int) -> int:
    return int(load_library().bitlinear_packed_bytes_trits(N, K))


def quantize_weights_trits(W: torch.Tensor, eps: float = 1e-5, packed: torch.Tensor | None = None,
                           gamma: torch.Tensor | None = None, stream=None):
    """bitlinear_quantize_weights_trits: fp32 [N, K] -> (base-3 packed uint8 buffer, gamma fp32[1])."""
    N, K = W.shape
    if packed is None:
        packed = torch.empty(packed_bytes_trits(N, K), dtype=torch.uint8, device=W.device)
    if gamma is None:
        gamma = torch.empty(1, dtype=torch.float32, device=W.device)
    st = load_library().bitlinear_quantize_weights_trits(_ptr(W), N, K, float(eps), _ptr(packed), _ptr(gamma), _stream(stream))
    _check(st, "bitlinear_quantize_weights_trits")
    return packed, gamma


def forward_trits(packed: torch.Tensor, gamma: torch.Tensor, X: torch.Tensor, N: int, Y: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """bitlinear_forward_trits: bf16 [M, K] (M <= 8) -> bf16 [M, N] on base-3 packed weights."""
    M, K = X.shape
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device)
    if workspace is None:
        workspace = alloc_workspace(M, N, K, X.device)
    st = load_library().bitlinear_forward_trits(_ptr(packed), _ptr(gamma), _ptr(X), M, K, N, _ptr(Y), _ptr(workspace),
                                                workspace.numel(), _stream(stream))
    _check(st, "bitlinear_forward_trits")
    return Y


def matmul_i32_trits(packed: torch.Tensor, Xq: torch.Tensor, N: int, workspace: torch.Tensor | None = None,
                     stream=None) -> torch.Tensor:
    """bitlinear_matmul_i32_trits (test hook): int8 [M, K] x base-3 packed [N, K] -> int32 [M, N]."""
    M, K = Xq.shape
    acc = torch.empty((M, N), dtype=torch.int32, device=Xq.device)
    if workspace is None:
        workspace = alloc_workspace(M, N, K, Xq.device)
    st = load_library().bitlinear_matmul_i32_trits(_ptr(packed), _ptr(Xq), M, K, N, _ptr(acc), _ptr(workspace),
                                                   workspace.numel(), _stream(stream))
    _check(st, "bitlinear_matmul_i32_trits")
    return acc


def unpack_weights_trits(packed: torch.Tensor, N: int, K: int, stream=None) -> torch.Tensor:
    """bitlinear_unpack_weights_trits (test hook): -> int8 [N, K] in {-1, 0, 1}."""
    T = torch.empty((N, K), dtype=torch.int8, device=packed.device)
    st = load_library().bitlinear_unpack_weights_trits(_ptr(packed), N, K, _ptr(T), _stream(stream))
    _check(st, "bitlinear_unpack_weights_trits")
    return T


def quantize_acts(X: torch.Tensor, stream=None):
    """bitlinear_quantize_acts: bf16 [M, K] -> (Xq int8 [M, K], beta fp32 [M], rowsum int32 [M])."""
    M, K = X.shape
    Xq = torch.empty((M, K), dtype=torch.int8, device=X.device)
    beta = torch.empty(max(M, 1), dtype=torch.float32, device=X.device)[:M]
    rowsum = torch.empty(max(M, 1), dtype=torch.int32, device=X.device)[:M]
    st = load_library().bitlinear_quantize_acts(_ptr(X), M, K, _ptr(Xq), _ptr(beta), _ptr(rowsum), _stream(stream))
    _check(st, "bitlinear_quantize_acts")
    return Xq, beta, rowsum


def rmsnorm_quantize_acts(H: torch.Tensor, gain: torch.Tensor, norm_eps: float, stream=None):
    """bitlinear_rmsnorm_quantize_acts: bf16 [M, K], fp32 gain [K] -> (Xq int8 [M, K], beta fp32 [M], rowsum int32 [M])."""
    M, K = H.shape
    Xq = torch.empty((M, K), dtype=torch.int8, device=H.device)
    beta = torch.empty(max(M, 1), dtype=torch.float32, device=H.device)[:M]
    rowsum = torch.empty(max(M, 1), dtype=torch.int32, device=H.device)[:M]
    st = load_library().bitlinear_rmsnorm_quantize_acts(_ptr(H), _ptr(gain), float(norm_eps), M, K, _ptr(Xq), _ptr(beta),
                                                        _ptr(rowsum), _stream(stream))
    _check(st, "bitlinear_rmsnorm_quantize_acts")
    return Xq, beta, rowsum


def forward_rmsnorm(packed: torch.Tensor, gamma: torch.Tensor, H: torch.Tensor, gain: torch.Tensor, norm_eps: float, N: int,
                    Y: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """bitlinear_forward_rmsnorm: BitLinear(RMSNorm(H)), bf16 [M, K] -> bf16 [M, N]."""
    M, K = H.shape
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.bfloat16, device=H.device)
    if workspace is None:
        workspace = alloc_workspace(M, N, K, H.device)
    st = load_library().bitlinear_forward_rmsnorm(_ptr(packed), _ptr(gamma), _ptr(H), _ptr(gain), float(norm_eps), M, K, N,
                                                  _ptr(Y), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "bitlinear_forward_rmsnorm")
    return Y


def quantize_acts_bits(X: torch.Tensor, act_bits: int, stream=None):
    """bitlinear_quantize_acts_bits: bf16 [M, K] -> (Xq int8 [M, K] with |q| <= 2^(act_bits-1) - 1, beta, rowsum)."""
    M, K = X.shape
    Xq = torch.empty((M, K), dtype=torch.int8, device=X.device)
    beta = torch.empty(max(M, 1), dtype=torch.float32, device=X.device)[:M]
    rowsum = torch.empty(max(M, 1), dtype=torch.int32, device=X.device)[:M]
    st = load_library().bitlinear_quantize_acts_bits(_ptr(X), M, K, int(act_bits), _ptr(Xq), _ptr(beta), _ptr(rowsum),
                                                     _stream(stream))
    _check(st, "bitlinear_quantize_acts_bits")
    return Xq, beta, rowsum


def forward_act_bits(packed: torch.Tensor, gamma: torch.Tensor, X: torch.Tensor, N: int, act_bits: int,
                     Y: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """bitlinear_forward_act_bits: the forward with act_bits-bit activations, bf16 [M, K] -> bf16 [M, N]."""
    M, K = X.shape
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device)
    if workspace is None:
        workspace = alloc_workspace(M, N, K, X.device)
    st = load_library().bitlinear_forward_act_bits(_ptr(packed), _ptr(gamma), _ptr(X), M, K, N, int(act_bits), _ptr(Y),
                                                   _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "bitlinear_forward_act_bits")
    return Y


def swiglu_quantize_acts(gate: torch.Tensor, up: torch.Tensor, stream=None):
    """bitlinear_swiglu_quantize_acts: bf16 gate, up [M, K] -> (Xq int8 [M, K], beta fp32 [M], rowsum int32 [M])."""
    M, K = gate.shape
    assert up.shape == gate.shape
    Xq = torch.empty((M, K), dtype=torch.int8, device=gate.device)
    beta = torch.empty(max(M, 1), dtype=torch.float32, device=gate.device)[:M]
    rowsum = torch.empty(max(M, 1), dtype=torch.int32, device=gate.device)[:M]
    st = load_library().bitlinear_swiglu_quantize_acts(_ptr(gate), _ptr(up), M, K, _ptr(Xq), _ptr(beta), _ptr(rowsum),
                                                       _stream(stream))
    _check(st, "bitlinear_swiglu_quantize_acts")
    return Xq, beta, rowsum


def forward_swiglu(packed: torch.Tensor, gamma: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, N: int,
                   Y: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """bitlinear_forward_swiglu: BitLinear(silu(gate) * up), bf16 [M, K] x 2 -> bf16 [M, N]."""
    M, K = gate.shape
    assert up.shape == gate.shape
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.bfloat16, device=gate.device)
    if workspace is None:
        workspace = alloc_workspace(M, N, K, gate.device)
    st = load_library().bitlinear_forward_swiglu(_ptr(packed), _ptr(gamma), _ptr(gate), _ptr(up), M, K, N, _ptr(Y),
                                                 _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "bitlinear_forward_swiglu")
    return Y


def forward(packed: torch.Tensor, gamma: torch.Tensor, X: torch.Tensor, N: int, Y: torch.Tensor | None = None,
            workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """bitlinear_forward: bf16 [M, K] -> bf16 [M, N]."""
    M, K = X.shape
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device)
    if workspace is None:
        workspace = alloc_workspace(M, N, K, X.device)
    st = load_library().bitlinear_forward(_ptr(packed), _ptr(gamma), _ptr(X), M, K, N, _ptr(Y), _ptr(workspace),
                                          workspace.numel(), _stream(stream))
    _check(st, "bitlinear_forward")
    return Y


def forward_static(packed: torch.Tensor, gamma: torch.Tensor, X: torch.Tensor, N: int, Y: torch.Tensor,
                   stream=None) -> torch.Tensor:
    """bitlinear_forward_static: the forward on the library's own scratch; the caller supplies Y, nothing is allocated."""
    M, K = X.shape
    st = load_library().bitlinear_forward_static(_ptr(packed), _ptr(gamma), _ptr(X), M, K, N, _ptr(Y), _stream(stream))
    _check(st, "bitlinear_forward_static")
    return Y


def matmul_i32(packed: torch.Tensor, Xq: torch.Tensor, N: int, path: int = PATH_AUTO,
               workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """bitlinear_matmul_i32 (test hook): int8 [M, K] x packed [N, K] -> int32 [M, N]."""
    M, K = Xq.shape
    acc = torch.empty((M, N), dtype=torch.int32, device=Xq.device)
    if workspace is None:
        workspace = alloc_workspace(M, N, K, Xq.device)
    st = load_library().bitlinear_matmul_i32(_ptr(packed), _ptr(Xq), M, K, N, _ptr(acc), int(path), _ptr(workspace),
                                             workspace.numel(), _stream(stream))
    _check(st, "bitlinear_matmul_i32")
    return acc


def unpack_weights(packed: torch.Tensor, N: int, K: int, stream=None) -> torch.Tensor:
    """bitlinear_unpack_weights (test hook): -> int8 [N, K] in {-1, 0, 1}."""
    T = torch.empty((N, K), dtype=torch.int8, device=packed.device)
    st = load_library().bitlinear_unpack_weights(_ptr(packed), N, K, _ptr(T), _stream(stream))
    _check(st, "bitlinear_unpack_weights")
    return T


def validate_packed(packed: torch.Tensor, N: int, K: int, stream=None) -> int:
    """bitlinear_validate_packed: -> number of 2-bit fields that hold the unused code 3 (0: the buffer is sound)."""
    bad = torch.empty(1, dtype=torch.int32, device=packed.device)
    st = load_library().bitlinear_validate_packed(_ptr(packed), N, K, _ptr(bad), _stream(stream))
    if st not in (OK, ERR_BADCODE):
        _check(st, "bitlinear_validate_packed")
    return int(bad.item())


def probe_int8_peak(iters: int, status: torch.Tensor, stream=None) -> int:
    """bitlinear_probe_int8_peak (measurement aid): enqueues the MMA issue loop; -> integer operations of the launch."""
    ops = ctypes.c_int64(0)
    st = load_library().bitlinear_probe_int8_peak(int(iters), _ptr(status), ctypes.byref(ops), _stream(stream))
    _check(st, "bitlinear_probe_int8_peak")
    return int(ops.value)


def test_expire_next_wait(limit_us: int, skip_arrive: bool):
    """bitlinear_test_expire_next_wait (test hook): arms the next matmul launch; see include/bitlinear.h."""
    load_library().bitlinear_test_expire_next_wait(int(limit_us), 1 if skip_arrive else 0)


def poll_status(workspace: torch.Tensor, stream=None) -> int:
    out = ctypes.c_int(0)
    st = load_library().bitlinear_poll_status(_ptr(workspace), _stream(stream), ctypes.byref(out))
    _check(st, "bitlinear_poll_status")
    return int(out.value)


class Sequence:
    """bitlinear_sequence_*: a fixed list of independent BitLinear forwards run by one persistent launch.

    `layers` is a list of (packed, gamma, X, Y, N) with torch tensors; the object keeps them alive.
    `gains` (optional): one fp32 gain vector [K] or None per layer; those layers get an RMSNorm with `norm_eps` in front
    of their activation quantiser (bitlinear_sequence_create_rmsnorm).
    `ups` (optional): one bf16 tensor [M, K] or None per layer; those layers quantise silu(X) * up
    (bitlinear_sequence_create_swiglu).
    `trits`: the packed weights are in the base-3 format (bitlinear_sequence_create_trits).
    """

    def __init__(self, layers, device="cuda", gains=None, norm_eps: float = 1e-5, ups=None, trits: bool = False):
        L = load_library()
        self._keep = list(layers)
        self._gains = list(gains) if gains is not None else None
        self._ups = list(ups) if ups is not None else None
        n = len(self._keep)
        arr = (LayerDesc * n)()
        for i, (packed, gamma, X, Y, N) in enumerate(self._keep):
            M, K = X.shape
            arr[i] = LayerDesc(_ptr(packed), _ptr(gamma), _ptr(X), _ptr(Y), M, K, N)
        nbytes = int(L.bitlinear_sequence_workspace_bytes(arr, n))
        if nbytes == 0:
            raise BitLinearError(ERR_SHAPE, "bitlinear_sequence_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        handle = ctypes.c_void_p()
        def pointers(tensors):
            assert len(tensors) == n
            return (ctypes.c_void_p * n)(*[(_ptr(x) if x is not None else None) for x in tensors])

        if trits:
            assert self._ups is None and self._gains is None
            st = L.bitlinear_sequence_create_trits(arr, n, _ptr(self.workspace), nbytes, ctypes.byref(handle))
        elif self._ups is not None:
            st = L.bitlinear_sequence_create_swiglu(arr, pointers(self._gains) if self._gains is not None else None,
                                                    pointers(self._ups), float(norm_eps), n, _ptr(self.workspace), nbytes,
                                                    ctypes.byref(handle))
        elif self._gains is None:
            st = L.bitlinear_sequence_create(arr, n, _ptr(self.workspace), nbytes, ctypes.byref(handle))
        else:
            assert len(self._gains) == n
            garr = (ctypes.c_void_p * n)(*[(_ptr(g) if g is not None else None) for g in self._gains])
            st = L.bitlinear_sequence_create_rmsnorm(arr, garr, float(norm_eps), n, _ptr(self.workspace), nbytes,
                                                     ctypes.byref(handle))
        _check(st, "bitlinear_sequence_create")
        self._handle = handle
        self.n = n

    def forward(self, stream=None):
        st = load_library().bitlinear_forward_sequence(self._handle, _stream(stream))
        _check(st, "bitlinear_forward_sequence")

    def forward_stage(self, stage: int, stream=None):
        """stage 1: activation quantiser; stage 2: matmul + dequantisation; 0: both."""
        st = load_library().bitlinear_forward_sequence_stage(self._handle, int(stage), _stream(stream))
        _check(st, "bitlinear_forward_sequence_stage")

    def close(self):
        if getattr(self, "_handle", None):
            load_library().bitlinear_sequence_destroy(self._handle)
            self._handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _refuse(where: str, why: str, status: int = ERR_ARG):
    error = BitLinearError(status, where)
    error.args = (f"{error.args[0]}: {why}",)
    raise error


def kv_cache_bytes(n_pages: int, kv_heads: int, head_dim: int, page_size: int, bits: int) -> int:
    return int(load_library().bitlinear_kv_cache_bytes(n_pages, kv_heads, head_dim, page_size, bits))


def _wait_for_fills(device):
    """Waits for what was just filled on the current stream, so that calls on any stream may use it (a capturing stream cannot be
    waited for: there the fills are part of the graph)."""
    if not torch.cuda.is_current_stream_capturing():
        torch.cuda.current_stream(device).synchronize()


class KVCache:
    """bitlinear_kv_cache: a paged cache of keys and values, bf16 (bits 16) or int8 codes with a scale per row (bits 8).

    `k`, `v`: [n_pages, kv_heads, page_size, head_dim rounded up to 16]; `k_scale`, `v_scale`: fp32
    [n_pages, kv_heads, page_size] or None; `status`: int32[1], see check().
    """

    def __init__(self, n_pages: int, kv_heads: int, head_dim: int, page_size: int = 16, bits: int = 16, device="cuda"):
        if kv_cache_bytes(n_pages, kv_heads, head_dim, page_size, bits) == 0:
            raise BitLinearError(ERR_SHAPE, "bitlinear_kv_cache_bytes")
        shape = (n_pages, kv_heads, page_size, (head_dim + 15) // 16 * 16)
        dtype = torch.bfloat16 if bits == 16 else torch.int8
        scales = [None, None] if bits == 16 else [torch.zeros(shape[:3], dtype=torch.float32, device=device) for _ in range(2)]
        self._set(torch.zeros(shape, dtype=dtype, device=device), torch.zeros(shape, dtype=dtype, device=device), head_dim, *scales)

    @classmethod
    def from_tensors(cls, k: torch.Tensor, v: torch.Tensor, head_dim: int, k_scale: torch.Tensor | None = None,
                     v_scale: torch.Tensor | None = None) -> "KVCache":
        """A cache over tensors that the caller allocated."""
        self = cls.__new__(cls)
        self._set(k, v, head_dim, k_scale, v_scale)
        return self

    def _set(self, k, v, head_dim, k_scale, v_scale):
        where = "bitlinear_kv_cache"
        if k.dim() != 4 or k.shape != v.shape or k.shape[3] != (head_dim + 15) // 16 * 16:
            _refuse(where, "k and v are [n_pages, kv_heads, page_size, head_dim rounded up to 16]", ERR_SHAPE)
        if k.dtype != v.dtype or k.dtype not in (torch.bfloat16, torch.int8):
            _refuse(where, "k and v are both bf16 or both int8")
        bits = 16 if k.dtype == torch.bfloat16 else 8
        for s in (k_scale, v_scale):
            if (s is None) != (bits == 16) or (s is not None and (s.shape != k.shape[:3] or s.dtype != torch.float32)):
                _refuse(where, "an int8 cache has fp32 scales [n_pages, kv_heads, page_size], a bf16 cache has none")
        if not all(t is None or (t.is_cuda and t.device == k.device and t.is_contiguous()) for t in (k, v, k_scale, v_scale)):
            _refuse(where, "the tensors are contiguous and on one CUDA device")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.kv_heads, self.page_size = k.shape[:3]
        self.head_dim, self.bits, self.device, self.index = head_dim, bits, k.device, k.get_device()
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self._desc = KVCacheDesc(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), _ptr(self.status), self.n_pages, self.kv_heads,
                                 head_dim, self.page_size, bits)
        self._address = ctypes.addressof(self._desc)
        _wait_for_fills(k.device)

    def check(self):
        """Waits for the device, whatever streams the calls ran on, and raises if one of them met a bad page, length, position or
        token row; clears the status."""
        torch.cuda.synchronize(self.device)
        status = int(self.status.item())
        if status != OK:
            self.status.zero_()
            torch.cuda.synchronize(self.device)  # (or the next call on another stream could report before it is cleared)
            raise BitLinearError(status, "bitlinear_kv_cache")


class KVBatch:
    """bitlinear_kv_batch: the sequences of a call.  page_table int32 [n_seqs, pages], kv_lens int32 [n_seqs] (with the new
    tokens), cu_tokens int32 [n_seqs + 1] or None (one token per sequence).  The tensors are kept, not copied: a program
    that writes new lengths and pages into them uses the same object again, in a captured graph too."""

    def __init__(self, page_table: torch.Tensor, kv_lens: torch.Tensor, cu_tokens: torch.Tensor | None = None):
        where = "bitlinear_kv_batch"
        n = kv_lens.numel()
        if page_table.dim() != 2 or page_table.shape[0] != n or kv_lens.dim() != 1 or \
                (cu_tokens is not None and (cu_tokens.dim() != 1 or cu_tokens.numel() != n + 1)):
            _refuse(where, "page_table is [n_seqs, pages], kv_lens [n_seqs], cu_tokens [n_seqs + 1]", ERR_SHAPE)
        for t in (page_table, kv_lens, cu_tokens):
            if t is not None and (t.dtype != torch.int32 or not t.is_cuda or t.device != kv_lens.device):
                _refuse(where, "page_table, kv_lens and cu_tokens are int32 and on one CUDA device")
        if (page_table.shape[1] > 1 and page_table.stride(1) != 1) or (n > 1 and kv_lens.stride(0) != 1) or \
                (cu_tokens is not None and n > 0 and cu_tokens.stride(0) != 1):
            _refuse(where, "kv_lens, cu_tokens and the rows of page_table are contiguous")
        self.page_table, self.kv_lens, self.cu_tokens, self.n_seqs = page_table, kv_lens, cu_tokens, n
        self.device, self.index = kv_lens.device, kv_lens.get_device()
        pages = page_table.shape[1]
        stride = page_table.stride(0) if n > 1 else pages
        self._desc = KVBatchDesc(_ptr(page_table), _ptr(kv_lens), _ptr(cu_tokens), n, stride, pages)
        self._address = ctypes.addressof(self._desc)


class KVMarks:
    """bitlinear_kv_marks of a cache that rows are evicted from: of every row the attention weight it has received (`mass`, fp32)
    and the position of its token (`pos`, int32), both [n_pages, kv_heads, page_size]."""

    def __init__(self, cache: KVCache):
        shape = (cache.n_pages, cache.kv_heads, cache.page_size)
        self._set(cache, torch.zeros(shape, dtype=torch.float32, device=cache.device), torch.zeros(shape, dtype=torch.int32, device=cache.device))
        _wait_for_fills(cache.device)

    @classmethod
    def from_tensors(cls, cache: KVCache, mass: torch.Tensor, pos: torch.Tensor) -> "KVMarks":
        """Marks over tensors that the caller allocated."""
        self = cls.__new__(cls)
        self._set(cache, mass, pos)
        return self

    def _set(self, cache, mass, pos):
        for t, dtype in ((mass, torch.float32), (pos, torch.int32)):
            if t.shape != cache.k.shape[:3] or t.dtype != dtype or t.device != cache.device or not t.is_contiguous():
                _refuse("bitlinear_kv_marks", "mass (fp32) and pos (int32) are contiguous [n_pages, kv_heads, page_size] on the cache's device")
        self.mass, self.pos, self.shape, self.index = mass, pos, tuple(mass.shape), cache.index
        self._desc = KVMarksDesc(_ptr(mass), _ptr(pos))
        self._address = ctypes.addressof(self._desc)


def _marks_of(cache: KVCache, marks: KVMarks, where: str) -> int:
    if marks.index != cache.index or marks.shape != (cache.n_pages, cache.kv_heads, cache.page_size):
        _refuse(where, "the marks belong to a cache of another shape or device")
    return marks._address


def rope_table(n_pos: int, head_dim: int, base: float = 10000.0, device="cuda", stream=None) -> torch.Tensor:
    """bitlinear_rope_table: -> fp32 [n_pos, head_dim / 2, 2], (cos, sin) of every position and pair."""
    if stream is not None:
        with _allocating_on(stream, device):
            return rope_table(n_pos, head_dim, base, device)
    table = torch.empty((n_pos, head_dim // 2, 2), dtype=torch.float32, device=device)
    if torch.cuda.current_device() != table.device.index:
        with torch.cuda.device(table.device):
            st = load_library().bitlinear_rope_table(_ptr(table), n_pos, head_dim, float(base), _stream(None))
    else:
        st = load_library().bitlinear_rope_table(_ptr(table), n_pos, head_dim, float(base), _stream(None))
    _check(st, "bitlinear_rope_table")
    return table


_BF16, _FP32 = torch.bfloat16, torch.float32


def _row_stride(t: torch.Tensor, shape: tuple, index: int, where: str) -> int:
    """Row stride of bf16 [rows, heads, head_dim] in elements; refuses what the kernels cannot address."""
    if t.shape != shape or t.dtype is not _BF16 or t.get_device() != index:
        _refuse(where, f"expected bf16 {list(shape)} on cuda:{index}, got {t.dtype} {list(t.shape)} on {t.device}")
    row, head, element = t.stride()
    if element != 1 or head != shape[2]:
        if element != 1 or shape[1] > 1:
            _refuse(where, "the heads of a row are contiguous")
    return row if shape[0] > 1 else (shape[1] * shape[2] + 7) // 8 * 8


def _empty_rows(rows: int, heads: int, head_dim: int, device) -> torch.Tensor:
    """bf16 [rows, heads, head_dim] whose rows start on 16-byte boundaries."""
    n = heads * head_dim
    t = torch.empty((rows, (n + 7) // 8 * 8), dtype=torch.bfloat16, device=device)
    return t.as_strided((rows, heads, head_dim), (t.shape[1], head_dim, 1))


def _allocating_on(stream, device):
    """Context in which `stream` is the current one: what a call allocates (and fills) for itself has to belong to the stream
    that uses it, or it is not filled in time and may be handed out again too early."""
    return torch.cuda.stream(torch.cuda.ExternalStream(_stream(stream), device=device))


# (what torch.cuda.current_device() and torch.cuda.current_stream(index).cuda_stream give, without the objects in between)
_current_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def kv_append(cache: KVCache, batch: KVBatch, k: torch.Tensor, v: torch.Tensor, q: torch.Tensor | None = None,
              rope: torch.Tensor | None = None, interleaved: bool = False, q_out: torch.Tensor | None = None, stream=None):
    """bitlinear_kv_append: rotates k [T, kv_heads, head_dim] and stores it with v in the cache; rotates q [T, heads, head_dim]
    into q_out (allocated if not given, may be q itself) and returns it (None without q)."""
    where = "bitlinear_kv_append"
    index = cache.index
    if batch.index != index:
        _refuse(where, f"the cache is on {cache.device}, the batch on {batch.device}")
    if _current_device() != index:
        with torch.cuda.device(index):
            return kv_append(cache, batch, k, v, q, rope, interleaved, q_out, stream)
    if stream is not None and q is not None and q_out is None:
        with _allocating_on(stream, cache.device):
            return kv_append(cache, batch, k, v, q, rope, interleaved)
    if k.dim() != 3 or (q is not None and q.dim() != 3):
        _refuse(where, "k, v and q are [tokens, heads, head_dim]", ERR_SHAPE)
    T, D = k.shape[0], cache.head_dim
    shape = (T, cache.kv_heads, D)
    ks = _row_stride(k, shape, index, where)
    vs = _row_stride(v, shape, index, where)
    heads = qs = os_ = positions = q_at = out_at = rope_at = 0
    if q is not None:
        heads = q.shape[1]
        shape = (T, heads, D)
        qs = _row_stride(q, shape, index, where)
        if q_out is None:
            q_out = _empty_rows(T, heads, D, cache.device)
        os_ = _row_stride(q_out, shape, index, where)
        q_at, out_at = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        _refuse(where, "q_out without q")
    if rope is not None:
        positions = rope.shape[0]
        if rope.shape != (positions, D // 2, 2) or rope.dtype is not _FP32 or not rope.is_contiguous() or rope.get_device() != index:
            _refuse(where, f"rope is a contiguous fp32 [positions, {D // 2}, 2] on {cache.device}")
        rope_at = rope.data_ptr()
    st = (_lib or load_library()).bitlinear_kv_append(cache._address, batch._address, k.data_ptr(), ks, v.data_ptr(), vs, q_at, qs, T, heads,
                                                      rope_at, positions, 1 if interleaved else 0, out_at, os_,
                                                      _raw_stream(index) if stream is None else _stream(stream))
    if st != OK:
        _check(st, where)
    return q_out


def attend_workspace_bytes(heads: int, kv_heads: int, head_dim: int, prompt: bool) -> int:
    return int(load_library().bitlinear_attend_workspace_bytes(heads, kv_heads, head_dim, 1 if prompt else 0))


def alloc_attend_workspace(heads: int, kv_heads: int, head_dim: int, prompt: bool, device="cuda") -> torch.Tensor:
    """A workspace for attend_decode (prompt False) or attend_prompt (prompt True), zeroed as its first use needs it and ready for
    calls on any stream."""
    workspace = _attend_workspace(heads, kv_heads, head_dim, prompt, device)
    _wait_for_fills(workspace.device)
    return workspace


def _attend_workspace(heads, kv_heads, head_dim, prompt, device):
    n = attend_workspace_bytes(heads, kv_heads, head_dim, prompt)
    if n == 0:
        raise BitLinearError(ERR_SHAPE, "bitlinear_attend_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def _attend(prompt: bool, cache: KVCache, batch: KVBatch, q, scale, out, workspace, stream):
    where = "bitlinear_attend_prompt" if prompt else "bitlinear_attend_decode"
    index = cache.index
    if batch.index != index:
        _refuse(where, f"the cache is on {cache.device}, the batch on {batch.device}")
    if _current_device() != index:
        with torch.cuda.device(index):
            return _attend(prompt, cache, batch, q, scale, out, workspace, stream)
    if stream is not None and (out is None or workspace is None):
        with _allocating_on(stream, cache.device):
            return _attend(prompt, cache, batch, q, scale, out, workspace, None)
    if q.dim() != 3:
        _refuse(where, "q is [tokens, heads, head_dim]", ERR_SHAPE)
    T, heads, _ = q.shape
    D = cache.head_dim
    if not prompt and T != batch.n_seqs:
        _refuse(where, f"{batch.n_seqs} sequences and {T} tokens", ERR_SHAPE)
    shape = (T, heads, D)
    qs = _row_stride(q, shape, index, where)
    if out is None:
        out = _empty_rows(T, heads, D, cache.device)
    os_ = _row_stride(out, shape, index, where)
    if workspace is None:
        workspace = _attend_workspace(heads, cache.kv_heads, D, prompt, cache.device)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        _refuse(where, f"the workspace is contiguous and on {cache.device}")
    scale = D ** -0.5 if scale is None else float(scale)
    nbytes = workspace.numel() * workspace.element_size()
    stream = _raw_stream(index) if stream is None else _stream(stream)
    L = _lib or load_library()
    if prompt:
        st = L.bitlinear_attend_prompt(cache._address, batch._address, q.data_ptr(), qs, T, heads, scale, out.data_ptr(), os_,
                                       workspace.data_ptr(), nbytes, stream)
    else:
        st = L.bitlinear_attend_decode(cache._address, batch._address, q.data_ptr(), qs, heads, scale, out.data_ptr(), os_,
                                       workspace.data_ptr(), nbytes, stream)
    if st != OK:
        _check(st, where)
    return out


def attend_decode(cache: KVCache, batch: KVBatch, q: torch.Tensor, scale: float | None = None, out: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """bitlinear_attend_decode: attention of the one new token of each sequence, bf16 [n_seqs, heads, head_dim] -> the same.
    scale: 1 / sqrt(head_dim) if not given."""
    return _attend(False, cache, batch, q, scale, out, workspace, stream)


def attend_prompt(cache: KVCache, batch: KVBatch, q: torch.Tensor, scale: float | None = None, out: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """bitlinear_attend_prompt: causal attention of the new tokens of prompts and prompt chunks, bf16 [T, heads, head_dim] ->
    the same; rows of out behind the last sequence keep what they held."""
    return _attend(True, cache, batch, q, scale, out, workspace, stream)


def _gain(gain, head_dim: int, index: int, where: str) -> int:
    if gain is None:
        return 0
    if gain.shape != (head_dim,) or gain.dtype is not _FP32 or gain.get_device() != index or gain.stride(0) != 1:
        _refuse(where, f"a gain is a contiguous fp32 [{head_dim}] on cuda:{index}")
    return gain.data_ptr()


def kv_append_rmsnorm(cache: KVCache, batch: KVBatch, k: torch.Tensor, v: torch.Tensor, q: torch.Tensor | None = None,
                      q_gain: torch.Tensor | None = None, k_gain: torch.Tensor | None = None, norm_eps: float = 1e-5,
                      rope: torch.Tensor | None = None, interleaved: bool = False, positions: torch.Tensor | None = None,
                      marks: KVMarks | None = None, q_out: torch.Tensor | None = None, stream=None):
    """bitlinear_kv_append_rmsnorm: kv_append with an RMS norm of every query and key head (gains fp32 [head_dim], None: not
    normalised) in front of the rotation.  positions: int32 [T], the positions of the tokens where they are not their places in the
    sequences; marks: the new rows' are set."""
    where = "bitlinear_kv_append_rmsnorm"
    index = cache.index
    if batch.index != index:
        _refuse(where, f"the cache is on {cache.device}, the batch on {batch.device}")
    if _current_device() != index:
        with torch.cuda.device(index):
            return kv_append_rmsnorm(cache, batch, k, v, q, q_gain, k_gain, norm_eps, rope, interleaved, positions, marks, q_out, stream)
    if stream is not None and q is not None and q_out is None:
        with _allocating_on(stream, cache.device):
            return kv_append_rmsnorm(cache, batch, k, v, q, q_gain, k_gain, norm_eps, rope, interleaved, positions, marks)
    if k.dim() != 3 or (q is not None and q.dim() != 3):
        _refuse(where, "k, v and q are [tokens, heads, head_dim]", ERR_SHAPE)
    T, D = k.shape[0], cache.head_dim
    shape = (T, cache.kv_heads, D)
    ks = _row_stride(k, shape, index, where)
    vs = _row_stride(v, shape, index, where)
    heads = qs = os_ = n_angles = q_at = out_at = rope_at = positions_at = marks_at = 0
    if q is not None:
        heads = q.shape[1]
        shape = (T, heads, D)
        qs = _row_stride(q, shape, index, where)
        if q_out is None:
            q_out = _empty_rows(T, heads, D, cache.device)
        os_ = _row_stride(q_out, shape, index, where)
        q_at, out_at = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None or q_gain is not None:
        _refuse(where, "q_out or q_gain without q")
    if rope is not None:
        n_angles = rope.shape[0]
        if rope.shape != (n_angles, D // 2, 2) or rope.dtype is not _FP32 or not rope.is_contiguous() or rope.get_device() != index:
            _refuse(where, f"rope is a contiguous fp32 [positions, {D // 2}, 2] on {cache.device}")
        rope_at = rope.data_ptr()
    if positions is not None:
        if positions.shape != (T,) or positions.dtype is not torch.int32 or positions.get_device() != index or (T > 1 and positions.stride(0) != 1):
            _refuse(where, f"positions is a contiguous int32 [{T}] on {cache.device}")
        positions_at = positions.data_ptr()
    if marks is not None:
        marks_at = _marks_of(cache, marks, where)
    st = (_lib or load_library()).bitlinear_kv_append_rmsnorm(
        cache._address, batch._address, k.data_ptr(), ks, v.data_ptr(), vs, q_at, qs, T, heads, _gain(q_gain, D, index, where),
        _gain(k_gain, D, index, where), norm_eps, rope_at, n_angles, 1 if interleaved else 0, positions_at, marks_at, out_at, os_,
        _raw_stream(index) if stream is None else _stream(stream))
    if st != OK:
        _check(st, where)
    return q_out


def attend_weigh_workspace_bytes(heads: int, kv_heads: int, head_dim: int, bits: int, n_seqs: int, max_keys: int) -> int:
    return int(load_library().bitlinear_attend_weigh_workspace_bytes(heads, kv_heads, head_dim, bits, n_seqs, max_keys))


def attend_shared_workspace_bytes(heads: int, kv_heads: int, head_dim: int, n_seqs: int) -> int:
    return int(load_library().bitlinear_attend_shared_workspace_bytes(heads, kv_heads, head_dim, n_seqs))


def _zeroed(nbytes: int, where: str, device) -> torch.Tensor:
    if nbytes == 0:
        raise BitLinearError(ERR_SHAPE, where)
    workspace = torch.zeros(nbytes, dtype=torch.uint8, device=device)
    _wait_for_fills(workspace.device)
    return workspace


def alloc_attend_weigh_workspace(heads: int, kv_heads: int, head_dim: int, bits: int, n_seqs: int, max_keys: int, device="cuda") -> torch.Tensor:
    """A workspace for attend_decode_weigh of up to n_seqs sequences with max_keys rows in all, zeroed and ready for calls on any stream."""
    return _zeroed(attend_weigh_workspace_bytes(heads, kv_heads, head_dim, bits, n_seqs, max_keys), "bitlinear_attend_weigh_workspace_bytes", device)


def alloc_attend_shared_workspace(heads: int, kv_heads: int, head_dim: int, n_seqs: int, device="cuda") -> torch.Tensor:
    """A workspace for attend_decode_shared of up to n_seqs sequences, zeroed and ready for calls on any stream."""
    return _zeroed(attend_shared_workspace_bytes(heads, kv_heads, head_dim, n_seqs), "bitlinear_attend_shared_workspace_bytes", device)


def _attend_more(where: str, call, cache: KVCache, batch: KVBatch, other, q, scale, more: tuple, out, workspace, stream):
    """What attend_decode_weigh and attend_decode_shared have in common: call(.., address of `other` (marks or groups), .., *more, ..)."""
    index = cache.index
    if batch.index != index or other.index != index:
        _refuse(where, f"not everything is on {cache.device}")
    if _current_device() != index:
        with torch.cuda.device(index):
            return _attend_more(where, call, cache, batch, other, q, scale, more, out, workspace, stream)
    if stream is not None and out is None:
        with _allocating_on(stream, cache.device):
            return _attend_more(where, call, cache, batch, other, q, scale, more, out, workspace, None)
    if q.dim() != 3:
        _refuse(where, "q is [tokens, heads, head_dim]", ERR_SHAPE)
    T, heads, _ = q.shape
    D = cache.head_dim
    if T != batch.n_seqs:
        _refuse(where, f"{batch.n_seqs} sequences and {T} tokens", ERR_SHAPE)
    shape = (T, heads, D)
    qs = _row_stride(q, shape, index, where)
    if out is None:
        out = _empty_rows(T, heads, D, cache.device)
    os_ = _row_stride(out, shape, index, where)
    if workspace.get_device() != index or not workspace.is_contiguous():
        _refuse(where, f"the workspace is contiguous and on {cache.device}")
    st = call(cache._address, batch._address, other._address, q.data_ptr(), qs, heads, D ** -0.5 if scale is None else float(scale),
              *more, out.data_ptr(), os_, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
              _raw_stream(index) if stream is None else _stream(stream))
    if st != OK:
        _check(st, where)
    return out


def attend_decode_weigh(cache: KVCache, batch: KVBatch, marks: KVMarks, q: torch.Tensor, scale: float | None = None,
                        out: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """bitlinear_attend_decode_weigh: attend_decode that also adds every row's weight to marks.mass.  The workspace
    (alloc_attend_weigh_workspace) depends on how many rows there are, so it has to be given."""
    where = "bitlinear_attend_decode_weigh"
    if workspace is None:
        _refuse(where, "a workspace is needed (alloc_attend_weigh_workspace)", ERR_WORKSPACE)
    _marks_of(cache, marks, where)
    return _attend_more(where, (_lib or load_library()).bitlinear_attend_decode_weigh, cache, batch, marks, q, scale, (), out, workspace, stream)


def attend_decode_shared(cache: KVCache, batch: KVBatch, groups: KVBatch, q: torch.Tensor, scale: float | None = None,
                         out: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None, share_from: int = -1) -> torch.Tensor:
    """bitlinear_attend_decode_shared: attend_decode for sequences that begin with the same rows.  groups: KVBatch(page_table [groups,
    pages] of the shared rows, kv_lens [groups] how many they are, cu_tokens [groups + 1] the bounds of each group's sequences).
    share_from: elements of keys from which on sharing is worth its cost; negative: the measured bound, 0: always."""
    where = "bitlinear_attend_decode_shared"
    if workspace is None:
        if stream is not None:
            with _allocating_on(stream, cache.device):
                return attend_decode_shared(cache, batch, groups, q, scale, out, share_from=share_from)
        workspace = torch.zeros(max(1, attend_shared_workspace_bytes(q.shape[1] if q.dim() == 3 else 0, cache.kv_heads, cache.head_dim, batch.n_seqs)),
                                dtype=torch.uint8, device=cache.device)
    return _attend_more(where, (_lib or load_library()).bitlinear_attend_decode_shared, cache, batch, groups, q, scale, (share_from,), out, workspace, stream)


def _int32(t: torch.Tensor, shape: tuple, index: int, where: str, name: str) -> int:
    if t.shape != shape or t.dtype is not torch.int32 or t.get_device() != index or not t.is_contiguous():
        _refuse(where, f"{name} is a contiguous int32 {list(shape)} on cuda:{index}")
    return t.data_ptr()


def kv_select(cache: KVCache, batch: KVBatch, marks: KVMarks, keep: int, recent: int = 0, source: torch.Tensor | None = None,
              new_lens: torch.Tensor | None = None, stream=None, any_order: bool = False):
    """bitlinear_kv_select: -> (source int32 [n_seqs, kv_heads, keep], new_lens int32 [n_seqs]), which rows stay when the sequences are
    cut to `keep` rows: those of the `recent` newest positions, then those of the largest mass.  The last row of a sequence has to be its
    newest, as it is behind an append; any_order (bitlinear_kv_select_any_order): rows may stand in any order, as they do when they
    were moved (kv_compact) and nothing was appended since."""
    where = "bitlinear_kv_select_any_order" if any_order else "bitlinear_kv_select"
    index = cache.index
    if batch.index != index:
        _refuse(where, f"the cache is on {cache.device}, the batch on {batch.device}")
    if _current_device() != index:
        with torch.cuda.device(index):
            return kv_select(cache, batch, marks, keep, recent, source, new_lens, stream, any_order)
    if stream is not None and (source is None or new_lens is None):
        with _allocating_on(stream, cache.device):
            return kv_select(cache, batch, marks, keep, recent, source, new_lens, any_order=any_order)
    if not 1 <= keep <= 1 << 30:
        _refuse(where, "keep is 1 .. 2^30", ERR_SHAPE)
    shape = (batch.n_seqs, cache.kv_heads, keep)
    if source is None:
        source = torch.empty(shape, dtype=torch.int32, device=cache.device)
    if new_lens is None:
        new_lens = torch.empty(shape[:1], dtype=torch.int32, device=cache.device)
    L = _lib or load_library()
    st = (L.bitlinear_kv_select_any_order if any_order else L.bitlinear_kv_select)(
        cache._address, batch._address, _marks_of(cache, marks, where), keep, recent, _int32(source, shape, index, where, "source"),
        _int32(new_lens, shape[:1], index, where, "new_lens"), _raw_stream(index) if stream is None else _stream(stream))
    if st != OK:
        _check(st, where)
    return source, new_lens


def kv_compact(cache: KVCache, batch: KVBatch, source: torch.Tensor, marks: KVMarks | None = None, stream=None):
    """bitlinear_kv_compact: moves the rows that `source` (from kv_select) names to the front; batch.kv_lens still holds the lengths
    before."""
    where = "bitlinear_kv_compact"
    index = cache.index
    if batch.index != index:
        _refuse(where, f"the cache is on {cache.device}, the batch on {batch.device}")
    if _current_device() != index:
        with torch.cuda.device(index):
            return kv_compact(cache, batch, source, marks, stream)
    if source.dim() != 3:
        _refuse(where, "source is [n_seqs, kv_heads, keep]", ERR_SHAPE)
    keep = source.shape[2]
    st = (_lib or load_library()).bitlinear_kv_compact(
        cache._address, batch._address, _int32(source, (batch.n_seqs, cache.kv_heads, keep), index, where, "source"), keep,
        0 if marks is None else _marks_of(cache, marks, where), _raw_stream(index) if stream is None else _stream(stream))
    if st != OK:
        _check(st, where)
