"""ctypes binding of librabit.so: argument marshalling only.

Every function has the name and meaning of the C entry point in
``include/rabit.h``.  PyTorch supplies device memory and the current stream;
all arithmetic runs in the HIP kernels.  Importing this module fails loudly if
the library has not been built - there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Sequence, Tuple

import numpy as np
import torch  # imported before the library so that both share one HIP runtime

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librabit.so")

RB_OK = 0
RB_ERR_NULL, RB_ERR_SHAPE, RB_ERR_ALIGN, RB_ERR_UNSUPPORTED = -1, -2, -3, -4
RB_ERR_HIP, RB_ERR_WORKSPACE, RB_ERR_VALUE, RB_ERR_HANDOVER = -5, -6, -7, -8
RB_F16, RB_BF16, RB_F32 = 0, 1, 2
_ERR_NAMES = {-1: "RB_ERR_NULL", -2: "RB_ERR_SHAPE", -3: "RB_ERR_ALIGN", -4: "RB_ERR_UNSUPPORTED",
              -5: "RB_ERR_HIP", -6: "RB_ERR_WORKSPACE", -7: "RB_ERR_VALUE", -8: "RB_ERR_HANDOVER"}

EXPORTS = [
    "rb_pack", "rb_unpack", "rb_native_bytes", "rb_repack_native", "rb_unpack_native",
    "rb_linear_gemv", "rb_linear_gemm", "rb_layer_stack", "rb_workspace_bytes",
    "rb_stack_prepare", "rb_stack_run", "rb_stack_forget", "rb_stack_status", "rb_stack_waited",
    "rb_stack_set_option", "rb_stack_gave_up",
    "rb_linear_gemm_noalloc", "rb_noalloc_scratch_bytes",
    "rb_couple", "rb_weight_grad", "rb_scale_grads", "rb_scale_grads_workspace_bytes",
    "rb_block_prepare", "rb_block_workspace_bytes", "rb_rmsnorm", "rb_silu_mul", "rb_add",
    "rb_derive_iterative", "rb_derive_workspace_bytes",
    "rb_attn_prompt", "rb_attn_prompt_grad", "rb_attn_grad_workspace_bytes", "rb_attn_paged", "rb_attn_paged_workspace_bytes", "rb_cache_append",
    "rb_cache8_append", "rb_cache8_read", "rb_attn_cache8", "rb_attn_cache8_workspace_bytes", "rb_sample", "rb_sample_workspace_bytes",
    "rb_dense_gemv_f16", "rb_stream_read", "rb_stream_read_groups", "rb_version", "rb_last_path",
]


class RabitError(RuntimeError):
    def __init__(self, fn: str, code: int):
        super().__init__(f"{fn} returned {_ERR_NAMES.get(code, code)}")
        self.code = code


class rb_layer(ctypes.Structure):
    _fields_ = [("out", ctypes.c_int), ("inn", ctypes.c_int), ("K", ctypes.c_int),
                ("bits", ctypes.c_void_p), ("g", ctypes.c_void_p), ("h", ctypes.c_void_p)]


class rb_stack_op(ctypes.Structure):
    _fields_ = [("layer", ctypes.c_int), ("src", ctypes.c_int), ("dst", ctypes.c_int)]


class rb_block_op(ctypes.Structure):
    _fields_ = [("layer", ctypes.c_int), ("src", ctypes.c_int), ("dst", ctypes.c_int),
                ("norm", ctypes.c_int), ("epilogue", ctypes.c_int), ("aux", ctypes.c_int)]


class rb_heads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("heads", "kv_heads", "dim", "dtype")] + \
               [(n, ctypes.c_longlong) for n in ("q_token", "q_head", "k_token", "k_head", "v_token", "v_head")]


class rb_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + \
               [(n, ctypes.c_int) for n in ("pages", "page_tokens", "kv_heads", "dim", "dtype")] + \
               [(n, ctypes.c_longlong) for n in ("page_stride", "token_stride", "head_stride")]


class rb_cache8(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_exp", "v_exp")] + \
               [(n, ctypes.c_int) for n in ("pages", "page_tokens", "kv_heads", "dim", "dtype")] + \
               [(n, ctypes.c_longlong) for n in ("page_stride", "token_stride", "head_stride")]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    lib = ctypes.CDLL(LIB_PATH)
    i, p, z = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    lib.rb_pack.argtypes = [p, i, i, i, p]
    lib.rb_unpack.argtypes = [p, i, i, i, p]
    lib.rb_native_bytes.argtypes = [i, i, i]
    lib.rb_native_bytes.restype = z
    lib.rb_repack_native.argtypes = [p, i, i, i, p]
    lib.rb_unpack_native.argtypes = [p, i, i, i, p]
    lib.rb_linear_gemv.argtypes = [ctypes.POINTER(rb_layer), p, p, p, z, p]
    lib.rb_linear_gemm.argtypes = [ctypes.POINTER(rb_layer), p, p, i, i, i, p, z, p]
    lib.rb_linear_gemm_noalloc.argtypes = [ctypes.POINTER(rb_layer), p, p, i, i, i, p]
    lib.rb_noalloc_scratch_bytes.argtypes = []
    lib.rb_noalloc_scratch_bytes.restype = z
    lib.rb_layer_stack.argtypes = [ctypes.POINTER(rb_layer), i, ctypes.POINTER(rb_stack_op), i,
                                   ctypes.POINTER(ctypes.c_void_p), i, i, p, z, p]
    lib.rb_stack_prepare.argtypes = lib.rb_layer_stack.argtypes
    lib.rb_stack_run.argtypes = [p, z, p]
    lib.rb_stack_forget.argtypes = [p]
    lib.rb_stack_set_option.argtypes = [i, i]
    lib.rb_stack_status.argtypes = [p, p]
    lib.rb_stack_waited.argtypes = [p, p, ctypes.POINTER(ctypes.c_ulonglong)]
    lib.rb_stack_gave_up.argtypes = [p, p, ctypes.POINTER(ctypes.c_int)]
    lib.rb_workspace_bytes.argtypes = [ctypes.POINTER(rb_layer), i, i, i]
    lib.rb_workspace_bytes.restype = z
    lib.rb_block_workspace_bytes.argtypes = [ctypes.POINTER(rb_layer), i, i, i]
    lib.rb_block_workspace_bytes.restype = z
    lib.rb_block_prepare.argtypes = [ctypes.POINTER(rb_layer), i, ctypes.POINTER(ctypes.c_void_p), i, ctypes.c_float,
                                     ctypes.POINTER(rb_block_op), i, ctypes.POINTER(ctypes.c_void_p), i, i, p, z, p]
    lib.rb_rmsnorm.argtypes = [p, p, p, i, i, ctypes.c_float, p]
    lib.rb_silu_mul.argtypes = [p, p, p, z, p]
    lib.rb_add.argtypes = [p, p, p, z, p]
    lib.rb_derive_workspace_bytes.argtypes = [i, i]
    lib.rb_derive_workspace_bytes.restype = z
    lib.rb_derive_iterative.argtypes = [p, p, p, i, i, i, i, p, p, p, p, p, z, p]
    lib.rb_couple.argtypes = [p, p, p, i, i, i, p, p, p, p]
    lib.rb_weight_grad.argtypes = [p, p, i, i, i, p, p]
    lib.rb_scale_grads_workspace_bytes.argtypes = [i, i, i]
    lib.rb_scale_grads_workspace_bytes.restype = z
    lib.rb_scale_grads.argtypes = [p, p, p, p, i, i, i, p, p, p, z, p]
    f, l = ctypes.c_float, ctypes.c_longlong
    lib.rb_attn_prompt.argtypes = [ctypes.POINTER(rb_heads), p, p, p, p, p, i, i, i, i, f, p, p, p]
    lib.rb_attn_grad_workspace_bytes.argtypes = [ctypes.POINTER(rb_heads), i, i]
    lib.rb_attn_grad_workspace_bytes.restype = z
    lib.rb_attn_prompt_grad.argtypes = [ctypes.POINTER(rb_heads), p, p, p, p, p, p, p, p, i, i, i, i, f, p, p, p, p, z, p]
    lib.rb_cache_append.argtypes = [ctypes.POINTER(rb_cache), ctypes.POINTER(rb_heads), p, p, p, p, p, i, i, i, p, p, p, i, i, i, p, p]
    lib.rb_attn_paged_workspace_bytes.argtypes = [ctypes.POINTER(rb_cache), i, i, i]
    lib.rb_attn_paged_workspace_bytes.restype = z
    lib.rb_attn_paged.argtypes = [ctypes.POINTER(rb_cache), p, l, l, i, p, p, p, i, i, i, f, p, p, z, p]
    lib.rb_cache8_append.argtypes = [ctypes.POINTER(rb_cache8), *lib.rb_cache_append.argtypes[1:]]
    lib.rb_cache8_read.argtypes = [ctypes.POINTER(rb_cache8), p, p, p, i, i, i, p, p, p]
    lib.rb_attn_cache8_workspace_bytes.argtypes = [ctypes.POINTER(rb_cache8), i, i, i]
    lib.rb_attn_cache8_workspace_bytes.restype = z
    lib.rb_attn_cache8.argtypes = [ctypes.POINTER(rb_cache8), *lib.rb_attn_paged.argtypes[1:]]
    lib.rb_sample.argtypes = [p, i, l, i, i, p, p, p, p, p, p, p, z, p]
    lib.rb_sample_workspace_bytes.argtypes = [i, i, i]
    lib.rb_sample_workspace_bytes.restype = z
    lib.rb_dense_gemv_f16.argtypes = [p, p, p, i, i, p]
    lib.rb_stream_read.argtypes = [p, z, p, p]
    lib.rb_stream_read_groups.argtypes = []
    lib.rb_version.argtypes = []
    lib.rb_last_path.argtypes = []
    for name in EXPORTS:
        if name not in ("rb_native_bytes", "rb_workspace_bytes", "rb_noalloc_scratch_bytes",
                        "rb_scale_grads_workspace_bytes", "rb_block_workspace_bytes", "rb_derive_workspace_bytes",
                        "rb_attn_paged_workspace_bytes", "rb_attn_grad_workspace_bytes", "rb_attn_cache8_workspace_bytes", "rb_sample_workspace_bytes"):
            getattr(lib, name).restype = i
    return lib


lib = _load()


def _check(fn: str, code: int) -> None:
    if code != RB_OK:
        raise RabitError(fn, code)


def _np_ptr(a: np.ndarray) -> ctypes.c_void_p:
    return a.ctypes.data_as(ctypes.c_void_p)


def _stream() -> int:
    """The current stream of the current device (torch.cuda.current_stream() without its stream object, 2 us of a call)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


_DTYPE_CODE = {torch.float16: RB_F16, torch.bfloat16: RB_BF16, torch.float32: RB_F32}


# ------------------------------------------------------------------ host ---
def rb_pack(signs: np.ndarray) -> np.ndarray:
    """int8 +1/-1 [K][out][in] (host) -> canonical uint32 [K][out][in/32] (host)."""
    signs = np.ascontiguousarray(signs, dtype=np.int8)
    K, out, inn = signs.shape
    packed = np.empty((K, out, max(inn // 32, 0)), dtype=np.uint32)
    _check("rb_pack", lib.rb_pack(_np_ptr(signs), K, out, inn, _np_ptr(packed)))
    return packed


def rb_unpack(packed: np.ndarray) -> np.ndarray:
    packed = np.ascontiguousarray(packed, dtype=np.uint32)
    K, out, W32 = packed.shape
    signs = np.empty((K, out, W32 * 32), dtype=np.int8)
    _check("rb_unpack", lib.rb_unpack(_np_ptr(packed), K, out, W32 * 32, _np_ptr(signs)))
    return signs


def rb_native_bytes(K: int, out: int, inn: int) -> int:
    return int(lib.rb_native_bytes(K, out, inn))


def rb_repack_native(packed: np.ndarray) -> np.ndarray:
    """canonical uint32 [K][out][in/32] -> native layout, flat uint32 (host)."""
    packed = np.ascontiguousarray(packed, dtype=np.uint32)
    K, out, W32 = packed.shape
    native = np.empty(rb_native_bytes(K, out, W32 * 32) // 4, dtype=np.uint32)
    _check("rb_repack_native", lib.rb_repack_native(_np_ptr(packed), K, out, W32 * 32, _np_ptr(native)))
    return native


def rb_unpack_native(native: np.ndarray, K: int, out: int, inn: int) -> np.ndarray:
    native = np.ascontiguousarray(native, dtype=np.uint32)
    packed = np.empty((K, out, inn // 32), dtype=np.uint32)
    _check("rb_unpack_native", lib.rb_unpack_native(_np_ptr(native), K, out, inn, _np_ptr(packed)))
    return packed


# ---------------------------------------------------------------- device ---
class Layer:
    """Device-resident frozen layer: native sign words + fp16 g [K][out], h [K][in]."""

    def __init__(self, bits: torch.Tensor, g: torch.Tensor, h: torch.Tensor, K: int, out: int, inn: int):
        assert bits.is_cuda and g.is_cuda and h.is_cuda
        assert g.dtype == torch.float16 and h.dtype == torch.float16
        assert tuple(g.shape) == (K, out) and tuple(h.shape) == (K, inn)
        assert bits.numel() * bits.element_size() == rb_native_bytes(K, out, inn)
        self.bits, self.g, self.h = bits.contiguous(), g.contiguous(), h.contiguous()
        self.K, self.out, self.inn = K, out, inn

    @classmethod
    def from_host(cls, signs: np.ndarray, g: np.ndarray, h: np.ndarray, device="cuda:0") -> "Layer":
        """Pack int8 signs [K][out][in] with rb_pack + rb_repack_native and upload."""
        K, out, inn = signs.shape
        native = rb_repack_native(rb_pack(signs))
        bits = torch.from_numpy(native.view(np.int32)).to(device)
        return cls(bits, torch.from_numpy(np.ascontiguousarray(g, dtype=np.float16)).to(device),
                   torch.from_numpy(np.ascontiguousarray(h, dtype=np.float16)).to(device), K, out, inn)

    def struct(self) -> rb_layer:
        return rb_layer(self.out, self.inn, self.K, self.bits.data_ptr(), self.g.data_ptr(),
                        self.h.data_ptr())

    @property
    def packed_bytes(self) -> int:
        """Bytes of sign bits of the unpadded matrix (K*out*in/8)."""
        return self.K * self.out * self.inn // 8


def _layer_array(layers: Sequence[Layer]):
    arr = (rb_layer * len(layers))()
    for n, L in enumerate(layers):
        arr[n] = L.struct()
    return arr


def rb_workspace_bytes(layers: Sequence[Layer], n_ops: int, T: int) -> int:
    return int(lib.rb_workspace_bytes(_layer_array(layers), len(layers), n_ops, T))


def _workspace(layers: Sequence[Layer], T: int, device, n_ops: int = 1) -> Tuple[torch.Tensor, int]:
    n = rb_workspace_bytes(layers, n_ops, T)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=device)
    return ws, n


def _call_workspace(s: rb_layer, T: int, device):
    """Scratch memory of one call on the layer of struct s: the tensor, which the caller holds until the call is enqueued, its
    address and size; nothing is allocated where nothing is asked for."""
    n = lib.rb_workspace_bytes(ctypes.byref(s), 1, 1, T)
    if n == 0:
        return None, 0, 0
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    return ws, ws.data_ptr(), n


def rb_linear_gemv(layer: Layer, x: torch.Tensor, y: torch.Tensor = None, workspace=None) -> torch.Tensor:
    """y = layer(x) for one fp16 token x [in]; returns fp16 [out]."""
    assert x.is_cuda and x.dtype == torch.float16 and x.is_contiguous() and x.numel() == layer.inn
    if y is None:
        y = torch.empty(layer.out, dtype=torch.float16, device=x.device)
    s = layer.struct()
    if workspace is None:
        ws, at, n = _call_workspace(s, 1, x.device)
    else:
        ws, n = workspace
        at = ws.data_ptr()
    _check("rb_linear_gemv", lib.rb_linear_gemv(ctypes.byref(s), x.data_ptr(), y.data_ptr(), at, n, _stream()))
    return y


def rb_linear_gemm(layer: Layer, X: torch.Tensor, out_dtype=torch.float16, Y: torch.Tensor = None,
                   workspace=None) -> torch.Tensor:
    """Y[t] = layer(X[t]); X [T][in] fp16 or bf16; returns [T][out] of out_dtype."""
    assert X.is_cuda and X.is_contiguous() and X.dim() == 2 and X.shape[1] == layer.inn
    T = X.shape[0]
    if Y is None:
        Y = torch.empty((T, layer.out), dtype=out_dtype, device=X.device)
    s = layer.struct()
    if workspace is None:
        ws, at, n = _call_workspace(s, T, X.device)
    else:
        ws, n = workspace
        at = ws.data_ptr()
    _check("rb_linear_gemm", lib.rb_linear_gemm(ctypes.byref(s), X.data_ptr(), Y.data_ptr(), T,
                                                _DTYPE_CODE[X.dtype], _DTYPE_CODE[Y.dtype], at, n, _stream()))
    return Y


def rb_linear_gemm_noalloc(layer: Layer, X: torch.Tensor, Y: torch.Tensor) -> torch.Tensor:
    """rb_linear_gemm_noalloc: like rb_linear_gemm, scratch memory inside the library; the caller
    passes the output tensor, so that nothing is allocated on the way."""
    assert X.is_cuda and X.is_contiguous() and X.dim() == 2 and X.shape[1] == layer.inn
    assert Y.is_cuda and Y.is_contiguous() and tuple(Y.shape) == (X.shape[0], layer.out)
    s = layer.struct()
    _check("rb_linear_gemm_noalloc", lib.rb_linear_gemm_noalloc(
        ctypes.byref(s), X.data_ptr(), Y.data_ptr(), X.shape[0], _DTYPE_CODE[X.dtype], _DTYPE_CODE[Y.dtype],
        _stream()))
    return Y


def rb_noalloc_scratch_bytes() -> int:
    return int(lib.rb_noalloc_scratch_bytes())


class Stack:
    """Marshalled arguments of rb_layer_stack, built once and reused per call."""

    def __init__(self, layers: Sequence[Layer], ops: Sequence[Tuple[int, int, int]],
                 bufs: Sequence[torch.Tensor], T: int):
        self.layers, self.bufs, self.T = list(layers), list(bufs), T
        for b in self.bufs:
            assert b.is_cuda and b.dtype == torch.float16 and b.is_contiguous()
        self._layers = _layer_array(self.layers)
        self._ops = (rb_stack_op * len(ops))(*[rb_stack_op(*o) for o in ops])
        self._bufs = (ctypes.c_void_p * len(bufs))(*[b.data_ptr() for b in self.bufs])
        self.n_ops = len(ops)
        self.ws, self.ws_bytes = _workspace(self.layers, T, self.bufs[0].device, n_ops=len(ops))

    def run(self) -> None:
        """rb_layer_stack: set-up and execution in one call."""
        _check("rb_layer_stack", lib.rb_layer_stack(
            self._layers, len(self.layers), self._ops, self.n_ops, self._bufs, len(self.bufs), self.T,
            self.ws.data_ptr(), self.ws_bytes, _stream()))

    def prepare(self) -> None:
        """rb_stack_prepare: everything that does not depend on the activations."""
        _check("rb_stack_prepare", lib.rb_stack_prepare(
            self._layers, len(self.layers), self._ops, self.n_ops, self._bufs, len(self.bufs), self.T,
            self.ws.data_ptr(), self.ws_bytes, _stream()))

    def run_prepared(self) -> None:
        """rb_stack_run: one pass of the prepared ops over the current buffer contents."""
        _check("rb_stack_run", lib.rb_stack_run(self.ws.data_ptr(), self.ws_bytes, _stream()))

    def status(self) -> int:
        """rb_stack_status: waits for the stream; RB_OK, or RB_ERR_HANDOVER if a run gave up a wait."""
        return int(lib.rb_stack_status(self.ws.data_ptr(), _stream()))

    def waited(self) -> int:
        """rb_stack_waited: input tiles, over all runs since prepare, that were requested before they
        were written and had to be waited for (waits for the stream)."""
        n = ctypes.c_ulonglong(0)
        _check("rb_stack_waited", lib.rb_stack_waited(self.ws.data_ptr(), _stream(), ctypes.byref(n)))
        return int(n.value)

    def gave_up(self) -> int:
        """rb_stack_gave_up: which bounded wait a run gave up (0: none); waits for the stream."""
        r = ctypes.c_int(0)
        _check("rb_stack_gave_up", lib.rb_stack_gave_up(self.ws.data_ptr(), _stream(), ctypes.byref(r)))
        return int(r.value)

    def forget(self) -> None:
        _check("rb_stack_forget", lib.rb_stack_forget(self.ws.data_ptr()))


RB_EPI_NONE, RB_EPI_ADD, RB_EPI_SILU_MUL = 0, 1, 2


class Block(Stack):
    """Marshalled arguments of rb_block_prepare; run, status, waited and forget are the stack's."""

    def __init__(self, layers: Sequence[Layer], norm_weights: Sequence[torch.Tensor], eps: float,
                 ops: Sequence[Tuple[int, int, int, int, int, int]], bufs: Sequence[torch.Tensor], T: int):
        self.layers, self.bufs, self.T = list(layers), list(bufs), T
        self.norm_weights, self.eps = list(norm_weights), float(eps)
        for b in self.bufs + self.norm_weights:
            assert b.is_cuda and b.dtype == torch.float16 and b.is_contiguous()
        self._layers = _layer_array(self.layers)
        self._ops = (rb_block_op * len(ops))(*[rb_block_op(*o) for o in ops])
        self._bufs = (ctypes.c_void_p * len(bufs))(*[b.data_ptr() for b in self.bufs])
        self._norms = (ctypes.c_void_p * max(len(self.norm_weights), 1))(*[w.data_ptr() for w in self.norm_weights])
        self.n_ops = len(ops)
        self.ws_bytes = int(lib.rb_block_workspace_bytes(self._layers, len(self.layers), self.n_ops, T))
        self.ws = torch.empty(max(self.ws_bytes, 16), dtype=torch.uint8, device=self.bufs[0].device)

    def run(self) -> None:
        self.prepare()
        self.run_prepared()

    def prepare(self) -> None:
        """rb_block_prepare: everything that does not depend on the activations."""
        _check("rb_block_prepare", lib.rb_block_prepare(
            self._layers, len(self.layers), self._norms, len(self.norm_weights), self.eps, self._ops, self.n_ops,
            self._bufs, len(self.bufs), self.T, self.ws.data_ptr(), self.ws_bytes, _stream()))


def rb_rmsnorm(x: torch.Tensor, w: torch.Tensor, eps: float, y: torch.Tensor = None) -> torch.Tensor:
    """y[t] = x[t] / sqrt(mean(x[t]^2) + eps) * w for fp16 x [T][n]."""
    assert x.is_cuda and x.dtype == torch.float16 and x.is_contiguous() and x.dim() == 2
    assert w.dtype == torch.float16 and w.numel() == x.shape[1]
    if y is None:
        y = torch.empty_like(x)
    _check("rb_rmsnorm", lib.rb_rmsnorm(x.data_ptr(), w.data_ptr(), y.data_ptr(), x.shape[0], x.shape[1], float(eps),
                                        _stream()))
    return y


def rb_silu_mul(gate: torch.Tensor, up: torch.Tensor, y: torch.Tensor = None) -> torch.Tensor:
    assert gate.is_cuda and gate.dtype == torch.float16 and up.dtype == torch.float16
    assert gate.is_contiguous() and up.is_contiguous() and gate.shape == up.shape
    if y is None:
        y = torch.empty_like(gate)
    _check("rb_silu_mul", lib.rb_silu_mul(gate.data_ptr(), up.data_ptr(), y.data_ptr(), gate.numel(), _stream()))
    return y


def rb_add(a: torch.Tensor, b: torch.Tensor, y: torch.Tensor = None) -> torch.Tensor:
    assert a.is_cuda and a.dtype == torch.float16 and b.dtype == torch.float16
    assert a.is_contiguous() and b.is_contiguous() and a.shape == b.shape
    if y is None:
        y = torch.empty_like(a)
    _check("rb_add", lib.rb_add(a.data_ptr(), b.data_ptr(), y.data_ptr(), a.numel(), _stream()))
    return y


def rb_layer_stack(layers: Sequence[Layer], ops: Sequence[Tuple[int, int, int]],
                   bufs: Sequence[torch.Tensor], T: int) -> None:
    """Run ops (layer, src, dst) in order over device fp16 buffers [T][width]."""
    Stack(layers, ops, bufs, T).run()


def rb_dense_gemv_f16(W: torch.Tensor, x: torch.Tensor, y: torch.Tensor = None) -> torch.Tensor:
    out, inn = W.shape
    assert W.dtype == torch.float16 and x.dtype == torch.float16 and W.is_contiguous()
    if y is None:
        y = torch.empty(out, dtype=torch.float16, device=W.device)
    _check("rb_dense_gemv_f16", lib.rb_dense_gemv_f16(W.data_ptr(), x.data_ptr(), y.data_ptr(), out, inn,
                                                      _stream()))
    return y


def rb_stream_read(src: torch.Tensor, sink: torch.Tensor = None) -> torch.Tensor:
    nbytes = src.numel() * src.element_size()
    if sink is None:
        sink = torch.empty(int(lib.rb_stream_read_groups()) * 16, dtype=torch.uint8, device=src.device)
    _check("rb_stream_read", lib.rb_stream_read(src.data_ptr(), nbytes, sink.data_ptr(), _stream()))
    return sink


RB_PATH_NONE, RB_PATH_SIGNADD, RB_PATH_MX, RB_PATH_GEMM, RB_PATH_BATCH = 0, 1, 2, 3, 4
RB_OPT_HANDOVER_PAUSE = 1


# -------------------------------------------------------- initialisation ---
def rb_derive_iterative(W: torch.Tensor, K: int, T_max: int, row_factors: torch.Tensor = None,
                        col_factors: torch.Tensor = None, want_err: bool = True):
    """Alg. 1 on the device: returns (packed int32 [K][out][in/32], g fp64 [K][out], h fp64 [K][in],
    err fp64 [T_max][K] or None)."""
    assert W.is_cuda and W.dtype == torch.float32 and W.is_contiguous() and W.dim() == 2
    out, inn = W.shape
    for f, n in ((row_factors, out), (col_factors, inn)):
        assert f is None or (f.is_cuda and f.dtype == torch.float64 and f.is_contiguous() and f.numel() == n)
    packed = torch.empty((K, out, inn // 32), dtype=torch.int32, device=W.device)
    g = torch.empty((K, out), dtype=torch.float64, device=W.device)
    h = torch.empty((K, inn), dtype=torch.float64, device=W.device)
    err = torch.empty((T_max, K), dtype=torch.float64, device=W.device) if want_err else None
    n = int(lib.rb_derive_workspace_bytes(out, inn))
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=W.device)
    _check("rb_derive_iterative", lib.rb_derive_iterative(
        W.data_ptr(), row_factors.data_ptr() if row_factors is not None else None,
        col_factors.data_ptr() if col_factors is not None else None, K, T_max, out, inn,
        packed.data_ptr(), g.data_ptr(), h.data_ptr(), err.data_ptr() if err is not None else None,
        ws.data_ptr(), n, _stream()))
    return packed, g, h, err


# -------------------------------------------------------------- training ---
def rb_couple(W: torch.Tensor, g: torch.Tensor, h: torch.Tensor, want_native: bool = True,
              want_residual: bool = False):
    """Alg. 2 forward loop on the device: W fp32 [out][in], g fp16 [K][out], h fp16 [K][in] ->
    (packed uint32 [K][out][in/32] as int32 tensor, native flat int32 tensor or None, residual or None)."""
    assert W.is_cuda and W.dtype == torch.float32 and W.is_contiguous()
    assert g.dtype == torch.float16 and h.dtype == torch.float16 and g.is_contiguous() and h.is_contiguous()
    out, inn = W.shape
    K = g.shape[0]
    packed = torch.empty((K, out, inn // 32), dtype=torch.int32, device=W.device)
    native = torch.empty(rb_native_bytes(K, out, inn) // 4, dtype=torch.int32, device=W.device) if want_native else None
    residual = torch.empty_like(W) if want_residual else None
    _check("rb_couple", lib.rb_couple(W.data_ptr(), g.data_ptr(), h.data_ptr(), K, out, inn, packed.data_ptr(),
                                      native.data_ptr() if native is not None else None,
                                      residual.data_ptr() if residual is not None else None, _stream()))
    return packed, native, residual


def rb_weight_grad(Delta: torch.Tensor, X: torch.Tensor) -> torch.Tensor:
    """G = Delta^T X in fp32: Delta fp16 [N][out], X fp16 [N][in]."""
    assert Delta.is_cuda and Delta.dtype == torch.float16 and X.dtype == torch.float16
    assert Delta.is_contiguous() and X.is_contiguous() and Delta.shape[0] == X.shape[0]
    N, out = Delta.shape
    inn = X.shape[1]
    G = torch.empty((out, inn), dtype=torch.float32, device=X.device)
    _check("rb_weight_grad", lib.rb_weight_grad(Delta.data_ptr(), X.data_ptr(), N, out, inn, G.data_ptr(), _stream()))
    return G


def rb_scale_grads(G: torch.Tensor, packed: torch.Tensor, g: torch.Tensor, h: torch.Tensor):
    """(grad_g fp32 [K][out], grad_h fp32 [K][in]) from G fp32 [out][in] and the canonical packed cores."""
    assert G.is_cuda and G.dtype == torch.float32 and G.is_contiguous() and packed.is_contiguous()
    out, inn = G.shape
    K = g.shape[0]
    n = int(lib.rb_scale_grads_workspace_bytes(K, out, inn))
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=G.device)
    gg = torch.empty((K, out), dtype=torch.float32, device=G.device)
    gh = torch.empty((K, inn), dtype=torch.float32, device=G.device)
    _check("rb_scale_grads", lib.rb_scale_grads(G.data_ptr(), packed.data_ptr(), g.data_ptr(), h.data_ptr(), K, out, inn,
                                                gg.data_ptr(), gh.data_ptr(), ws.data_ptr(), n, _stream()))
    return gg, gh


# -------------------------------------------------- attention, its cache ---
# (A call of these is a few microseconds of kernel: each attribute of a tensor is asked for once.)
_I32 = torch.int32


def _heads(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> rb_heads:
    """Shapes and strides of q [tokens][heads][dim] and k, v [tokens][kv_heads][dim], elements of a head contiguous."""
    qs, ks, vs, dtype = q.stride(), k.stride(), v.stride(), k.dtype
    tokens, heads, dim = q.shape
    tokens_k, kv_heads, dim_k = k.shape
    assert k.is_cuda and v.is_cuda and q.is_cuda and q.dtype is dtype and v.dtype is dtype and k.shape == v.shape
    assert qs[2] == ks[2] == vs[2] == 1 and dim_k == dim
    H = rb_heads(heads, kv_heads, dim, _DTYPE_CODE[dtype], qs[0], qs[1], ks[0], ks[1], vs[0], vs[1])
    # one token or head: torch's stride says nothing and may be anything
    if tokens == 1:
        H.q_token = dim
    if heads == 1:
        H.q_head = dim
    if tokens_k <= 1:
        H.k_token = H.v_token = dim
    if kv_heads == 1:
        H.k_head = H.v_head = dim
    return H


def _starts(first: torch.Tensor, first_k: torch.Tensor = None):
    """Address of first int32 [n_seqs + 1], of first_k of the same length or None, and n_seqs."""
    n = first.shape[0]
    assert first.is_cuda and first.dtype is _I32 and first.dim() == 1 and first.is_contiguous()
    if first_k is None:
        return first.data_ptr(), None, n - 1
    assert first_k.is_cuda and first_k.dtype is _I32 and first_k.shape == first.shape and first_k.is_contiguous()
    return first.data_ptr(), first_k.data_ptr(), n - 1


def rb_attn_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, first: torch.Tensor, first_k: torch.Tensor = None,
                   causal: bool = True, scale: float = None, want_lse: bool = False, o: torch.Tensor = None):
    """Attention over packed sequences: q [tokens][heads][dim], k and v [tokens][kv_heads][dim] (fp16 or bf16, any
    strides of tokens and heads), first int32 [n_seqs + 1]; returns o [tokens][heads][dim], or (o, lse fp32 [tokens][heads])."""
    H = _heads(q, k, v)
    at, at_k, n = _starts(first, first_k)
    shape = q.shape
    if o is None:
        o = torch.empty(shape, dtype=q.dtype, device=q.device)
    else:
        assert o.is_cuda and o.dtype is q.dtype and o.shape == shape and o.is_contiguous()
    lse = torch.empty(shape[:2], dtype=torch.float32, device=q.device) if want_lse else None
    _check("rb_attn_prompt", lib.rb_attn_prompt(
        ctypes.byref(H), q.data_ptr(), k.data_ptr(), v.data_ptr(), at, at_k, n, shape[0], k.shape[0], causal,
        shape[2] ** -0.5 if scale is None else scale, o.data_ptr(), lse.data_ptr() if want_lse else None, _stream()))
    return (o, lse) if want_lse else o


def rb_attn_prompt_grad(go: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor,
                        first: torch.Tensor, first_k: torch.Tensor = None, causal: bool = True, scale: float = None):
    """(dq, dk, dv) of rb_attn_prompt, given go, the gradient of its result o, and its lse."""
    H = _heads(q, k, v)
    at, at_k, n = _starts(first, first_k)
    shape, dtype, device = q.shape, q.dtype, q.device
    for x in (go, o):
        assert x.is_cuda and x.dtype is dtype and x.shape == shape and x.is_contiguous()
    assert lse.is_cuda and lse.dtype is torch.float32 and lse.shape == shape[:2] and lse.is_contiguous()
    if k.shape[0] == 0:
        return torch.zeros(shape, dtype=dtype, device=device), torch.empty_like(k), torch.empty_like(v)
    dq, dk, dv = (torch.empty(s, dtype=dtype, device=device) for s in (shape, k.shape, k.shape))
    need = lib.rb_attn_grad_workspace_bytes(ctypes.byref(H), shape[0], k.shape[0])
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
    _check("rb_attn_prompt_grad", lib.rb_attn_prompt_grad(
        ctypes.byref(H), go.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), at, at_k, n, shape[0], k.shape[0],
        causal, shape[2] ** -0.5 if scale is None else scale, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), need, _stream()))
    return dq, dk, dv


class Cache:
    """A paged cache over two tensors [pages][page_tokens][kv_heads][dim] of equal strides (fp16 or bf16)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        assert k.is_cuda and v.is_cuda and k.dim() == 4 and k.shape == v.shape and k.dtype is v.dtype
        self.k, self.v, self.dtype = k, v, k.dtype
        pages, page_tokens, self.kv_heads, self.dim = k.shape
        strides = [(page if pages > 1 else page_tokens * token, token, head if self.kv_heads > 1 else self.dim, one)      # (of a single page or head torch's says nothing)
                   for page, token, head, one in (k.stride(), v.stride())]
        assert strides[0] == strides[1] and strides[0][3] == 1
        self._struct = rb_cache(k.data_ptr(), v.data_ptr(), pages, page_tokens, self.kv_heads, self.dim, _DTYPE_CODE[k.dtype], *strides[0][:3])

    @classmethod
    def zeros(cls, pages: int, page_tokens: int, kv_heads: int, dim: int, dtype=torch.float16, device="cuda:0") -> "Cache":
        return cls(*(torch.zeros((pages, page_tokens, kv_heads, dim), dtype=dtype, device=device) for _ in range(2)))

    def struct(self) -> rb_cache:
        return self._struct


def _sequences(first: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor):
    """Addresses of first int32 [n_seqs + 1], lengths [n_seqs] and table [n_seqs][width]; width, n_seqs."""
    n, width = table.shape
    assert first.is_cuda and lengths.is_cuda and table.is_cuda and first.dtype is _I32 and lengths.dtype is _I32 and table.dtype is _I32
    assert first.shape == (n + 1,) and lengths.shape == (n,)
    assert first.is_contiguous() and lengths.is_contiguous() and table.is_contiguous()
    return first.data_ptr(), lengths.data_ptr(), table.data_ptr(), width, n


class Cache8:
    """A paged cache in 8 bits: k and v float8_e4m3fn [pages][page_tokens][kv_heads][dim] of equal strides, k_exp and v_exp uint8 [pages][kv_heads][page_tokens],
    an element being e4m3 * 2^(byte - 127); dtype: fp16 or bf16, of the tokens that enter it and of the queries."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_exp: torch.Tensor, v_exp: torch.Tensor, dtype: torch.dtype = torch.float16):
        assert k.is_cuda and v.is_cuda and k_exp.is_cuda and v_exp.is_cuda and k.dim() == 4 and k.shape == v.shape
        assert k.dtype is v.dtype is torch.float8_e4m3fn and k_exp.dtype is v_exp.dtype is torch.uint8
        self.k, self.v, self.k_exp, self.v_exp, self.dtype = k, v, k_exp, v_exp, dtype
        pages, page_tokens, self.kv_heads, self.dim = k.shape
        assert k_exp.shape == v_exp.shape == (pages, self.kv_heads, page_tokens) and k_exp.is_contiguous() and v_exp.is_contiguous()
        strides = [(page if pages > 1 else page_tokens * token, token, head if self.kv_heads > 1 else self.dim, one) for page, token, head, one in (k.stride(), v.stride())]
        assert strides[0] == strides[1] and strides[0][3] == 1
        self._struct = rb_cache8(k.data_ptr(), v.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(), pages, page_tokens, self.kv_heads, self.dim, _DTYPE_CODE[dtype],
                                 *strides[0][:3])

    @classmethod
    def zeros(cls, pages: int, page_tokens: int, kv_heads: int, dim: int, dtype=torch.float16, device="cuda:0") -> "Cache8":
        bytes_of = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device=device)
        return cls(*(bytes_of(pages, page_tokens, kv_heads, dim).view(torch.float8_e4m3fn) for _ in range(2)), *(bytes_of(pages, kv_heads, page_tokens) for _ in range(2)),
                   dtype)

    def struct(self) -> rb_cache8:
        return self._struct


def rb_cache_append(cache: Cache, k: torch.Tensor, v: torch.Tensor, first: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor,
                    q: torch.Tensor = None, cos: torch.Tensor = None, sin: torch.Tensor = None, interleaved: bool = False,
                    q_out: torch.Tensor = None):
    """New tokens k, v [tokens][kv_heads][dim] become the last of each sequence's lengths int32 [n_seqs] positions of the
    cache, with the rotary embedding of cos, sin fp32 [rows][rotary / 2] on k and q [tokens][heads][dim]; returns the turned q."""
    return _append("rb_cache_append", lib.rb_cache_append, cache, k, v, first, lengths, table, q, cos, sin, interleaved, q_out)


def rb_cache8_append(cache: Cache8, k: torch.Tensor, v: torch.Tensor, first: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor,
                     q: torch.Tensor = None, cos: torch.Tensor = None, sin: torch.Tensor = None, interleaved: bool = False,
                     q_out: torch.Tensor = None):
    """rb_cache_append into a cache in 8 bits."""
    return _append("rb_cache8_append", lib.rb_cache8_append, cache, k, v, first, lengths, table, q, cos, sin, interleaved, q_out)


def _append(name, entry, cache, k, v, first, lengths, table, q, cos, sin, interleaved, q_out):
    at = _sequences(first, lengths, table)
    H = _heads(k if q is None else q, k, v)
    assert H.kv_heads == cache.kv_heads and H.dim == cache.dim and k.dtype is cache.dtype
    tokens, from_q, to_q = k.shape[0], None, None
    if q is not None:
        shape = q.shape
        assert shape[0] == tokens
        if q_out is None:
            q_out = torch.empty(shape, dtype=q.dtype, device=q.device)
        else:
            assert q_out.is_cuda and q_out.dtype is q.dtype and q_out.shape == shape and q_out.is_contiguous()
        from_q, to_q = q.data_ptr(), q_out.data_ptr()
    assert (q is None) == (q_out is None) and (cos is None) == (sin is None)
    at_cos = at_sin = None
    rows = half = 0
    if cos is not None:
        rows, half = cos.shape
        assert cos.is_cuda and sin.is_cuda and cos.dtype is sin.dtype is torch.float32 and sin.shape == cos.shape
        assert cos.is_contiguous() and sin.is_contiguous()
        at_cos, at_sin = cos.data_ptr(), sin.data_ptr()
    _check(name, entry(ctypes.byref(cache._struct), ctypes.byref(H), from_q, k.data_ptr(), v.data_ptr(), at_cos, at_sin, rows, 2 * half, interleaved,
                       *at, tokens, to_q, _stream()))
    return q_out


def rb_cache8_read(cache: Cache8, first: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor, tokens: int, k: torch.Tensor = None, v: torch.Tensor = None):
    """The last first[s + 1] - first[s] of each sequence's lengths[s] positions, `tokens` in all (first[n_seqs], or more), as
    k and v [tokens][kv_heads][dim] of the cache's dtype."""
    at = _sequences(first, lengths, table)
    shape = (tokens, cache.kv_heads, cache.dim)
    if k is None:
        k = torch.empty(shape, dtype=cache.dtype, device=cache.k.device)
    if v is None:
        v = torch.empty_like(k)
    for x in (k, v):
        assert x.is_cuda and x.dtype is cache.dtype and x.shape == shape and x.is_contiguous()
    _check("rb_cache8_read", lib.rb_cache8_read(ctypes.byref(cache._struct), *at, tokens, k.data_ptr(), v.data_ptr(), _stream()))
    return k, v


def rb_attn_paged(cache: Cache, q: torch.Tensor, first: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor, scale: float = None,
                  o: torch.Tensor = None, workspace: torch.Tensor = None) -> torch.Tensor:
    """Attention of new tokens q [tokens][heads][dim], the last of each sequence's lengths positions, over the cache."""
    return _over_cache("rb_attn_paged", lib.rb_attn_paged, lib.rb_attn_paged_workspace_bytes, cache, q, first, lengths, table, scale, o, workspace)


def rb_attn_cache8(cache: Cache8, q: torch.Tensor, first: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor, scale: float = None,
                   o: torch.Tensor = None, workspace: torch.Tensor = None) -> torch.Tensor:
    """rb_attn_paged over a cache in 8 bits."""
    return _over_cache("rb_attn_cache8", lib.rb_attn_cache8, lib.rb_attn_cache8_workspace_bytes, cache, q, first, lengths, table, scale, o, workspace)


def _over_cache(name, entry, workspace_bytes, cache, q, first, lengths, table, scale, o, workspace):
    at = _sequences(first, lengths, table)
    shape, strides = q.shape, q.stride()
    tokens, heads, dim = shape
    assert q.is_cuda and q.dtype is cache.dtype and dim == cache.dim and strides[2] == 1
    if o is None:
        o = torch.empty(shape, dtype=q.dtype, device=q.device)
    else:
        assert o.is_cuda and o.dtype is q.dtype and o.shape == shape and o.is_contiguous()
    C = ctypes.byref(cache._struct)
    if workspace is None:
        need = workspace_bytes(C, heads, at[4], tokens)
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    else:
        assert workspace.is_cuda and workspace.is_contiguous()
    at_ws, size = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    _check(name, entry(C, q.data_ptr(), strides[0] if tokens > 1 else dim, strides[1] if heads > 1 else dim, heads, *at, tokens,
                       dim ** -0.5 if scale is None else scale, o.data_ptr(), at_ws, size, _stream()))
    return o


# -------------------------------------------------------------- sampling ---
def rb_sample(logits: torch.Tensor, u: torch.Tensor, temperature: torch.Tensor = None, top_k: torch.Tensor = None, top_p: torch.Tensor = None,
              min_p: torch.Tensor = None, tokens: torch.Tensor = None, workspace: torch.Tensor = None) -> torch.Tensor:
    """The next token int32 [rows] of logits [rows][vocab] (fp16, bf16 or fp32, any stride of rows), drawn with u fp32 [rows] in [0, 1); temperature, top_p and
    min_p fp32 [rows], top_k int32 [rows], None: not filtered.  -1: the row has no logit above minus infinity."""
    rows, vocab = logits.shape
    stride, one = logits.stride()
    assert logits.is_cuda and (one == 1 or vocab == 1)
    if tokens is None:
        tokens = torch.empty(rows, dtype=_I32, device=logits.device)
    at = []
    for x, dtype in ((u, torch.float32), (temperature, torch.float32), (top_k, _I32), (top_p, torch.float32), (min_p, torch.float32), (tokens, _I32)):
        assert x is None or (x.is_cuda and x.dtype is dtype and x.shape == (rows,) and x.is_contiguous())
        at.append(None if x is None else x.data_ptr())
    dtype = _DTYPE_CODE[logits.dtype]
    if workspace is None:
        need = lib.rb_sample_workspace_bytes(dtype, rows, vocab)
        workspace = torch.empty(need, dtype=torch.uint8, device=logits.device) if need else None
    else:
        assert workspace.is_cuda and workspace.is_contiguous()
    at_ws, size = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    _check("rb_sample", lib.rb_sample(logits.data_ptr(), dtype, stride if rows > 1 else vocab, rows, vocab, *at, at_ws, size, _stream()))
    return tokens


def rb_stack_set_option(option: int, value: int) -> None:
    _check("rb_stack_set_option", lib.rb_stack_set_option(option, value))


def rb_last_path() -> int:
    return int(lib.rb_last_path())


def rb_version() -> int:
    return int(lib.rb_version())
