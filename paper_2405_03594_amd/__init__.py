"""Python binding of libspl, the gfx950 sparse linear library (C ABI in ``include/spl.h``).

Argument marshalling only: every step of the computation runs in the HIP
kernels of ``libspl.so``.  PyTorch supplies device memory and the stream.
There is no fallback: if the library is missing or a call fails, an
exception is raised.

Names follow the C ABI without its ``spl_`` prefix:

* ``pack_sparse(W, mask)`` -> :class:`SparseMatrix` (bitmask, packed values,
  row offsets; paper section 2.4.1);
* ``sparse_linear(X, Wc)`` -> ``Y = X (W . Mask)^T`` for fp16/bf16 (section 2.4.2);
* ``sparse_linear_int8(Xq, x_scales, Wqc, w_scales)`` -> fp16 ``Y`` (section 3.4);
* ``sparse_linear_group`` / ``dense_linear_group``: several independent
  linears (e.g. q, k, v) of one batch size in one launch;
* ``unpack``, ``dense_linear``, ``dense_linear_int8``: decoder and dense comparators;
* ``sparse_weight_grad[_group]``, ``sparse_input_grad``, ``sparse_sgd_update``:
  the training step with the mask held fixed (Algorithm 1);
* ``block_tables``, ``qk_norm_rope[_grad|_append]``, ``cache_read``,
  ``attention_fp4`` over a :class:`KVCache`: the attention half of a layer,
  between the q, k, v projections and o;
* ``quantize_fp8[_both]``, ``linear_fp8[_grad]``, ``linear_fp8_grouped[_grad]``
  over an :class:`Fp8Matrix`: dense linears in 8-bit floats, and of experts;
* ``adamw_plan``, ``adamw_step``: the optimizer step over many tensors.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspl.so")

F16, BF16, I8 = 1, 2, 3
LAYOUT = {"rows": 0, "tile16": 1}
ALGO = {"auto": 0, "decode": 1, "prefill": 2}
_STATUS = {0: "ok", 1: "invalid argument", 2: "unsupported", 3: "overflow", 4: "HIP runtime error"}
I4 = 4                                  # 4-bit codes, two per byte (values held as uint8)
F32 = 5                                 # of the 8-bit float linears and the optimizer step
_TORCH_DTYPE = {torch.float16: F16, torch.bfloat16: BF16, torch.int8: I8, torch.uint8: I4}
_CODE_DTYPE = {F16: torch.float16, BF16: torch.bfloat16, I8: torch.int8, I4: torch.uint8}


class SplError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn}: {_STATUS.get(status, status)} (status {status})")
        self.status = status


class _Matrix(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int64),
        ("cols", ctypes.c_int64),
        ("dtype", ctypes.c_int32),
        ("layout", ctypes.c_int32),
        ("nnz", ctypes.c_int64),
        ("bitmask", ctypes.c_void_p),
        ("values", ctypes.c_void_p),
        ("row_offsets", ctypes.c_void_p),
        ("tile_offsets", ctypes.c_void_p),
        ("values_bytes", ctypes.c_int64),
    ]


class _SparseTask(ctypes.Structure):
    _fields_ = [("X", ctypes.c_void_p), ("W", ctypes.POINTER(_Matrix)), ("Y", ctypes.c_void_p)]


class _DenseTask(ctypes.Structure):
    _fields_ = [("X", ctypes.c_void_p), ("W", ctypes.c_void_p), ("N", ctypes.c_int64), ("K", ctypes.c_int64),
                ("Y", ctypes.c_void_p)]


class _Int8Task(ctypes.Structure):
    _fields_ = [("Xq", ctypes.c_void_p), ("x_scales", ctypes.c_void_p), ("Wq", ctypes.POINTER(_Matrix)),
                ("w_scales", ctypes.c_void_p), ("Y", ctypes.c_void_p), ("acc_out", ctypes.c_void_p)]


class _WeightGradTask(ctypes.Structure):
    _fields_ = [("dY", ctypes.c_void_p), ("X", ctypes.c_void_p), ("W", ctypes.POINTER(_Matrix)),
                ("grad_values", ctypes.c_void_p)]


class _Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("heads", ctypes.c_int32)]


class _KVCache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("pages", ctypes.c_int64), ("data_bytes", ctypes.c_int64),
                ("page", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class _Fp8(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("count", ctypes.c_int64), ("codes_bytes", ctypes.c_int64),
                ("scales_bytes", ctypes.c_int64), ("block", ctypes.c_int32)]


class _AdamwTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("m_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p), ("copy", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("decay", ctypes.c_double)]


class _AdamwTypes(ctypes.Structure):
    _fields_ = [("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32), ("copy_dtype", ctypes.c_int32),
                ("state_bits", ctypes.c_int32)]


class _DenseInt8Task(ctypes.Structure):
    _fields_ = [("Xq", ctypes.c_void_p), ("x_scales", ctypes.c_void_p), ("Wq", ctypes.c_void_p),
                ("w_scales", ctypes.c_void_p), ("N", ctypes.c_int64), ("K", ctypes.c_int64), ("Y", ctypes.c_void_p),
                ("acc_out", ctypes.c_void_p)]


MAX_GROUP = 16
_lib = None


def lib() -> ctypes.CDLL:
    """Load libspl.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
    L = ctypes.CDLL(LIB_PATH)
    P, I64, I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    MP = ctypes.POINTER(_Matrix)
    sigs = {
        "spl_version": (I32, []),
        "spl_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "spl_read_probe": (ctypes.c_int, [P, I64, P, P]),
        "spl_check_matrix": (ctypes.c_int, [MP]),
        "spl_validate": (ctypes.c_int, [MP, P]),
        "spl_values_bytes": (I64, [I32, I64]),
        "spl_tile16_count": (I64, [I64, I64]),
        "spl_retile16": (ctypes.c_int, [MP, P, P, P, P]),
        "spl_pack_count": (ctypes.c_int, [P, I32, P, I64, I64, I32, P, ctypes.POINTER(I64), P]),
        "spl_pack_sparse": (ctypes.c_int, [P, I32, P, I64, I64, I32, P, P, P, P]),
        "spl_unpack": (ctypes.c_int, [MP, P, P]),
        "spl_sparse_linear": (ctypes.c_int, [P, I64, MP, P, P]),
        "spl_sparse_linear_ex": (ctypes.c_int, [P, I64, MP, P, I32, P]),
        "spl_sparse_linear_expanded_workspace_bytes": (I64, [MP]),
        "spl_sparse_linear_expanded": (ctypes.c_int, [P, I64, MP, P, P, P]),
        "spl_sparse_linear_group_scratch_bytes": (I64, [ctypes.POINTER(_SparseTask), I32, I64]),
        "spl_sparse_linear_group_scratch": (ctypes.c_int, [ctypes.POINTER(_SparseTask), I32, I64, P, I64, P]),
        "spl_sparse_linear_silu_mul_scratch_bytes": (I64, [I64, MP, MP]),
        "spl_sparse_linear_silu_mul_scratch": (ctypes.c_int, [P, I64, MP, MP, P, P, I64, P]),
        "spl_sparse_linear_int8_group_scratch_bytes": (I64, [ctypes.POINTER(_Int8Task), I32, I64]),
        "spl_sparse_linear_int8_group_scratch": (ctypes.c_int, [ctypes.POINTER(_Int8Task), I32, I64, P, I64, P]),
        "spl_sparse_input_grad_scratch_bytes": (I64, [I64, MP]),
        "spl_sparse_input_grad_scratch": (ctypes.c_int, [P, I64, MP, P, P, I64, P]),
        "spl_sparse_linear_int8": (ctypes.c_int, [P, P, I64, MP, P, P, P, P]),
        "spl_sparse_linear_int8_expanded": (ctypes.c_int, [P, P, I64, MP, P, P, P, P, P]),
        "spl_quantize_rows_i8": (ctypes.c_int, [P, ctypes.c_int32, I64, I64, P, P, P]),
        "spl_sparse_linear_silu_mul": (ctypes.c_int, [P, I64, MP, MP, P, I32, P]),
        "spl_magnitude_mask_workspace_bytes": (I64, []),
        "spl_magnitude_mask": (ctypes.c_int, [P, I32, I64, I64, I64, P, P, P]),
        "spl_magnitude_mask_noalloc": (ctypes.c_int, [P, I32, I64, I64, I64, P, P]),
        "spl_transpose16": (ctypes.c_int, [P, I64, I64, P, P]),
        "spl_int4_values_bytes": (I64, [I64]),
        "spl_pack_int4": (ctypes.c_int, [MP, P, P, P]),
        "spl_sparse_linear_int4": (ctypes.c_int, [P, P, I64, MP, P, P, P, P]),
        "spl_gather_tiled": (ctypes.c_int, [P, MP, P, P]),
        "spl_sparse_weight_grad_workspace_bytes": (I64, [I64, I64, I64]),
        "spl_sparse_weight_grad": (ctypes.c_int, [P, P, I64, MP, P, P, P]),
        "spl_sparse_weight_grad_group": (ctypes.c_int, [ctypes.POINTER(_WeightGradTask), I32, I64, P, P]),
        "spl_sparse_input_grad_workspace_bytes": (I64, [I64, MP]),
        "spl_sparse_input_grad": (ctypes.c_int, [P, I64, MP, P, P, P]),
        "spl_sparse_sgd_update": (ctypes.c_int, [MP, P, ctypes.c_float, P]),
        "spl_transpose_perm_workspace_bytes": (I64, [I64, I64, I64]),
        "spl_transpose_perm": (ctypes.c_int, [MP, MP, P, P, P]),
        "spl_permute_values": (ctypes.c_int, [P, P, I64, P, P]),
        "spl_dense_linear": (ctypes.c_int, [P, I64, P, I32, I64, I64, P, P]),
        "spl_dense_linear_ex": (ctypes.c_int, [P, I64, P, I32, I64, I64, P, I32, P]),
        "spl_dense_linear_int8": (ctypes.c_int, [P, P, I64, P, P, I64, I64, P, P, P]),
        "spl_sparse_linear_group": (ctypes.c_int, [ctypes.POINTER(_SparseTask), I32, I64, I32, P]),
        "spl_dense_linear_group": (ctypes.c_int, [ctypes.POINTER(_DenseTask), I32, I64, I32, I32, P]),
        "spl_sparse_linear_int8_group": (ctypes.c_int, [ctypes.POINTER(_Int8Task), I32, I64, P]),
        "spl_dense_linear_int8_group": (ctypes.c_int, [ctypes.POINTER(_DenseInt8Task), I32, I64, P]),
    }
    HP, CP, F32 = ctypes.POINTER(_Heads), ctypes.POINTER(_KVCache), ctypes.c_float
    sigs.update({
        "spl_kv_page_bytes": (I64, [I32, I32]),
        "spl_block_tables": (ctypes.c_int, [P, P, I64, I64, I32, P, I64, P, I64, P, P, P, P, P, P, P]),
        "spl_qk_norm_rope": (ctypes.c_int, [HP, HP, I64, I32, I32, P, P, F32, P, P, I64, I32, I32, P, P, P]),
        "spl_qk_norm_rope_grad_workspace_bytes": (I64, [I64, I32, I32, I32]),
        "spl_qk_norm_rope_grad": (ctypes.c_int, [HP, HP, HP, HP, I64, I32, I32, P, P, F32, P, P, I64, I32, I32, P, P, P,
                                                 P, P, P]),
        "spl_qk_norm_rope_append": (ctypes.c_int, [HP, HP, HP, I64, P, P, F32, P, P, I64, I32, I32, P, CP, P, P, P]),
        "spl_cache_read": (ctypes.c_int, [CP, P, I64, P, P, P]),
        "spl_attention_fp4_workspace_bytes": (I64, [CP, I64, I32, I64, I64, I64, I64]),
        "spl_attention_fp4": (ctypes.c_int, [HP, I64, CP, P, I64, I64, P, P, I64, I64, F32, I32, P, P, P, P]),
    })
    MQ, F64 = ctypes.POINTER(_Fp8), ctypes.c_double
    TP, YP = ctypes.POINTER(_AdamwTensor), ctypes.POINTER(_AdamwTypes)
    sigs.update({
        "spl_fp8_codes_bytes": (I64, [I64, I64, I64]),
        "spl_fp8_scales_bytes": (I64, [I64, I64, I64, I32]),
        "spl_fp8_grouped_cols": (I64, [I64, I64]),
        "spl_quantize_fp8": (ctypes.c_int, [P, I32, I64, I64, I64, I64, P, I64, MQ, MQ, P]),
        "spl_dequantize_fp8": (ctypes.c_int, [MQ, I32, P, P]),
        "spl_linear_fp8_workspace_bytes": (I64, [I64, I64, I64]),
        "spl_linear_fp8": (ctypes.c_int, [MQ, MQ, I32, P, P, P]),
        "spl_linear_fp8_rows_workspace_bytes": (I64, [I64, I64, I64]),
        "spl_linear_fp8_rows": (ctypes.c_int, [P, I32, I64, I64, MQ, I32, P, P, P]),
        "spl_linear_fp8_grouped": (ctypes.c_int, [MQ, MQ, P, I32, P, P]),
        "spl_linear_fp8_grouped_rows_workspace_bytes": (I64, [I64, I64, I64, I64]),
        "spl_linear_fp8_grouped_rows": (ctypes.c_int, [P, I32, I64, I64, MQ, P, I32, P, P, P]),
        "spl_linear_fp8_grouped_weight_grad": (ctypes.c_int, [MQ, MQ, P, I64, I64, I32, P, P]),
        "spl_linear_fp8_grad_workspace_bytes": (I64, [I64, I64, I64, I64]),
        "spl_linear_fp8_grad": (ctypes.c_int, [P, I64, P, I64, I32, I64, MQ, P, I32, P, P, P, P]),
        "spl_linear_fp8_kernel": (I32, [I32, I64, I64, I64, I64, I32, I32]),
        "spl_adamw_plan_chunks": (I64, [TP, I64, YP]),
        "spl_adamw_plan_bytes": (I64, [TP, I64, YP]),
        "spl_adamw_plan": (ctypes.c_int, [TP, I64, YP, P]),
        "spl_adamw_step": (ctypes.c_int, [P, I64, YP, F64, F64, F64, F64, I64, P, P, ctypes.c_uint32, P]),
    })
    for name, (res, args) in sigs.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise SplError(fn, status)


def _ptr(t: torch.Tensor | None):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _lends(M: int, n: int, k: int) -> bool:
    """Whether a call of more rows than the streaming kernels take is offered scratch memory (the library says how
    much it can use): not for a matrix so small that it is always expanded in place."""
    return k > 1024 or M * n > 1 << 20


def _scratch(need: int, device, stream) -> torch.Tensor | None:
    """`need` bytes from the caching allocator for one call on `stream` (None: the current one): a block of that
    stream's own pool, so it is reused only behind the call.  `device` is that of a stream known by its handle
    alone.  None where none is needed or free (the call then runs without)."""
    if need <= 0:
        return None
    try:
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
        if stream is None or stream == torch.cuda.current_stream():
            return torch.empty((need,), dtype=torch.uint8, device="cuda")
        with torch.cuda.stream(stream):
            return torch.empty((need,), dtype=torch.uint8, device=stream.device)
    except torch.OutOfMemoryError:
        return None


def _dev_tensor(t: torch.Tensor, name: str) -> torch.Tensor:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _arg(t, name: str, shape=None, dtype=None, min_numel: int | None = None, device: bool = True) -> torch.Tensor:
    """An argument tensor's shape, dtype, length and contiguity, checked before
    its device: the C ABI sees only pointers, so a mismatch here would make a
    kernel read or write past a buffer."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a tensor")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if min_numel is not None and (t.dim() != 1 or t.numel() < min_numel):
        raise ValueError(f"{name} must be 1-D with at least {min_numel} entries")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return _dev_tensor(t, name) if device else t


def _q_args(Xq, x_scales, N: int, K: int, w_scales, M: int, device: bool = True) -> None:
    """int8 activations [M][K] and their per-row scales, per-channel weight scales [N]."""
    _arg(Xq, "Xq", shape=(M, K), dtype=torch.int8, device=False)
    _arg(x_scales, "x_scales", dtype=torch.float32, min_numel=M, device=False)
    _arg(w_scales, "w_scales", dtype=torch.float32, min_numel=N, device=False)
    if device:
        for t, nm in ((Xq, "Xq"), (x_scales, "x_scales"), (w_scales, "w_scales")):
            _dev_tensor(t, nm)


def _q_outs(out, acc_out, M: int, N: int, device: bool = True) -> None:
    _arg(out, "out", shape=(M, N), dtype=torch.float16, device=False)
    if acc_out is not None:
        _arg(acc_out, "acc_out", shape=(M, N), dtype=torch.int32, device=False)
    if device:
        _dev_tensor(out, "out")
        if acc_out is not None:
            _dev_tensor(acc_out, "acc_out")


def _rows_of(X, name: str) -> int:
    if not isinstance(X, torch.Tensor) or X.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor")
    return X.shape[0]


@dataclass
class SparseMatrix:
    """A compressed [N][K] matrix in one of the two layouts of include/spl.h:
    "rows" (row-layout bitmask, values, row_offsets) or "tile16" (16 x 32
    submatrices: tile-major bitmask, values, tile_offsets)."""

    bitmask: torch.Tensor              # int32 view of the uint32 bitmask words
    values: torch.Tensor               # payloads (fp16 / bf16 / int8), length >= nnz (+16 bytes of tail)
    row_offsets: torch.Tensor | None   # int32 [N+1] (rows layout)
    tile_offsets: torch.Tensor | None  # int32 [B*S+1] (tile16 layout)
    rows: int
    cols: int
    nnz: int
    layout: str = "rows"

    @property
    def dtype(self) -> torch.dtype:
        return self.values.dtype

    def view(self) -> _Matrix:
        return _Matrix(self.rows, self.cols, _TORCH_DTYPE[self.values.dtype], LAYOUT[self.layout], self.nnz,
                       self.bitmask.data_ptr(), self.values.data_ptr(),
                       self.row_offsets.data_ptr() if self.row_offsets is not None else 0,
                       self.tile_offsets.data_ptr() if self.tile_offsets is not None else 0,
                       self.values.numel() * self.values.element_size())

    def compressed_bytes(self) -> int:
        """Bytes of the encoding: payloads + bitmask + offsets."""
        offs = self.row_offsets if self.layout == "rows" else self.tile_offsets
        payload = (self.nnz + 1) // 2 if self.values.dtype == torch.uint8 else self.nnz * self.values.element_size()
        return payload + self.bitmask.numel() * 4 + offs.numel() * 4


def _values_buffer(nnz: int, dtype: torch.dtype, device) -> torch.Tensor:
    # spl_values_bytes: payloads rounded up to 16 bytes plus 16 readable bytes of
    # tail (kernels may read, never write, up to 16 bytes past the last payload)
    esz = torch.empty((), dtype=dtype).element_size()
    return torch.zeros(int(lib().spl_values_bytes(_TORCH_DTYPE[dtype], nnz)) // esz, dtype=dtype, device=device)


def pack_sparse(W: torch.Tensor, mask: torch.Tensor | None = None, layout: str = "tile16",
                stream=None) -> SparseMatrix:
    """Compress W [N][K] (fp16/bf16/int8) under `mask` (uint8/bool, non-zero = kept;
    None = keep the non-zero payloads) with spl_pack_count + spl_pack_sparse.
    layout="tile16" (default) is the layout the linear kernels read; "rows" is
    the row-layout interchange format."""
    L = lib()
    if not isinstance(W, torch.Tensor) or W.dim() != 2 or W.dtype not in _TORCH_DTYPE or W.dtype == torch.uint8:
        raise ValueError("W must be a 2-D fp16/bf16/int8 tensor")
    if layout not in LAYOUT:
        raise ValueError(f"unknown layout {layout!r}")
    N, K = W.shape
    if mask is not None:
        if mask.dtype == torch.bool:
            mask = mask.view(torch.uint8)
        _arg(mask, "mask", shape=(N, K), dtype=torch.uint8)
    _dev_tensor(W, "W")
    code = _TORCH_DTYPE[W.dtype]
    if layout == "rows":
        blocks = N
        bitmask = torch.empty((N, (K + 31) // 32), dtype=torch.int32, device=W.device)
    else:
        blocks = int(L.spl_tile16_count(N, K))
        bitmask = torch.empty(blocks * 16, dtype=torch.int32, device=W.device)
    offsets = torch.empty(blocks + 1, dtype=torch.int32, device=W.device)
    nnz = ctypes.c_int64(0)
    s = _stream(stream)
    _check("spl_pack_count", L.spl_pack_count(_ptr(W), code, _ptr(mask), N, K, LAYOUT[layout], _ptr(offsets),
                                              ctypes.byref(nnz), s))
    values = _values_buffer(nnz.value, W.dtype, W.device)
    _check("spl_pack_sparse", L.spl_pack_sparse(_ptr(W), code, _ptr(mask), N, K, LAYOUT[layout], _ptr(offsets),
                                                _ptr(bitmask), _ptr(values), s))
    if layout == "rows":
        return SparseMatrix(bitmask, values, offsets, None, N, K, nnz.value, "rows")
    return SparseMatrix(bitmask, values, None, offsets, N, K, nnz.value, "tile16")


def validate(Wc: SparseMatrix, stream=None) -> bool:
    """Device check of the view's format (spl_validate): True if consistent."""
    view = Wc.view()
    st = lib().spl_validate(ctypes.byref(view), _stream(stream))
    if st == 1:
        return False
    _check("spl_validate", st)
    return True


def retile16(Wc: SparseMatrix, stream=None) -> SparseMatrix:
    """Row layout -> tile layout (16 x 32 submatrices)."""
    L = lib()
    if Wc.layout != "rows":
        raise ValueError("retile16 expects the row layout")
    T = int(L.spl_tile16_count(Wc.rows, Wc.cols))
    dev = Wc.values.device
    bitmask = torch.empty(T * 16, dtype=torch.int32, device=dev)
    tile_offsets = torch.empty(T + 1, dtype=torch.int32, device=dev)
    values = _values_buffer(Wc.nnz, Wc.dtype, dev)
    view = Wc.view()
    _check("spl_retile16", L.spl_retile16(ctypes.byref(view), _ptr(bitmask), _ptr(values), _ptr(tile_offsets),
                                          _stream(stream)))
    return SparseMatrix(bitmask, values, None, tile_offsets, Wc.rows, Wc.cols, Wc.nnz, "tile16")


def unpack(Wc: SparseMatrix, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    L = lib()
    if out is None:
        out = torch.empty((Wc.rows, Wc.cols), dtype=Wc.dtype, device=Wc.values.device)
    view = Wc.view()
    _check("spl_unpack", L.spl_unpack(ctypes.byref(view), _ptr(out), _stream(stream)))
    return out


def sparse_linear(X: torch.Tensor, Wc: SparseMatrix, out: torch.Tensor | None = None, algo: str = "auto",
                  stream=None) -> torch.Tensor:
    """Y [M][N] = X [M][K] (W . Mask)^T, fp32 accumulation, output in X's dtype.

    Above 128 rows algo="auto" may multiply through a decoded copy of W: 2 bytes an entry from the caching allocator,
    for the call (a captured graph's pool keeps them), also where `out` is given.  Without the memory, or with
    algo="prefill", the tiles are expanded in place."""
    L = lib()
    M = _rows_of(X, "X")
    _arg(X, "X", shape=(M, Wc.cols), dtype=Wc.dtype, device=False)
    if out is None:
        out = torch.empty((M, Wc.rows), dtype=X.dtype, device=X.device)
    _arg(out, "out", shape=(M, Wc.rows), dtype=Wc.dtype)
    _dev_tensor(X, "X")
    view = Wc.view()
    if algo == "auto" and M > 128 and _lends(M, Wc.rows, Wc.cols):
        _linear_group(L, (_SparseTask * 1)(_SparseTask(X.data_ptr(), ctypes.pointer(view), out.data_ptr())), 1, M,
                      X.device, stream)
        return out
    _check("spl_sparse_linear_ex", L.spl_sparse_linear_ex(_ptr(X), M, ctypes.byref(view), _ptr(out), ALGO[algo],
                                                          _stream(stream)))
    return out


def _linear_group(L, tasks, n: int, M: int, device, stream) -> None:
    """AUTO on a task array, with scratch."""
    ws = _scratch(L.spl_sparse_linear_group_scratch_bytes(tasks, n, M), device, stream)
    _check("spl_sparse_linear_group_scratch",
           L.spl_sparse_linear_group_scratch(tasks, n, M, _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)))


def sparse_linear_expanded(X: torch.Tensor, Wc: SparseMatrix, out: torch.Tensor | None = None,
                           workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """sparse_linear through a decoded copy of W in `workspace` (see
    spl_sparse_linear_expanded): for large batches."""
    L = lib()
    M = _rows_of(X, "X")
    _arg(X, "X", shape=(M, Wc.cols), dtype=Wc.dtype, device=False)
    if out is None:
        out = torch.empty((M, Wc.rows), dtype=X.dtype, device=X.device)
    _arg(out, "out", shape=(M, Wc.rows), dtype=Wc.dtype)
    _dev_tensor(X, "X")
    view = Wc.view()
    need = L.spl_sparse_linear_expanded_workspace_bytes(ctypes.byref(view))
    if need < 0:
        raise ValueError("spl_sparse_linear_expanded: the matrix view is invalid")
    if workspace is None:
        workspace = torch.empty((need,), dtype=torch.uint8, device=X.device)
    _dev_tensor(workspace, "workspace")
    if workspace.numel() * workspace.element_size() < need:
        raise ValueError(f"workspace holds {workspace.numel() * workspace.element_size()} bytes, needs {need}")
    _check("spl_sparse_linear_expanded", L.spl_sparse_linear_expanded(_ptr(X), M, ctypes.byref(view), _ptr(out),
                                                                      _ptr(workspace), _stream(stream)))
    return out


def sparse_linear_silu_mul(X: torch.Tensor, Wgate: SparseMatrix, Wup: SparseMatrix, out: torch.Tensor | None = None,
                           algo: str = "auto", stream=None) -> torch.Tensor:
    """Y [M][N] = silu(X Wgate^T) * (X Wup^T): the gated half of a Llama MLP in
    one launch (see spl_sparse_linear_silu_mul).  Above 112 rows algo="auto" may take memory for a decoded copy of
    both matrices as in sparse_linear."""
    L = lib()
    if (Wup.rows, Wup.cols, Wup.dtype) != (Wgate.rows, Wgate.cols, Wgate.dtype):
        raise ValueError("gate and up must share shape and dtype")
    M = _rows_of(X, "X")
    _arg(X, "X", shape=(M, Wgate.cols), dtype=Wgate.dtype, device=False)
    if out is None:
        out = torch.empty((M, Wgate.rows), dtype=X.dtype, device=X.device)
    _arg(out, "out", shape=(M, Wgate.rows), dtype=Wgate.dtype)
    _dev_tensor(X, "X")
    vg, vu = Wgate.view(), Wup.view()
    if algo == "auto" and M > 112 and _lends(M, 2 * Wgate.rows, Wgate.cols):
        ws = _scratch(L.spl_sparse_linear_silu_mul_scratch_bytes(M, ctypes.byref(vg), ctypes.byref(vu)), X.device,
                      stream)
        _check("spl_sparse_linear_silu_mul_scratch",
               L.spl_sparse_linear_silu_mul_scratch(_ptr(X), M, ctypes.byref(vg), ctypes.byref(vu), _ptr(out),
                                                    _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)))
        return out
    _check("spl_sparse_linear_silu_mul", L.spl_sparse_linear_silu_mul(_ptr(X), M, ctypes.byref(vg), ctypes.byref(vu),
                                                                      _ptr(out), ALGO[algo], _stream(stream)))
    return out


def read_probe(buf: torch.Tensor, sink: torch.Tensor, stream=None) -> None:
    """Stream-read every byte of `buf` (a measurement helper; see spl_read_probe)."""
    L = lib()
    _dev_tensor(buf, "buf")
    _dev_tensor(sink, "sink")
    nbytes = buf.numel() * buf.element_size()
    if sink.numel() * sink.element_size() < 4:
        raise ValueError("sink needs 4 bytes")
    _check("spl_read_probe", L.spl_read_probe(_ptr(buf), nbytes, _ptr(sink), _stream(stream)))


def magnitude_mask(W: torch.Tensor, prune: int, out: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Keep-mask (uint8 [N][K]) zeroing exactly `prune` entries of smallest |w|,
    ties by ascending row-major index (see spl_magnitude_mask)."""
    L = lib()
    _dev_tensor(W, "W")
    N, K = W.shape
    if out is None:
        out = torch.empty((N, K), dtype=torch.uint8, device=W.device)
    if workspace is None:
        workspace = torch.empty((L.spl_magnitude_mask_workspace_bytes(),), dtype=torch.uint8, device=W.device)
    _check("spl_magnitude_mask", L.spl_magnitude_mask(_ptr(W), _TORCH_DTYPE[W.dtype], N, K, int(prune), _ptr(out),
                                                      _ptr(workspace), _stream(stream)))
    return out


def magnitude_mask_noalloc(W: torch.Tensor, prune: int, out: torch.Tensor, stream=None) -> torch.Tensor:
    """magnitude_mask through the entry point that allocates nothing (see
    spl_magnitude_mask_noalloc): the caller passes the uint8 [N][K] output;
    the scratch is the library's own, shared by every call on the device."""
    L = lib()
    if W.dim() != 2:
        raise ValueError(f"W: expected a 2-D tensor, got shape {tuple(W.shape)}")
    N, K = W.shape
    if W.dtype not in (torch.float16, torch.bfloat16):
        raise ValueError(f"W has dtype {W.dtype}, expected float16 or bfloat16")
    _arg(out, "out", shape=(N, K), dtype=torch.uint8, device=False)
    _dev_tensor(W, "W")
    _dev_tensor(out, "out")
    _check("spl_magnitude_mask_noalloc", L.spl_magnitude_mask_noalloc(_ptr(W), _TORCH_DTYPE[W.dtype], N, K,
                                                                      int(prune), _ptr(out), _stream(stream)))
    return out


def transpose16(A: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """out [C][R] = A [R][C]^T for a 16-bit matrix (see spl_transpose16)."""
    L = lib()
    _dev_tensor(A, "A")
    R, C = A.shape
    if out is None:
        out = torch.empty((C, R), dtype=A.dtype, device=A.device)
    _check("spl_transpose16", L.spl_transpose16(_ptr(A), R, C, _ptr(out), _stream(stream)))
    return out


def gather_tiled(W: torch.Tensor, pattern: SparseMatrix, out: torch.Tensor | None = None, stream=None):
    """The entries of dense W [N][K] at the kept positions of `pattern`, in its value order."""
    L = lib()
    _dev_tensor(W, "W")
    if out is None:
        out = torch.empty_like(pattern.values)
    view = pattern.view()
    _check("spl_gather_tiled", L.spl_gather_tiled(_ptr(W), ctypes.byref(view), _ptr(out), _stream(stream)))
    return out


def _wgrad_args(dY, X, Wc: SparseMatrix, out, M: int, name: str = "") -> None:
    _arg(dY, "dY" + name, shape=(M, Wc.rows), dtype=Wc.dtype, device=False)
    _arg(X, "X" + name, shape=(M, Wc.cols), dtype=Wc.dtype, device=False)
    if out is not None:
        _arg(out, "out" + name, dtype=Wc.dtype, min_numel=Wc.nnz, device=False)


def _workspace(L, workspace, need: int, device) -> torch.Tensor:
    if need < 0:
        raise ValueError("the workspace-size function rejected the shape")
    if workspace is None:
        return torch.empty((max(need, 1),), dtype=torch.uint8, device=device)
    _dev_tensor(workspace, "workspace")
    if workspace.numel() * workspace.element_size() < need:
        raise ValueError(f"workspace holds {workspace.numel() * workspace.element_size()} bytes, needs {need}")
    return workspace


def sparse_weight_grad(dY: torch.Tensor, X: torch.Tensor, Wc: SparseMatrix, out: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Kept entries of dY^T X in Wc's value order (see spl_sparse_weight_grad)."""
    L = lib()
    M = _rows_of(X, "X")
    _wgrad_args(dY, X, Wc, out, M)
    _dev_tensor(dY, "dY")
    _dev_tensor(X, "X")
    if out is None:
        out = torch.empty_like(Wc.values)
    _dev_tensor(out, "out")
    workspace = _workspace(L, workspace, L.spl_sparse_weight_grad_workspace_bytes(M, Wc.rows, Wc.cols), X.device)
    view = Wc.view()
    _check("spl_sparse_weight_grad", L.spl_sparse_weight_grad(_ptr(dY), _ptr(X), M, ctypes.byref(view), _ptr(out),
                                                              _ptr(workspace), _stream(stream)))
    return out


def sparse_weight_grad_group(dYs, Xs, mats, outs=None, workspace: torch.Tensor | None = None,
                             stream=None) -> list:
    """Weight gradients of several layers of one batch in one call (see
    spl_sparse_weight_grad_group); outs[i] gets mats[i]'s kept entries."""
    L = lib()
    if not (len(dYs) == len(Xs) == len(mats)) or not 1 <= len(mats) <= MAX_GROUP:
        raise ValueError("dYs, Xs and mats: one entry per task, 1..MAX_GROUP tasks")
    if outs is not None and len(outs) != len(mats):
        raise ValueError("outs: one entry per task")
    M = _rows_of(Xs[0], "X")
    for i, (dY, X, Wc) in enumerate(zip(dYs, Xs, mats)):
        _wgrad_args(dY, X, Wc, outs[i] if outs is not None else None, M, f"[{i}]")
    for i, (dY, X) in enumerate(zip(dYs, Xs)):
        _dev_tensor(dY, f"dY[{i}]")
        _dev_tensor(X, f"X[{i}]")
    if outs is None:
        outs = [torch.empty_like(Wc.values) for Wc in mats]
    for i, o in enumerate(outs):
        _dev_tensor(o, f"out[{i}]")
    need = max(L.spl_sparse_weight_grad_workspace_bytes(M, Wc.rows, Wc.cols) for Wc in mats)
    workspace = _workspace(L, workspace, need, Xs[0].device)
    views = [Wc.view() for Wc in mats]
    tasks = (_WeightGradTask * len(mats))(*[
        _WeightGradTask(dY.data_ptr(), X.data_ptr(), ctypes.pointer(v), o.data_ptr())
        for dY, X, v, o in zip(dYs, Xs, views, outs)])
    _check("spl_sparse_weight_grad_group", L.spl_sparse_weight_grad_group(tasks, len(mats), M, _ptr(workspace),
                                                                          _stream(stream)))
    return outs


def sparse_input_grad(dY: torch.Tensor, Wc: SparseMatrix, out: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """dX [M][K] = dY [M][N] (W . Mask) from W's packed tiles (see spl_sparse_input_grad).  Without a `workspace`, and
    where it is the faster way, through W's decoded transpose: 2 bytes an entry from the caching allocator, for the
    call (a captured graph's pool keeps them)."""
    L = lib()
    M = _rows_of(dY, "dY")
    _arg(dY, "dY", shape=(M, Wc.rows), dtype=Wc.dtype, device=False)
    if out is not None:
        _arg(out, "out", shape=(M, Wc.cols), dtype=Wc.dtype, device=False)
    _dev_tensor(dY, "dY")
    if out is None:
        out = torch.empty((M, Wc.cols), dtype=dY.dtype, device=dY.device)
    _dev_tensor(out, "out")
    view = Wc.view()
    if workspace is None:
        ws = _scratch(L.spl_sparse_input_grad_scratch_bytes(M, ctypes.byref(view)), dY.device, stream)
        if ws is not None:
            _check("spl_sparse_input_grad_scratch",
                   L.spl_sparse_input_grad_scratch(_ptr(dY), M, ctypes.byref(view), _ptr(out), _ptr(ws), ws.numel(),
                                                   _stream(stream)))
            return out
    need = L.spl_sparse_input_grad_workspace_bytes(M, ctypes.byref(view))
    if need < 0:
        raise ValueError("spl_sparse_input_grad_workspace_bytes rejected the shape")
    if need > 0 or workspace is not None:
        workspace = _workspace(L, workspace, need, dY.device)
    _check("spl_sparse_input_grad", L.spl_sparse_input_grad(_ptr(dY), M, ctypes.byref(view), _ptr(out),
                                                            _ptr(workspace), _stream(stream)))
    return out


def sparse_sgd_update(Wc: SparseMatrix, grad_values: torch.Tensor, lr: float, stream=None) -> None:
    """Wc.values <- Wc.values - lr * grad_values in place (see spl_sparse_sgd_update)."""
    L = lib()
    view = Wc.view()
    _check("spl_sparse_sgd_update", L.spl_sparse_sgd_update(ctypes.byref(view), _ptr(grad_values), float(lr),
                                                            _stream(stream)))


def transpose_perm(W: SparseMatrix, Wt: SparseMatrix, stream=None) -> torch.Tensor:
    """perm (int32 [nnz]): value i of Wt is value perm[i] of W (see spl_transpose_perm)."""
    L = lib()
    perm = torch.empty((max(W.nnz, 1),), dtype=torch.int32, device=W.values.device)
    ws = torch.empty((max(L.spl_transpose_perm_workspace_bytes(W.rows, W.cols, W.nnz), 1),), dtype=torch.uint8,
                     device=W.values.device)
    vw, vt = W.view(), Wt.view()
    _check("spl_transpose_perm", L.spl_transpose_perm(ctypes.byref(vw), ctypes.byref(vt), _ptr(perm), _ptr(ws),
                                                      _stream(stream)))
    return perm


def permute_values(src: torch.Tensor, perm: torch.Tensor, nnz: int, out: torch.Tensor, stream=None) -> torch.Tensor:
    """out[i] = src[perm[i]] for i < nnz (see spl_permute_values)."""
    L = lib()
    _check("spl_permute_values", L.spl_permute_values(_ptr(src), _ptr(perm), int(nnz), _ptr(out), _stream(stream)))
    return out


def pack_int4(W8: SparseMatrix, stream=None, check: bool = True) -> SparseMatrix:
    """The 4-bit form of an int8 tile-layout matrix whose codes lie in [-8, 7]
    (see spl_pack_int4): same pattern, values as uint8 bytes of two nibbles.
    With check, the library counts codes outside [-8, 7] and a nonzero count
    raises ValueError (this waits for the stream)."""
    L = lib()
    if W8.dtype != torch.int8 or W8.layout != "tile16":
        raise ValueError("pack_int4 takes an int8 matrix in the tile layout")
    dev = W8.values.device
    v4 = torch.zeros((L.spl_int4_values_bytes(W8.nnz),), dtype=torch.uint8, device=dev)
    bad = torch.zeros((1,), dtype=torch.int32, device=dev) if check else None
    view = W8.view()
    _check("spl_pack_int4", L.spl_pack_int4(ctypes.byref(view), _ptr(v4), _ptr(bad), _stream(stream)))
    if check:
        (stream if stream is not None else torch.cuda.current_stream()).synchronize()
        n = int(bad.item())
        if n:
            raise ValueError(f"pack_int4: {n} codes outside [-8, 7]")
    return SparseMatrix(W8.bitmask, v4, None, W8.tile_offsets, W8.rows, W8.cols, W8.nnz, "tile16")


def sparse_linear_int4(Xq: torch.Tensor, x_scales: torch.Tensor, W4: SparseMatrix, w_scales: torch.Tensor,
                       out: torch.Tensor | None = None, acc_out: torch.Tensor | None = None,
                       stream=None) -> torch.Tensor:
    """fp16 Y from 4-bit sparse weights and int8 activations, M <= 16 (see spl_sparse_linear_int4)."""
    L = lib()
    M = _rows_of(Xq, "Xq")
    _q_args(Xq, x_scales, W4.rows, W4.cols, w_scales, M, device=False)
    if out is None:
        out = torch.empty((M, W4.rows), dtype=torch.float16, device=Xq.device)
    _q_outs(out, acc_out, M, W4.rows)
    _q_args(Xq, x_scales, W4.rows, W4.cols, w_scales, M)
    view = W4.view()
    _check("spl_sparse_linear_int4", L.spl_sparse_linear_int4(_ptr(Xq), _ptr(x_scales), M, ctypes.byref(view),
                                                              _ptr(w_scales), _ptr(out), _ptr(acc_out),
                                                              _stream(stream)))
    return out


def quantize_rows_i8(X: torch.Tensor, out: torch.Tensor | None = None, scales: torch.Tensor | None = None,
                     stream=None):
    """Per-token int8 codes and binary32 scales of fp16/bf16 activations X [M][K]
    (section 3.4; see spl_quantize_rows_i8).  Returns (Xq int8 [M][K], x_scales f32 [M])."""
    L = lib()
    M = _rows_of(X, "X")
    K = X.shape[1]
    if X.dtype not in (torch.float16, torch.bfloat16):
        raise ValueError("X must be fp16 or bf16")
    if out is None:
        out = torch.empty((M, K), dtype=torch.int8, device=X.device)
    if scales is None:
        scales = torch.empty((M,), dtype=torch.float32, device=X.device)
    _arg(out, "out", shape=(M, K), dtype=torch.int8, device=False)
    _arg(scales, "scales", dtype=torch.float32, min_numel=M, device=False)
    for t, nm in ((X, "X"), (out, "out"), (scales, "scales")):
        _dev_tensor(t, nm)
    _check("spl_quantize_rows_i8", L.spl_quantize_rows_i8(_ptr(X), _TORCH_DTYPE[X.dtype], M, K, _ptr(out),
                                                          _ptr(scales), _stream(stream)))
    return out, scales


def sparse_linear_int8(Xq: torch.Tensor, x_scales: torch.Tensor, Wqc: SparseMatrix, w_scales: torch.Tensor,
                       out: torch.Tensor | None = None, acc_out: torch.Tensor | None = None,
                       stream=None) -> torch.Tensor:
    """fp16 Y = dequant(int32 Xq (Wq . Mask)^T) with per-token and per-channel scales.

    From 128 rows on most matrices are multiplied through a decoded copy: 1 byte an entry from the caching allocator,
    for the call (a captured graph's pool keeps them).  Without the memory the tiles are expanded in place."""
    L = lib()
    M = _rows_of(Xq, "Xq")
    _q_args(Xq, x_scales, Wqc.rows, Wqc.cols, w_scales, M, device=False)
    if out is None:
        out = torch.empty((M, Wqc.rows), dtype=torch.float16, device=Xq.device)
    _q_outs(out, acc_out, M, Wqc.rows)
    _q_args(Xq, x_scales, Wqc.rows, Wqc.cols, w_scales, M)
    view = Wqc.view()
    if M > 127 and _lends(M, Wqc.rows, Wqc.cols):
        task = _Int8Task(Xq.data_ptr(), x_scales.data_ptr(), ctypes.pointer(view), w_scales.data_ptr(),
                         out.data_ptr(), None if acc_out is None else acc_out.data_ptr())
        _int8_group(L, (_Int8Task * 1)(task), 1, M, Xq.device, stream)
        return out
    _check("spl_sparse_linear_int8", L.spl_sparse_linear_int8(_ptr(Xq), _ptr(x_scales), M, ctypes.byref(view),
                                                              _ptr(w_scales), _ptr(out), _ptr(acc_out),
                                                              _stream(stream)))
    return out


def _int8_group(L, tasks, n: int, M: int, device, stream) -> None:
    ws = _scratch(L.spl_sparse_linear_int8_group_scratch_bytes(tasks, n, M), device, stream)
    _check("spl_sparse_linear_int8_group_scratch",
           L.spl_sparse_linear_int8_group_scratch(tasks, n, M, _ptr(ws), 0 if ws is None else ws.numel(),
                                                  _stream(stream)))


def sparse_linear_int8_expanded(Xq: torch.Tensor, x_scales: torch.Tensor, Wqc: SparseMatrix, w_scales: torch.Tensor,
                                out: torch.Tensor | None = None, acc_out: torch.Tensor | None = None,
                                workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """sparse_linear_int8 through a decoded copy of the codes in `workspace`
    (see spl_sparse_linear_int8_expanded): for large batches."""
    L = lib()
    M = _rows_of(Xq, "Xq")
    _q_args(Xq, x_scales, Wqc.rows, Wqc.cols, w_scales, M, device=False)
    if out is None:
        out = torch.empty((M, Wqc.rows), dtype=torch.float16, device=Xq.device)
    _q_outs(out, acc_out, M, Wqc.rows)
    _q_args(Xq, x_scales, Wqc.rows, Wqc.cols, w_scales, M)
    view = Wqc.view()
    need = L.spl_sparse_linear_expanded_workspace_bytes(ctypes.byref(view))
    if need < 0:
        raise ValueError("spl_sparse_linear_int8_expanded: the matrix view is invalid")
    if workspace is None:
        workspace = torch.empty((need,), dtype=torch.uint8, device=Xq.device)
    _dev_tensor(workspace, "workspace")
    if workspace.numel() * workspace.element_size() < need:
        raise ValueError(f"workspace holds {workspace.numel() * workspace.element_size()} bytes, needs {need}")
    _check("spl_sparse_linear_int8_expanded",
           L.spl_sparse_linear_int8_expanded(_ptr(Xq), _ptr(x_scales), M, ctypes.byref(view), _ptr(w_scales),
                                             _ptr(out), _ptr(acc_out), _ptr(workspace), _stream(stream)))
    return out


def dense_linear(X: torch.Tensor, W: torch.Tensor, out: torch.Tensor | None = None, algo: str = "auto",
                 stream=None) -> torch.Tensor:
    """Dense comparator: Y = X W^T with the same kernel families."""
    L = lib()
    M = _rows_of(X, "X")
    _rows_of(W, "W")
    N, K = W.shape
    _arg(X, "X", shape=(M, K), dtype=W.dtype, device=False)
    _arg(W, "W", shape=(N, K), device=False)
    if out is None:
        out = torch.empty((M, N), dtype=X.dtype, device=X.device)
    _arg(out, "out", shape=(M, N), dtype=W.dtype)
    _dev_tensor(X, "X")
    _dev_tensor(W, "W")
    _check("spl_dense_linear_ex", L.spl_dense_linear_ex(_ptr(X), M, _ptr(W), _TORCH_DTYPE[W.dtype], N, K,
                                                        _ptr(out), ALGO[algo], _stream(stream)))
    return out


def dense_linear_int8(Xq: torch.Tensor, x_scales: torch.Tensor, Wq: torch.Tensor, w_scales: torch.Tensor,
                      out: torch.Tensor | None = None, acc_out: torch.Tensor | None = None,
                      stream=None) -> torch.Tensor:
    L = lib()
    M = _rows_of(Xq, "Xq")
    _rows_of(Wq, "Wq")
    N, K = Wq.shape
    _arg(Wq, "Wq", shape=(N, K), dtype=torch.int8, device=False)
    _q_args(Xq, x_scales, N, K, w_scales, M, device=False)
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=Xq.device)
    _q_outs(out, acc_out, M, N)
    _dev_tensor(Wq, "Wq")
    _q_args(Xq, x_scales, N, K, w_scales, M)
    _check("spl_dense_linear_int8", L.spl_dense_linear_int8(_ptr(Xq), _ptr(x_scales), M, _ptr(Wq),
                                                            _ptr(w_scales), N, K, _ptr(out), _ptr(acc_out),
                                                            _stream(stream)))
    return out


def sparse_linear_group(Xs, Wcs, outs=None, algo: str = "auto", stream=None):
    """Y_i = X_i (W_i . Mask_i)^T for up to MAX_GROUP independent layers sharing the
    batch size and dtype, in one launch (decode) or one launch per layer (prefill).  Above
    128 rows algo="auto" may take memory for decoded copies of all of them, as in sparse_linear."""
    L = lib()
    n = len(Xs)
    if n != len(Wcs) or not 1 <= n <= MAX_GROUP:
        raise ValueError("need 1..MAX_GROUP (X, W) pairs")
    M = _rows_of(Xs[0], "X")
    if outs is None:
        outs = [torch.empty((M, W.rows), dtype=X.dtype, device=X.device) for X, W in zip(Xs, Wcs)]
    if len(outs) != n:
        raise ValueError("one output per layer")
    views = [W.view() for W in Wcs]
    tasks = (_SparseTask * n)()
    for i, (X, W, Y) in enumerate(zip(Xs, Wcs, outs)):
        if W.dtype != Wcs[0].dtype:
            raise ValueError("every layer of a group shares M and the fp16/bf16 dtype")
        _arg(X, "X", shape=(M, W.cols), dtype=W.dtype, device=False)
        _arg(Y, "out", shape=(M, W.rows), dtype=W.dtype, device=False)
    for i, (X, W, Y) in enumerate(zip(Xs, Wcs, outs)):
        _dev_tensor(X, "X")
        _dev_tensor(Y, "out")
        tasks[i].X = X.data_ptr()
        tasks[i].W = ctypes.pointer(views[i])
        tasks[i].Y = Y.data_ptr()
    if algo == "auto" and M > 128:
        _linear_group(L, tasks, n, M, Xs[0].device, stream)
        return outs
    _check("spl_sparse_linear_group", L.spl_sparse_linear_group(tasks, n, M, ALGO[algo], _stream(stream)))
    return outs


def dense_linear_group(Xs, Ws, outs=None, algo: str = "auto", stream=None):
    """Dense comparator of :func:`sparse_linear_group`."""
    L = lib()
    n = len(Xs)
    if n != len(Ws) or not 1 <= n <= MAX_GROUP:
        raise ValueError("need 1..MAX_GROUP (X, W) pairs")
    M = _rows_of(Xs[0], "X")
    if outs is None:
        outs = [torch.empty((M, W.shape[0]), dtype=X.dtype, device=X.device) for X, W in zip(Xs, Ws)]
    if len(outs) != n:
        raise ValueError("one output per layer")
    tasks = (_DenseTask * n)()
    for i, (X, W, Y) in enumerate(zip(Xs, Ws, outs)):
        _rows_of(W, "W")
        if W.dtype != Xs[0].dtype:
            raise ValueError("every layer of a group shares M and the fp16/bf16 dtype")
        _arg(W, "W", device=False)
        _arg(X, "X", shape=(M, W.shape[1]), dtype=W.dtype, device=False)
        _arg(Y, "out", shape=(M, W.shape[0]), dtype=W.dtype, device=False)
    for i, (X, W, Y) in enumerate(zip(Xs, Ws, outs)):
        for t, nm in ((X, "X"), (W, "W"), (Y, "out")):
            _dev_tensor(t, nm)
        tasks[i].X = X.data_ptr()
        tasks[i].W = W.data_ptr()
        tasks[i].N, tasks[i].K = W.shape
        tasks[i].Y = Y.data_ptr()
    _check("spl_dense_linear_group", L.spl_dense_linear_group(tasks, n, M, _TORCH_DTYPE[Xs[0].dtype], ALGO[algo],
                                                              _stream(stream)))
    return outs


def sparse_linear_int8_group(Xqs, x_scales, Wqcs, w_scales, outs=None, acc_outs=None, stream=None):
    """fp16 Y_i = dequant(int32 Xq_i (Wq_i . Mask_i)^T) for up to MAX_GROUP independent
    int8 layers sharing the batch size, in one launch; from 128 rows on through decoded
    copies of all of them, as in sparse_linear_int8."""
    L = lib()
    n = len(Xqs)
    if not (n == len(x_scales) == len(Wqcs) == len(w_scales)) or not 1 <= n <= MAX_GROUP:
        raise ValueError("need 1..MAX_GROUP (Xq, x_scales, Wq, w_scales) tuples")
    M = _rows_of(Xqs[0], "Xq")
    if outs is None:
        outs = [torch.empty((M, W.rows), dtype=torch.float16, device=X.device) for X, W in zip(Xqs, Wqcs)]
    accs = acc_outs if acc_outs is not None else [None] * n
    if len(outs) != n or len(accs) != n:
        raise ValueError("one output per layer")
    views = [W.view() for W in Wqcs]
    tasks = (_Int8Task * n)()
    for i in range(n):
        _q_args(Xqs[i], x_scales[i], Wqcs[i].rows, Wqcs[i].cols, w_scales[i], M, device=False)
        _q_outs(outs[i], accs[i], M, Wqcs[i].rows, device=False)
    for i in range(n):
        _q_args(Xqs[i], x_scales[i], Wqcs[i].rows, Wqcs[i].cols, w_scales[i], M)
        _q_outs(outs[i], accs[i], M, Wqcs[i].rows)
        tasks[i].Xq, tasks[i].x_scales = Xqs[i].data_ptr(), x_scales[i].data_ptr()
        tasks[i].Wq = ctypes.pointer(views[i])
        tasks[i].w_scales, tasks[i].Y = w_scales[i].data_ptr(), outs[i].data_ptr()
        tasks[i].acc_out = None if accs[i] is None else accs[i].data_ptr()
    if M > 127:
        _int8_group(L, tasks, n, M, Xqs[0].device, stream)
        return outs
    _check("spl_sparse_linear_int8_group", L.spl_sparse_linear_int8_group(tasks, n, M, _stream(stream)))
    return outs


def dense_linear_int8_group(Xqs, x_scales, Wqs, w_scales, outs=None, acc_outs=None, stream=None):
    """Dense comparator of :func:`sparse_linear_int8_group`."""
    L = lib()
    n = len(Xqs)
    if not (n == len(x_scales) == len(Wqs) == len(w_scales)) or not 1 <= n <= MAX_GROUP:
        raise ValueError("need 1..MAX_GROUP (Xq, x_scales, Wq, w_scales) tuples")
    M = _rows_of(Xqs[0], "Xq")
    if outs is None:
        outs = [torch.empty((M, W.shape[0]), dtype=torch.float16, device=X.device) for X, W in zip(Xqs, Wqs)]
    accs = acc_outs if acc_outs is not None else [None] * n
    if len(outs) != n or len(accs) != n:
        raise ValueError("one output per layer")
    tasks = (_DenseInt8Task * n)()
    for i in range(n):
        _rows_of(Wqs[i], "Wq")
        _arg(Wqs[i], "Wq", dtype=torch.int8, device=False)
        _q_args(Xqs[i], x_scales[i], Wqs[i].shape[0], Wqs[i].shape[1], w_scales[i], M, device=False)
        _q_outs(outs[i], accs[i], M, Wqs[i].shape[0], device=False)
    for i in range(n):
        _dev_tensor(Wqs[i], "Wq")
        _q_args(Xqs[i], x_scales[i], Wqs[i].shape[0], Wqs[i].shape[1], w_scales[i], M)
        _q_outs(outs[i], accs[i], M, Wqs[i].shape[0])
        tasks[i].Xq, tasks[i].x_scales, tasks[i].Wq = Xqs[i].data_ptr(), x_scales[i].data_ptr(), Wqs[i].data_ptr()
        tasks[i].w_scales, tasks[i].Y = w_scales[i].data_ptr(), outs[i].data_ptr()
        tasks[i].N, tasks[i].K = Wqs[i].shape
        tasks[i].acc_out = None if accs[i] is None else accs[i].data_ptr()
    _check("spl_dense_linear_int8_group", L.spl_dense_linear_int8_group(tasks, n, M, _stream(stream)))
    return outs


# ------------------------------------------------------------------------------ the attention half of a layer


_HEAD_TYPES = (torch.float16, torch.bfloat16)


class KVCache:
    """Keys and values in 4 bits (format and layout: spl_kv_cache), in pages of `page` tokens.

    data: uint8 [pages, heads, kv_page_bytes(head_dim, page)]; dtype: the type (fp16 or bf16) of what is stored and read
    back.  ``KVCache.empty`` allocates one."""

    __slots__ = ("data", "page", "head_dim", "dtype")

    def __init__(self, data: torch.Tensor, page: int, head_dim: int, dtype: torch.dtype):
        self.data, self.page, self.head_dim, self.dtype = data, page, head_dim, dtype
        self.view()

    @property
    def pages(self) -> int:
        return self.data.shape[0]

    @property
    def heads(self) -> int:
        return self.data.shape[1]

    def view(self) -> _KVCache:
        """The cache as a call takes it: of the attributes as they are now, so that it follows another `data`."""
        data, page, dim = self.data, self.page, self.head_dim
        if self.dtype not in _HEAD_TYPES:
            raise ValueError("a cache holds fp16 or bf16 keys and values")
        size = kv_page_bytes(dim, page)
        shape = data.shape if isinstance(data, torch.Tensor) else ()
        if len(shape) != 3 or shape[2] != size:
            raise ValueError(f"data must be [pages, heads, {size}]")
        if data.dtype != torch.uint8 or not data.is_contiguous():
            _arg(data, "data", dtype=torch.uint8, device=False)
        pages, heads, _ = shape
        return _KVCache(data.data_ptr(), pages, pages * heads * size, page, heads, dim, _TORCH_DTYPE[self.dtype])

    @classmethod
    def empty(cls, pages: int, heads: int, head_dim: int, page: int, dtype: torch.dtype, device="cuda") -> "KVCache":
        return cls(torch.zeros((pages, heads, kv_page_bytes(head_dim, page)), dtype=torch.uint8, device=device), page,
                   head_dim, dtype)


@functools.lru_cache(maxsize=None)
def kv_page_bytes(head_dim: int, page: int) -> int:
    """Bytes of one head's region of a page (see spl_kv_page_bytes)."""
    size = lib().spl_kv_page_bytes(_int32(head_dim, "head_dim"), _int32(page, "page"))
    if size == 0:
        raise ValueError(f"no cache of {head_dim} channels in pages of {page} tokens: 64, 96, 128 or 256 channels, a "
                         "power of two from 16 to 256 tokens")
    return size


@functools.lru_cache(maxsize=1024)
def _attention_workspace(page, cache_heads, head_dim, tokens, heads, requests, width, max_new, max_len) -> int:
    """spl_attention_fp4_workspace_bytes, a function of these sizes (and of the device, whose CUs are the same for all)."""
    view = _KVCache(16, 1, 1 << 62, page, cache_heads, head_dim, F16)
    _int32(max_new, "max_new"), _int32(max_len, "max_len")
    need = lib().spl_attention_fp4_workspace_bytes(view, tokens, heads, requests, width, max_new, max_len)
    if need < 0:
        raise ValueError("spl_attention_fp4_workspace_bytes rejected the arguments")
    return need


@dataclass
class BlockPlan:
    """A step's rows and slots (see spl_block_tables)."""

    row_start: torch.Tensor            # int32 [requests + 1]
    lens: torch.Tensor                 # int32 [requests]
    positions: torch.Tensor            # int32 [tokens]
    slots: torch.Tensor                # int32 [tokens]
    free_head: torch.Tensor            # int32 [1]: free_head of the next step
    missing: torch.Tensor              # int32 [1]: new tokens without a row or a slot


def _on(stream) -> int:
    """_stream for the calls of this section, whose smallest take a few microseconds: the handle of the current
    stream without the stream object."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _int32(n: int, name: str) -> int:
    """A number that the library takes in 32 bits, of which ctypes would pass the low ones of a larger one."""
    if not -1 << 31 <= n < 1 << 31:
        raise ValueError(f"{name} is {n}, past 32 bits")
    return n


def _on_device(names: str, *tensors) -> None:
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError(f"{names}: device tensors only")


def _ints(t, name: str, n: int) -> int:
    """The address of an int32 vector of n entries."""
    if not isinstance(t, torch.Tensor) or t.shape != (n,) or t.dtype != torch.int32 or not t.is_contiguous():
        _arg(t, name, shape=(n,), dtype=torch.int32, device=False)
    return t.data_ptr()


def _table(table) -> tuple[int, int]:
    """(requests, width) of a page table."""
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise ValueError("table must be [requests, width]")
    if table.dtype != torch.int32 or not table.is_contiguous():
        _arg(table, "table", dtype=torch.int32, device=False)
    return table.shape


def _workspace_on(need: int, device, stream) -> torch.Tensor:
    """As _scratch, for a call that cannot do without."""
    ws = _scratch(need, device, stream)
    if ws is None:
        raise torch.OutOfMemoryError(f"no {need} bytes of workspace")
    return ws


def _result(shape, dtype, device, stream) -> torch.Tensor:
    """A result to be written on `stream` (None: the current one): from that stream's own pool, as a block of the current
    one's may still be in use there, and not reused before the current stream is done with it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    here = torch.cuda.current_stream(device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    if stream != here:
        t.record_stream(here)
    return t


def block_tables(cached: torch.Tensor, new: torch.Tensor, table: torch.Tensor, free_pages: torch.Tensor,
                 free_head: torch.Tensor, page: int, tokens: int, stream=None) -> BlockPlan:
    """Pages from the free list for each request's `new` tokens after its `cached` ones, written into `table`
    [requests, width], and the row, position and slot of every new token (see spl_block_tables).  `tokens` is the rows
    of the step's tensors; nothing waits for the GPU."""
    R, width = _table(table)
    args = (_ints(cached, "cached", R), _ints(new, "new", R))
    if not isinstance(free_pages, torch.Tensor) or free_pages.dim() != 1:
        raise ValueError("free_pages must be 1-D")
    free = _ints(free_pages, "free_pages", free_pages.shape[0])
    head = _ints(free_head, "free_head", 1)
    if tokens < 0:
        raise ValueError("tokens must not be negative")
    _int32(page, "page")
    _on_device("cached, new, table, free_pages, free_head", cached, new, table, free_pages, free_head)
    # one allocation for all results
    buf = _result((2 * R + 2 * tokens + 3,), torch.int32, table.device, stream)
    p = buf.data_ptr()
    _check("spl_block_tables",
           lib().spl_block_tables(*args, R, tokens, page, table.data_ptr(), width, free, free_pages.shape[0], head, p,
                                  p + 4 * (R + 1), p + 4 * (2 * R + 1), p + 4 * (2 * R + 1 + tokens),
                                  p + 4 * (2 * R + 1 + 2 * tokens), _on(stream)))
    return BlockPlan(*buf.split_with_sizes((R + 1, R, tokens, tokens, 1, 1)))


def _heads(x: torch.Tensor, name: str, tokens: int | None = None, dim: int | None = None, dtype=None) -> _Heads:
    """A [tokens, heads, dim] view with contiguous channels and other strides that are multiples of 8."""
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        raise ValueError(f"{name} must be [tokens, heads, dim]")
    T, H, D = x.shape
    st, sh, sd = x.stride()
    at = x.data_ptr()
    if (T == tokens or tokens is None) and (D == dim or dim is None) and (
            x.dtype == dtype or (dtype is None and x.dtype in _HEAD_TYPES)):
        if sd == 1 and not (st | sh) & 7 and not at & 15:
            return _Heads(at, st, sh, H)
        st, sh = 0 if T <= 1 else st, 0 if H == 1 else sh
        if (sd == 1 or D == 1) and not (st | sh) & 7 and not at & 15:
            return _Heads(at, st, sh, H)
        raise ValueError(f"{name}: channels must be contiguous, the other strides multiples of 8, the start 16-byte "
                         "aligned")
    raise ValueError(f"{name} is {x.dtype} {tuple(x.shape)}, expected {dtype or 'fp16 or bf16'} [{tokens}, heads, {dim}]")


def _weight(w, name: str, dim: int, dtype) -> int | None:
    if w is None:
        return None
    if not isinstance(w, torch.Tensor) or w.shape != (dim,) or w.dtype != dtype or not w.is_contiguous():
        _arg(w, name, shape=(dim,), dtype=dtype, device=False)
    return w.data_ptr()


def _turn_args(tokens: int, positions, rope):
    """The rotation's arguments: (positions, angles, rows of angles, rotated channels)."""
    if rope is None:
        return None, None, 0, 0
    if not isinstance(rope, torch.Tensor) or rope.dim() != 3 or rope.shape[2] != 2:
        raise ValueError("rope must be float32 [positions, rot / 2, 2] (cosine, sine)")
    if rope.dtype != torch.float32 or not rope.is_contiguous():
        _arg(rope, "rope", dtype=torch.float32, device=False)
    rows, half, _ = rope.shape
    return _ints(positions, "positions", tokens), rope.data_ptr(), rows, 2 * half


def _heads_out(out, like: torch.Tensor, name: str, stream) -> torch.Tensor:
    if out is None:
        if stream is None:
            return torch.empty_like(like, memory_format=torch.contiguous_format)
        return _result(like.shape, like.dtype, like.device, stream)
    return _arg(out, name, shape=like.shape, dtype=like.dtype)


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor | None, rope: torch.Tensor | None,
                 q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, eps: float = 1e-6,
                 interleaved: bool = False, q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None,
                 stream=None):
    """(q_out, k_out): the RMS norm of every head of q [tokens, heads, dim] and k, with the weights given, then the
    rotation by rope[position] (see spl_qk_norm_rope).  rope: float32 [positions, rot / 2, 2], or None for none.  q and
    k may be slices of one fused product."""
    hq = _heads(q, "q")
    T, _, D = q.shape
    hk = _heads(k, "k", T, D, q.dtype)
    wq, wk = _weight(q_weight, "q_weight", D, q.dtype), _weight(k_weight, "k_weight", D, q.dtype)
    at, angles, rows, rot = _turn_args(T, positions, rope)
    _on_device("q, k, weights, positions, rope", q, k, q_weight, k_weight, positions, rope)
    q_out, k_out = _heads_out(q_out, q, "q_out", stream), _heads_out(k_out, k, "k_out", stream)
    _check("spl_qk_norm_rope",
           lib().spl_qk_norm_rope(hq, hk, T, D, _TORCH_DTYPE[q.dtype], wq, wk, eps, at, angles, rows, rot, interleaved,
                                  q_out.data_ptr(), k_out.data_ptr(), _on(stream)))
    return q_out, k_out


def qk_norm_rope_grad(dq: torch.Tensor, dk: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                      positions: torch.Tensor | None, rope: torch.Tensor | None,
                      q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, eps: float = 1e-6,
                      interleaved: bool = False, dq_out: torch.Tensor | None = None,
                      dk_out: torch.Tensor | None = None, stream=None):
    """(dq, dk, dq_weight, dk_weight) of the inputs of qk_norm_rope from the gradients dq, dk of its results; the
    weights' are float32, None without a weight (see spl_qk_norm_rope_grad)."""
    L = lib()
    hq = _heads(q, "q")
    T, H, D = q.shape
    hk = _heads(k, "k", T, D, q.dtype)
    hdq, hdk = _heads(dq, "dq", T, D, q.dtype), _heads(dk, "dk", T, D, q.dtype)
    if hdq.heads != H or hdk.heads != hk.heads:
        raise ValueError("a gradient has its input's heads")
    wq, wk = _weight(q_weight, "q_weight", D, q.dtype), _weight(k_weight, "k_weight", D, q.dtype)
    at, angles, rows, rot = _turn_args(T, positions, rope)
    _on_device("q, k, dq, dk, weights, positions, rope", q, k, dq, dk, q_weight, k_weight, positions, rope)
    need = L.spl_qk_norm_rope_grad_workspace_bytes(T, H, hk.heads, D)
    if need < 0:
        raise ValueError("the workspace-size function rejected the shape")
    dq_out, dk_out = _heads_out(dq_out, q, "dq_out", stream), _heads_out(dk_out, k, "dk_out", stream)
    dwq, dwk = (None if w is None else _result((D,), torch.float32, q.device, stream) for w in (q_weight, k_weight))
    ws = _workspace_on(need, q.device, stream) if need else None
    _check("spl_qk_norm_rope_grad",
           L.spl_qk_norm_rope_grad(hdq, hdk, hq, hk, T, D, _TORCH_DTYPE[q.dtype], wq, wk, eps, at, angles, rows, rot,
                                   interleaved, dq_out.data_ptr(), dk_out.data_ptr(), _ptr(dwq), _ptr(dwk), _ptr(ws),
                                   _on(stream)))
    return dq_out, dk_out, dwq, dwk


def qk_norm_rope_append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor | None,
                        rope: torch.Tensor | None, slots: torch.Tensor, cache: KVCache,
                        q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None,
                        eps: float = 1e-6, interleaved: bool = False, q_out: torch.Tensor | None = None,
                        k_out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """q_out of qk_norm_rope; its keys and the values v go to `slots` of the cache in the same launch (and the keys to
    k_out, where given; see spl_qk_norm_rope_append)."""
    view = cache.view()
    D, dtype, heads = cache.head_dim, cache.dtype, view.heads
    hq = _heads(q, "q", None, D, dtype)
    T = q.shape[0]
    hk, hv = _heads(k, "k", T, D, dtype), _heads(v, "v", T, D, dtype)
    if hk.heads != heads or hv.heads != heads:
        raise ValueError(f"k and v have {hk.heads} and {hv.heads} heads, the cache has {heads}")
    to = _ints(slots, "slots", T)
    wq, wk = _weight(q_weight, "q_weight", D, dtype), _weight(k_weight, "k_weight", D, dtype)
    at, angles, rows, rot = _turn_args(T, positions, rope)
    _on_device("q, k, v, slots, the cache, weights, positions, rope", q, k, v, slots, cache.data, q_weight, k_weight,
               positions, rope)
    q_out = _heads_out(q_out, q, "q_out", stream)
    if k_out is not None:
        k_out = _heads_out(k_out, k, "k_out", stream)
    _check("spl_qk_norm_rope_append",
           lib().spl_qk_norm_rope_append(hq, hk, hv, T, wq, wk, eps, at, angles, rows, rot, interleaved, to,
                                         view, q_out.data_ptr(), _ptr(k_out), _on(stream)))
    return q_out


def cache_read(cache: KVCache, slots: torch.Tensor, stream=None):
    """(keys, values) [tokens, heads, head_dim] that the cache holds at `slots` (see spl_cache_read)."""
    if not isinstance(slots, torch.Tensor) or slots.dim() != 1:
        raise ValueError("slots must be 1-D")
    T = slots.shape[0]
    at, view = _ints(slots, "slots", T), cache.view()
    _on_device("slots, the cache", slots, cache.data)
    k = _result((T, view.heads, cache.head_dim), cache.dtype, slots.device, stream)
    v = _heads_out(None, k, "v", stream)
    _check("spl_cache_read", lib().spl_cache_read(view, at, T, k.data_ptr(), v.data_ptr(), _on(stream)))
    return k, v


def attention_fp4(q: torch.Tensor, cache: KVCache, table: torch.Tensor, lens: torch.Tensor, row_start: torch.Tensor,
                  scale: float | None = None, window: int = 0, max_new: int = 0, max_len: int = 0,
                  out: torch.Tensor | None = None, lse: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Causal attention of the rows q [tokens, heads, head_dim] over the 4-bit cache, whose pages `table` [requests,
    width] lists (see spl_attention_fp4).  `row_start` [requests + 1] and `lens` [requests] are those of block_tables;
    scale is 1 / sqrt(head_dim) unless given.  max_new (the most rows of a request) and max_len (about the most tokens)
    let the call choose its launch without asking the GPU.  lse: float32 [tokens, heads], written if given."""
    L, D, view = lib(), cache.head_dim, cache.view()
    hq = _heads(q, "q", None, D, cache.dtype)
    T, H, _ = q.shape
    if H % view.heads:
        raise ValueError(f"q has {H} heads, not a multiple of the cache's {view.heads}")
    R, width = _table(table)
    _int32(window, "window")
    ends, starts = _ints(lens, "lens", R), _ints(row_start, "row_start", R + 1)
    if lse is not None:
        _arg(lse, "lse", shape=(T, H), dtype=torch.float32, device=False)
    _on_device("q, the cache, table, lens, row_start, lse", q, cache.data, table, lens, row_start, lse)
    out = _heads_out(out, q, "out", stream)
    need = _attention_workspace(cache.page, view.heads, D, T, H, R, width, max_new, max_len)
    ws = _workspace_on(need, q.device, stream) if need else None
    _check("spl_attention_fp4",
           L.spl_attention_fp4(hq, T, view, table.data_ptr(), R, width, ends, starts, max_new, max_len,
                               D ** -0.5 if scale is None else scale, window, out.data_ptr(), _ptr(lse), _ptr(ws),
                               _on(stream)))
    return out


# ------------------------------------------------------------------------------ linears in 8-bit floats


_FLOAT_TYPES = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}
_CODE_TYPES = (torch.uint8, torch.float8_e4m3fn)


def _here(names: str, stream, *tensors) -> torch.device:
    """The device of the call, which is the current one: every tensor is on it, and so is the stream."""
    first = tensors[0]
    at = torch._C._cuda_getDevice() if first.is_cuda else -1
    for t in tensors:
        if t is not None and (t.get_device() != at or at < 0):
            raise ValueError(f"{names}: tensors of the current device only")
    if stream is not None and isinstance(stream, torch.cuda.Stream) and stream.device_index != at:
        raise ValueError("the stream must be of the current device")
    return first.device


class Fp8Matrix:
    """A matrix [rows, cols] (or `count` of them) in 8-bit floats with a power-of-two scale for each block of 128 columns
    of one row (block 1) or of 128 rows (block 128); format: spl_fp8_matrix.

    codes: uint8 or float8_e4m3fn [rows, pitch] or [count, rows, pitch], pitch = cols rounded up to 128; scales: uint8
    [..., ceil(rows / block), spitch], spitch = pitch / 128 rounded up to 4.  ``quantize_fp8`` makes one, ``Fp8Matrix.of``
    takes codes and scales that come from elsewhere."""

    __slots__ = ("codes", "scales", "cols", "block")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, cols: int, block: int = 1):
        self.codes, self.scales, self.cols, self.block = codes, scales, cols, block
        self.view()

    @property
    def rows(self) -> int:
        return self.codes.shape[-2]

    @property
    def count(self) -> int:
        return 1 if self.codes.dim() == 2 else self.codes.shape[0]

    def block_scales(self) -> torch.Tensor:
        """The scale bytes (e + 127) without the padding of their rows: [..., ceil(rows / block), ceil(cols / 128)]."""
        scales, blocks = self.scales, (self.cols + 127) // 128
        return scales if scales.shape[-1] == blocks else scales[..., :blocks]

    def view(self) -> _Fp8:
        """The matrix as a call takes it: of the attributes as they are now."""
        codes, scales, cols, block = self.codes, self.scales, self.cols, self.block
        shape = codes.shape
        if block not in (1, 128):
            raise ValueError("block must be 1 or 128")
        pitch = (cols + 127) // 128 * 128
        if cols < 1 or len(shape) not in (2, 3) or shape[-1] != pitch or codes.dtype not in _CODE_TYPES or \
                not codes.is_contiguous():
            raise ValueError(f"codes must be contiguous 8-bit floats [rows, {pitch}] or [count, rows, {pitch}]")
        want = (*shape[:-2], (shape[-2] + block - 1) // block, (pitch // 128 + 3) // 4 * 4)
        if scales.shape != want or scales.dtype != torch.uint8 or not scales.is_contiguous():
            raise ValueError(f"scales must be contiguous uint8 {list(want)}")
        return _Fp8(codes.data_ptr(), scales.data_ptr(), shape[-2], cols, 1 if len(shape) == 2 else shape[0],
                    codes.numel(), scales.numel(), block)

    @classmethod
    def empty(cls, rows: int, cols: int, block: int = 1, count: int | None = None, device="cuda", stream=None):
        return cls._made(rows, cols, block, count, device, stream)[0]

    @classmethod
    def _made(cls, rows: int, cols: int, block: int, count: int | None, device, stream):
        """A matrix to be written, and its view (right as made: view()'s checks are 1 us of a short call's 10.6)."""
        n = 1 if count is None else count
        scales_bytes = _fp8_workspace("spl_fp8_scales_bytes", rows, cols, n, block)   # refuses the sizes
        blocks = (cols + 127) // 128
        codes, scales = (rows, 128 * blocks), ((rows + block - 1) // block, (blocks + 3) // 4 * 4)
        if count is not None:
            codes, scales = (count, *codes), (count, *scales)
        m = object.__new__(cls)
        m.codes, m.scales = _result(codes, torch.uint8, device, stream), _result(scales, torch.uint8, device, stream)
        m.cols, m.block = cols, block
        return m, _Fp8(m.codes.data_ptr(), m.scales.data_ptr(), rows, cols, n, n * rows * 128 * blocks, scales_bytes, block)

    @classmethod
    def of(cls, codes: torch.Tensor, scales: torch.Tensor, cols: int, block: int) -> "Fp8Matrix":
        """From codes [..., rows, cols or more] and scale bytes [..., ceil(rows / block), ceil(cols / 128)], copied where
        they are not laid out as here."""
        if codes.dtype not in _CODE_TYPES or scales.dtype != torch.uint8 or block not in (1, 128) or cols < 1:
            raise ValueError("codes of 8-bit floats, scales of uint8, block 1 or 128, at least one column")
        blocks, rows = (cols + 127) // 128, codes.shape[-2]
        if codes.shape[-1] < cols or scales.shape != (*codes.shape[:-2], (rows + block - 1) // block, blocks):
            raise ValueError(f"codes {list(codes.shape)} and scales {list(scales.shape)} are not of {cols} columns")
        codes = codes.view(torch.uint8)
        if codes.shape[-1] != cols or cols != 128 * blocks or not codes.is_contiguous():   # zeros behind the columns
            wide = torch.zeros((*codes.shape[:-1], 128 * blocks), dtype=torch.uint8, device=codes.device)
            wide[..., :cols] = codes[..., :cols]
            codes = wide
        spitch = (blocks + 3) // 4 * 4
        if spitch != blocks or not scales.is_contiguous():
            wide = torch.zeros((*scales.shape[:-1], spitch), dtype=torch.uint8, device=scales.device)
            wide[..., :blocks] = scales
            scales = wide
        return cls(codes, scales, cols, block)


def _dense(X, name: str):
    """(rows, cols, row stride, count) of a float matrix, or of several one after another."""
    if not isinstance(X, torch.Tensor) or X.dim() not in (2, 3) or X.dtype not in _FLOAT_TYPES:
        raise ValueError(f"{name} must be fp16, bf16 or fp32 [rows, cols] or [count, rows, cols]")
    rows, cols = X.shape[-2:]
    stride = X.stride(-2) if rows > 1 else max(cols, 1)
    count = 1 if X.dim() == 2 else X.shape[0]
    if cols < 1 or (cols > 1 and X.stride(-1) != 1) or stride < cols or (
            X.dim() == 3 and count > 1 and X.stride(0) != rows * stride):
        raise ValueError(f"{name}: columns must be contiguous, matrices one after another")
    return rows, cols, stride, count


def _starts(starts, experts: int | None = None) -> int:
    """The groups of starts [groups + 1]."""
    if not isinstance(starts, torch.Tensor) or starts.dim() != 1 or starts.shape[0] < 2:
        raise ValueError("starts must be int32 [experts + 1]")
    _ints(starts, "starts", starts.shape[0] if experts is None else experts + 1)
    return starts.shape[0] - 1


def _quantize(X, block, rows_too, cols_too, starts, stream):
    rows, cols, stride, count = _dense(X, "X")
    groups = 0 if starts is None else _starts(starts)
    if rows < 1:
        raise ValueError("X has no rows")
    if block not in (1, 128):
        raise ValueError("block must be 1 or 128")
    if starts is not None and (X.dim() != 2 or block != 1):
        raise ValueError("starts is for one matrix with blocks of one row")
    device = _here("X, starts", stream, X, starts)
    L, lead = lib(), None if X.dim() == 2 else count
    out, view = Fp8Matrix._made(rows, cols, block, lead, device, stream) if rows_too else (None, None)
    out_t = view_t = None
    if cols_too:
        wide = rows if starts is None else L.spl_fp8_grouped_cols(rows, groups)
        if wide < 0:
            raise ValueError("too many rows or groups")
        out_t, view_t = Fp8Matrix._made(cols, wide, block, lead, device, stream)
    _check("spl_quantize_fp8",
           L.spl_quantize_fp8(X.data_ptr(), _FLOAT_TYPES[X.dtype], rows, cols, stride, count,
                              None if starts is None else starts.data_ptr(), groups,
                              view, view_t, _on(stream)))
    return out, out_t


def quantize_fp8(X: torch.Tensor, block: int = 1, transposed: bool = False, starts: torch.Tensor | None = None,
                 stream=None) -> Fp8Matrix:
    """X [rows, cols] (or [count, rows, cols]; fp16, bf16 or fp32) in 8-bit floats, or its transpose (see
    spl_quantize_fp8).  block 1: a scale for 128 columns of a row, block 128: for 128 x 128 entries.  starts (int32
    [groups + 1], transposed): each group's rows begin at a multiple of 128 of the result's columns."""
    if starts is not None and not transposed:
        raise ValueError("starts is for the transposed form")
    return _quantize(X, block, not transposed, transposed, starts, stream)[transposed]


def quantize_fp8_both(X: torch.Tensor, block: int = 1, starts: torch.Tensor | None = None, stream=None):
    """(quantize_fp8(X), quantize_fp8(X, transposed=True)) in one pass over X.  With starts, rows of no group are in
    neither."""
    return _quantize(X, block, True, True, starts, stream)


def dequantize_fp8(A: Fp8Matrix, dtype: torch.dtype = torch.float32, stream=None) -> torch.Tensor:
    """What A stands for, [rows, cols] or [count, rows, cols] of dtype (see spl_dequantize_fp8)."""
    if dtype not in _FLOAT_TYPES:
        raise ValueError("dtype must be fp16, bf16 or fp32")
    view, device = A.view(), _here("A", stream, A.codes, A.scales)
    out = _result((*A.codes.shape[:-1], A.cols), dtype, device, stream)
    _check("spl_dequantize_fp8", lib().spl_dequantize_fp8(view, _FLOAT_TYPES[dtype], out.data_ptr(), _on(stream)))
    return out


@functools.lru_cache(maxsize=1024)
def _fp8_workspace(name: str, *sizes) -> int:
    """A workspace-size function of sizes alone."""
    need = getattr(lib(), name)(*sizes)
    if need < 0:
        raise ValueError(f"{name} rejected the sizes {sizes}")
    return need


def _fp8_out(out, M: int, N: int, dtype, X, device, stream) -> torch.Tensor:
    """The result of a product, in dtype, else `out`'s, else X's type (bf16 where X holds codes)."""
    if out is not None:
        if dtype is not None and out.dtype != dtype:
            raise ValueError(f"out has dtype {out.dtype}, expected {dtype}")
        if out.dtype not in _FLOAT_TYPES:
            raise ValueError("out must be fp16, bf16 or fp32")
        _arg(out, "out", shape=(M, N), device=False)
        _here("out", None, out)
        return out
    dtype = dtype or (torch.bfloat16 if isinstance(X, Fp8Matrix) else X.dtype)
    if dtype not in _FLOAT_TYPES:
        raise ValueError("dtype must be fp16, bf16 or fp32")
    if stream is None:
        return torch.empty((M, N), dtype=dtype, device=device)
    return _result((M, N), dtype, device, stream)


def _fp8_rows(X, cols: int, name: str = "X"):
    """(rows, row stride) of the activations of a product: 16-bit floats."""
    if not isinstance(X, torch.Tensor) or X.dim() != 2 or X.dtype not in _HEAD_TYPES or X.shape[1] != cols:
        raise ValueError(f"{name} must be an Fp8Matrix or fp16 / bf16 [rows, {cols}]")
    rows = X.shape[0]
    stride, step = X.stride()
    if rows <= 1:
        stride = cols
    if (step != 1 and cols > 1) or stride < cols:
        raise ValueError(f"{name}: columns must be contiguous")
    return rows, stride


def linear_fp8(X, W: Fp8Matrix, dtype: torch.dtype | None = None, out: torch.Tensor | None = None,
               stream=None) -> torch.Tensor:
    """Y [M, N] = X W^T in 8-bit floats (see spl_linear_fp8).  X: an Fp8Matrix, or fp16 / bf16 activations [M, K] that are
    quantized on the way, a scale for 128 columns of a row.  Y: dtype, else that of out, else X's (bf16 for codes).  Sums
    of 16-bit results are off by up to 2^-9 of each block's largest product, those of fp32 results by fp32's roundings only:
    where large products cancel and what is left counts, ask for torch.float32."""
    L, w = lib(), W.view()
    if w.count != 1:
        raise ValueError("W is several matrices: linear_fp8_grouped")
    N, K = w.rows, w.cols
    if isinstance(X, Fp8Matrix):
        x = X.view()
        if x.count != 1 or x.cols != K:
            raise ValueError(f"X has {x.cols} columns, W {K}")
        device = _here("X, W", stream, X.codes, X.scales, W.codes, W.scales)
        out = _fp8_out(out, x.rows, N, dtype, X, device, stream)
        need = _fp8_workspace("spl_linear_fp8_workspace_bytes", x.rows, N, K)
        ws = _workspace_on(need, device, stream) if need else None
        _check("spl_linear_fp8",
               L.spl_linear_fp8(x, w, _FLOAT_TYPES[out.dtype], out.data_ptr(), _ptr(ws), _on(stream)))
        return out
    M, stride = _fp8_rows(X, K)
    device = _here("X, W", stream, X, W.codes, W.scales)
    out = _fp8_out(out, M, N, dtype, X, device, stream)
    need = _fp8_workspace("spl_linear_fp8_rows_workspace_bytes", M, N, K)
    ws = _workspace_on(need, device, stream) if need else None
    _check("spl_linear_fp8_rows",
           L.spl_linear_fp8_rows(X.data_ptr(), _TORCH_DTYPE[X.dtype], M, stride, w, _FLOAT_TYPES[out.dtype],
                                 out.data_ptr(), _ptr(ws), _on(stream)))
    return out


def _gradients(dY, X, Wt: Fp8Matrix, starts, grad_dtype, stream):
    for t, name in ((dY, "dY"), (X, "X")):
        if not isinstance(t, torch.Tensor) or t.dim() != 2 or t.dtype not in _HEAD_TYPES:
            raise ValueError(f"{name} must be fp16 or bf16 [rows, columns]")
    view = Wt.view()
    K, N, E = view.rows, view.cols, view.count
    M = X.shape[0]
    if dY.shape[0] != M or X.dtype != dY.dtype or X.shape[1] != K or dY.shape[1] != N:
        raise ValueError(f"dY {list(dY.shape)}, X {list(X.shape)} and the transposed weight [{K}, {N}] do not belong "
                         "together")
    if grad_dtype not in _FLOAT_TYPES:
        raise ValueError("grad_dtype must be fp16, bf16 or fp32")
    if starts is None and E != 1:
        raise ValueError("Wt is several matrices: linear_fp8_grouped_grad")
    (_, dys), (_, xs) = _fp8_rows(dY, N, "dY"), _fp8_rows(X, K)
    device = _here("dY, X, Wt, starts", stream, dY, X, Wt.codes, Wt.scales, starts)
    dX = _result((M, K), dY.dtype, device, stream)
    dW = _result((N, K) if starts is None else (E, N, K), grad_dtype, device, stream)
    need = _fp8_workspace("spl_linear_fp8_grad_workspace_bytes", M, N, K, 0 if starts is None else E)
    ws = _workspace_on(need, device, stream) if need else None
    _check("spl_linear_fp8_grad",
           lib().spl_linear_fp8_grad(dY.data_ptr(), dys, X.data_ptr(), xs, _TORCH_DTYPE[X.dtype], M, view,
                                     None if starts is None else starts.data_ptr(), _FLOAT_TYPES[grad_dtype],
                                     dX.data_ptr(), dW.data_ptr(), _ptr(ws), _on(stream)))
    return dX, dW


def linear_fp8_grad(dY: torch.Tensor, X: torch.Tensor, Wt: Fp8Matrix, grad_dtype: torch.dtype = torch.float32,
                    stream=None):
    """(dX, dW) of Y = X W^T from dY [M, N] and X [M, K] (fp16 or bf16): dX = dY W in their type, dW = dY^T X in
    grad_dtype, both sums in 8-bit floats (see spl_linear_fp8_grad).  Wt: the transposed weight [K, N], as
    quantize_fp8_both makes it.  A dW of 16 bits is summed at twice the rate of an fp32 one."""
    return _gradients(dY, X, Wt, None, grad_dtype, stream)


def linear_fp8_grouped(X, W: Fp8Matrix, starts: torch.Tensor, dtype: torch.dtype | None = None,
                       out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Y [M, N]: row m of X, starts[e] <= m < starts[e + 1], times matrix e of W (see spl_linear_fp8_grouped).  starts:
    int32 [experts + 1] on the device.  X and Y as in linear_fp8.  Rows of no expert are not written: pass `out` where
    there are some."""
    L, w = lib(), W.view()
    N, K = w.rows, w.cols
    _starts(starts, w.count)
    at = starts.data_ptr()
    if isinstance(X, Fp8Matrix):
        x = X.view()
        if x.count != 1 or x.cols != K:
            raise ValueError(f"X has {x.cols} columns, W {K}")
        device = _here("X, W, starts", stream, X.codes, X.scales, W.codes, W.scales, starts)
        out = _fp8_out(out, x.rows, N, dtype, X, device, stream)
        _check("spl_linear_fp8_grouped",
               L.spl_linear_fp8_grouped(x, w, at, _FLOAT_TYPES[out.dtype], out.data_ptr(), _on(stream)))
        return out
    M, stride = _fp8_rows(X, K)
    device = _here("X, W, starts", stream, X, W.codes, W.scales, starts)
    out = _fp8_out(out, M, N, dtype, X, device, stream)
    need = _fp8_workspace("spl_linear_fp8_grouped_rows_workspace_bytes", M, N, K, w.count)
    ws = _workspace_on(need, device, stream) if need else None
    _check("spl_linear_fp8_grouped_rows",
           L.spl_linear_fp8_grouped_rows(X.data_ptr(), _TORCH_DTYPE[X.dtype], M, stride, w, at,
                                         _FLOAT_TYPES[out.dtype], out.data_ptr(), _ptr(ws), _on(stream)))
    return out


def linear_fp8_grouped_grad(dY: torch.Tensor, X: torch.Tensor, Wt: Fp8Matrix, starts: torch.Tensor,
                            grad_dtype: torch.dtype = torch.float32, stream=None):
    """(dX, dW) of linear_fp8_grouped as linear_fp8_grad's, Wt the transposed weights [experts, K, N], dW [experts, N, K]
    with zeros for an expert without rows.  Rows of no expert are zeros in dX."""
    _starts(starts, Wt.count)
    return _gradients(dY, X, Wt, starts, grad_dtype, stream)


def linear_fp8_grouped_weight_grad(dYt: Fp8Matrix, Xt: Fp8Matrix, starts: torch.Tensor, tokens: int,
                                   dtype: torch.dtype = torch.float32, stream=None) -> torch.Tensor:
    """dW [experts, N, K] from the transposes of dY and X, `tokens` rows each, that quantize_fp8 made with the same starts
    (see spl_linear_fp8_grouped_weight_grad): for a program that quantizes X once for both passes."""
    a, b, E = dYt.view(), Xt.view(), _starts(starts)
    if dtype not in _FLOAT_TYPES:
        raise ValueError("dtype must be fp16, bf16 or fp32")
    device = _here("dYt, Xt, starts", stream, dYt.codes, dYt.scales, Xt.codes, Xt.scales, starts)
    dW = _result((E, a.rows, b.rows), dtype, device, stream)
    _check("spl_linear_fp8_grouped_weight_grad",
           lib().spl_linear_fp8_grouped_weight_grad(a, b, starts.data_ptr(), E, tokens, _FLOAT_TYPES[dtype],
                                                    dW.data_ptr(), _on(stream)))
    return dW


# ------------------------------------------------------------------------------ the optimizer step


class Fp8Vector:
    """An optimizer state of n elements in 8 bits: codes uint8 [128 * ceil(n / 128)] and a scale byte for every 128."""

    __slots__ = ("codes", "scales", "n")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, n: int):
        blocks = (n + 127) // 128
        _arg(codes, "codes", shape=(128 * blocks,), dtype=torch.uint8, device=False)
        _arg(scales, "scales", shape=(blocks,), dtype=torch.uint8, device=False)
        self.codes, self.scales, self.n = codes, scales, n

    @classmethod
    def zeros(cls, n: int, device="cuda") -> "Fp8Vector":
        blocks = (n + 127) // 128
        return cls(torch.zeros((128 * blocks,), dtype=torch.uint8, device=device),
                   torch.zeros((blocks,), dtype=torch.uint8, device=device), n)


class AdamwPlan:
    """The tensors of adamw_step, made by adamw_plan: it keeps them, and the list of their addresses on the device."""

    __slots__ = ("tensors", "table", "chunks", "types", "device")

    def __init__(self, tensors, table, chunks, types, device):
        self.tensors, self.table, self.chunks, self.types, self.device = tensors, table, chunks, types, device


def _one_type(tensors, name: str, allowed) -> int:
    kinds = {t.dtype if isinstance(t, torch.Tensor) else type(t) for t in tensors}
    if len(kinds) > 1 or not kinds <= set(allowed):
        raise ValueError(f"{name}: tensors of one type of {', '.join(str(k) for k in allowed)}, got {kinds or 'none'}")
    return allowed[kinds.pop()] if kinds else F32


def adamw_plan(params, grads, exp_avg, exp_avg_sq, weight_decay=0.01, copies=None) -> AdamwPlan:
    """The plan of adamw_step for lists of contiguous tensors (see spl_adamw_plan): params and grads in fp32, bf16 or
    fp16 (one type for each list), both states float32 tensors or both Fp8Vector (exp_avg_sq then holds square roots),
    copies (fp16 or bf16, or None) what receives the rounded params.  weight_decay: a number, or one for each tensor.
    The plan keeps the tensors; where one gets another address, a new plan is needed.  Waits for the device once."""
    lists = [list(x) for x in (params, grads, exp_avg, exp_avg_sq)] + ([] if copies is None else [list(copies)])
    count = len(lists[0])
    decays = [float(weight_decay)] * count if isinstance(weight_decay, (int, float)) else [float(d) for d in weight_decay]
    if any(len(x) != count for x in lists) or len(decays) != count:
        raise ValueError("params, grads, states, copies and weight_decay: one entry for each tensor")
    P, G, M, V = lists[:4]
    C = lists[4] if copies is not None else None
    eight = any(isinstance(x, Fp8Vector) for x in M + V)
    for i in range(count):
        _arg(P[i], f"params[{i}]", device=False)
        n = P[i].numel()
        _arg(G[i], f"grads[{i}]", shape=P[i].shape, device=False)
        if C is not None:
            _arg(C[i], f"copies[{i}]", shape=P[i].shape, device=False)
        for x, name in ((M[i], "exp_avg"), (V[i], "exp_avg_sq")):
            if eight:
                if not isinstance(x, Fp8Vector) or x.n != n:
                    raise ValueError(f"{name}[{i}] must be an Fp8Vector of {n} elements, as the others")
            else:
                _arg(x, f"{name}[{i}]", shape=P[i].shape, dtype=torch.float32, device=False)
    types = _AdamwTypes(_one_type(P, "params", _FLOAT_TYPES), _one_type(G, "grads", _FLOAT_TYPES),
                        0 if C is None else _one_type(C, "copies", {torch.float16: F16, torch.bfloat16: BF16}),
                        8 if eight else 32)
    if copies is not None and count == 0:
        types.copy_dtype = 0
    states = [t for x in M + V for t in ((x.codes, x.scales) if eight else (x,))]
    every = [*P, *G, *states, *(C or [])]
    device = _here("params, grads, states, copies", None, *every) if every else torch.device("cuda")
    rows = (_AdamwTensor * max(count, 1))()
    for i in range(count):
        m, v = M[i], V[i]
        rows[i] = _AdamwTensor(P[i].data_ptr(), G[i].data_ptr(), (m.codes if eight else m).data_ptr(),
                               (v.codes if eight else v).data_ptr(), m.scales.data_ptr() if eight else None,
                               v.scales.data_ptr() if eight else None, C[i].data_ptr() if C is not None else None,
                               P[i].numel(), decays[i])
    L = lib()
    need, chunks = L.spl_adamw_plan_bytes(rows, count, types), L.spl_adamw_plan_chunks(rows, count, types)
    if need < 0:
        raise ValueError("spl_adamw_plan_bytes rejected the tensors (addresses of their type's alignment, 8-bit codes 16-byte "
                         "aligned, finite weight decay, fewer than 2^24 chunks of 8192 elements)")
    host = torch.zeros((max(need, 16),), dtype=torch.uint8)
    st = L.spl_adamw_plan(rows, count, types, host.data_ptr())
    if st == 1:
        raise ValueError("two arrays of the plan overlap")
    _check("spl_adamw_plan", st)
    table = host.to(device) if every else host
    return AdamwPlan(every, table, chunks, types, device)


def adamw_step(plan: AdamwPlan, lr: float, betas=(0.9, 0.999), eps: float = 1e-8, step: int | torch.Tensor = 1,
               grad_scale: torch.Tensor | None = None, seed: int = 0, stream=None) -> None:
    """One AdamW step over the tensors of the plan, in one launch (see spl_adamw_step).  step: this step's number, from 1
    on, or an int32 tensor [1] on the device that holds it when the step runs.  grad_scale: float32 [1] on the device that
    the gradients are multiplied with (a clipping factor, the inverse of a loss scale); where it is not finite, nothing
    is updated.  seed: of the rounding of 8-bit states."""
    at, number = None, 1
    if isinstance(step, torch.Tensor):
        at = _ints(step, "step", 1)
    else:
        number = step
    scale = None if grad_scale is None else _arg(grad_scale, "grad_scale", shape=(1,), dtype=torch.float32,
                                                 device=False).data_ptr()
    if not plan.chunks:
        return
    _here("the plan, step, grad_scale", stream, plan.table, step if at is not None else None, grad_scale)
    _check("spl_adamw_step",
           lib().spl_adamw_step(plan.table.data_ptr(), plan.chunks, plan.types, lr, betas[0], betas[1], eps, number, at,
                                scale, seed & 0xFFFFFFFF, _on(stream)))
