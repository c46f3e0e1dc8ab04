"""The output head over an embedding table: thin binding, like the package's
other entry points (device pointers and the current HIP stream to the C ABI of
``include/embbag.h``, a status code back, buffer sizes checked first).

4-bit microscaled tables (``Mx4Table``, ``Mx4Tables``): ``embbag_mx4_quantize``,
``embbag_mx4_dequantize``, ``embbag_mx4_forward`` (bags), ``embbag_mx4_matmul``
(scores of every row; ``embbag_mx4_matmul_x8`` from 8-bit rows) and
``embbag_mx4_matmul_grad``.  Between rows and scores:
``embbag_rmsnorm`` (into FP32, BF16 or 8-bit rows, ``Mx8Rows``), ``embbag_rmsnorm_grad``,
``embbag_mx8_dequantize``.  Logits:
``embbag_logits_process`` (penalties, biases, masks) and ``embbag_distill`` (loss
and gradient against a teacher's top logits).  ``embbag_xent``: loss on labels over an
FP32 or BF16 table, with the gradients of both sides, in pieces of the vocabulary (the logits stay in the workspace
only where they are few).
"""
from __future__ import annotations

import ctypes as C
import struct

from . import (EMBBAG_POOL_SUM, _check_bags, _check_numel, _dt, _I32, _need, _ptr, _status_ptr,
               _stream, _U32, lib)

EMBBAG_F32 = 0
EMBBAG_BF16 = 1


class _Mx4Tables(C.Structure):
    _fields_ = [("num_tables", C.c_int32), ("dim", C.c_int32), ("rows", C.POINTER(C.c_int64)),
                ("codes", C.POINTER(C.c_void_p)), ("scales", C.POINTER(C.c_void_p))]


class _Logits(C.Structure):
    _fields_ = [("rows", C.c_int32), ("vocab", C.c_int32), ("type", C.c_int32),
                ("logits", C.c_void_p), ("logits_stride", C.c_int64),
                ("out", C.c_void_p), ("out_stride", C.c_int64),
                ("seen", C.c_void_p), ("seen_offsets", C.c_void_p), ("num_seen", C.c_int64),
                ("prompt_lens", C.c_void_p), ("repetition", C.c_void_p),
                ("frequency", C.c_void_p), ("presence", C.c_void_p),
                ("bias_ids", C.c_void_p), ("bias_offsets", C.c_void_p), ("biases", C.c_void_p),
                ("num_biases", C.c_int64),
                ("masks", C.c_void_p), ("mask_stride", C.c_int64), ("num_masks", C.c_int32),
                ("mask_ids", C.c_void_p)]


class _Distill(C.Structure):
    _fields_ = [("rows", C.c_int32), ("vocab", C.c_int32), ("type", C.c_int32),
                ("logits", C.c_void_p), ("logits_stride", C.c_int64), ("top", C.c_int32),
                ("ids", C.c_void_p), ("teacher_type", C.c_int32), ("teacher", C.c_void_p),
                ("temperature", C.c_float), ("row_weights", C.c_void_p), ("loss", C.c_void_p),
                ("grad", C.c_void_p), ("grad_stride", C.c_int64)]


class _RmsNorm(C.Structure):
    _fields_ = [("rows", C.c_int64), ("dim", C.c_int32), ("eps", C.c_float),
                ("x_type", C.c_int32), ("x", C.c_void_p), ("x_stride", C.c_int64),
                ("residual_type", C.c_int32), ("residual", C.c_void_p),
                ("residual_stride", C.c_int64), ("sum_out", C.c_void_p), ("sum_stride", C.c_int64),
                ("weight_type", C.c_int32), ("weight", C.c_void_p), ("out_type", C.c_int32),
                ("out", C.c_void_p), ("out_stride", C.c_int64), ("codes", C.c_void_p),
                ("scales", C.c_void_p)]


class _RmsNormGrad(C.Structure):
    _fields_ = [("rows", C.c_int64), ("dim", C.c_int32), ("eps", C.c_float),
                ("dy_type", C.c_int32), ("dy", C.c_void_p), ("dy_stride", C.c_int64),
                ("h_type", C.c_int32), ("h", C.c_void_p), ("h_stride", C.c_int64),
                ("weight_type", C.c_int32), ("weight", C.c_void_p), ("dsum", C.c_void_p),
                ("dsum_stride", C.c_int64), ("dh", C.c_void_p), ("dh_stride", C.c_int64),
                ("dweight", C.c_void_p)]


class _Xent(C.Structure):
    _fields_ = [("rows", C.c_int32), ("dim", C.c_int32), ("vocab", C.c_int64),
                ("x_type", C.c_int32), ("x", C.c_void_p), ("x_stride", C.c_int64),
                ("table_type", C.c_int32), ("table", C.c_void_p), ("table_stride", C.c_int64),
                ("labels", C.c_void_p), ("row_weights", C.c_void_p), ("scale", C.c_float),
                ("loss", C.c_void_p), ("grad_x", C.c_void_p), ("grad_x_stride", C.c_int64),
                ("grad_table", C.c_void_p), ("grad_table_stride", C.c_int64)]


# A call's arguments as the bytes of its structure (0.2 us; a ctypes object of 22 fields 1.0).
_CODES = {C.c_int32: "i", C.c_int64: "q", C.c_void_p: "P", C.c_float: "f"}


def _packer(cls):
    fmt = struct.Struct("@" + "".join(_CODES[t] for _, t in cls._fields_))
    assert fmt.size == C.sizeof(cls), cls

    def pack(*fields):
        try:
            return fmt.pack(*fields)
        except struct.error as e:
            raise ValueError(f"an argument is out of range: {e}") from None
    return pack


_pack_logits, _pack_distill = _packer(_Logits), _packer(_Distill)
_pack_xent = _packer(_Xent)
_pack_norm, _pack_norm_grad = _packer(_RmsNorm), _packer(_RmsNormGrad)

_ready = None


def _lib():
    global _ready
    if _ready is None:
        _load_types()
        L = lib()
        p, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        L.embbag_mx4_quantize.argtypes = [p, i32, i64, i64, i32, p, i64, p, p, p, p]
        L.embbag_mx4_dequantize.argtypes = [p, p, i64, i32, p, i32, i64, p]
        L.embbag_mx4_forward.argtypes = [p, i32, p, p, i64, p, i32, p, i32, p, p]
        L.embbag_mx4_matmul_workspace_bytes.argtypes = [i32, i64, i32]
        L.embbag_mx4_matmul.argtypes = [p, i32, i64, i32, p, p, i64, i32, p, i32, i64, p, sz, p]
        L.embbag_mx4_matmul_x8_workspace_bytes.argtypes = [i32, i64, i32]
        L.embbag_mx4_matmul_x8.argtypes = [p, p, i32, p, p, i64, i32, p, i32, i64, p, sz, p]
        L.embbag_mx4_matmul_grad_workspace_bytes.argtypes = [i32, i64, i32]
        L.embbag_mx4_matmul_grad.argtypes = [p, i32, i64, i32, p, p, i64, i32, p, i32, i64, p, sz,
                                             p]
        L.embbag_logits_process.argtypes = [p, p, p]
        L.embbag_distill_workspace_bytes.argtypes = [i32, i32, i32]
        L.embbag_distill.argtypes = [p, p, sz, p, p]
        L.embbag_mx8_dequantize.argtypes = [p, p, i64, i32, p, i32, i64, p]
        L.embbag_rmsnorm.argtypes = [p, p]
        L.embbag_rmsnorm_grad_workspace_bytes.argtypes = [i64, i32]
        L.embbag_rmsnorm_grad.argtypes = [p, p, sz, p]
        L.embbag_xent_workspace_bytes.argtypes = [i32, i64, i32, i32, i32]
        L.embbag_xent.argtypes = [p, p, sz, p, p]
        for n in ("xent", "mx8_dequantize", "mx4_matmul_x8", "rmsnorm", "rmsnorm_grad", "mx4_quantize", "mx4_dequantize", "mx4_forward", "mx4_matmul",
                  "mx4_matmul_grad", "logits_process", "distill"):
            getattr(L, "embbag_" + n).restype = C.c_int
        for n in ("xent", "rmsnorm_grad", "mx4_matmul_x8", "mx4_matmul", "mx4_matmul_grad", "distill"):
            getattr(L, f"embbag_{n}_workspace_bytes").restype = sz
        _ready = L
    return _ready


# ---- marshalling helpers ---------------------------------------------------
def _i32(n):
    """A size as the C ABI's 32 bits take it: ctypes would wrap a larger one into their range, -1 is out
    of every size's."""
    return n if -2 ** 31 <= n < 2 ** 31 else -1


def _types():
    import torch
    return {torch.float32: EMBBAG_F32, torch.bfloat16: EMBBAG_BF16}


_type_of = _I32_T = _F32_T = None


def _load_types():
    global _type_of, _I32_T, _F32_T
    import torch
    _I32_T, _F32_T = torch.int32, torch.float32
    _type_of = _types()


def _matrix(t, cols, name):
    """(pointer, type, row stride) of a 2-D FP32 or BF16 GPU tensor of `cols`
    columns whose rows are contiguous."""
    if _type_of is None:
        _load_types()
    code = _type_of.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: dtype {t.dtype}, expected float32 or bfloat16")
    if not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    shape = t.shape
    if len(shape) != 2 or shape[1] != cols:
        raise ValueError(f"{name}: shape {tuple(shape)}, expected 2-D with {cols} columns")
    s0, s1 = t.stride()
    if shape[0] <= 1:
        s0 = (cols + 3) // 4 * 4  # no second row: any stride
    if s1 != 1 and cols > 1:
        raise TypeError(f"{name}: rows must be contiguous")
    if s0 < cols:
        raise TypeError(f"{name}: rows overlap (stride {s0} for {cols} columns)")
    return t.data_ptr(), code, s0


def _vector(t, n, name, dtype):
    """Pointer of a contiguous GPU tensor of n elements of `dtype` (None: 0; n
    None: any number)."""
    if t is None:
        return 0
    if t.dtype is dtype and t.is_cuda and t.is_contiguous() and (n is None or t.numel() == n):
        return t.data_ptr()
    if n is not None:
        _check_numel(t, n, name)
    return _ptr(t, (dtype,), name)


def _list(entries, offsets, rows, name):
    """Pointers and length of a list per row (None: 0)."""
    if offsets is None:
        if entries is not None:
            raise ValueError(f"{name}: entries without offsets")
        return 0, 0, 0
    if entries is None:
        raise ValueError(f"{name}: offsets without entries")
    return (_vector(entries, None, name, _I32_T),
            _vector(offsets, rows + 1, name + " offsets", _I32_T), entries.numel())


def _status(t):
    if t is not None and t.dtype is _I32_T and t.is_cuda and t.is_contiguous() and t.numel() >= 1:
        return t.data_ptr()
    return _status_ptr(t)


def _check_rows(t, rows, name):
    if t.shape[0] != rows:
        raise ValueError(f"{name}: {t.shape[0]} rows, expected {rows}")


def _ws(workspace):
    if workspace is None:
        return None, 0
    return _ptr(workspace, None, "workspace"), workspace.numel() * workspace.element_size()


def mx4_code_bytes(dim: int) -> int:
    """Bytes of a row of codes (EMBBAG_MX4_CODE_BYTES)."""
    return (dim + 31) // 32 * 16


def mx4_scale_bytes(dim: int) -> int:
    """Bytes of a row of scales (EMBBAG_MX4_SCALE_BYTES)."""
    return (dim + 127) // 128 * 4


class Mx4Table:
    """A 4-bit microscaled table: ``codes`` [M, mx4_code_bytes(dim)] and ``scales``
    [M, mx4_scale_bytes(dim)], contiguous uint8 GPU tensors, which must keep
    their storage while the object is in use."""

    def __init__(self, codes, scales, dim):
        dim = int(dim)
        _need(dim < 2 ** 31, f"dim: {dim} does not fit 32 bits")
        _need(len(codes.shape) == 2 and codes.shape[1] == mx4_code_bytes(dim),
              f"codes: shape {tuple(codes.shape)}, expected [rows, {mx4_code_bytes(dim)}]")
        _need(tuple(scales.shape) == (codes.shape[0], mx4_scale_bytes(dim)),
              f"scales: shape {tuple(scales.shape)}, expected "
              f"[{codes.shape[0]}, {mx4_scale_bytes(dim)}]")
        self.codes_ptr = _ptr(codes, _dt("uint8"), "codes")
        self.scales_ptr = _ptr(scales, _dt("uint8"), "scales")
        self.codes, self.scales, self.dim, self.rows = codes, scales, dim, int(codes.shape[0])

    @classmethod
    def empty(cls, rows, dim, device="cuda"):
        """A table of zeros."""
        import torch
        return cls(torch.zeros(rows, mx4_code_bytes(dim), dtype=torch.uint8, device=device),
                   torch.zeros(rows, mx4_scale_bytes(dim), dtype=torch.uint8, device=device), dim)


def mx8_code_bytes(dim: int) -> int:
    """Bytes of a row of 8-bit codes (EMBBAG_MX8_CODE_BYTES)."""
    return (dim + 127) // 128 * 128


class Mx8Rows:
    """8-bit microscaled rows: ``codes`` [rows, mx8_code_bytes(dim)] and ``scales``
    [rows, mx4_scale_bytes(dim)], contiguous uint8 GPU tensors, which must keep
    their storage while the object is in use."""

    def __init__(self, codes, scales, dim):
        dim = int(dim)
        _need(dim < 2 ** 31, f"dim: {dim} does not fit 32 bits")
        _need(len(codes.shape) == 2 and codes.shape[1] == mx8_code_bytes(dim),
              f"codes: shape {tuple(codes.shape)}, expected [rows, {mx8_code_bytes(dim)}]")
        _need(tuple(scales.shape) == (codes.shape[0], mx4_scale_bytes(dim)),
              f"scales: shape {tuple(scales.shape)}, expected "
              f"[{codes.shape[0]}, {mx4_scale_bytes(dim)}]")
        self.codes_ptr = _ptr(codes, _dt("uint8"), "codes")
        self.scales_ptr = _ptr(scales, _dt("uint8"), "scales")
        self.codes, self.scales, self.dim, self.rows = codes, scales, dim, int(codes.shape[0])

    @classmethod
    def empty(cls, rows, dim, device="cuda"):
        """Rows of zeros."""
        import torch
        return cls(torch.zeros(rows, mx8_code_bytes(dim), dtype=torch.uint8, device=device),
                   torch.zeros(rows, mx4_scale_bytes(dim), dtype=torch.uint8, device=device), dim)


class Mx4Tables:
    """Microscaled tables of one width with their C descriptor built once."""

    def __init__(self, tables):
        self.tables = list(tables)
        T = len(self.tables)
        self.dim = self.tables[0].dim if T else 0
        for i, t in enumerate(self.tables):
            _need(t.dim == self.dim, f"table {i}: dim {t.dim}, expected {self.dim} like table 0")
        n = max(T, 1)
        rows = (C.c_int64 * n)(*[t.rows for t in self.tables])
        codes = (C.c_void_p * n)(*[t.codes_ptr for t in self.tables])
        scales = (C.c_void_p * n)(*[t.scales_ptr for t in self.tables])
        self._keep = (rows, codes, scales)
        pp = C.POINTER(C.c_void_p)
        self.struct = _Mx4Tables(T, self.dim, C.cast(rows, C.POINTER(C.c_int64)),
                                 C.cast(codes, pp), C.cast(scales, pp))

    def __len__(self):
        return len(self.tables)

    def __getitem__(self, i):
        return self.tables[i]

    def __iter__(self):
        return iter(self.tables)


# ---- entry points (same names as the C ABI) --------------------------------
def embbag_mx4_quantize(src, table, row_ids=None, d_status=None, stream=None) -> int:
    """Rows of ``src`` ([M, dim] FP32 or BF16) into ``table``: all of them, or those
    that the int32 tensor ``row_ids`` names."""
    p, ty, ld = _matrix(src, table.dim, "src")
    _check_rows(src, table.rows, "src")
    ids = _ptr(row_ids, _dt(*_I32), "row_ids")
    n = 0 if row_ids is None else row_ids.numel()
    if row_ids is not None and n == 0:
        return 0
    return _lib().embbag_mx4_quantize(p, ty, ld, table.rows, table.dim, ids, n, table.codes_ptr,
                                      table.scales_ptr, _status(d_status), _stream(stream))


def embbag_mx4_dequantize(table, dst, stream=None) -> int:
    """All rows of ``table`` as values into ``dst`` ([M, dim] FP32 or BF16)."""
    p, ty, ld = _matrix(dst, table.dim, "dst")
    _check_rows(dst, table.rows, "dst")
    return _lib().embbag_mx4_dequantize(table.codes_ptr, table.scales_ptr, table.rows, table.dim, p,
                                        ty, ld, _stream(stream))


def embbag_mx4_forward(tables, batch, indices, offsets, pooled_out, per_sample_weights=None,
                       pooling=EMBBAG_POOL_SUM, d_status=None, stream=None) -> int:
    """``embbag_forward_pooled`` from ``Mx4Tables`` into FP32 or BF16 ``pooled_out``."""
    T, dim = len(tables), tables.dim
    _check_bags(T, batch, offsets)
    _check_numel(pooled_out, T * batch * dim, "pooled_out (num_tables x batch x dim)")
    _check_numel(per_sample_weights, indices.numel(), "per_sample_weights")
    out = _ptr(pooled_out, _dt("float32", "bfloat16"), "pooled_out")
    return _lib().embbag_mx4_forward(
        C.byref(tables.struct), _i32(int(batch)), _ptr(indices, _dt(*_I32), "indices"),
        _ptr(offsets, _dt(*_I32), "offsets"), indices.numel(),
        _ptr(per_sample_weights, _dt("float32"), "per_sample_weights"), int(pooling), out,
        EMBBAG_BF16 if pooled_out.element_size() == 2 else EMBBAG_F32, _status(d_status),
        _stream(stream))


def embbag_mx4_matmul_workspace_bytes(m, n, k) -> int:
    return int(_lib().embbag_mx4_matmul_workspace_bytes(_i32(int(m)), int(n), _i32(int(k))))


def embbag_mx4_matmul(x, table, out, workspace, stream=None) -> int:
    """Scores of every row of ``table``: ``out`` [m, M] = q(``x`` [m, dim]) W^T."""
    p, ty, ld = _matrix(x, table.dim, "x")
    q, tq, lq = _matrix(out, table.rows, "out")
    m = x.shape[0]
    _check_rows(out, m, "out")
    w, n = _ws(workspace)
    return _lib().embbag_mx4_matmul(p, ty, ld, _i32(m), table.codes_ptr, table.scales_ptr, table.rows,
                                    table.dim, q, tq, lq, w, n, _stream(stream))


def embbag_mx4_matmul_x8_workspace_bytes(m, n, k) -> int:
    return int(_lib().embbag_mx4_matmul_x8_workspace_bytes(_i32(int(m)), int(n), _i32(int(k))))


def embbag_mx4_matmul_x8(x, table, out, workspace, stream=None) -> int:
    """Scores of every row of ``table`` from 8-bit rows ``x`` (``Mx8Rows``): ``out`` [m, M] = x W^T."""
    if x.dim != table.dim:
        raise ValueError(f"x: rows of {x.dim}, expected {table.dim} like the table's")
    q, tq, lq = _matrix(out, table.rows, "out")
    _check_rows(out, x.rows, "out")
    w, n = _ws(workspace)
    return _lib().embbag_mx4_matmul_x8(x.codes_ptr, x.scales_ptr, _i32(x.rows), table.codes_ptr,
                                       table.scales_ptr, table.rows, table.dim, q, tq, lq, w, n,
                                       _stream(stream))


def embbag_mx4_matmul_grad_workspace_bytes(m, n, k) -> int:
    return int(_lib().embbag_mx4_matmul_grad_workspace_bytes(_i32(int(m)), int(n), _i32(int(k))))


def embbag_mx4_matmul_grad(dy, table, dx, workspace, stream=None) -> int:
    """Gradient of ``embbag_mx4_matmul`` with respect to x: ``dx`` = ``dy`` W."""
    p, ty, ld = _matrix(dy, table.rows, "dy")
    q, tq, lq = _matrix(dx, table.dim, "dx")
    m = dy.shape[0]
    _check_rows(dx, m, "dx")
    w, n = _ws(workspace)
    return _lib().embbag_mx4_matmul_grad(p, ty, ld, _i32(m), table.codes_ptr, table.scales_ptr,
                                         table.rows, table.dim, q, tq, lq, w, n, _stream(stream))


def embbag_mx8_dequantize(rows8, dst, stream=None) -> int:
    """All rows of ``rows8`` (``Mx8Rows``) as values into ``dst`` ([rows, dim] FP32 or BF16)."""
    p, ty, ld = _matrix(dst, rows8.dim, "dst")
    _check_rows(dst, rows8.rows, "dst")
    return _lib().embbag_mx8_dequantize(rows8.codes_ptr, rows8.scales_ptr, rows8.rows, rows8.dim, p,
                                        ty, ld, _stream(stream))


def _weight(t, dim, name):
    """(pointer, type) of a vector of `dim` weights (None: none)."""
    if t is None:
        return 0, EMBBAG_F32
    code = _type_of.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: dtype {t.dtype}, expected float32 or bfloat16")
    return _vector(t, dim, name, t.dtype), code


def _same_rows(t, shape, name, code=None, like=""):
    """_matrix of a tensor of the shape `shape` and of the type `code` (None: any; no tensor: zeros)."""
    if t is None:
        return 0, EMBBAG_F32 if code is None else code, 0
    own = _type_of.get(t.dtype)
    if t.shape == shape and own is not None and t.is_cuda and (code is None or own == code):
        s0, s1 = t.stride()
        if s1 == 1 and s0 >= shape[1]:
            return t.data_ptr(), own, s0
    m = _matrix(t, shape[1], name)
    _check_rows(t, shape[0], name)
    if code is not None and m[1] != code:
        raise TypeError(f"{name}: dtype {t.dtype}, expected that of {like}")
    return m


def embbag_rmsnorm(x, weight, eps, out=None, mx8=None, residual=None, sum_out=None, stream=None) -> int:
    """RMS norm of ``x`` [rows, dim] plus ``residual``, times ``weight`` ([dim], None: ones), into
    ``out`` and/or the 8-bit rows ``mx8`` (``Mx8Rows``); the sum itself into ``sum_out`` (which may
    be ``residual``, and has its type)."""
    shape = x.shape
    p, ty, ld = _matrix(x, shape[1] if len(shape) == 2 else -1, "x")
    rows, dim = shape
    r, tr, lr = _same_rows(residual, shape, "residual")
    s, ts, ls = _same_rows(sum_out, shape, "sum_out", None if residual is None else tr, "residual")
    q, tq, lq = _same_rows(out, shape, "out")
    w, tw = _weight(weight, dim, "weight")
    codes = scales = 0
    if mx8 is not None:
        if mx8.rows != rows or mx8.dim != dim:
            raise ValueError(f"mx8: {mx8.rows} rows of {mx8.dim}, expected {rows} of {dim}")
        codes, scales = mx8.codes_ptr, mx8.scales_ptr
    a = _pack_norm(rows, dim, eps, ty, p, ld, ts, r, lr, s, ls, tw, w, tq, q, lq, codes, scales)
    return _lib().embbag_rmsnorm(a, _stream(stream))


def embbag_rmsnorm_grad_workspace_bytes(rows, dim) -> int:
    return int(_lib().embbag_rmsnorm_grad_workspace_bytes(int(rows), _i32(int(dim))))


def embbag_rmsnorm_grad(dy, h, weight, eps, dh, workspace, dweight=None, dsum=None, stream=None) -> int:
    """Gradients of ``embbag_rmsnorm``: ``dh`` (that of x and of the residual) and ``dweight`` from the
    output's gradient ``dy``, the sum ``h`` and the sum's own gradient ``dsum``."""
    shape = h.shape
    p, th, lh = _matrix(h, shape[1] if len(shape) == 2 else -1, "h")
    rows, dim = shape
    y, ty, ly = _same_rows(dy, shape, "dy")
    d, _, ld = _same_rows(dh, shape, "dh", th, "h")
    s, _, ls = _same_rows(dsum, shape, "dsum", th, "h")
    w, tw = _weight(weight, dim, "weight")
    g, tg = _weight(dweight, dim, "dweight")
    if dweight is not None and tg != (ty if weight is None else tw):
        raise TypeError(f"dweight: dtype {dweight.dtype}, expected that of "
                        f"{'dy' if weight is None else 'weight'}")
    a = _pack_norm_grad(rows, dim, eps, ty, y, ly, th, p, lh, tw, w, s, ls, d, ld, g)
    ws, n = _ws(workspace)
    return _lib().embbag_rmsnorm_grad(a, ws, n, _stream(stream))


def embbag_logits_process(logits, out, seen=None, seen_offsets=None, prompt_lens=None,
                          repetition=None, frequency=None, presence=None, bias_ids=None,
                          bias_offsets=None, biases=None, masks=None, mask_ids=None, d_status=None,
                          stream=None) -> int:
    """Penalties for seen tokens, biases and masks: ``logits`` [rows, vocab] into
    ``out`` (which may be ``logits``).  Every argument after ``out`` is optional."""
    vocab = logits.shape[1] if len(logits.shape) == 2 else -1
    p, ty, ld = _matrix(logits, vocab, "logits")
    q, tq, lq = _matrix(out, vocab, "out")
    if tq != ty:
        raise TypeError(f"out: dtype {out.dtype}, expected {logits.dtype} like logits")
    rows = logits.shape[0]
    _check_rows(out, rows, "out")
    seen_p, seen_o, num_seen = _list(seen, seen_offsets, rows, "seen")
    bias_p, bias_o, num_biases = _list(bias_ids, bias_offsets, rows, "bias_ids")
    if bias_ids is not None and biases is None:
        raise ValueError("bias_ids without biases")
    masks_p, num_masks, mask_stride = 0, 0, 0
    if masks is not None:
        if len(masks.shape) != 2 or masks.shape[1] * 32 < vocab:
            raise ValueError(f"masks: shape {tuple(masks.shape)}, expected 2-D with at least "
                             f"{(vocab + 31) // 32} words a row")
        masks_p = _ptr(masks, _dt(*_U32), "masks")
        num_masks, mask_stride = masks.shape
        if mask_ids is None and num_masks < rows:
            raise ValueError(f"masks: {num_masks} for {rows} rows and no mask_ids")
    a = _pack_logits(
        rows, vocab, ty, p, ld, q, lq, seen_p, seen_o, num_seen,
        _vector(prompt_lens, rows, "prompt_lens", _I32_T),
        _vector(repetition, rows, "repetition", _F32_T),
        _vector(frequency, rows, "frequency", _F32_T),
        _vector(presence, rows, "presence", _F32_T), bias_p, bias_o,
        _vector(biases, num_biases, "biases", _F32_T), num_biases, masks_p, mask_stride,
        num_masks, _vector(mask_ids, rows, "mask_ids", _I32_T))
    return _lib().embbag_logits_process(a, _status(d_status), _stream(stream))


def embbag_distill_workspace_bytes(rows, vocab, top) -> int:
    return int(_lib().embbag_distill_workspace_bytes(_i32(int(rows)), _i32(int(vocab)), _i32(int(top))))


def embbag_distill(logits, teacher_ids, teacher_logits, temperature, loss, workspace, grad=None,
                   row_weights=None, d_status=None, stream=None) -> int:
    """Loss of every row of ``logits`` [rows, vocab] against a teacher's top logits
    ([rows, top]; an id below 0 is no entry) and, with ``grad``, its gradient (into
    ``logits`` itself if that is given)."""
    vocab = logits.shape[1] if len(logits.shape) == 2 else -1
    p, ty, ld = _matrix(logits, vocab, "logits")
    rows = logits.shape[0]
    if len(teacher_ids.shape) != 2 or teacher_ids.shape[0] != rows:
        raise ValueError(f"teacher_ids: shape {tuple(teacher_ids.shape)}, expected [{rows}, top]")
    top = teacher_ids.shape[1]
    if teacher_logits.shape != teacher_ids.shape and (len(teacher_logits.shape) == 2 or
                                                      teacher_logits.numel() != rows * top):
        raise ValueError(f"teacher_logits: shape {tuple(teacher_logits.shape)}, expected "
                         f"{tuple(teacher_ids.shape)} like teacher_ids")
    q, lq = 0, 0
    if grad is not None:
        q, tq, lq = _matrix(grad, vocab, "grad")
        if tq != ty:
            raise TypeError(f"grad: dtype {grad.dtype}, expected {logits.dtype} like logits")
        _check_rows(grad, rows, "grad")
    a = _pack_distill(
        rows, vocab, ty, p, ld, top, _vector(teacher_ids, None, "teacher_ids", _I32_T),
        EMBBAG_BF16 if teacher_logits.element_size() == 2 else EMBBAG_F32,
        _ptr(teacher_logits, _dt("float32", "bfloat16"), "teacher_logits"),
        C.c_float(temperature).value, _vector(row_weights, rows, "row_weights", _F32_T),
        _vector(loss, rows, "loss", _F32_T), q, lq)
    w, n = _ws(workspace)
    return _lib().embbag_distill(a, w, n, _status(d_status), _stream(stream))


def embbag_xent_workspace_bytes(rows, vocab, dim, type, backward) -> int:
    """``type``: EMBBAG_F32 if x or the table is FP32, else EMBBAG_BF16; ``backward``: whether a
    gradient is wanted."""
    return int(_lib().embbag_xent_workspace_bytes(_i32(int(rows)), int(vocab), _i32(int(dim)),
                                                  int(type), 1 if backward else 0))


def embbag_xent(x, table, labels, loss, workspace, grad_x=None, grad_table=None, row_weights=None,
                scale=1.0, d_status=None, stream=None) -> int:
    """Loss of every row of ``x`` [rows, dim] on its label among the rows of ``table`` [vocab, dim]
    (scores ``scale`` x table^T; a negative label is no row to learn) and, into ``grad_x`` and
    ``grad_table``, the gradients of the losses' sum."""
    shape, tshape = x.shape, table.shape
    p, ty, ld = _matrix(x, shape[1] if len(shape) == 2 else -1, "x")
    rows, dim = shape
    w, tw, lw = _matrix(table, dim, "table")
    vocab = tshape[0]
    g, _, lg = _same_rows(grad_x, shape, "grad_x", ty, "x")
    h, _, lh = _same_rows(grad_table, tshape, "grad_table", tw, "table")
    a = _pack_xent(_i32(rows), dim, vocab, ty, p, ld, tw, w, lw, _vector(labels, rows, "labels", _I32_T),
                   _vector(row_weights, rows, "row_weights", _F32_T), scale,
                   _vector(loss, rows, "loss", _F32_T), g, lg, h, lh)
    ws, n = _ws(workspace)
    return _lib().embbag_xent(a, ws, n, _status(d_status), _stream(stream))
