"""Binding of the row operators (the C ABI declared in include/uccl_rows.h): norm of rows, products grouped by expert,
combination of rows, and their gradients.

Argument marshalling only, as in the package's main module, whose names for streams and errors hold here too.  Matrices
are torch tensors on the GPU whose last dimension is contiguous; leading dimensions are rows, a constant number of bytes
apart.  The library checks types, shapes and alignment; what only the tensors know (an index as long as the rows it is
for, say) is checked here and raises ValueError.  Outputs are the caller's tensors and come first.
"""
import ctypes as C
import os
import struct

UCCL_E4M3, UCCL_MX4 = 16, 17
ROWS_HEADER_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "uccl_rows.h")


class uccl_rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_uint64), ("scales", C.c_void_p), ("scale_stride", C.c_uint64),
                ("rows", C.c_uint32), ("cols", C.c_uint32), ("dtype", C.c_uint32), ("reserved", C.c_uint32)]


class uccl_norm_opts(C.Structure):
    _fields_ = [("eps", C.c_float), ("reserved", C.c_uint32 * 3)]


# Rows are passed as the struct's bytes, which take a third of the time of a ctypes structure's making.
_pack_rows = struct.Struct("@QQQQIIII").pack
assert len(_pack_rows(*[0] * 8)) == C.sizeof(uccl_rows)

_R, _P, _U32 = C.c_void_p, C.c_void_p, C.c_uint32

ROWS_SIGNATURES = {
    "uccl_norm_rows": (C.c_int, [_R, _R, _P, _R, _R, _P, _P, _P]),
    "uccl_norm_rows_grad": (C.c_int, [_R, _P, _R, _R, _R, _P, _P, _P, C.c_uint64, _P]),
    "uccl_norm_rows_scratch": (C.c_uint64, [_U32, _U32]),
    "uccl_group_product": (C.c_int, [_R, _R, _P, _R, _P, _U32, _P]),
    "uccl_group_product_grad_x": (C.c_int, [_R, _R, _R, _P, _U32, _P]),
    "uccl_group_product_grad_w": (C.c_int, [_R, _R, _R, _P, _P, _U32, _P]),
    "uccl_combine_rows": (C.c_int, [_R, _R, _P, _P, _U32, _R, _P]),
    "uccl_combine_rows_grad": (C.c_int, [_R, _P, _R, _R, _P, _P, _U32, _P]),
}

_types = {}   # torch dtype -> (number of the type, bytes), filled on first use


def _type(dtype):
    if not _types:
        import torch
        from . import UCCL_BF16, UCCL_F16, UCCL_F32
        _types.update({torch.float32: (UCCL_F32, 4), torch.bfloat16: (UCCL_BF16, 2), torch.float16: (UCCL_F16, 2),
                       torch.float8_e4m3fn: (UCCL_E4M3, 1), "scale": torch.float32})
        four, block = getattr(torch, "float4_e2m1fn_x2", None), getattr(torch, "float8_e8m0fnu", None)
        if four is not None and block is not None:   # a torch without them has no tensors of 4 bits, and all others
            _types.update({four: (UCCL_MX4, 1), "block": block})
    if dtype not in _types:
        raise ValueError(f"rows of {dtype} are not supported")
    return _types[dtype]


_reader = None   # the extension, if it reads tensors; False: it does not


def _find_reader():
    """The extension, if it reads a matrix and a vector as this module does."""
    global _reader
    import torch
    from . import _load_extension
    extension, table = _load_extension(), getattr(torch.Tensor, "__dlpack_c_exchange_api__", None)
    _reader = False
    if extension and table is not None and extension.read_tensors(table, torch.Tensor, torch.nn.Parameter):
        matrix, vector = torch.zeros(3, 8, dtype=torch.bfloat16)[1:, :5], torch.zeros(7, dtype=torch.int32)
        want, address = _rows(matrix), vector.data_ptr()
        if extension.matrix_rows(matrix) == want and extension.vector_address(vector, False, 7) == address:
            _reader = extension
    return _reader


def _rows(t, scales=None, cols_in_4_bits=None):
    """The bytes of a HOST uccl_rows for a tensor, as an argument; None for None.  Rows of 4 bits have two elements in each of the tensor's, or
    one in the last, if ``cols_in_4_bits`` says so."""
    if t is None:
        return None
    if scales is None:
        reader = _find_reader() if _reader is None else _reader
        if reader:
            made = reader.matrix_rows(t)
            if made is not None:
                return made
    number, size = _types.get(t.dtype) or _type(t.dtype)
    shape = t.shape
    if len(shape) == 2:
        rows, cols = shape
        step, last = t.stride()
    elif len(shape) == 3:
        groups, each, cols = shape
        apart, step, last = t.stride()
        rows = groups * each
        if each == 1:
            step = apart
        elif groups > 1 and rows and cols and apart != each * step:
            raise ValueError("the rows of a three-dimensional tensor have to be the same distance apart throughout")
    else:
        raise ValueError("a tensor of rows has two or three dimensions")
    if last != 1 and cols > 1:
        raise ValueError("the last dimension of a tensor of rows has to be contiguous")
    if rows > 0xFFFFFFFF or cols > 0xFFFFFFFF:
        raise ValueError("a tensor of rows has fewer than 2^32 rows and columns")
    if scales is None:
        return _pack_rows(t.data_ptr(), step * size, 0, 0, rows, cols, number, 0)
    if number == UCCL_MX4:
        return _rows_in_4_bits(t, step, rows, cols, scales, cols_in_4_bits)
    if scales.dtype is not _types["scale"] or scales.numel() != rows:
        raise ValueError("scales are float32, one for every row")
    lengths, apart = scales.shape, scales.stride()
    if len(lengths) > 1 and lengths[-1] == 1:   # a last dimension of one scale
        lengths, apart = lengths[:-1], apart[:-1]
    if len(lengths) == 2 and lengths[0] > 1 and lengths[1] > 1 and apart[0] != lengths[1] * apart[1] or len(lengths) > 2:
        raise ValueError("scales have to be the same distance apart throughout")
    between = 0 if not lengths else 4 * (apart[0] if lengths[-1] == 1 else apart[-1])
    return _pack_rows(t.data_ptr(), step * size, scales.data_ptr(), between, rows, cols, number, 0)


def _rows_in_4_bits(t, step, rows, pairs, scales, cols):
    cols = 2 * pairs if cols is None else cols
    blocks = -(-cols // 32)
    if (cols + 1) // 2 != pairs:
        raise ValueError(f"{cols} elements are {(cols + 1) // 2} pairs in 4 bits")
    lengths, apart = scales.shape, scales.stride()
    if scales.dtype is not _types["block"] or len(lengths) not in (2, 3) or scales.numel() != rows * blocks or lengths[-1] != blocks:
        raise ValueError("scales are float8_e8m0fnu, one for every 32 elements of a row")
    if (apart[-1] != 1 and blocks > 1) or len(lengths) == 3 and lengths[0] > 1 and lengths[1] > 1 and apart[0] != lengths[1] * apart[1]:
        raise ValueError("a row's scales have to be contiguous, and the rows' the same distance apart throughout")
    between = apart[0] if lengths[-2] == 1 else apart[-2]
    return _pack_rows(t.data_ptr(), step, scales.data_ptr(), between, rows, cols, UCCL_MX4, 0)


def _vector(t, kind, n, what):
    """The address of `n` contiguous elements of `kind` (i: int32, f: float32); None for None."""
    if t is None:
        return None
    if _reader:
        address = _reader.vector_address(t, kind == "f", n)
        if address is not None:
            return address
    if t.element_size() != 4 or t.is_floating_point() != (kind == "f") or not t.is_contiguous() or t.numel() != n:
        raise ValueError(f"{what}: {n} contiguous elements of {'float32' if kind == 'f' else 'int32'} are wanted")
    return t.data_ptr()


def _count(t):
    """Rows of a tensor of rows."""
    return t.shape[0] * t.shape[1] if t.dim() == 3 else t.shape[0]


def _weight(t, like):
    if t.dtype != like.dtype or t.numel() != like.shape[-1] or not t.is_contiguous():
        raise ValueError("the weight has the rows' type and one element for every column")
    return t.data_ptr()


def uccl_norm_rows(y, x, weight, eps, residual=None, h=None, rstd=None, scales=None, stream=None):
    """y = norm(x + residual) * weight by rows; h: the sum, rstd: 1 / root of its mean square.  A float8_e4m3fn ``y`` takes
    a scale for every row in ``scales``."""
    _call("uccl_norm_rows", _rows(y, scales), _rows(h), _vector(rstd, "f", _count(x), "rstd"), _rows(x), _rows(residual),
          _weight(weight, x), C.byref(uccl_norm_opts(eps)), _stream(stream))


def uccl_norm_rows_scratch(rows, cols) -> int:
    """Bytes of scratch memory that the gradient of a norm of that many rows and columns needs."""
    return load().uccl_norm_rows_scratch(int(rows), int(cols))


def uccl_norm_rows_grad(dx, dweight, dy, h, rstd, weight, scratch, dh=None, stream=None):
    """dx: gradient of x and of the residual alike; dweight: float32.  ``dh`` is what arrives along the residual."""
    _call("uccl_norm_rows_grad", _rows(dx), _vector(dweight, "f", h.shape[-1], "dweight"), _rows(dy), _rows(dh), _rows(h),
          _vector(rstd, "f", _count(h), "rstd"), _weight(weight, h), _ptr(scratch), _nbytes(scratch), _stream(stream))


def uccl_group_product(y, x, w, offsets, index=None, x_scales=None, w_scales=None, stream=None):
    """y[i] = x[index[i]] @ w[g].T for the rows offsets[g] <= i < offsets[g + 1]; ``w``: groups x n x k."""
    cols = x.shape[-1] if w_scales is not None and x_scales is None else None   # 16-bit rows with weights in 4 bits
    _call("uccl_group_product", _rows(y), _rows(x, x_scales), _vector(index, "i", _count(y), "index"), _rows(w, w_scales, cols),
          _vector(offsets, "i", w.shape[0] + 1, "offsets"), w.shape[0], _stream(stream))


def uccl_group_product_grad_x(dx, dy, w, offsets, stream=None):
    """dx[i] = dy[i] @ w[g], by rows as the product read them."""
    _call("uccl_group_product_grad_x", _rows(dx), _rows(dy), _rows(w), _vector(offsets, "i", w.shape[0] + 1, "offsets"), w.shape[0],
          _stream(stream))


def uccl_group_product_grad_w(dw, dy, x, offsets, index=None, stream=None):
    """dw[g] = dy[rows of g].T @ x[index[rows of g]]; ``dw``: groups x n x k, zeros for a group without rows."""
    _call("uccl_group_product_grad_w", _rows(dw), _rows(dy), _rows(x), _vector(index, "i", _count(dy), "index"),
          _vector(offsets, "i", dw.shape[0] + 1, "offsets"), dw.shape[0], _stream(stream))


def _slots(pos, tokens):
    if pos.dim() != 2 or pos.shape[0] != tokens:
        raise ValueError("pos: one row of slots for every token")
    return pos.shape[1]


def uccl_combine_rows(out, y, pos, weights=None, residual=None, stream=None):
    """out[t] = residual[t] + sum_j weights[t, j] y[pos[t, j]]; a ``pos`` that is no row of y adds nothing."""
    slots = _slots(pos, _count(out))
    n = slots * pos.shape[0]
    _call("uccl_combine_rows", _rows(out), _rows(y), _vector(pos, "i", n, "pos"), _vector(weights, "f", n, "weights"), slots, _rows(residual),
          _stream(stream))


def uccl_combine_rows_grad(dy, dweights, dout, y, pos, weights=None, stream=None):
    """dy[pos[t, j]] = weights[t, j] dout[t]; dweights[t, j] = dout[t] . y[pos[t, j]] (None: not wanted)."""
    slots = _slots(pos, _count(dout))
    n = slots * pos.shape[0]
    _call("uccl_combine_rows_grad", _rows(dy), _vector(dweights, "f", n, "dweights"), _rows(dout), _rows(y), _vector(pos, "i", n, "pos"),
          _vector(weights, "f", n, "weights"), slots, _stream(stream))


from . import _call, _nbytes, _ptr, _stream, load  # noqa: E402  (the package imports this module at its end)
