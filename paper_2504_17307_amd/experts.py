"""Binding of routing, microscaled 4 bits and clipping (the C ABI declared in include/uccl_experts.h).

Argument marshalling only, in the manner of the row operators' module: outputs are the caller's tensors and come first, matrices are torch
tensors on the GPU whose last dimension is contiguous, the library checks types, shapes and alignment, and what only the tensors
know is checked here and raises ValueError.  Rows in 4 bits are float4_e2m1fn_x2 tensors, two elements a byte, with a float8_e8m0fnu tensor of one
scale for every 32 elements of a row.
"""
import ctypes as C
import os
import struct

from . import rows
from .rows import _count, _find_reader, _rows, _vector

EXPERTS_HEADER_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "uccl_experts.h")


class uccl_route_opts(C.Structure):
    _fields_ = [("slots", C.c_uint32), ("normalise", C.c_uint32), ("scale", C.c_float), ("reserved", C.c_uint32)]


class uccl_balance_opts(C.Structure):
    _fields_ = [("tokens", C.c_uint64), ("slots", C.c_uint32), ("coef", C.c_float)]


class uccl_clip_opts(C.Structure):
    _fields_ = [("most", C.c_float), ("reserved", C.c_uint32 * 3)]


_R, _P, _U32, _U64 = C.c_void_p, C.c_void_p, C.c_uint32, C.c_uint64

EXPERTS_SIGNATURES = {
    "uccl_route_rows": (C.c_int, [_P, _P, _P, _P, _R, _P, _P, _P, _U64, _P]),
    "uccl_route_rows_scratch": (_U64, [_U32, _U32]),
    "uccl_route_rows_grad": (C.c_int, [_R, _R, _P, _P, _P, _P, _P]),
    "uccl_balance_loss": (C.c_int, [_P, _P, _P, _P, _U32, _P, _P]),
    "uccl_plan_rows": (C.c_int, [_P, _P, _P, _P, _U32, _U32, _U32, _P, _U64, _P]),
    "uccl_plan_rows_scratch": (_U64, [_U64, _U32]),
    "uccl_quantise_rows": (C.c_int, [_R, _R, _R, _P]),
    "uccl_gradient_norm": (C.c_int, [_P, _R, _U32, _P, _U64, _P]),
    "uccl_gradient_norm_scratch": (_U64, [_U32]),
    "uccl_gradient_clip": (C.c_int, [_R, _R, _U32, _P, _P, _P]),
}

# passed as the structs' bytes
_pack_route, _pack_balance, _pack_clip = struct.Struct("@IIfI").pack, struct.Struct("@QIf").pack, struct.Struct("@f3I").pack


def _choices(t, kind, tokens, what):
    """The address and the slots of a tensor of tokens x slots."""
    if t.dim() != 2 or t.shape[0] != tokens:
        raise ValueError(f"{what}: one row of slots for every token")
    return _vector(t, kind, t.numel(), what), t.shape[1]


def uccl_route_rows(experts, weights, scores, bias=None, normalise=False, scale=1.0, counts=None, sums=None, scratch=None, stream=None):
    """The ``experts`` (int32, tokens x slots; -1: none) with the greatest scores + bias of every token, and their ``weights``: scale softmax(scores),
    over all experts or, ``normalise``, over the token's own.  ``counts`` (int32) and ``sums`` (float32) of the experts' tokens and probabilities."""
    tokens, n = _count(scores), scores.shape[-1]
    chosen, slots = _choices(experts, "i", tokens, "experts")
    w, same = _choices(weights, "f", tokens, "weights")
    if same != slots:
        raise ValueError("experts and weights have the same slots")
    _call("uccl_route_rows", chosen, w, _vector(counts, "i", n, "counts"), _vector(sums, "f", n, "sums"), _rows(scores), _vector(bias, "f", n, "bias"),
          _pack_route(slots, int(bool(normalise)), scale, 0), _ptr(scratch), _nbytes(scratch), _stream(stream))


def uccl_route_rows_scratch(tokens, n_experts) -> int:
    """Bytes of scratch memory that counts and sums of that many tokens and experts need."""
    return load().uccl_route_rows_scratch(int(tokens), int(n_experts))


def uccl_route_rows_grad(dscores, scores, experts=None, dweights=None, dsums=None, normalise=False, scale=1.0, slots=None, stream=None):
    """The gradient of the scores for ``dweights`` of the weights that went to ``experts``, and ``dsums`` of the sums of probabilities (either may be None).
    ``slots``: where there are no experts, 1 will do."""
    tokens, n = _count(scores), scores.shape[-1]
    chosen, d = None, None
    if experts is not None:
        chosen, slots = _choices(experts, "i", tokens, "experts")
    if dweights is not None:
        d, same = _choices(dweights, "f", tokens, "dweights")
        if same != slots:
            raise ValueError("experts and dweights have the same slots")
    _call("uccl_route_rows_grad", _rows(dscores), _rows(scores), chosen, d, _vector(dsums, "f", n, "dsums"),
          _pack_route(1 if slots is None else slots, int(bool(normalise)), scale, 0), _stream(stream))


def uccl_balance_loss(loss, dsums, counts, sums, tokens, slots, coef, stream=None):
    """loss = coef E / (slots tokens^2) sum of counts sums; ``dsums``: its gradient.  ``tokens``: of all ranks whose counts and sums were added up."""
    n = counts.numel()
    _call("uccl_balance_loss", _vector(loss, "f", 1, "loss"), _vector(dsums, "f", n, "dsums"), _vector(counts, "i", n, "counts"),
          _vector(sums, "f", n, "sums"), n, _pack_balance(tokens, slots, coef), _stream(stream))


def uccl_plan_rows(index, offsets, pos, experts, scratch=None, stream=None):
    """``experts`` (tokens x slots) to the ``index`` (the token of every row, -1 behind the last) and ``offsets`` (n_experts + 1) of the products and the
    ``pos`` (every choice's row, -1: none) of the combination; index and pos may be None."""
    tokens, slots = experts.shape[0], experts.shape[-1]
    chosen, _ = _choices(experts, "i", tokens, "experts")
    _call("uccl_plan_rows", _vector(index, "i", tokens * slots, "index"), _vector(offsets, "i", offsets.numel(), "offsets"),
          _vector(pos, "i", tokens * slots, "pos"), chosen, tokens, slots, offsets.numel() - 1, _ptr(scratch), _nbytes(scratch), _stream(stream))


def uccl_plan_rows_scratch(choices, n_experts) -> int:
    """Bytes of scratch memory that the order of that many choices (tokens x slots) needs."""
    return load().uccl_plan_rows_scratch(int(choices), int(n_experts))


def uccl_quantise_rows(q, scales, x, values=None, stream=None):
    """``x`` in microscaled 4 bits; ``values``: what they stand for, in x's type."""
    _call("uccl_quantise_rows", _rows(q, scales, x.shape[-1]), _rows(values), _rows(x), _stream(stream))


_LONGEST = 1 << 30   # columns of a matrix


def _matrices(tensors, like=None):
    """The bytes of a HOST array of uccl_rows for ``tensors``, of another for those of ``like``, which have their shapes and types (by default they themselves), and how many matrices there
    are: a contiguous tensor is one row, or whole rows and what is left; two tensors are cut alike."""
    like = tensors if like is None else like
    if hasattr(tensors, "__next__") or hasattr(like, "__next__"):   # gone through once, and nothing of it is left for a prepared call to hold
        raise ValueError("a list of tensors is wanted, not an iterator")
    if type(tensors) is list and type(like) is list:
        reader = _find_reader() if rows._reader is None else rows._reader
        made = reader.contiguous_rows(tensors, like, _LONGEST) if reader else None
        if made is not None:
            return (*made, len(tensors))
    made = [], []
    for pair in zip(tensors, like):
        if pair[0].shape != pair[1].shape or pair[0].dtype != pair[1].dtype:
            raise ValueError("outputs have the gradients' shapes and types")
        whole = pair[0].is_contiguous() and pair[1].is_contiguous()
        for to, t in zip(made, pair):
            if not whole:
                to.append(_rows(t))
                continue
            flat = t.view(-1)
            n = flat.shape[0]
            if n > _LONGEST:
                at = n // _LONGEST * _LONGEST
                to.append(_rows(flat[:at].view(-1, _LONGEST)))
                flat = flat[at:]
            to.append(_rows(flat.view(1, -1)))
    return b"".join(made[0]), b"".join(made[1]), len(made[0])


def uccl_gradient_norm(norm, grads, scratch, stream=None):
    """The root of the sum of the squares of all elements of ``grads``, a list of tensors."""
    m, _, n = _matrices(grads)
    _call("uccl_gradient_norm", _vector(norm, "f", 1, "norm"), m, n, _ptr(scratch), _nbytes(scratch), _stream(stream))


def uccl_gradient_norm_scratch(n) -> int:
    """Bytes of scratch memory that the norm of n tensors of up to 2^30 elements each needs."""
    return load().uccl_gradient_norm_scratch(int(n))


def uccl_gradient_clip(outs, grads, norm, most, stream=None):
    """outs = grads min(1, most / norm), tensor by tensor; ``outs`` may be ``grads``."""
    if len(outs) != len(grads):
        raise ValueError("an output for every gradient")
    to, of, n = _matrices(outs, grads)
    _call("uccl_gradient_clip", to, of, n, _vector(norm, "f", 1, "norm"), _pack_clip(most, 0, 0, 0), _stream(stream))


from . import _call, _nbytes, _ptr, _stream, load  # noqa: E402  (the package imports this module at its end)
