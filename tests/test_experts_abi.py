"""The C ABI of routing, microscaled 4 bits and clipping without a GPU: exports, layouts, refusals, which come before anything is enqueued, and what the
library asks of the HIP runtime (tests/hip_stub.c: nothing runs)."""
import ctypes as C
import os
import re
import struct
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path[:0] = [HERE, os.path.dirname(HERE)]
import paper_2504_17307_amd as pkg  # noqa: E402
from test_rows_abi import A, B, BF16, D, E4M3, EALIGN, EINVAL, F16, F32, I32, M, OK, S, q8, rows  # noqa: E402

MX4 = pkg.UCCL_MX4
TOOBIG = pkg.UCCL_ETOOBIG


def q4(n, cols, data=A, stride=None, scales=S, scale_stride=None):
    stride = -(-cols // 32) * 16 if stride is None else stride
    return C.byref(pkg.uccl_rows(data, stride, scales, -(-cols // 128) * 4 if scale_stride is None else scale_stride, n, cols, MX4, 0))


def route(slots=2, normalise=0, scale=1.0, reserved=0):
    return C.byref(pkg.uccl_route_opts(slots, normalise, scale, reserved))


def test_every_declared_function_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(pkg.EXPERTS_HEADER_PATH).read(), flags=re.S)
    names = set(re.findall(r"\b(uccl_[a-z_]+)\s*\(", text))
    assert names == set(pkg.EXPERTS_SIGNATURES) and len(names) == 10
    lib = pkg.load()
    for n in names:
        assert hasattr(lib, n) and hasattr(pkg, n), n
    assert "#define UCCL_MX4 %d" % MX4 in open(pkg.ROWS_HEADER_PATH).read()
    assert [C.sizeof(t) for t in (pkg.uccl_route_opts, pkg.uccl_balance_opts, pkg.uccl_clip_opts)] == [16, 16, 16]


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("change,code", [
    (dict(experts=None), EINVAL), (dict(weights=None), EINVAL), (dict(scores=None), EINVAL), (dict(opts=None), EINVAL),
    (dict(scores=rows(9, 8, I32)), EINVAL), (dict(scores=q8(9, 8)), EINVAL), (dict(scores=q4(9, 8)), EINVAL), (dict(scores=rows(9, 1025)), EINVAL), (dict(scores=rows(9, 0)), EINVAL),
    (dict(scores=rows(9, 8, data=None)), EINVAL), (dict(scores=rows(9, 8, data=A + 8)), EALIGN), (dict(scores=rows(9, 8, stride=24)), EALIGN),
    (dict(opts=route(0)), EINVAL), (dict(opts=route(9)), EINVAL), (dict(scores=rows(9, 64), opts=route(33)), EINVAL), (dict(opts=route(2, 2)), EINVAL),
    (dict(opts=route(2, 0, INF)), EINVAL), (dict(opts=route(2, 0, NAN)), EINVAL), (dict(opts=route(2, 0, 1.0, 1)), EINVAL),
    (dict(experts=M + 2), EALIGN), (dict(weights=M + 1), EALIGN), (dict(counts=M + 2), EALIGN), (dict(sums=M + 3), EALIGN), (dict(bias=M + 2), EALIGN),
    (dict(scores=rows(9000, 8), counts=M), EINVAL), (dict(scores=rows(9000, 8), sums=M, scratch=B, scratch_bytes=8), EINVAL),
    (dict(scores=rows(9000, 8), sums=M, scratch=B + 8, scratch_bytes=1 << 20), EALIGN),
    (dict(scores=rows(1 << 28, 8)), TOOBIG), (dict(scores=rows(1 << 26, 512)), TOOBIG),
    (dict(scores=rows(0, 8), experts=None, weights=None), OK),
])
def test_route_refusals(change, code):
    a = dict(experts=M, weights=D, counts=None, sums=None, scores=rows(9, 8), bias=None, opts=route(), scratch=None, scratch_bytes=0, stream=None)
    a.update(change)
    assert pkg.load().uccl_route_rows(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(dscores=None), EINVAL), (dict(scores=None), EINVAL), (dict(opts=None), EINVAL), (dict(experts=None), EINVAL), (dict(dweights=None), EINVAL),
    (dict(dscores=rows(9, 9)), EINVAL), (dict(dscores=rows(8, 8)), EINVAL), (dict(dscores=rows(9, 8, F16)), EINVAL), (dict(opts=route(9)), EINVAL),
    (dict(scores=rows(9, 2000), dscores=rows(9, 2000)), EINVAL), (dict(dscores=rows(9, 8, data=A + 4)), EALIGN),
    (dict(experts=M + 2), EALIGN), (dict(dweights=M + 2), EALIGN), (dict(dsums=M + 2), EALIGN),
    (dict(scores=rows(1 << 28, 8), dscores=rows(1 << 28, 8)), TOOBIG),
    (dict(scores=rows(0, 8), dscores=rows(0, 8), experts=None), OK),
])
def test_route_grad_refusals(change, code):
    a = dict(dscores=rows(9, 8), scores=rows(9, 8), experts=M, dweights=D, dsums=None, opts=route(), stream=None)
    a.update(change)
    assert pkg.load().uccl_route_rows_grad(*a.values()) == code


def balance(tokens=9, slots=2, coef=0.1):
    return C.byref(pkg.uccl_balance_opts(tokens, slots, coef))


@pytest.mark.parametrize("change,code", [
    (dict(counts=None), EINVAL), (dict(sums=None), EINVAL), (dict(opts=None), EINVAL), (dict(opts=balance(0)), EINVAL), (dict(opts=balance(9, 0)), EINVAL),
    (dict(opts=balance(9, 2, NAN)), EINVAL), (dict(opts=balance(9, 2, -INF)), EINVAL), (dict(n=1 << 31), EINVAL),
    (dict(loss=M + 2), EALIGN), (dict(dsums=M + 1), EALIGN), (dict(counts=M + 2), EALIGN), (dict(sums=M + 2), EALIGN),
    (dict(loss=None, dsums=None), OK), (dict(loss=None, n=0, counts=None, sums=None), OK),
])
def test_balance_refusals(change, code):
    a = dict(loss=M, dsums=D, counts=M, sums=D, n=8, opts=balance(), stream=None)
    a.update(change)
    assert pkg.load().uccl_balance_loss(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(offsets=None), EINVAL), (dict(experts=None), EINVAL), (dict(n=0), EINVAL), (dict(n=1025), EINVAL), (dict(tokens=1 << 31, slots=1), EINVAL), (dict(tokens=1 << 20, slots=1 << 20), EINVAL),
    (dict(index=A), EINVAL), (dict(index=D), EINVAL),                      # where the experts are read, or the rows written
    (dict(index=M + 2), EALIGN), (dict(offsets=B + 1), EALIGN), (dict(pos=D + 2), EALIGN), (dict(experts=A + 2), EALIGN),
    (dict(tokens=9000), EINVAL), (dict(tokens=9000, scratch=S, scratch_bytes=64), EINVAL), (dict(tokens=9000, scratch=S + 4, scratch_bytes=1 << 20), EALIGN),
])
def test_plan_refusals(change, code):
    a = dict(index=M, offsets=B, pos=D, experts=A, tokens=9, slots=2, n=8, scratch=None, scratch_bytes=0, stream=None)
    a.update(change)
    assert pkg.load().uccl_plan_rows(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(q=None), EINVAL), (dict(x=None), EINVAL), (dict(q=q8(9, 70)), EINVAL), (dict(q=rows(9, 70)), EINVAL), (dict(x=q4(9, 70)), EINVAL), (dict(x=rows(9, 70, I32)), EINVAL),
    (dict(q=q4(8, 70)), EINVAL), (dict(q=q4(9, 71)), EINVAL), (dict(values=rows(9, 70, F16)), EINVAL), (dict(values=rows(9, 69)), EINVAL), (dict(q=q4(9, 70, scales=None)), EINVAL),
    (dict(q=q4(9, 70, stride=32)), EINVAL), (dict(q=q4(9, 70, scale_stride=0)), EINVAL), (dict(q=q4(9, 200, scale_stride=4), x=rows(9, 200)), EINVAL),
    (dict(q=q4(9, 70, data=A + 8)), EALIGN), (dict(q=q4(9, 70, stride=40)), EALIGN), (dict(q=q4(9, 70, scales=S + 2)), EALIGN), (dict(q=q4(9, 70, scale_stride=6)), EALIGN),
    (dict(x=rows(9, 70, data=A + 2)), EALIGN), (dict(values=rows(9, 70, stride=148)), EALIGN),
    (dict(q=q4(0, 70), x=rows(0, 70)), OK), (dict(q=q4(9, 0), x=rows(9, 0)), OK),
])
def test_quantise_refusals(change, code):
    a = dict(q=q4(9, 70), values=None, x=rows(9, 70), stream=None)
    a.update(change)
    assert pkg.load().uccl_quantise_rows(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(w=q4(12, 24)), EINVAL), (dict(w=q8(12, 16)), EINVAL), (dict(x=rows(7, 16, F32)), EINVAL), (dict(x=q8(7, 16)), EINVAL), (dict(x=q4(7, 16), w=rows(12, 16)), EINVAL),
    (dict(x=q4(7, 16), w=q8(12, 16)), EINVAL), (dict(x=q4(7, 16, scales=None)), EINVAL), (dict(w=q4(12, 16, scales=None)), EINVAL), (dict(y=q4(7, 3)), EINVAL),
    (dict(x=q4(7, 16, data=A + 8)), EALIGN), (dict(w=q4(12, 16, scales=S + 2)), EALIGN), (dict(w=q4(12, 16, scale_stride=2)), EALIGN), (dict(w=q4(12, 16, stride=8)), EALIGN),
    (dict(x=q4(6, 16)), EINVAL), (dict(n_groups=5), EINVAL), (dict(offsets=None), EINVAL),
    (dict(x=q4(0, 16), y=rows(0, 3), offsets=None), OK),
])
def test_product_refusals(change, code):
    a = dict(y=rows(7, 3), x=rows(7, 16), index=None, w=q4(12, 16), offsets=M, n_groups=4, stream=None)
    a.update(change)
    assert pkg.load().uccl_group_product(*a.values()) == code


def test_other_row_operators_do_not_take_4_bits():
    lib, eps = pkg.load(), C.byref(pkg.uccl_norm_opts(1e-6))
    assert lib.uccl_norm_rows(q4(2, 32), None, None, rows(2, 32), None, B, eps, None) == EINVAL
    assert lib.uccl_norm_rows(q4(2, 32), None, None, q4(2, 32), None, B, eps, None) == EINVAL
    assert lib.uccl_group_product_grad_x(rows(7, 16), rows(7, 3), q4(12, 16), M, 4, None) == EINVAL
    assert lib.uccl_group_product_grad_w(q4(12, 16), rows(7, 3), rows(7, 16), None, M, 4, None) == EINVAL
    assert lib.uccl_combine_rows(q4(4, 32), q4(9, 32), M, None, 2, None, None) == EINVAL


def many(*m):
    return (pkg.uccl_rows * len(m))(*[r._obj for r in m])


def clip(most=1.0, reserved=0):
    return C.byref(pkg.uccl_clip_opts(most, (C.c_uint32 * 3)(0, reserved, 0)))


SCRATCH = 1 << 20


@pytest.mark.parametrize("change,code", [
    (dict(norm=None), EINVAL), (dict(grads=None), EINVAL), (dict(n=1 << 31), EINVAL), (dict(scratch=None), EINVAL), (dict(scratch_bytes=32768), EINVAL),
    (dict(grads=many(rows(9, 8), q8(9, 8))), EINVAL), (dict(grads=many(rows(9, 8), q4(9, 32))), EINVAL), (dict(grads=many(rows(9, 8), rows(9, 8, data=None))), EINVAL),
    (dict(grads=many(rows(9, 8), rows(9, 8, data=A + 2))), EALIGN), (dict(grads=many(rows(9, 8), rows(9, 8, stride=20))), EALIGN), (dict(norm=M + 2), EALIGN), (dict(scratch=B + 8), EALIGN),
])
def test_gradient_norm_refusals(change, code):
    a = dict(norm=M, grads=many(rows(9, 8), rows(3, 5, F32)), n=2, scratch=B, scratch_bytes=SCRATCH, stream=None)
    a.update(change)
    assert pkg.load().uccl_gradient_norm(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(out=None), EINVAL), (dict(grads=None), EINVAL), (dict(norm=None), EINVAL), (dict(opts=None), EINVAL), (dict(opts=clip(0.0)), EINVAL), (dict(opts=clip(-1.0)), EINVAL),
    (dict(opts=clip(INF)), EINVAL), (dict(opts=clip(NAN)), EINVAL), (dict(opts=clip(1.0, 1)), EINVAL), (dict(out=many(rows(9, 8), rows(3, 6, F32))), EINVAL),
    (dict(out=many(rows(9, 8), rows(3, 5))), EINVAL), (dict(out=many(rows(9, 8), q8(3, 5))), EINVAL), (dict(out=many(rows(9, 8, data=A + 4), rows(3, 5, F32))), EALIGN), (dict(norm=M + 1), EALIGN),
    (dict(out=None, grads=None, n=0, norm=None), OK), (dict(out=many(rows(0, 8)), grads=many(rows(0, 8)), n=1), OK),
])
def test_gradient_clip_refusals(change, code):
    a = dict(out=many(rows(9, 8), rows(3, 5, F32)), grads=many(rows(9, 8), rows(3, 5, F32)), n=2, norm=M, opts=clip(), stream=None)
    a.update(change)
    assert pkg.load().uccl_gradient_clip(*a.values()) == code


def test_scratch_sizes():
    f, g, h = pkg.uccl_route_rows_scratch, pkg.uccl_plan_rows_scratch, pkg.uccl_gradient_norm_scratch
    assert f(0, 8) == f(32, 8) == 0 and f(33, 8) == 2 * 8 * 8 and f(1 << 31, 1024) == 512 * 8 * 1024
    assert g(0, 8) == 0 and g(1 << 30, 1024) <= 1 << 20 and g(1 << 20, 3) % 16 == 0
    assert h(0) > 0 and h(1000) - h(0) >= 8000 and h(7) % 16 == 0


def test_the_binding_refuses_what_only_the_tensors_know():
    """On CPU tensors: every call here raises before the library is asked."""
    import torch
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)      # noqa: E731
    f = torch.zeros
    b4 = lambda *s: torch.zeros(*s, dtype=torch.uint8).view(torch.float4_e2m1fn_x2)  # noqa: E731
    s8 = lambda *s: torch.zeros(*s, dtype=torch.uint8).view(torch.float8_e8m0fnu)    # noqa: E731
    for call in (
        lambda: pkg.uccl_route_rows(i(3, 2), f(3, 2), bf(4, 8), stream=0),
        lambda: pkg.uccl_route_rows(i(4, 2), f(4, 3), bf(4, 8), stream=0),
        lambda: pkg.uccl_route_rows(i(8), f(4, 2), bf(4, 8), stream=0),
        lambda: pkg.uccl_route_rows(i(4, 2).long(), f(4, 2), bf(4, 8), stream=0),
        lambda: pkg.uccl_route_rows(f(4, 2), f(4, 2), bf(4, 8), stream=0),
        lambda: pkg.uccl_route_rows(i(4, 4)[:, ::2], f(4, 2), bf(4, 8), stream=0),
        lambda: pkg.uccl_route_rows(i(4, 2), f(4, 2), bf(4, 8), bias=f(7), stream=0),
        lambda: pkg.uccl_route_rows(i(4, 2), f(4, 2), bf(4, 8), bias=bf(8), stream=0),
        lambda: pkg.uccl_route_rows(i(4, 2), f(4, 2), bf(4, 8), counts=i(9), stream=0),
        lambda: pkg.uccl_route_rows(i(4, 2), f(4, 2), bf(8, 4).t(), stream=0),
        lambda: pkg.uccl_route_rows_grad(bf(4, 8), bf(4, 8), i(4, 2), f(4, 3), stream=0),
        lambda: pkg.uccl_route_rows_grad(bf(4, 8), bf(4, 8), i(4, 2), f(4, 2), dsums=f(9), stream=0),
        lambda: pkg.uccl_balance_loss(f(1), f(8), i(8), f(9), 4, 2, 0.1, stream=0),
        lambda: pkg.uccl_balance_loss(f(2), f(8), i(8), f(8), 4, 2, 0.1, stream=0),
        lambda: pkg.uccl_plan_rows(i(7), i(9), i(4, 2), i(4, 2), stream=0),
        lambda: pkg.uccl_plan_rows(i(8), i(9), i(4, 2), i(8), stream=0),
        lambda: pkg.uccl_plan_rows(i(8), f(9), i(4, 2), i(4, 2), stream=0),
        lambda: pkg.uccl_quantise_rows(b4(4, 34), s8(4, 3), bf(4, 70), stream=0),
        lambda: pkg.uccl_quantise_rows(b4(4, 35), s8(4, 2), bf(4, 70), stream=0),
        lambda: pkg.uccl_quantise_rows(b4(4, 35), f(4, 3), bf(4, 70), stream=0),
        lambda: pkg.uccl_quantise_rows(b4(4, 35), s8(12), bf(4, 70), stream=0),
        lambda: pkg.uccl_quantise_rows(b4(4, 35), s8(3, 4).t(), bf(4, 70), stream=0),
        lambda: pkg.uccl_group_product(bf(4, 3), bf(4, 70), b4(2, 3, 34), i(3), w_scales=s8(2, 3, 3), stream=0),
        lambda: pkg.uccl_group_product(bf(4, 3), bf(4, 70), b4(2, 3, 35), i(3), w_scales=s8(2, 3, 2), stream=0),
        lambda: pkg.uccl_gradient_norm(f(2), [f(4)], f(100), stream=0),
        lambda: pkg.uccl_gradient_norm(f(1), [f(4).double()], f(100), stream=0),
        lambda: pkg.uccl_gradient_norm(f(1), [f(4, 4).t()[:2]], f(100), stream=0),
        lambda: pkg.uccl_gradient_clip([f(4)], [f(4), f(4)], f(1), 1.0, stream=0),
        lambda: pkg.uccl_gradient_clip([f(5)], [f(4)], f(1), 1.0, stream=0),
        lambda: pkg.uccl_gradient_clip([bf(4)], [f(4)], f(1), 1.0, stream=0),
    ):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(pkg.UcclError) as e:
        pkg.uccl_route_rows(i(4, 9), f(4, 9), bf(4, 8), stream=0)
    assert e.value.code == EINVAL


def test_tensors_are_read_as_the_interpreter_reads_them(monkeypatch):
    """By the extension and without it: matrices, vectors and lists, and what neither takes."""
    import torch
    from paper_2504_17307_amd import experts, rows as r
    reader = r._find_reader()
    assert reader
    matrices = [torch.zeros(s, dtype=t) for s in ((3, 8), (1, 7), (0, 4), (4, 0), (2, 3, 8), (2, 1, 5), (1, 1, 1)) for t in (torch.float32, torch.bfloat16, torch.float16)]
    matrices += [torch.zeros(6, 16)[::2, :5], torch.zeros(4, 6, 8)[:, :1], torch.zeros(2, 4, 8)[1:, :2], torch.zeros(9, 1).expand(9, 1), torch.nn.Parameter(torch.zeros(3, 4)), torch.zeros(5, 8).t()[:1].t()]
    vectors = [torch.zeros(7), torch.zeros(7, dtype=torch.int32), torch.zeros(7, 1), torch.zeros(14)[::2], torch.zeros(7, dtype=torch.float64), torch.zeros(7, dtype=torch.int64), torch.zeros(6), torch.zeros(7, dtype=torch.uint32)]
    lists = [[torch.zeros(3, 4), torch.zeros(5, dtype=torch.bfloat16)], [torch.zeros(()), torch.zeros(0)], [torch.nn.Parameter(torch.zeros(3)), torch.zeros(3)], [torch.zeros(8, 8)[:, :4]], [torch.zeros(4, dtype=torch.float16)] * 3, []]
    kept = [list(x) for x in lists]

    def answers():
        got = []
        for call in [lambda m=m: r._rows(m) for m in matrices] + [lambda v=v, k=k: r._vector(v, k, 7, "v") for v in vectors for k in "if"] + [lambda x=x: experts._matrices(x) for x in lists] + [lambda x=x, k=k: experts._matrices(x, [t.detach().clone() for t in kept[k]])[::2] for k, x in enumerate(lists)]:
            try:
                got.append(call())
            except ValueError as e:
                got.append(str(e))
        return got
    fast = answers()
    monkeypatch.setattr(r, "_reader", False)
    assert fast == answers()
    for thing in (None, 3, "x", [1], object()):                              # not taken for tensors
        assert reader.matrix_rows(thing) is None and reader.vector_address(thing, False, 7) is None and reader.contiguous_rows([thing], [thing], 9) is None


@pytest.mark.parametrize("reads", [True, False])
def test_lists_of_tensors_are_no_iterators(monkeypatch, reads):
    """Whatever can be gone through again is taken whole; an iterator, which cannot, and of which a prepared call would hold nothing, is refused."""
    import torch
    from paper_2504_17307_amd import experts, rows as r
    r._find_reader()
    if not reads:
        monkeypatch.setattr(r, "_reader", False)
    grads = [torch.ones(5) * k for k in range(5)]
    want = experts._matrices(grads)
    assert want[2] == 5
    for again in (tuple(grads), dict(enumerate(grads)).values(), torch.nn.ParameterList(grads)):
        assert experts._matrices(again)[2] == 5 and (again.__class__ is torch.nn.ParameterList or experts._matrices(again) == want)
    f = torch.zeros
    for once in (lambda: iter(grads), lambda: (g for g in grads), lambda: map(torch.clone, grads), lambda: iter([])):
        for call in (lambda: pkg.uccl_gradient_norm(f(1), once(), f(100), stream=0), lambda: pkg.uccl_prepare(pkg.uccl_gradient_norm, f(1), once(), f(100), stream=0),
                     lambda: experts._matrices(grads, once()), lambda: experts._matrices(once(), grads)):
            with pytest.raises(ValueError):
                call()
        for outs, of in ((grads, once()), (once(), grads), (once(), once())):
            with pytest.raises((ValueError, TypeError)):
                pkg.uccl_gradient_clip(outs, of, f(1), 1.0, stream=0)


@pytest.mark.parametrize("missing", [("float4_e2m1fn_x2", "float8_e8m0fnu"), ("float4_e2m1fn_x2",), ("float8_e8m0fnu",)])
def test_rows_of_other_types_need_no_torch_with_4_bits(monkeypatch, missing):
    import torch
    from paper_2504_17307_amd import rows as r
    tensors = [torch.zeros(4, 32, dtype=t) for t in (torch.float32, torch.bfloat16, torch.float16)]
    eight, four = torch.zeros(4, 32, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(4, 16, dtype=torch.uint8).view(torch.float4_e2m1fn_x2)
    want = [r._rows(t) for t in tensors] + [r._rows(eight, torch.zeros(4))[4 * 8:]]
    monkeypatch.setattr(r, "_types", {})
    monkeypatch.setattr(r, "_reader", False)
    for name in missing:
        monkeypatch.delattr(torch, name)
    assert [r._rows(t) for t in tensors] + [r._rows(eight, torch.zeros(4))[4 * 8:]] == want
    with pytest.raises(ValueError):
        r._rows(four, torch.zeros(4, 1, dtype=torch.uint8))


@pytest.mark.parametrize("extension", [True, False])
def test_a_prepared_call_keeps_the_tensors_of_its_lists(monkeypatch, extension):
    """Also when the lists hold others by then: the call has the addresses of those that it was prepared with."""
    import gc
    import weakref
    import torch
    if not extension:
        monkeypatch.setattr(pkg, "_extension", False)
    make = lambda: [torch.zeros(64) for _ in range(3)]  # noqa: E731
    outs, grads, norm = make(), make(), torch.zeros(1)
    for prepare in (lambda: pkg.uccl_prepare(pkg.uccl_gradient_clip, outs, grads, norm, 1.0, stream=0), lambda: pkg.uccl_prepare(pkg.uccl_gradient_norm, norm, grads=grads, scratch=torch.zeros(1 << 16), stream=0)):
        outs[:], grads[:] = make(), make()
        call = prepare()
        there = [weakref.ref(t) for t in (grads + outs if "clip" in call.__name__ else grads)]
        outs.clear(), grads.clear()
        gc.collect()
        assert all(t() is not None for t in there)
        del call
        gc.collect()
        assert all(t() is None for t in there)


def test_kernels_use_no_scratch_memory(tmp_path):
    """The library's code objects of routing and clipping, and of 4 bits."""
    lib, at, blocks = open(pkg.LIB_PATH, "rb").read(), -1, []
    while (at := lib.find(b"__CLANG_OFFLOAD_BUNDLE__", at + 1)) >= 0:
        n, = struct.unpack_from("<Q", lib, at + 24)
        entry = at + 32
        for _ in range(n):
            off, size, length = struct.unpack_from("<QQQ", lib, entry)
            if b"gfx950" in lib[entry + 24:entry + 24 + length]:
                path = tmp_path / f"{at}.elf"
                path.write_bytes(lib[at + off:at + off + size])
                blocks.append(subprocess.run(["/opt/rocm/llvm/bin/llvm-readelf", "--notes", str(path)], capture_output=True, text=True, check=True).stdout)
            entry += 24 + length
    for part in ("route_kernel", "quantise_kernel"):
        notes, = [b for b in blocks if part in b]
        assert set(re.findall(r"\.private_segment_fixed_size: +(\d+)", notes)) == {"0"}
        assert set(re.findall(r"\.vgpr_spill_count: +(\d+)", notes)) == {"0"}


# ---- what the library is asked to launch: the HIP runtime of tests/hip_stub.c reports it, nothing runs --------------------------------

START, STOP, BAD = 0x6000, 0x7000, 0x5000
SHAPES = [(1500, 2, 1030, 4000), (700, 5, 520, 2600), (4500, 3, 2060, 1300), (90, 3, 200, 5000), (1300, 1, 4100, 1500), (400, 1, 1900, 3000), (6000, 1, 4200, 900), (4300, 2, 2040, 1000)]   # of tests/test_gpu_experts.py


def in_process(scenario, tmp_path):
    stub = str(tmp_path / "libamdhip64.so.7")
    subprocess.check_call(["gcc", "-O1", "-shared", "-fPIC", "-w", "-I/opt/rocm/include", "-Wl,-soname,libamdhip64.so.7", os.path.join(HERE, "hip_stub.c"), "-o", stub])
    r = subprocess.run([sys.executable, os.path.abspath(__file__), scenario, stub], cwd=os.path.dirname(HERE), capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "SCENARIO DONE" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
    return r.stdout


def product(rt, kind, n, groups, wide, cols):
    make = {"mx4": q4, "bf16": rows, "f16": lambda n, c: rows(n, c, F16)}[kind]
    rt.symbols.clear()
    assert rt.lib.uccl_group_product(rows(n, wide), make(n, cols), None, q4(groups * wide, cols), M, groups, None) == OK
    (symbol,), shape = rt.symbols, re.compile(r"(few|tile|wide)_kernelI(?:LNS_7Mx4RowsE\d|Lb\d)?E?Lj(\d+)ELj(\d+)E")
    return shape.search(symbol).groups()


def product_kernels(rt):
    """Rows of a tile, or columns of one of 16 rows, by what is multiplied; the shapes of the GPU's tests and those that were measured."""
    few, least, lower, small, middle, large, wide = ("few", "32", "4"), ("tile", "64", "64"), ("tile", "64", "128"), ("tile", "128", "128"), ("tile", "192", "256"), ("tile", "256", "256"), ("wide", "128", "256")
    few16, few64, least16, low, square = ("few", "16", "4"), ("few", "64", "4"), ("wide", "64", "64"), ("wide", "64", "128"), ("wide", "128", "128")
    for shape, four, bf16, f16 in zip(SHAPES, (lower, least, middle, few, small, least, large, middle), (low, least16, square, few16, wide, least16, wide, square), (low, few64, square, few16, wide, least16, wide, square)):
        assert [product(rt, kind, *shape) for kind in ("mx4", "bf16", "f16")] == [four, bf16, f16], shape
    for shape, four, sixteen in (((500, 1, 520, 600), least, least16), ((1500, 2, 1030, 600), lower, low), ((150, 8, 1000, 2600), few, few64)):
        assert [product(rt, kind, *shape) for kind in ("mx4", "bf16", "f16")] == [four, sixteen, sixteen], shape
    for shape, four, sixteen in (((16, 32, 2048, 7168), few, few64), ((128, 32, 2048, 7168), few, few64), ((1, 1, 2048, 7168), few, few16), ((300, 8, 2048, 7168), least, least16), ((1000, 16, 2048, 7168), small, square),
                                 ((4096, 16, 2048, 7168), middle, square), ((4000, 4, 2048, 7168), small, wide), ((8190, 16, 7168, 2048), large, wide), ((2999, 24, 1003, 2044), small, low), ((500, 8, 2048, 7168), lower, low), ((8192, 1, 8192, 8192), large, wide)):
        assert [product(rt, kind, *shape) for kind in ("mx4", "bf16")] == [four, sixteen], (shape, product(rt, "mx4", *shape), product(rt, "bf16", *shape))
    # narrow outputs of very many rows: by 16 rows while that fits a launch, by tiles where these do, refused where nothing does
    for n, kind in ((1 << 26, "few"), ((1 << 29) - 1024, None)):
        for x in ("mx4", "bf16"):
            assert (product(rt, x, n, 1, 5, 500)[0] == "few") == (kind == "few")
    rt.launches.clear()
    big = (1 << 31) - 1
    assert rt.lib.uccl_group_product(rows(big, 8 << 20), q4(big, 64), None, q4(8 << 20, 64), M, 1, None) == TOOBIG and rt.launches == []


def test_which_kernel_a_product_is_launched_as(tmp_path):
    in_process("product_kernels", tmp_path)


def one_round_of_small_tiles(rt):
    """64 x 64 while every tile of one group has a compute unit."""
    for rows, wide, small in ((1024, 1024, True), (1024, 1088, False), (832, 1280, False), (256, 4224, False), (256, 4096, True)):
        for cols in (512, 2048, 5000):
            for kind in ("mx4", "bf16", "f16"):
                assert (product(rt, kind, rows, 1, wide, cols)[1:] == ("64", "64")) == small, (kind, rows, wide, cols)


def test_one_round_of_small_tiles(tmp_path):
    in_process("one_round_of_small_tiles", tmp_path)


def timing_events(rt):
    """A call's start event is on its first launch and its stop on its last; what HIP refuses comes back."""
    events = []
    rt.refuse = lambda kernel, stream, start, stop: bool(events.append((start, stop)))
    lib, grads = rt.lib, many(*[rows(5, 8) for _ in range(130)])
    most, gaps = many(*[rows(5, 8) for _ in range(320)]), many(rows(1, 9), *[rows(5, 8, stride=32) for _ in range(130)])
    calls = {
        "route": (1, lambda: lib.uccl_route_rows(M, D, None, None, rows(9000, 8), None, route(), None, 0, None)),
        "route, one group's sums": (1, lambda: lib.uccl_route_rows(M, D, M, D, rows(9, 8), None, route(), None, 0, None)),
        "route with sums": (2, lambda: lib.uccl_route_rows(M, D, M, D, rows(9000, 8), None, route(), B, 1 << 20, None)),
        "sums of nothing": (1, lambda: lib.uccl_route_rows(None, None, M, D, rows(0, 8), None, route(), None, 0, None)),
        "route_grad": (1, lambda: lib.uccl_route_rows_grad(rows(9, 8), rows(9, 8), M, D, None, route(), None)),
        "balance": (1, lambda: lib.uccl_balance_loss(M, D, M, D, 8, balance(), None)),
        "plan": (1, lambda: lib.uccl_plan_rows(M, B, D, A, 9, 2, 8, None, 0, None)),
        "plan of many": (2, lambda: lib.uccl_plan_rows(M, B, D, A, 90000, 2, 8, S, 1 << 20, None)),
        "quantise": (1, lambda: lib.uccl_quantise_rows(q4(9, 70), None, rows(9, 70), None)),
        "product": (1, lambda: lib.uccl_group_product(rows(9, 3), q4(9, 64), None, q4(12, 64), M, 4, None)),
        "norm": (2, lambda: lib.uccl_gradient_norm(M, grads, 130, B, 1 << 20, None)),
        "norm of nothing": (1, lambda: lib.uccl_gradient_norm(M, None, 0, B, 1 << 20, None)),
        "clip": (1, lambda: lib.uccl_gradient_clip(grads, grads, 130, M, clip(), None)),
        "norm of many": (4, lambda: lib.uccl_gradient_norm(M, most, 320, B, 1 << 20, None)),
        "clip of many": (3, lambda: lib.uccl_gradient_clip(most, most, 320, M, clip(), None)),
        "clip of rows with gaps": (4, lambda: lib.uccl_gradient_clip(gaps, gaps, 131, M, clip(), None)),
    }
    for name, (launches, call) in calls.items():
        events.clear()
        assert lib.uccl_time_next_launch(START, STOP) == OK and call() == OK, name
        assert len(events) == launches and events[0][0] == START and events[-1][1] == STOP and not any(start for start, _ in events[1:]), (name, events)
        events.clear()
        assert call() == OK and not any(map(any, events)), (name, events)   # once only
    rt.refuse = lambda kernel, stream, start, stop: BAD in (start, stop)
    for name, (launches, call) in calls.items():
        for start, stop in ((START, BAD), (BAD, STOP)):
            rt.launches.clear()
            assert lib.uccl_time_next_launch(start, stop) == OK and call() == pkg.UCCL_ELAUNCH and not rt.launches, name
    rt.refuse = lambda *a: True
    for name, (_, call) in calls.items():
        assert call() == pkg.UCCL_ELAUNCH, name
    assert b"as the test asked" in lib.uccl_last_error_detail()


def test_timing_events_span_a_call_of_several_launches(tmp_path):
    in_process("timing_events", tmp_path)


if __name__ == "__main__":
    import test_host_launches
    runtime = test_host_launches.Runtime(sys.argv[2])
    for name, (res, args) in {**pkg.ROWS_SIGNATURES, **pkg.EXPERTS_SIGNATURES}.items():
        fn = getattr(runtime.lib, name)
        fn.restype, fn.argtypes = res, args
    globals()[sys.argv[1]](runtime)
    print("SCENARIO DONE")
