"""The row operators' C ABI without a GPU: exports, layouts, and refusals, which come before anything is enqueued."""
import ctypes as C
import re
import struct
import subprocess

import pytest

import paper_2504_17307_amd as pkg

F32, BF16, F16, I32, E4M3 = pkg.UCCL_F32, pkg.UCCL_BF16, pkg.UCCL_F16, pkg.UCCL_I32, pkg.UCCL_E4M3
SIZE = {F32: 4, BF16: 2, F16: 2, E4M3: 1, I32: 4, 9: 4}
A, B, D, M, S = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000   # never dereferenced: every call fails on the host, or has nothing to do


def rows(n, cols, dtype=BF16, data=A, stride=None, scales=None, scale_stride=4, reserved=0):
    stride = -(-cols * SIZE[dtype] // 16) * 16 if stride is None else stride
    return C.byref(pkg.uccl_rows(data, stride, scales, scale_stride, n, cols, dtype, reserved))


def q8(n, cols, **kw):
    return rows(n, cols, E4M3, scales=S, **kw)


def test_every_declared_function_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(pkg.ROWS_HEADER_PATH).read(), flags=re.S)
    names = set(re.findall(r"\b(uccl_[a-z_]+)\s*\(", text))
    assert names == set(pkg.ROWS_SIGNATURES) and len(names) == 8
    lib = pkg.load()
    for n in names:
        assert hasattr(lib, n) and hasattr(pkg, n), n
    assert C.sizeof(pkg.uccl_rows) == 48
    assert [getattr(pkg.uccl_rows, f).offset for f, _ in pkg.uccl_rows._fields_] == [0, 8, 16, 24, 32, 36, 40, 44]
    assert "#define UCCL_E4M3 %d" % E4M3 in open(pkg.ROWS_HEADER_PATH).read()


OK, EINVAL, EALIGN = pkg.UCCL_OK, pkg.UCCL_EINVAL, pkg.UCCL_EALIGN


@pytest.mark.parametrize("y,h,rstd,x,r,weight,eps,code", [
    (None, None, None, rows(2, 8), None, B, 1e-6, EINVAL),
    (rows(2, 8), None, None, None, None, B, 1e-6, EINVAL),
    (rows(2, 8), None, None, rows(2, 8, data=None), None, B, 1e-6, EINVAL),
    (rows(2, 8), None, None, rows(2, 8), None, None, 1e-6, EINVAL),
    (rows(2, 8), None, None, rows(2, 9), None, B, 1e-6, EINVAL),               # shapes
    (rows(3, 8), None, None, rows(2, 8), None, B, 1e-6, EINVAL),
    (rows(2, 8), rows(2, 7), None, rows(2, 8), None, B, 1e-6, EINVAL),
    (rows(2, 8), None, None, rows(2, 8), rows(1, 8), B, 1e-6, EINVAL),
    (rows(2, 8, F16), None, None, rows(2, 8), None, B, 1e-6, EINVAL),          # types
    (rows(2, 8), rows(2, 8, F32), None, rows(2, 8), None, B, 1e-6, EINVAL),
    (rows(2, 8), None, None, rows(2, 8), rows(2, 8, F16), B, 1e-6, EINVAL),
    (rows(2, 8, I32), None, None, rows(2, 8, I32), None, B, 1e-6, EINVAL),
    (rows(2, 8, 9), None, None, rows(2, 8, 9), None, B, 1e-6, EINVAL),
    (q8(2, 16), None, None, q8(2, 16), None, B, 1e-6, EINVAL),
    (rows(2, 8, E4M3), None, None, rows(2, 8), None, B, 1e-6, EINVAL),         # no scales
    (rows(2, 8, scales=S), None, None, rows(2, 8), None, B, 1e-6, EINVAL),     # scales that no type has
    (rows(2, 8), None, None, rows(2, 8, reserved=1), None, B, 1e-6, EINVAL),
    (rows(2, 8), None, None, rows(2, 8), None, B, -1.0, EINVAL),
    (rows(2, 8), None, None, rows(2, 8), None, B, float("nan"), EINVAL),
    (rows(2, 8), None, None, rows(2, 8), None, B, float("inf"), EINVAL),
    (rows(2, 9, stride=16), None, None, rows(2, 9), None, B, 1e-6, EINVAL),    # rows overlap
    (rows(2, 8, data=A + 8), None, None, rows(2, 8), None, B, 1e-6, EALIGN),
    (rows(2, 8, stride=24), None, None, rows(2, 8), None, B, 1e-6, EALIGN),
    (rows(2, 8), None, None, rows(2, 8), rows(2, 8, data=A + 2), B, 1e-6, EALIGN),
    (rows(2, 8), None, None, rows(2, 8), None, B + 8, 1e-6, EALIGN),
    (rows(2, 8), None, D + 2, rows(2, 8), None, B, 1e-6, EALIGN),
    (rows(2, 8, E4M3, scales=S + 2), None, None, rows(2, 8), None, B, 1e-6, EALIGN),
    (q8(2, 8, scale_stride=6), None, None, rows(2, 8), None, B, 1e-6, EALIGN),
    (rows(0, 8), None, None, rows(0, 8, data=None), None, None, 1e-6, OK),
    (rows(2, 0), None, None, rows(2, 0, data=None), None, None, 1e-6, OK),
    (rows(1 << 31, 8), None, None, rows(1 << 31, 8), None, B, 1e-6, EINVAL),
    (rows(1, (1 << 30) + 8), None, None, rows(1, (1 << 30) + 8), None, B, 1e-6, EINVAL),
])
def test_norm_refusals(y, h, rstd, x, r, weight, eps, code):
    assert pkg.load().uccl_norm_rows(y, h, rstd, x, r, weight, C.byref(pkg.uccl_norm_opts(eps)), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(dx=None), EINVAL), (dict(dy=None), EINVAL), (dict(h=None), EINVAL), (dict(rstd=None), EINVAL), (dict(weight=None), EINVAL),
    (dict(scratch=None), EINVAL), (dict(scratch_bytes=4 * 2 * 8 - 1), EINVAL), (dict(dweight=None), EINVAL),
    (dict(dx=rows(2, 8, F32)), EINVAL), (dict(dy=rows(2, 8, F16)), EINVAL), (dict(dh=rows(2, 8, F16)), EINVAL),
    (dict(dx=rows(1, 8)), EINVAL), (dict(dy=rows(2, 9)), EINVAL), (dict(dh=rows(3, 8)), EINVAL),
    (dict(dx=rows(2, 8, data=A + 4)), EALIGN), (dict(dh=rows(2, 8, stride=40)), EALIGN), (dict(rstd=D + 1), EALIGN),
    (dict(weight=B + 8), EALIGN), (dict(scratch=S + 8), EALIGN), (dict(dweight=M + 2), EALIGN),
    (dict(dx=rows(2, 0), dy=rows(2, 0), h=rows(2, 0)), OK),
])
def test_norm_grad_refusals(change, code):
    a = dict(dx=rows(2, 8), dweight=M, dy=rows(2, 8), dh=None, h=rows(2, 8), rstd=D, weight=B, scratch=S, scratch_bytes=64, stream=None, **{})
    a.update(change)
    assert pkg.load().uccl_norm_rows_grad(*a.values()) == code


def test_norm_options_are_wanted_and_what_is_reserved_is_0():
    f, o = pkg.load().uccl_norm_rows, pkg.uccl_norm_opts(1e-6)
    o.reserved[2] = 1
    for opts in (None, C.byref(o)):
        assert f(rows(2, 8), None, None, rows(2, 8), None, B, opts, None) == EINVAL


def test_norm_grad_scratch_grows_with_the_rows_up_to_a_limit():
    f = pkg.uccl_norm_rows_scratch
    assert f(0, 8) == f(8, 0) == 0 and f(1, 3) == 16 and f(2, 8) == 64
    assert f(1 << 30, 7168) == f(1 << 20, 7168) < 1 << 26 and f(1 << 20, 7168) % 16 == 0


@pytest.mark.parametrize("change,code", [
    (dict(y=None), EINVAL), (dict(x=None), EINVAL), (dict(w=None), EINVAL), (dict(offsets=None), EINVAL),
    (dict(n_groups=0), EINVAL), (dict(n_groups=5), EINVAL),                               # 12 rows of weights
    (dict(y=rows(7, 4)), EINVAL), (dict(w=rows(12, 24)), EINVAL), (dict(x=rows(7, 24)), EINVAL),
    (dict(x=rows(6, 16)), EINVAL),                                                        # fewer rows than y, and no index
    (dict(x=rows(7, 16, F32), w=rows(12, 16, F32)), EINVAL), (dict(w=rows(12, 16, F16)), EINVAL),
    (dict(y=rows(7, 3, I32)), EINVAL), (dict(y=q8(7, 3)), EINVAL), (dict(x=q8(7, 16)), EINVAL),
    (dict(x=rows(7, 16, E4M3), w=q8(12, 16)), EINVAL), (dict(x=q8(7, 16), w=rows(12, 16, E4M3)), EINVAL),
    (dict(x=rows(7, 16, data=A + 8)), EALIGN), (dict(w=rows(12, 16, stride=40)), EALIGN), (dict(y=rows(7, 3, data=D + 4)), EALIGN),
    (dict(offsets=M + 2), EALIGN), (dict(index=B + 1), EALIGN),
    (dict(y=rows(0, 3), x=rows(0, 16), offsets=None), OK), (dict(y=rows(7, 0), w=rows(0, 16)), OK),
    (dict(y=rows(7, 3), w=rows(0, 16), n_groups=0, offsets=None), OK),
])
def test_product_refusals(change, code):
    a = dict(y=rows(7, 3), x=rows(7, 16), index=None, w=rows(12, 16), offsets=M, n_groups=4, stream=None)
    a.update(change)
    assert pkg.load().uccl_group_product(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(dx=None), EINVAL), (dict(dy=None), EINVAL), (dict(w=None), EINVAL), (dict(offsets=None), EINVAL), (dict(n_groups=5), EINVAL),
    (dict(dx=rows(6, 16)), EINVAL), (dict(dx=rows(7, 15)), EINVAL), (dict(dy=rows(7, 4)), EINVAL), (dict(w=rows(12, 8)), EINVAL),
    (dict(dy=q8(7, 3), w=q8(12, 16)), EINVAL), (dict(dy=rows(7, 3, F16)), EINVAL), (dict(dy=rows(7, 3, F32), w=rows(12, 16, F32)), EINVAL),
    (dict(dx=q8(7, 16)), EINVAL), (dict(dx=rows(7, 16, data=A + 2)), EALIGN), (dict(dy=rows(7, 3, stride=24)), EALIGN), (dict(offsets=M + 1), EALIGN),
    (dict(dx=rows(0, 16), dy=rows(0, 3), offsets=None), OK),
])
def test_product_grad_x_refusals(change, code):
    a = dict(dx=rows(7, 16), dy=rows(7, 3), w=rows(12, 16), offsets=M, n_groups=4, stream=None)
    a.update(change)
    assert pkg.load().uccl_group_product_grad_x(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(dw=None), EINVAL), (dict(dy=None), EINVAL), (dict(x=None), EINVAL), (dict(offsets=None), EINVAL), (dict(n_groups=5), EINVAL),
    (dict(dw=rows(12, 17)), EINVAL), (dict(dy=rows(7, 4)), EINVAL), (dict(x=rows(6, 16)), EINVAL), (dict(x=rows(7, 16, F16)), EINVAL),
    (dict(dy=q8(7, 3), x=q8(7, 16)), EINVAL), (dict(dw=q8(12, 16)), EINVAL), (dict(dw=rows(12, 16, data=A + 2)), EALIGN),
    (dict(index=B + 2), EALIGN), (dict(offsets=M + 2), EALIGN), (dict(dw=rows(0, 16), dy=rows(7, 0)), OK),
    (dict(dy=rows(0, 3), x=rows(0, 16), offsets=None), EINVAL),                            # the zeros still need to know the groups
])
def test_product_grad_w_refusals(change, code):
    a = dict(dw=rows(12, 16), dy=rows(7, 3), x=rows(7, 16), index=None, offsets=M, n_groups=4, stream=None)
    a.update(change)
    assert pkg.load().uccl_group_product_grad_w(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(out=None), EINVAL), (dict(y=None), EINVAL), (dict(pos=None), EINVAL), (dict(y=rows(9, 15)), EINVAL), (dict(y=rows(9, 16, F16)), EINVAL),
    (dict(r=rows(3, 16)), EINVAL), (dict(r=rows(4, 16, F32)), EINVAL), (dict(out=q8(4, 16), y=q8(9, 16)), EINVAL), (dict(slots=1 << 31), EINVAL),
    (dict(out=rows(4, 16, data=A + 2)), EALIGN), (dict(pos=M + 2), EALIGN), (dict(weights=M + 2), EALIGN), (dict(r=rows(4, 16, stride=40)), EALIGN),
    (dict(out=rows(0, 16), pos=None), OK), (dict(out=rows(4, 0), y=rows(9, 0)), OK),
])
def test_combine_refusals(change, code):
    a = dict(out=rows(4, 16), y=rows(9, 16), pos=M, weights=D, slots=2, r=None, stream=None)
    a.update(change)
    assert pkg.load().uccl_combine_rows(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(dy=None), EINVAL), (dict(dout=None), EINVAL), (dict(y=None), EINVAL), (dict(pos=None), EINVAL), (dict(dy=rows(8, 16)), EINVAL),
    (dict(dy=rows(9, 16, F32)), EINVAL), (dict(dout=rows(4, 15)), EINVAL), (dict(dout=rows(4, 16, F16)), EINVAL),
    (dict(dweights=D + 2), EALIGN), (dict(pos=M + 1), EALIGN), (dict(weights=M + 3), EALIGN), (dict(dy=rows(9, 16, data=A + 4)), EALIGN),
    (dict(dout=rows(0, 16), pos=None), OK), (dict(slots=0), OK),
])
def test_combine_grad_refusals(change, code):
    a = dict(dy=rows(9, 16), dweights=D, dout=rows(4, 16), y=rows(9, 16), pos=M, weights=S, slots=2, stream=None)
    a.update(change)
    assert pkg.load().uccl_combine_rows_grad(*a.values()) == code


def test_the_binding_refuses_what_only_the_tensors_know():
    """On CPU tensors: every call here raises before the library is asked."""
    import torch
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)    # noqa: E731
    w, off = bf(4, 3, 16), i32(5)
    for call in (
        lambda: pkg.uccl_norm_rows(bf(2, 8), bf(2, 8), bf(7), 1e-6, stream=0),
        lambda: pkg.uccl_norm_rows(bf(2, 8), bf(2, 8), torch.zeros(8), 1e-6, stream=0),
        lambda: pkg.uccl_norm_rows(bf(2, 8), bf(8, 2).t(), bf(8), 1e-6, stream=0),
        lambda: pkg.uccl_norm_rows(bf(2, 8), bf(2, 8), bf(8), 1e-6, rstd=torch.zeros(3), stream=0),
        lambda: pkg.uccl_norm_rows(bf(2, 8), bf(8), bf(8), 1e-6, stream=0),
        lambda: pkg.uccl_norm_rows(torch.zeros(2, 8, dtype=torch.float64), torch.zeros(2, 8, dtype=torch.float64), bf(8), 1e-6, stream=0),
        lambda: pkg.uccl_norm_rows(torch.zeros(2, 8, dtype=torch.float8_e4m3fn), bf(2, 8), bf(8), 1e-6, scales=torch.zeros(3), stream=0),
        lambda: pkg.uccl_group_product(bf(7, 3), bf(7, 16), w, i32(4), stream=0),
        lambda: pkg.uccl_group_product(bf(7, 3), bf(7, 16), w, torch.zeros(5), stream=0),
        lambda: pkg.uccl_group_product(bf(7, 3), bf(7, 16), w, i32(10)[::2], stream=0),
        lambda: pkg.uccl_group_product(bf(7, 3), bf(7, 16), w, torch.zeros(5, dtype=torch.int64), stream=0),
        lambda: pkg.uccl_group_product(bf(7, 3), bf(9, 16), w, off, index=i32(9), stream=0),
        lambda: pkg.uccl_group_product(bf(7, 3), bf(7, 16), bf(8, 3, 16)[::2], off, stream=0),
        lambda: pkg.uccl_combine_rows(bf(4, 16), bf(9, 16), i32(3, 2), stream=0),
        lambda: pkg.uccl_combine_rows(bf(4, 16), bf(9, 16), i32(4, 2), weights=torch.zeros(4, 3), stream=0),
        lambda: pkg.uccl_combine_rows_grad(bf(9, 16), torch.zeros(4, 1), bf(4, 16), bf(9, 16), i32(4, 2), stream=0),
    ):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(pkg.UcclError) as e:
        pkg.uccl_group_product(bf(7, 8), bf(7, 16), w, off, stream=0)
    assert e.value.code == EINVAL


def test_the_binding_refuses_more_rows_than_the_struct_can_say():
    """2^32 rows and more do not come down to what is left of them: no rows, or one."""
    import torch
    one = torch.zeros(1, 8, dtype=torch.bfloat16)
    for n in (1 << 32, (1 << 32) + 1):
        many = one.expand(n, 8)
        with pytest.raises(ValueError):
            pkg.uccl_norm_rows(many, many, one[0], 1e-6, stream=0)
        with pytest.raises(ValueError):
            pkg.uccl_combine_rows(one[:0], many, torch.zeros(0, 2, dtype=torch.int32), stream=0)


def test_prepared_calls_hold_their_structs():
    """The bytes of a uccl_rows live as long as the prepared call does."""
    import gc
    import torch
    x, eps = torch.zeros(3, 8, dtype=torch.bfloat16), 1e-6
    call = pkg.uccl_prepare(pkg.uccl_norm_rows, x, x, torch.zeros(8, dtype=torch.bfloat16), eps, stream=0, h=x[:2])   # refused: shapes
    gc.collect()
    junk = [bytes(48) for _ in range(1000)]
    for _ in range(3):
        with pytest.raises(pkg.UcclError) as e:
            call()
        assert e.value.code == EINVAL
    assert junk


def test_calls_can_be_prepared():
    import torch
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    call = pkg.uccl_prepare(pkg.uccl_norm_rows, bf(0, 8), bf(0, 8), bf(8), 1e-6, stream=0)
    call()
    call()
    assert call.__name__ == "uccl_norm_rows"


def test_kernels_use_no_scratch_memory(tmp_path):
    """The code object of the row operators, the library's second one."""
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
    notes, = [b for b in blocks if "norm_kernel" in b]
    assert len(re.findall(r"\.name: +_Z\S*kernel", notes)) > 10
    assert set(re.findall(r"\.private_segment_fixed_size: +(\d+)", notes)) == {"0"}
    assert set(re.findall(r"\.vgpr_spill_count: +(\d+)", notes)) == {"0"}


# ---- which kernel a product is launched as: the HIP runtime of tests/hip_stub.c reports it, nothing runs ----------------

def product_kernels(rt):
    """(what is multiplied, kernel as it is named in the library) of products by rows, groups, columns and depth."""
    for dtype, rows_, groups, wide, cols, out, kernel in (
        (BF16, 1, 1, 2048, 7168, BF16, "few_kernelILNS_10ArithmeticE0ELj16ELj8E"),
        (BF16, 16, 32, 2048, 7168, BF16, "few_kernelILNS_10ArithmeticE0ELj32ELj4E"),
        (F16, 128, 32, 2048, 7168, F16, "few_kernelILNS_10ArithmeticE1ELj32ELj4E"),
        (E4M3, 128, 32, 2048, 7168, BF16, "few_kernelILNS_10ArithmeticE2ELj32ELj4E"),
        (E4M3, 4096, 16, 2048, 7168, BF16, "tile_kernelILNS_10ArithmeticE3ELNS_7ProductE0ELj256ELj256E"),
        (E4M3, 2048, 16, 2048, 7168, BF16, "tile_kernelILNS_10ArithmeticE3ELNS_7ProductE0ELj128ELj256E"),
        (E4M3, 4096, 16, 2048, 7168, F32, "tile_kernelILNS_10ArithmeticE2ELNS_7ProductE0ELj128ELj128E"),   # exact where it can be seen
        (E4M3, 4096, 16, 2048, 500, BF16, "tile_kernelILNS_10ArithmeticE2ELNS_7ProductE0ELj128ELj128E"),
        (E4M3, 512, 1, 2048, 7168, BF16, "tile_kernelILNS_10ArithmeticE3ELNS_7ProductE0ELj128ELj256E"),
        (E4M3, 4000, 4, 2048, 7168, BF16, "tile_kernelILNS_10ArithmeticE3ELNS_7ProductE0ELj256ELj256E"),
        # few rows: by 16 while that is cheaper than the tiles that leave the machine idle
        (BF16, 20, 1, 2048, 7168, BF16, "few_kernelILNS_10ArithmeticE0ELj16ELj8E"),
        (BF16, 100, 1, 2048, 7168, BF16, "few_kernelILNS_10ArithmeticE0ELj32ELj4E"),
        (E4M3, 20, 8, 1200, 3000, BF16, "few_kernelILNS_10ArithmeticE2ELj32ELj4E"),
        (BF16, 400, 1, 2048, 7168, BF16, "tile_kernelILNS_10ArithmeticE0ELNS_7ProductE0ELj128ELj128E"),
        (E4M3, 200, 1, 2048, 7168, BF16, "few_kernelILNS_10ArithmeticE2ELj32ELj4E"),
        (BF16, 4096, 3, 5, 500, BF16, "few_kernelILNS_10ArithmeticE0ELj32ELj4E"),
        (BF16, 4096, 16, 2048, 7168, BF16, "tile_kernelILNS_10ArithmeticE0ELNS_7ProductE0ELj256ELj256E"),
        (F16, 2999, 24, 1003, 2043, F16, "tile_kernelILNS_10ArithmeticE1ELNS_7ProductE0ELj128ELj256E"),
        (BF16, 512, 1, 2048, 2048, BF16, "tile_kernelILNS_10ArithmeticE0ELNS_7ProductE0ELj128ELj128E"),
        # those of tests/test_gpu_rows.py that are there for the large tiles
        (BF16, 3001, 3, 4100, 40, BF16, "tile_kernelILNS_10ArithmeticE0ELNS_7ProductE0ELj256ELj256E"),
        (BF16, 1299, 1, 4103, 40, BF16, "tile_kernelILNS_10ArithmeticE0ELNS_7ProductE0ELj128ELj256E"),
        (E4M3, 3001, 3, 4100, 521, BF16, "tile_kernelILNS_10ArithmeticE3ELNS_7ProductE0ELj256ELj256E"),
        (E4M3, 1299, 1, 4103, 521, BF16, "tile_kernelILNS_10ArithmeticE3ELNS_7ProductE0ELj128ELj256E"),
        (BF16, 647, 4, 2050, 40, BF16, "tile_kernelILNS_10ArithmeticE0ELNS_7ProductE0ELj128ELj128E"),
    ):
        rt.launches.clear(), rt.symbols.clear()
        make = (lambda n, c: q8(n, c)) if dtype == E4M3 else (lambda n, c: rows(n, c, dtype))
        y, x, w = rows(rows_, wide, out), make(rows_, cols), make(groups * wide, cols)
        assert rt.lib.uccl_group_product(y, x, None, w, M, groups, None) == OK
        assert len(rt.symbols) == 1 and kernel in rt.symbols[0], (rt.symbols, kernel)
    for rows_, groups, wide, cols, x_kernel, w_kernel in (
        (4096, 16, 2048, 7168, "ProductE1ELj256ELj256E", "ProductE2ELj256ELj256E"),
        (1299, 1, 40, 4103, "ProductE1ELj128ELj256E", "ProductE2ELj128ELj128E"),
        (199, 3, 2900, 2300, "ProductE1ELj128ELj128E", "ProductE2ELj256ELj256E"),
        (199, 3, 630, 4100, "ProductE1ELj128ELj128E", "ProductE2ELj128ELj256E"),
    ):
        rt.symbols.clear()
        dy, x, w = rows(rows_, wide), rows(rows_, cols), rows(groups * wide, cols)
        assert rt.lib.uccl_group_product_grad_x(x, dy, w, M, groups, None) == OK
        assert rt.lib.uccl_group_product_grad_w(w, dy, x, None, M, groups, None) == OK
        assert x_kernel in rt.symbols[0] and w_kernel in rt.symbols[1], rt.symbols
    # the grid: a workgroup for every tile that there could be, by eights, and a launch that HIP could not take is refused
    rt.launches.clear()
    assert rt.lib.uccl_group_product(rows(512, 2048), rows(512, 2048), None, rows(2048, 2048), M, 1, None) == OK
    assert rt.launches[-1][1:3] == ((512 // 128 + 1) * 16 + 8, 512)      # a group's tiles together: an XCD's eighth may be one more
    assert rt.lib.uccl_group_product(rows(500, 700), rows(500, 2048), None, rows(5600, 2048), M, 8, None) == OK
    assert rt.launches[-1][1:3] == (3 * 6 + 6 + 8 * 6, 512)              # full tiles and those that groups end in, by eights
    # narrow outputs of very many rows go by 16 rows while that fits a launch, and by tiles where these do
    for n, kernel in ((1 << 26, "few_kernel"), ((1 << 29) - 1024, "tile_kernel")):
        rt.symbols.clear()
        assert rt.lib.uccl_group_product(rows(n, 5), rows(n, 500), None, rows(5, 500), M, 1, None) == OK
        assert kernel in rt.symbols[0]
    rt.launches.clear()
    big = (1 << 31) - 1
    assert rt.lib.uccl_group_product(rows(big, 8 << 20), rows(big, 64), None, rows(8 << 20, 64), M, 1, None) == pkg.UCCL_ETOOBIG
    assert rt.launches == []
    assert rt.lib.uccl_combine_rows(rows(big, 1 << 20), rows(9, 1 << 20), M, None, 2, None, None) == pkg.UCCL_ETOOBIG
    norm = lambda n, c: rt.lib.uccl_norm_rows(rows(n, c), None, None, rows(n, c), None, B, C.byref(pkg.uccl_norm_opts(1e-6)), None)
    assert [norm(n, c) for n, c in ((1 << 26, 128), ((1 << 22) - 1, 1 << 20), (1 << 22, 1 << 20))] == [pkg.UCCL_ETOOBIG, OK, pkg.UCCL_ETOOBIG]
    assert len(rt.launches) == 1
    rt.launches.clear()
    wide = 1 << 28
    assert rt.lib.uccl_norm_rows_grad(rows(1, wide), D, rows(1, wide), None, rows(1, wide), D, B, S, 4 * wide, None) == pkg.UCCL_ETOOBIG
    assert rt.lib.uccl_combine_rows_grad(rows(9, 8), None, rows(1 << 24, 8), rows(9, 8), M, None, 1, None) == pkg.UCCL_ETOOBIG
    assert rt.launches == []
    # launches that the runtime refuses come back as such
    rt.refuse = lambda *a: True
    assert rt.lib.uccl_group_product(rows(512, 2048), rows(512, 2048), None, rows(2048, 2048), M, 1, None) == pkg.UCCL_ELAUNCH
    assert rt.lib.uccl_norm_rows(rows(2, 8), None, None, rows(2, 8), None, B, C.byref(pkg.uccl_norm_opts(1e-6)), None) == pkg.UCCL_ELAUNCH
    assert b"as the test asked" in rt.lib.uccl_last_error_detail()


def test_which_kernel_a_product_is_launched_as(tmp_path):
    import os
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    stub = str(tmp_path / "libamdhip64.so.7")
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", "-Wl,-soname,libamdhip64.so.7", "-I/opt/rocm/include", os.path.join(here, "hip_stub.c"), "-o", stub])
    code = (f"import sys; sys.path[:0] = [{here!r}, {os.path.dirname(here)!r}]\n"
            f"import test_host_launches as h, test_rows_abi as t\n"
            f"rt = h.Runtime({stub!r})\n"
            f"for n, (r, a) in t.pkg.ROWS_SIGNATURES.items():\n    f = getattr(rt.lib, n); f.restype, f.argtypes = r, a\n"
            f"t.product_kernels(rt)\n")
    subprocess.run([sys.executable, "-c", code], check=True)
