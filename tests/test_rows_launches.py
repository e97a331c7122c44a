"""What the row operators ask of the HIP runtime, launch by launch: kernels and timing events.  The runtime is tests/hip_stub.c, so nothing runs and no
GPU is needed; each test's body runs in a process of its own, where the stub is loaded first and serves the library by its soname."""
import ctypes as C
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path[:0] = [HERE, os.path.dirname(HERE)]
import paper_2504_17307_amd as pkg  # noqa: E402
from test_rows_abi import B, BF16, D, E4M3, EINVAL, F16, F32, M, OK, S, q8, rows  # noqa: E402

START, STOP, BAD = 0x6000, 0x7000, 0x5000
EPS = C.byref(pkg.uccl_norm_opts(1e-6))


def in_process(scenario, tmp_path):
    stub = str(tmp_path / "libamdhip64.so.7")
    subprocess.check_call(["gcc", "-O1", "-shared", "-fPIC", "-w", "-I/opt/rocm/include", "-Wl,-soname,libamdhip64.so.7", os.path.join(HERE, "hip_stub.c"), "-o", stub])
    r = subprocess.run([sys.executable, os.path.abspath(__file__), scenario, stub], cwd=os.path.dirname(HERE), capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "SCENARIO DONE" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]


def norm_grad(rt, n, cols, dtype=BF16, dh=False):
    scratch = rt.lib.uccl_norm_rows_scratch(n, cols)
    return rt.lib.uccl_norm_rows_grad(rows(n, cols, dtype), D, rows(n, cols, dtype), rows(n, cols, dtype) if dh else None, rows(n, cols, dtype), D, B, S, scratch, None)


def timing_events(rt):
    events = []
    rt.refuse = lambda kernel, stream, start, stop: bool(events.append((start, stop)))
    calls = {
        "norm": lambda: rt.lib.uccl_norm_rows(rows(2, 8), None, None, rows(2, 8), None, B, EPS, None),
        "norm_grad": lambda: norm_grad(rt, 300, 640),
        "norm_grad long": lambda: norm_grad(rt, 3, 40000, dh=True),
        "norm_grad of nothing": lambda: norm_grad(rt, 0, 64),
        "product": lambda: rt.lib.uccl_group_product(rows(9, 8), rows(9, 64), None, rows(16, 64), M, 2, None),
        "combine": lambda: rt.lib.uccl_combine_rows(rows(9, 8), rows(9, 8), M, None, 2, None, None),
    }
    for name, call in calls.items():
        events.clear()
        assert rt.lib.uccl_time_next_launch(START, STOP) == OK and call() == OK
        assert events[0][0] == START and events[-1][1] == STOP and not any(start for start, _ in events[1:]), (name, events)
        assert len(events) == (2 if name in ("norm_grad", "norm_grad long") else 1), (name, events)
        events.clear()
        assert call() == OK and not any(map(any, events)), (name, events)   # once only
    # a launch that fails takes them too, and an event that HIP does not take fails the call before anything is enqueued
    rt.refuse = lambda kernel, stream, start, stop: BAD in (start, stop)
    for start, stop in ((START, BAD), (BAD, STOP), (BAD, None), (None, BAD)):
        rt.launches.clear()
        assert rt.lib.uccl_time_next_launch(start, stop) == OK
        assert norm_grad(rt, 300, 640) == pkg.UCCL_ELAUNCH and not rt.launches, (start, stop)
        assert norm_grad(rt, 300, 640) == OK and len(rt.launches) == 2


def test_timing_events_span_a_call_of_two_launches(tmp_path):
    in_process("timing_events", tmp_path)


class Seen:
    """The stub's runtime, which also notes of every product whether it is launched with a group's tiles together."""

    def __init__(self, rt):
        self.rt, self.together, self.product = rt, [], None
        self.was = rt._launch
        on_launch = C.CFUNCTYPE(C.c_int, C.c_char_p, C.c_uint, C.c_uint, C.c_uint, C.c_void_p, C.POINTER(C.c_void_p), C.c_void_p, C.c_void_p)
        self.keep = on_launch(self._launch)
        rt.stub.stub_callbacks(self.keep, rt.keep[1])

    def _launch(self, kernel, grid, block, lds, stream, args, start, stop):
        if b"product_" in kernel:   # ProductArgs: three matrices of 32 bytes, two pointers, six numbers
            self.together.append(C.cast(args[0] + 136, C.POINTER(C.c_uint32))[0])
        return self.was(kernel, grid, block, lds, stream, args, start, stop)


TYPE = {F32: "IfL", BF16: "IDF16bL", F16: "IDF16_L"}


def kernels(rt):
    """The shapes of tests/test_gpu_rows_large.py, and what they are there for."""
    lib = rt.lib
    for dtype, n, cols, shape, once in (
        (BF16, 1, 7168, "1024ELj1", 0), (BF16, 512, 7168, "1024ELj1", 0), (BF16, 513, 7168, "512ELj2", 0), (BF16, 600, 7168, "512ELj2", 0), (BF16, 2500, 7168, "512ELj2", 1),
        (F16, 2500, 7171, "512ELj2", 1), (BF16, 4096, 7168, "512ELj2", 1), (BF16, 2340, 7168, "512ELj2", 0), (BF16, 2341, 7168, "512ELj2", 1), (BF16, 40000, 500, "64ELj1", 1),
        (BF16, 9000, 2043, "256ELj1", 1), (BF16, 4500, 4093, "512ELj1", 1), (BF16, 1100, 16381, "512ELj4", 1), (F32, 600, 4093, "512ELj2", 0), (F32, 2100, 4093, "512ELj2", 1),
        (F32, 1300, 7168, "512ELj4", 1), (F32, 40000, 250, "64ELj1", 1), (F32, 9000, 1021, "256ELj1", 1), (F32, 4500, 2043, "512ELj1", 1), (F32, 3, 9000, None, 0), (BF16, 3, 16385, None, 0),
    ):
        for out, e8 in ((rows(n, cols, dtype), 0), (q8(n, cols), 1)):
            rt.symbols.clear()
            x = rows(n, cols, dtype)
            assert lib.uccl_norm_rows(out, x, None, x, None, B, EPS, None) == OK
            t = TYPE[dtype][:-1]
            want = f"norm_long_kernel{t}Lb{e8}E" if shape is None else f"norm_kernel{t}Lb{e8}ELj{shape}ELb{once}E"
            assert len(rt.symbols) == 1 and want in rt.symbols[0], (want, rt.symbols)
    # an output in 8 bits is a half or a quarter of h, which may be there or not
    for n, once in ((4681, 0), (4682, 1)):
        rt.symbols.clear()
        assert lib.uccl_norm_rows(q8(n, 7168), None, None, rows(n, 7168), None, B, EPS, None) == OK and f"norm_kernelIDF16bLb1ELj512ELj2ELb{once}E" in rt.symbols[0]
    for dtype, n, cols, shape, once in (
        (BF16, 2, 255, "256ELj1", 0), (BF16, 9000, 2043, "256ELj1", 1), (BF16, 4500, 4093, "512ELj1", 1), (BF16, 600, 7168, "1024ELj1", 0), (BF16, 2500, 7168, "1024ELj1", 1), (F16, 2500, 7171, "1024ELj1", 1),
        (BF16, 530, 8208, "512ELj4", 0), (BF16, 1100, 16381, "512ELj4", 1), (F32, 600, 4093, "1024ELj1", 0), (F32, 2100, 4093, "1024ELj1", 1), (F32, 1300, 7168, "512ELj4", 1), (F32, 1100, 8188, "512ELj4", 1),
        (F32, 9000, 1021, "256ELj1", 1), (F32, 4500, 2043, "512ELj1", 1), (F32, 300, 9000, None, 0), (BF16, 300, 20000, None, 0),
    ):
        rt.symbols.clear(), rt.launches.clear()
        assert norm_grad(rt, n, cols, dtype, dh=True) == OK
        want = f"norm_grad_long_kernel{TYPE[dtype][:-1]}E" if shape is None else f"norm_grad_kernel{TYPE[dtype]}j{shape}ELb{once}E"
        assert want in rt.symbols[0] and "column_sum_kernel" in rt.symbols[1] and rt.launches[0][1] == min(n, 256), (want, rt.symbols)
    for dtype, tokens, slots, cols, once, once_grad in ((BF16, 2500, 2, 7168, 1, 1), (F16, 2500, 3, 7171, 1, 1), (BF16, 700, 9, 7171, 0, 1), (F32, 1300, 2, 7168, 1, 1), (F32, 400, 9, 7171, 0, 1), (BF16, 70, 4, 20, 0, 0)):
        rt.symbols.clear()
        y = rows(tokens * slots * 7 // 8, cols, dtype)
        assert lib.uccl_combine_rows(rows(tokens, cols, dtype), y, M, D, slots, None, None) == OK
        assert lib.uccl_combine_rows_grad(y, D, rows(tokens, cols, dtype), y, M, D, slots, None) == OK
        assert f"combine_kernel{TYPE[dtype]}j128ELb{once}E" in rt.symbols[0] and f"combine_grad_kernel{TYPE[dtype]}b{once_grad}E" in rt.symbols[1], rt.symbols
    # more than 64 groups, together
    seen = Seen(rt)
    few, tiles = sum((5 * i) % 17 for i in range(150)), sum((29 * i) % 81 for i in range(70))
    for dtype in (BF16, E4M3):
        make = (lambda n, c: q8(n, c)) if dtype == E4M3 else (lambda n, c: rows(n, c, dtype))
        rt.symbols.clear(), seen.together.clear()
        assert lib.uccl_group_product(rows(few, 1280), make(few, 72), M, make(150 * 1280, 72), M, 150, None) == OK
        assert lib.uccl_group_product(rows(tiles, 14336), make(tiles, 40), M, make(70 * 14336, 40), M, 70, None) == OK
        assert "few_kernel" in rt.symbols[0] and "tile_kernel" in rt.symbols[1] and seen.together == [1, 1], (rt.symbols, seen.together)
    rt.symbols.clear(), seen.together.clear()
    assert lib.uccl_group_product_grad_x(rows(tiles, 14336), rows(tiles, 40), rows(70 * 40, 14336), M, 70, None) == OK
    assert "tile_kernel" in rt.symbols[0] and seen.together == [1]
    assert lib.uccl_group_product(rows(2743, 777), rows(2743, 40), None, rows(67 * 777, 40), M, 67, None) == OK and seen.together == [1, 0]


def test_which_kernel_a_row_operator_is_launched_as(tmp_path):
    in_process("kernels", tmp_path)


def largest_launches(rt):
    """Just fewer than 2^22 tiles of 128 x 128: 65535 groups of 128 rows by 8192 columns, which the order by size has a launch for and the order by group
    has not."""
    seen, groups = Seen(rt), 65535
    y, x, w = rows(128 * groups, 8192), q8(128 * groups, 496), q8(8192 * groups, 496)
    assert rt.lib.uccl_group_product(y, x, None, w, M, groups, None) == OK
    assert "ArithmeticE2ELNS_7ProductE0ELj128ELj128E" in rt.symbols[-1] and seen.together == [0] and rt.launches[-1][1] * rt.launches[-1][2] < 2 ** 32, (rt.symbols, seen.together)
    seen.together.clear()
    groups = 30000
    assert rt.lib.uccl_group_product(rows(128 * groups, 8192), q8(128 * groups, 496), None, q8(8192 * groups, 496), M, groups, None) == OK and seen.together == [1]


def test_the_largest_products_fit_a_launch(tmp_path):
    in_process("largest_launches", tmp_path)


if __name__ == "__main__":
    import test_host_launches
    runtime = test_host_launches.Runtime(sys.argv[2])
    for name, (res, args) in pkg.ROWS_SIGNATURES.items():
        fn = getattr(runtime.lib, name)
        fn.restype, fn.argtypes = res, args
    globals()[sys.argv[1]](runtime)
    print("SCENARIO DONE")
