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


if __name__ == "__main__":
    import test_host_launches
    runtime = test_host_launches.Runtime(sys.argv[2])
    for name, (res, args) in pkg.ROWS_SIGNATURES.items():
        fn = getattr(runtime.lib, name)
        fn.restype, fn.argtypes = res, args
    globals()[sys.argv[1]](runtime)
    print("SCENARIO DONE")
