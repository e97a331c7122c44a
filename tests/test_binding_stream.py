"""How the binding finds torch's current stream, without a GPU: torch's functions are replaced, in a process of its own."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FORK = """
import os, torch
import paper_2504_17307_amd as pkg
torch.cuda.is_available, torch.cuda.init = lambda: True, lambda: None
torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream = lambda: 1, lambda device: 70 + device
assert pkg._stream(None) == 71                      # a process that has made a call
child = os.fork()
if child == 0:
    def init():                                     # as torch does where the parent has initialised the GPU
        raise RuntimeError("Cannot re-initialize CUDA in forked subprocess")
    torch.cuda.init = init
    try:
        pkg._stream(None)
    except RuntimeError:
        os._exit(7)
    os._exit(1)
_, status = os.waitpid(child, 0)
assert os.WEXITSTATUS(status) == 7, status
assert pkg._stream(None) == 71
print("DONE")
"""


def test_a_forked_child_gets_torchs_own_refusal():
    """HIP does not work in a child of a process that uses it: torch says so, and the binding asks torch there anew."""
    r = subprocess.run([sys.executable, "-c", FORK], cwd=ROOT, capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "DONE" in r.stdout, r.stdout + r.stderr
