"""Routing, microscaled 4 bits and clipping where values are infinite, the greatest or the least of their type, and where calls are large enough for every kernel.

Tolerances as in tests/test_gpu_experts.py.
"""
import pytest
import torch

from test_gpu_experts import E2M1, E8M0, gen, random_mx4
from test_gpu_rows import aligned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def uccl(gpu_lib):
    return gpu_lib


def grouped(q, groups):
    return q.view(torch.uint8).unflatten(0, (groups, -1))


# ---- products of weights in 4 bits ----------------------------------------------------------------


def multiply(uccl, x, xs, w, ws, wide):
    """Of one group, to f32."""
    y, offsets = aligned(x.shape[0], wide, torch.float32), torch.tensor([0, x.shape[0]], dtype=torch.int32, device="cuda")
    uccl.uccl_group_product(y, x, grouped(w, 1).view(E2M1), offsets, x_scales=xs, w_scales=grouped(ws, 1).view(E8M0))
    return y


@pytest.mark.parametrize("rows", [1, 2, 90, 600, 3000])
def test_product_of_the_greatest_f16_by_large_weights(uccl, rows):
    """Products below binary32's greatest number whose f16 factor rounds up to a power of two in 8 bits."""
    wide, cols = 300, 64
    w, ws = random_mx4(gen(rows), wide, cols)
    w.view(torch.uint8)[:], ws.view(torch.uint8)[:] = 0, 127
    w.view(torch.uint8)[:, 20] = 2                                          # element 40: 1 by 2^112
    ws.view(torch.uint8)[:, 1] = 127 + 112
    x = aligned(rows, cols, torch.float16)
    x[:] = 0.0
    x[:, 40] = 65504.0
    x[1::2, 40] = -65504.0
    y = multiply(uccl, x, None, w, ws, wide)
    want = torch.full((rows, wide), 65504.0 * 2.0 ** 112, dtype=torch.float64, device="cuda")
    want[1::2] *= -1
    assert torch.equal(y.double(), want)
