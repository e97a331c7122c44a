"""Routing, microscaled 4 bits and clipping where values are infinite, the greatest or the least of their type, and where calls are large enough for every kernel.

Tolerances as in tests/test_gpu_experts.py.
"""
import pytest
import torch

from test_gpu_experts import DEEP, E2M1, E8M0, INF, decode, f32, gen, i32, product_reference, random_mx4, softmax
from test_gpu_rows import T, aligned, close, normal

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


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("more", [0, 17, 40, 64, 100])
@pytest.mark.parametrize("rows,groups,wide,cols", DEEP)
def test_product_of_infinities(uccl, kind, rows, groups, wide, cols, more):
    """A row with an infinity, and every weight beside it another number than 0: an infinity with the sign of the product in every column, also where a column of the same
    wavefront has scales that f16 does not hold, and where the sum ends within a block.  By every kernel (tests/test_experts_abi.py has which)."""
    g, cols = gen(rows + cols + more), cols + more + more % 2
    w, ws = random_mx4(g, groups * wide, cols)
    w.view(torch.uint8).bitwise_or_(0x11)                                   # no zeros
    ws.view(torch.uint8)[3::16, ::3] = 0
    ws.view(torch.uint8)[9::16, -1] = 200
    x = normal(g, rows, cols, T[kind], pad=1)
    broken = torch.arange(0, rows, 3, device="cuda")
    at = torch.randint(0, cols, (len(broken),), device="cuda", generator=g)
    at[0], at[-1] = cols - 1, 0
    sign = torch.where(torch.rand(len(broken), device="cuda", generator=g) < 0.5, -1.0, 1.0)
    x[broken, at] = (INF * sign).to(T[kind])
    ends = [rows * k // groups for k in range(groups + 1)]
    y = aligned(rows, wide, torch.float32)
    uccl.uccl_group_product(y, x, grouped(w, groups).view(E2M1), torch.tensor(ends, dtype=torch.int32, device="cuda"), w_scales=grouped(ws, groups).view(E8M0))
    dw = decode(w, ws, cols).view(groups, wide, cols)
    want, mag = product_reference(torch.where(x.isinf(), 0.0, x.double()), dw, None, ends)
    of = torch.bucketize(broken, torch.tensor(ends[1:], device="cuda"), right=True)
    want[broken] = INF * sign[:, None].double() * dw[of, :, at].sign()
    mag[broken] = 0.0
    close(y, want, mag, cols, kind)
    assert torch.equal(y[broken].double(), want[broken])


# ---- routing --------------------------------------------------------------------------------------


@pytest.mark.parametrize("normalise", [False, True])
@pytest.mark.parametrize("tokens", [5, 3000])
@pytest.mark.parametrize("n", [3, 61, 64, 100, 250, 700])
@pytest.mark.parametrize("dtype", list(T))
def test_route_grad_of_infinite_gradients_of_the_sums(uccl, dtype, n, tokens, normalise):
    """An infinity for one expert's sum: its probability's share is an infinity for every other expert, and what lies behind a row's last expert is not in it."""
    scores = normal(gen(n), tokens, n, T[dtype])
    experts, dw = i32(tokens, 2, fill=0), f32(tokens, 2, fill=0.0)
    for at in (0, n - 1):
        ds = torch.randn(n, device="cuda", generator=gen(1))
        ds[at] = INF
        out = aligned(tokens, n, T[dtype])
        uccl.uccl_route_rows_grad(out, scores, experts, dw, dsums=ds, normalise=normalise)
        p = softmax(scores)
        want = p * (ds.double() - (p * ds.double()).sum(1, keepdim=True))     # infinity less infinity for the expert itself
        assert bool(want[:, at].isnan().all()) and bool((want[:, torch.arange(n, device="cuda") != at] == -INF).all())
        assert torch.equal(out.double().nan_to_num(nan=7.0), want.nan_to_num(nan=7.0))
