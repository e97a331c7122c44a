"""Row operators on inputs whose results binary32 has exactly, whatever the order of the sums: equality, and no tolerance that a dropped
term could hide in."""
import numpy as np
import pytest
import torch

from test_gpu_rows import E8, T, aligned, gen, offsets_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def uccl(gpu_lib):
    return gpu_lib


# rows by group, columns, depth: by 16 rows, by tiles of 128 x 128 (8 bits: short sums), 128 x 256 and 256 x 256
SUMS = {"few": ([7, 0, 20], 600, 7168), "128x128": ([700, 0, 613], 4103, 500), "128x256": ([1299], 4103, 521), "128x256 deep": ([130] * 16, 2048, 7168),
        "256x256": ([1100, 0, 1901], 4100, 521), "256x256 deep": ([1000] * 4, 2048, 7168)}


@pytest.mark.parametrize("out", list(T))
@pytest.mark.parametrize("dtype", ["e4m3", "bf16"])
@pytest.mark.parametrize("shape", list(SUMS))
def test_small_terms_beside_large_ones_that_cancel(uccl, shape, dtype, out):
    """Integers of at most 2, and up to 40 pairs of columns that bring 448 x 448 and its opposite next to them.  The magnitudes of a row's terms add up to less than
    2^24, so every partial sum is an integer that binary32 has; scales are powers of two.  What is left is the one rounding to the output's type."""
    counts, n, k = SUMS[shape]
    g, rows, groups = gen(k + n), sum(counts), len(counts)
    small = lambda r: torch.randint(-2, 3, (r, k), device="cuda", generator=g).float()  # noqa: E731
    x, w = small(rows + 3), small(groups * n)
    for c in (torch.randperm(k // 8, device="cuda", generator=g)[:40] * 8).tolist():
        a, b = c + c // 8 % 7, c + 7
        x[:, a], x[:, b], w[:, a], w[:, b] = 448.0, -448.0, 448.0, 448.0
    assert 80 * 448 ** 2 + 4 * k < 2 ** 24
    t = E8 if dtype == "e4m3" else torch.bfloat16
    xt, wt = aligned(rows + 3, k, t), aligned(groups * n, k, t)
    for to, v in ((xt, x), (wt, w)):
        to.view(torch.uint8 if t == E8 else t).copy_(v.to(t).view(torch.uint8 if t == E8 else t))
    xs = ws = None
    ex, ew = x.double(), w.double()
    if t == E8:
        xs, ws = (torch.exp2(torch.randint(-4, 1, (r, 1), device="cuda", generator=g).float()) for r in (rows + 3, groups * n))
        ex, ew = ex * xs, ew * ws
    index = torch.randint(0, rows + 3, (rows,), device="cuda", generator=g).to(torch.int32)
    y = aligned(rows, n, T[out])
    uccl.uccl_group_product(y, xt, wt.unflatten(0, (groups, n)), offsets_of(counts), index=index, x_scales=xs, w_scales=ws)
    at = 0
    for e, c in enumerate(counts):
        want = ex[index[at:at + c].long()] @ ew[e * n:(e + 1) * n].T
        assert torch.equal(y[at:at + c], want.to(T[out])), f"group {e}: off by up to {float((y[at:at + c].double() - want).abs().max())}"
        at += c


def elements(y, scales):
    """The e4m3 elements of binary32 rows: their binary32 quotients by the scales (a quotient in 64 bits rounds to those), to nearest even."""
    return (y.double() / scales.double()).float().to(E8).view(torch.uint8)


# columns that take one piece a thread, one wavefront; several; two and four pieces; rows of any length
@pytest.mark.parametrize("cols", [256, 1024, 2048, 4096, 8192, 32768])
@pytest.mark.parametrize("rows", [2, 520])
def test_8_bit_outputs_are_the_quotients_by_the_scale(uccl, rows, cols):
    """Ones have a mean square of one, and eps 0 leaves them so: y is the weight.  It holds products of a scale of few bits with the ties between e4m3 values and their
    neighbours in binary32; the greatest, 448 times the scale, is among them."""
    vals = torch.arange(0, 127, dtype=torch.uint8).view(E8).double()
    ties = (vals[1:] + vals[:-1]) / 2
    r = np.random.default_rng(cols)
    x = aligned(rows, cols, torch.float32)
    x.fill_(1.0)
    y, s, rstd = aligned(rows, cols, E8), torch.zeros(rows, 1, device="cuda"), torch.zeros(rows, device="cuda")
    for power in (0, -20, -63, -117, 100):
        for _ in range(8):
            scale = float(np.ldexp(r.integers(2 ** 18, 2 ** 19) | 1, power - 18))
            v = (ties * scale).float()                       # 4 bits and 19: exact
            v = torch.cat([v, (vals * scale).float(), torch.nextafter(v, torch.tensor(torch.inf)), torch.nextafter(v, torch.tensor(0.0))])
            v = v[torch.from_numpy(r.integers(0, len(v), cols))] * torch.from_numpy(r.choice([-1.0, 1.0], cols)).float()
            v[int(r.integers(0, cols))] = 448 * scale
            w = v.cuda()
            uccl.uccl_norm_rows(y, x, w, 0.0, rstd=rstd, scales=s)
            assert bool((rstd == 1.0).all()) and bool((s == scale).all())
            assert torch.equal(y.view(torch.uint8), elements(w.expand(rows, cols), s)), (power, scale)


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("rows,cols", [(3000, 2043), (1000, 7168), (40, 20000)])
def test_8_bit_outputs_of_many_rows_are_the_quotients(uccl, dtype, rows, cols):
    """y from the call's own 1 / root, with the kernel's two roundings."""
    g, t = gen(cols), T[dtype]
    x, w = aligned(rows, cols, t), aligned(1, cols, t)[0]
    x.copy_(torch.randn(rows, cols, device="cuda", generator=g))
    w.copy_(torch.randn(cols, device="cuda", generator=g))
    y, s, rstd = aligned(rows, cols, E8), torch.zeros(rows, 1, device="cuda"), torch.zeros(rows, device="cuda")
    uccl.uccl_norm_rows(y, x, w, 1e-6, rstd=rstd, scales=s)
    e = x.float() * rstd[:, None] * w.float()
    assert torch.equal(s, (e.abs().amax(1, keepdim=True).double() / 448.0).float())
    assert torch.equal(y.view(torch.uint8), elements(e, s))
