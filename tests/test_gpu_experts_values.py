"""Routing, microscaled 4 bits and clipping where values are infinite, the greatest or the least of their type, and where calls are large enough for every kernel.

Tolerances as in tests/test_gpu_experts.py.
"""
import pytest
import torch

from test_gpu_experts import (DEEP, E2M1, E8M0, INF, NAN, bytes_, choice, codes_of, decode, f32, gen, grad_reference, i32, mx4_rows, product_reference, quantise_reference, random_mx4, softmax,
                              spread, weights_of)
from test_gpu_rows import T, aligned, close, margin, normal

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


@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 2, 90, 600, 3000])
@pytest.mark.parametrize("byte", [0, 1, 103, 104, 140, 141, 200, 251, 252, 253, 254])
def test_product_by_weights_of_one_scale(uccl, kind, rows, byte):
    """Every element by scales from the least to the greatest: exact, for a sum has one term; beside rows in 16 bits infinities or NaN from 2^128 on."""
    wide, cols = 16, 96
    w, ws = random_mx4(gen(rows), wide, cols)
    w.view(torch.uint8)[:], ws.view(torch.uint8)[:] = 0, byte
    w.view(torch.uint8)[:, 35] = torch.arange(16, device="cuda") << 4        # element 71
    by = 2.0 ** (20 if byte < 100 else -20 if byte > 150 else 0)
    if kind == "mx4":
        x, xs = random_mx4(gen(1), rows, cols)
        x.view(torch.uint8)[:], xs.view(torch.uint8)[:] = 0, 127 + (20 if byte < 100 else -20 if byte > 150 else 0)
        x.view(torch.uint8)[:, 35] = 3 << 4                                  # 1.5
    else:
        x, xs = aligned(rows, cols, T[kind]), None
        by = 2.0 ** (15 if byte < 100 else -14 if byte > 150 else 0) if kind == "f16" else by
        x[:] = 0.0
        x[:, 71] = 1.5 * by
    y = multiply(uccl, x, xs, w, ws, wide)
    dw = decode(w, ws, cols)[:, 71]
    held = torch.ones(16, dtype=torch.bool, device="cuda") if kind == "mx4" else dw.abs() < 2.0 ** 128
    want = (1.5 * by * dw).expand(rows, wide)
    assert torch.equal(y.double()[:, held], want[:, held])
    assert bool((~y[:, ~held].isfinite()).all())


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


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("tokens,n,slots", [(20481, 61, 6), (40001, 256, 8), (33001, 300, 5), (9001, 700, 8), (2501, 100, 6), (2501, 128, 4), (2499, 200, 8)])
def test_route_of_more_tokens_than_all_workgroups_have_at_once(uccl, dtype, tokens, n, slots):
    """Workgroups that add up sums go round, the last time not all of them whole; and every shape of a token's lanes where there are many tokens.  With sums and without, and the gradient."""
    g, t = gen(tokens + n), T[dtype]
    scores = normal(g, tokens, n, t, 2.0, pad=1)
    scores.masked_fill_(torch.rand(tokens, n, device="cuda", generator=g) < 0.1, -INF)
    scores[5], scores[tokens - 1, 1:] = -INF, -INF
    bias = torch.randn(n, device="cuda", generator=g)
    want = choice(scores, bias, slots)
    for normalise, scale in ((True, 2.5), (False, 1.0)):
        ew = weights_of(scores, want, normalise, scale)
        for wanted in (True, False):
            experts, w, counts, sums = i32(tokens, slots), f32(tokens, slots), i32(n), f32(n)
            scratch = bytes_(uccl.uccl_route_rows_scratch(tokens, n))
            uccl.uccl_route_rows(experts, w, scores, bias=bias, normalise=normalise, scale=scale, **(dict(counts=counts, sums=sums, scratch=scratch) if wanted else {}))
            assert torch.equal(experts.long(), want)
            close(w, ew, ew.abs() * (1 + spread(scores)), n + 8, "weights")
        assert int(uccl.uccl_route_rows_scratch(tokens, n)) <= scratch.numel()
    uccl.uccl_route_rows(experts, w, scores, bias=bias, counts=counts, sums=sums, scratch=scratch)
    assert torch.equal(counts.long(), torch.bincount(want[want >= 0], minlength=n))
    p = softmax(scores)
    es = p.sum(0)
    close(sums, es, es * (1 + spread(scores)), n + tokens + 8, "sums")
    dw, ds = torch.randn(tokens, slots, device="cuda", generator=g), torch.randn(n, device="cuda", generator=g)
    for normalise in (True, False):
        out = aligned(tokens, n, t, 2)
        around = margin(out)
        uccl.uccl_route_rows_grad(out, scores, want.to(torch.int32), dw, dsums=ds, normalise=normalise, scale=0.5)
        dz, mag = grad_reference(scores, want.to(torch.int32), dw, ds, normalise, 0.5)
        close(out, dz, mag * (1 + spread(scores)), 2 * n + slots + 16, "dscores")
        assert torch.equal(margin(out), around)


# ---- rows in 4 bits -------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("rows,cols", [(4100, 515), (2500, 4099), (4300, 4099), (9000, 1000), (1100, 8192)])
def test_quantise_of_many_pieces_with_values(uccl, dtype, rows, cols):
    """Four pieces a thread; values of up to and above 32 MiB, into rows with gaps and over the rows themselves."""
    t, g = T[dtype], gen(rows)
    x = normal(g, rows, cols, t, pad=1)
    x.mul_(torch.exp2(torch.randint(-8, 8, (rows, 1), device="cuda", generator=g).to(t)))
    x[7], x[-1, -1], x[3, cols - 2] = 0.0, INF, NAN
    wire, q, scales = mx4_rows(rows, cols)
    before, values = wire.clone(), aligned(rows, cols, t, 2)
    around = margin(values)
    uccl.uccl_quantise_rows(q, scales, x, values=values)
    number, byte = quantise_reference(x)
    assert torch.equal(scales.view(torch.uint8).cpu().long(), byte) and torch.equal(codes_of(q, cols).cpu().long(), number)
    n, at = -(-cols // 2), -(-cols // 32) * 16
    assert torch.equal(wire[:, n:at], before[:, n:at]) and torch.equal(wire[:, at - (-cols // 32):], before[:, at - (-cols // 32):])
    if cols % 2:
        assert bool((q.view(torch.uint8)[:, -1] >> 4 == 0).all())
    want = decode(q, scales, cols)
    assert torch.equal(values.double().nan_to_num(nan=1e300), want.nan_to_num(nan=1e300)) and torch.equal(margin(values), around)
    _, again, s = mx4_rows(rows, cols)
    uccl.uccl_quantise_rows(again, s, x)
    assert torch.equal(again.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s.view(torch.uint8), scales.view(torch.uint8))
    _, again, s = mx4_rows(rows, cols)
    beside = margin(x)
    uccl.uccl_quantise_rows(again, s, x, values=x)
    assert torch.equal(again.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s.view(torch.uint8), scales.view(torch.uint8))
    assert torch.equal(x.double().nan_to_num(nan=1e300), want.nan_to_num(nan=1e300)) and torch.equal(margin(x), beside)


@pytest.mark.parametrize("dtype", list(T))
def test_quantise_gives_the_values_of_the_lowest_and_of_the_greatest_exponents(uccl, dtype):
    """Where a block's greatest element is any power of two of the type, subnormal ones too, beside elements of every code and its middles: values are exact."""
    t = T[dtype]
    low, high = {"f32": (-149, 127), "bf16": (-133, 127), "f16": (-24, 15)}[dtype]
    e = torch.arange(low, high + 1, device="cuda")
    parts = torch.tensor([1.0, 1.5, 0.75, 0.625, 0.5, 0.4375, 0.375, 0.3125, 0.25, 0.1875, 0.125, 0.0625, 0.0, 1.75, 1.25, 0.0624], device="cuda", dtype=torch.float64)
    x = torch.zeros(len(e), 32, dtype=t, device="cuda")
    x[:, :16] = (torch.exp2(e.double())[:, None] * parts).to(t)
    x[:, 16:] = -x[:, :16]
    assert bool(x.isfinite().all())
    values, (_, q, s) = torch.full_like(x, 7.0), mx4_rows(len(e), 32)
    uccl.uccl_quantise_rows(q, s, x, values=values)
    number, byte = quantise_reference(x)
    assert torch.equal(s.view(torch.uint8).cpu().long(), byte) and torch.equal(codes_of(q, 32).cpu().long(), number)
    want = decode(q, s, 32)
    # below 2^-127 scales are that, and a half of it is 2^-128: f32 and bf16 hold all of these, and f16 what its own elements make
    assert torch.equal(values.double(), want)
