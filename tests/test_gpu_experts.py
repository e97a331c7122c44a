"""Routing, the order of rows, microscaled 4 bits and clipping on the GPU against plain implementations in 64 bits.

Tolerances are those of tests/test_gpu_rows.py: half a step of the result's type, and (n + 4) 2^-24 of the sum of the terms' magnitudes for n
operations in binary32.  An exponential's argument z - m is rounded once, which is (z - m) 2^-24 of the exponential; it and its quotient by a sum
of E of them are off by E + 8 more at most.  Choices, orders, 4-bit values and clipped gradients have one right answer each.
"""
import numpy as np
import pytest
import torch

from test_gpu_rows import T, aligned, close, gen, margin, normal

pytestmark = pytest.mark.gpu
E2M1, E8M0 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def uccl(gpu_lib):
    return gpu_lib


def i32(*shape, fill=-7):
    return torch.full(shape, fill, dtype=torch.int32, device="cuda")


def f32(*shape, fill=NAN):
    return torch.full(shape, fill, device="cuda")


def bytes_(n):
    return torch.full((max(n, 16),), 0xA5, dtype=torch.uint8, device="cuda")


# ---- routing --------------------------------------------------------------------------------------


def choice(scores, bias, slots):
    """The experts by the definition: binary32 keys, the greatest first, of equal ones the lowest."""
    key = scores.float() + (bias if bias is not None else 0.0)
    key = torch.where(key.isnan(), -INF, key)
    n = key.shape[1]
    at, out = torch.arange(n, device="cuda"), []
    for _ in range(slots):
        most = key.amax(1, keepdim=True)
        e = torch.where(key == most, at, n).amin(1)
        out.append(torch.where(most[:, 0] > -INF, e, -1))
        key = torch.where(at == e[:, None], -INF, key)
    return torch.stack(out, 1)


def softmax(scores):
    z = scores.double()
    return torch.where((z == -INF).all(1, keepdim=True), 0.0, torch.softmax(z, 1))


def weights_of(scores, experts, normalise, scale):
    """Weights in 64 bits, by the definition."""
    there = experts >= 0
    z = scores.double().gather(1, experts.clamp(min=0).long())
    if normalise:
        z = torch.where(there, z, -INF)
        w = torch.where(there.any(1, keepdim=True), torch.softmax(z, 1), 0.0)
        w = torch.where(scores.isnan().any(1, keepdim=True), NAN, w)
    else:
        w = softmax(scores).gather(1, experts.clamp(min=0).long())
    return torch.where(there, scale * w, 0.0)


def spread(scores):
    z = torch.where(scores.isinf() | scores.isnan(), 0.0, scores.double())
    return float(z.amax() - z.amin()) + 2.0


ROUTES = [(1, 1, 1), (3, 2, 2), (5, 8, 3), (33, 31, 6), (17, 61, 17), (300, 64, 8), (7, 65, 4), (40, 128, 32), (9, 129, 8), (1, 256, 8), (1025, 256, 8), (70, 250, 9), (11, 257, 8), (19, 512, 20),
          (13, 513, 5), (21, 1000, 32), (600, 1024, 8), (9001, 32, 2), (4097, 256, 6)]


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("tokens,n,slots", ROUTES)
def test_route(uccl, dtype, tokens, n, slots):
    g, t = gen(tokens + n), T[dtype]
    scores = normal(g, tokens, n, t, 2.0, pad=1)
    if n > 2:
        scores.masked_fill_(torch.rand(tokens, n, device="cuda", generator=g) < 0.2, -INF)
    if tokens > 4:
        scores[3] = -INF                                                  # nothing left
        scores[4, 1:] = -INF                                              # fewer than slots
    bias = torch.randn(n, device="cuda", generator=g)
    for b, normalise, scale, wanted in ((None, False, 1.0, True), (bias, True, 2.5, True), (bias, False, -0.5, False), (None, True, 1.0, False)):
        experts, w, counts, sums = i32(tokens, slots), f32(tokens, slots), i32(n), f32(n)
        scratch = bytes_(uccl.uccl_route_rows_scratch(tokens, n))
        uccl.uccl_route_rows(experts, w, scores, bias=b, normalise=normalise, scale=scale, **(dict(counts=counts, sums=sums, scratch=scratch) if wanted else {}))
        want = choice(scores, b, slots)
        assert torch.equal(experts.long(), want)
        ew = weights_of(scores, want, normalise, scale)
        close(w, ew, ew.abs() * (1 + spread(scores)), n + 8, "weights")
        if wanted:
            assert torch.equal(counts.long(), torch.bincount(want[want >= 0], minlength=n))
            es = softmax(scores).sum(0)
            close(sums, es, es * (1 + spread(scores)), n + tokens + 8, "sums")


def test_route_of_equal_scores_takes_the_lowest_expert(uccl):
    for dtype, t in T.items():
        scores = aligned(64, 200, t)
        scores.copy_((torch.rand(64, 200, device="cuda", generator=gen(1)) * 4).floor())
        scores[::2] *= -0.0                                              # zeros of both signs are equal
        experts, w = i32(64, 32), f32(64, 32)
        uccl.uccl_route_rows(experts, w, scores)
        assert torch.equal(experts.long(), choice(scores, None, 32)) and torch.equal(experts[0].long(), torch.arange(32, device="cuda"))


@pytest.mark.parametrize("n", [40, 256, 700])
def test_route_of_scores_that_are_not_finite(uccl, n):
    slots = 4
    scores = normal(gen(n), 8, n, torch.float32)
    scores[0, 5] = NAN
    scores[1, :] = NAN
    scores[2, 7] = INF
    scores[3, 9], scores[3, 11] = NAN, INF
    scores[4, :] = -INF
    scores[4, 0] = NAN
    bias = torch.zeros(n, device="cuda")
    bias[2], bias[3], bias[4] = -INF, NAN, INF
    scores[6, 4] = -INF                                                   # with a bias of +infinity: NaN, not chosen
    for normalise in (False, True):
        for b in (None, bias):
            experts, w, counts, sums = i32(8, slots), f32(8, slots), i32(n), f32(n)
            uccl.uccl_route_rows(experts, w, scores, bias=b, normalise=normalise, counts=counts, sums=sums, scratch=bytes_(uccl.uccl_route_rows_scratch(8, n)))
            want = choice(scores, b, slots)
            assert torch.equal(experts.long(), want)
            assert bool((w[experts < 0] == 0).all())
            broken = torch.tensor([0, 1, 2, 3], device="cuda")
            assert bool(w[broken][experts[broken] >= 0].isnan().all())
            ew = weights_of(scores, want, normalise, 1.0)
            whole = [4, 5, 6, 7]
            assert bool((w[4] == 0).all())
            close(w[whole[1:]], ew[whole[1:]], ew[whole[1:]].abs() * 20, n + 8, "weights")
            assert bool(sums.isnan().all()) and torch.equal(counts.long(), torch.bincount(want[want >= 0], minlength=n))


@pytest.mark.parametrize("tokens", [9, 2500])
@pytest.mark.parametrize("n", [40, 100, 256, 700])
@pytest.mark.parametrize("dtype", T)
def test_route_without_sums_is_route_with_them(uccl, dtype, n, tokens):
    """Normalised weights without sums are made without the sum over all experts: NaN and infinities of experts that are not chosen still count."""
    scores = normal(gen(tokens + n), tokens, n, T[dtype])
    scores[0, n - 1], scores[1, n - 1], scores[2, 0], scores[3, n // 2] = NAN, -INF, INF, NAN
    scores[4, :], scores[5, :], scores[6, 1:] = -INF, NAN, -INF
    scores[tokens - 1, n - 2] = NAN
    bias = torch.zeros(n, device="cuda")
    bias[n - 1] = -INF
    for normalise in (False, True):
        for b in (None, bias):
            experts, w, alike, v = i32(tokens, 4), f32(tokens, 4), i32(tokens, 4), f32(tokens, 4)
            uccl.uccl_route_rows(experts, w, scores, bias=b, normalise=normalise)
            uccl.uccl_route_rows(alike, v, scores, bias=b, normalise=normalise, counts=i32(n), sums=f32(n), scratch=bytes_(uccl.uccl_route_rows_scratch(tokens, n)))
            assert torch.equal(experts, alike) and torch.equal(w.view(torch.int32) << 1 == 0, v.view(torch.int32) << 1 == 0)
            assert torch.equal(w.isnan(), v.isnan()) and torch.equal(w.nan_to_num(), v.nan_to_num())
            for row in (0, 2, 3, 5, tokens - 1):
                assert bool(w[row][experts[row] >= 0].isnan().all()), row
            for row in (1, 4, 6, 7):
                assert not bool(w[row].isnan().any()), row


def test_route_by_a_bias_to_experts_whose_probability_is_nothing(uccl):
    """Normalised weights are relative to the chosen."""
    scores = aligned(2, 64, torch.float32)
    scores[:] = 0.0
    scores[:, 8:12] = torch.tensor([-200.0, -201.0, -203.0, -300.0], device="cuda")
    bias = torch.zeros(64, device="cuda")
    bias[8:12] = 1000.0
    experts, w = i32(2, 4), f32(2, 4)
    uccl.uccl_route_rows(experts, w, scores, bias=bias, normalise=True)
    assert experts.tolist() == [[8, 9, 10, 11]] * 2
    want = torch.softmax(torch.tensor([-200.0, -201.0, -203.0, -300.0], dtype=torch.float64, device="cuda"), 0).expand(2, 4)
    close(w, want, want * 4, 20, "weights")
    d, dz = f32(2, 4, fill=1.0), aligned(2, 64, torch.float32)
    d[:, 1] = 3.0
    uccl.uccl_route_rows_grad(dz, scores, experts, d, normalise=True)
    g = want * (d.double() - (want * d.double()).sum(1, keepdim=True))
    close(dz[:, 8:12], g, want * 16, 20, "dscores")
    assert bool((dz[:, :8] == 0).all()) and bool((dz[:, 12:] == 0).all())


def grad_reference(scores, experts, dweights, dsums, normalise, scale):
    """dscores in 64 bits, and the sum of the magnitudes of its terms."""
    p = softmax(scores)
    dz, mag = torch.zeros_like(p), torch.zeros_like(p)
    if dsums is not None:
        d = dsums.double()
        dz += p * (d - (p * d).sum(1, keepdim=True))
        mag += p * (d.abs() + (p * d.abs()).sum(1, keepdim=True))
    if experts is not None:
        there = (experts >= 0) & (experts < scores.shape[1])
        e = torch.where(there, experts, 0).long()
        g = torch.where(there, scale * dweights.double(), 0.0)
        q = torch.where(there, weights_of(scores, torch.where(there, experts, -1).long(), normalise, 1.0), 0.0)
        along, size = (q * g).sum(1, keepdim=True), (q * g.abs()).sum(1, keepdim=True)
        dz.scatter_add_(1, e, q * (g - along) if normalise else q * g)
        mag.scatter_add_(1, e, q * (g.abs() + size))
        if not normalise:
            dz -= p * along
            mag += p * size
    return dz, mag


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("tokens,n,slots", ROUTES)
def test_route_grad(uccl, dtype, tokens, n, slots):
    g, t = gen(tokens * 3 + n), T[dtype]
    scores = normal(g, tokens, n, t, 2.0, pad=1)
    if tokens > 4:
        scores[3] = -INF
        scores[4, 1:] = -INF
    experts = choice(scores, torch.randn(n, device="cuda", generator=g), slots).to(torch.int32)
    if tokens > 8:
        experts[7, 0], experts[8, -1] = n, 1 << 30                        # no experts
        experts[6] = experts[6, 0].item()                                 # the same one in every slot
    dw, ds = torch.randn(tokens, slots, device="cuda", generator=g), torch.randn(n, device="cuda", generator=g)
    for e, d, s, normalise, scale in ((experts, dw, ds, True, 2.5), (experts, dw, None, False, 1.0), (experts, dw, ds, False, -1.5), (experts, dw, None, True, 1.0), (None, None, ds, False, 1.0)):
        out = aligned(tokens, n, t, 2)
        around = margin(out)
        uccl.uccl_route_rows_grad(out, scores, e, d, dsums=s, normalise=normalise, scale=scale)
        want, mag = grad_reference(scores, e, d, s, normalise, scale)
        close(out, want, mag * (1 + spread(scores)), 2 * n + slots + 16, "dscores")
        assert torch.equal(margin(out), around)
    same = aligned(tokens, n, t).copy_(scores)
    uccl.uccl_route_rows_grad(same, same, experts, dw, dsums=ds)             # in place
    out = aligned(tokens, n, t)
    uccl.uccl_route_rows_grad(out, scores, experts, dw, dsums=ds)
    assert torch.equal(same, out)


@pytest.mark.parametrize("normalise", [False, True])
def test_route_grad_against_differences(uccl, normalise):
    """Of weights and balance loss together along random directions, from the definition in 64 bits with the choice held."""
    tokens, n, slots, coef, scale = 37, 24, 4, 0.3, 1.7
    g = gen(5)
    scores = normal(g, tokens, n, torch.float32)
    experts, w, counts, sums = i32(tokens, slots), f32(tokens, slots), i32(n), f32(n)
    scratch = bytes_(uccl.uccl_route_rows_scratch(tokens, n))
    uccl.uccl_route_rows(experts, w, scores, normalise=normalise, scale=scale, counts=counts, sums=sums, scratch=scratch)
    loss, ds = f32(1), f32(n)
    uccl.uccl_balance_loss(loss, ds, counts, sums, tokens, slots, coef)
    dw, dz = torch.randn(tokens, slots, device="cuda", generator=g), aligned(tokens, n, torch.float32)
    uccl.uccl_route_rows_grad(dz, scores, experts, dw, dsums=ds, normalise=normalise, scale=scale)

    def value(z):
        p = torch.softmax(z, 1)
        mine = p.gather(1, experts.long())
        if normalise:
            mine = mine / mine.sum(1, keepdim=True)
        balance = coef * n / (slots * tokens ** 2) * (counts.double() * p.sum(0)).sum()
        return float((scale * mine * dw.double()).sum() + balance)
    for seed in range(3):
        way = torch.randn(tokens, n, dtype=torch.float64, device="cuda", generator=gen(seed))
        h = 1e-5
        slope = (value(scores.double() + h * way) - value(scores.double() - h * way)) / (2 * h)
        along = float((dz.double() * way).sum())
        # the difference is off by h^2 of the third derivative, about 1e-10 of the terms, and by 2^-52 / h of the value
        size = float((dz.double() * way).abs().sum())
        assert abs(slope - along) <= size * (1e-6 + (2 * n + 32) * 2.0 ** -24) + 1e-8


@pytest.mark.parametrize("n,tokens,slots", [(1, 1, 1), (8, 100, 2), (256, 32768, 8), (1000, 7, 32), (5000, 1 << 40, 3)])
def test_balance_loss(uccl, n, tokens, slots):
    g = gen(n)
    counts = torch.randint(0, 10000, (n,), dtype=torch.int32, device="cuda", generator=g)
    sums = torch.rand(n, device="cuda", generator=g) * 100
    loss, ds = f32(1), f32(n)
    uccl.uccl_balance_loss(loss, ds, counts, sums, tokens, slots, 0.01)
    c = float(torch.tensor(0.01))                                          # as binary32 has it
    ed = c * n / (slots * float(tokens) ** 2) * counts.double()
    close(ds, ed, ed, 0, "dsums")
    close(loss, (ed * sums.double()).sum()[None], (ed * sums.double()).sum()[None] * 1e-6, 0, "loss")
    again = sums.clone()
    uccl.uccl_balance_loss(None, again, counts, again, tokens, slots, 0.01)
    assert torch.equal(again, ds)
    alone = f32(1)
    uccl.uccl_balance_loss(alone, None, counts, sums, tokens, slots, 0.01)
    assert torch.equal(alone, loss)


def test_balance_loss_of_even_use_is_its_coefficient(uccl):
    loss, n, tokens, slots = f32(1), 64, 128, 4
    uccl.uccl_balance_loss(loss, None, torch.full((n,), tokens * slots // n, dtype=torch.int32, device="cuda"), torch.full((n,), tokens / n, device="cuda"), tokens, slots, 0.25)
    assert loss.item() == 0.25
    uccl.uccl_balance_loss(loss, None, i32(0), f32(0), 1, 1, 0.25)         # no experts
    assert loss.item() == 0.0


# ---- the order of rows ----------------------------------------------------------------------------


def plan_reference(experts, n):
    flat = experts.cpu().numpy().reshape(-1).astype(np.int64)
    key = np.where((flat < 0) | (flat >= n), n, flat)
    order = np.argsort(key, kind="stable")
    offsets = np.searchsorted(key[order], np.arange(n + 1))
    pos = np.empty_like(flat)
    pos[order] = np.arange(len(flat))
    slots = experts.shape[1]
    return np.where(key[order] < n, order // max(slots, 1), -1), offsets, np.where(key == n, -1, pos).reshape(experts.shape)


PLANS = [(1, 1, 1), (1, 8, 256), (5, 3, 2), (63, 1, 7), (64, 1, 1024), (511, 2, 1), (512, 2, 33), (1025, 1, 64), (1023, 3, 1000), (4096, 8, 256), (40000, 4, 61), (32768, 8, 256), (150001, 1, 5), (70000, 6, 1024)]


@pytest.mark.parametrize("tokens,slots,n", PLANS)
@pytest.mark.parametrize("how", ["even", "skewed", "missing", "sorted"])
def test_plan(uccl, tokens, slots, n, how):
    r = np.random.default_rng(tokens + n)
    e = r.integers(0, n, (tokens, slots))
    if how == "skewed":
        e = np.minimum(e, r.integers(0, n, (tokens, slots)) ** 2 // max(n, 1))
    if how == "missing":
        e = np.where(r.random((tokens, slots)) < 0.5, r.choice([-1, n, -2 ** 31, 2 ** 31 - 1], (tokens, slots)), e)
    if how == "sorted":
        e = np.sort(e.reshape(-1)).reshape(tokens, slots)
    experts = torch.from_numpy(e.astype(np.int32)).cuda()
    index, offsets, pos = i32(tokens * slots), i32(n + 1), i32(tokens, slots)
    scratch = bytes_(uccl.uccl_plan_rows_scratch(tokens * slots, n))
    uccl.uccl_plan_rows(index, offsets, pos, experts, scratch)
    wi, wo, wp = plan_reference(experts, n)
    assert np.array_equal(offsets.cpu().numpy(), wo) and np.array_equal(pos.cpu().numpy(), wp) and np.array_equal(index.cpu().numpy(), wi)
    alone, only = i32(n + 1), i32(tokens * slots)
    uccl.uccl_plan_rows(None, alone, None, experts, scratch)
    assert torch.equal(alone, offsets)
    uccl.uccl_plan_rows(only, alone, None, experts, scratch)
    assert torch.equal(only, index)
    same = experts.clone()
    uccl.uccl_plan_rows(None, alone, same, same, scratch)                    # in place
    assert torch.equal(same, pos)


def test_plan_of_nothing(uccl):
    for tokens, slots in ((0, 4), (4, 0)):
        offsets = i32(5)
        uccl.uccl_plan_rows(i32(0), offsets, i32(tokens, slots), i32(tokens, slots))
        assert offsets.tolist() == [0] * 5


# ---- rows in 4 bits -------------------------------------------------------------------------------

MAGNITUDES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def mx4_rows(rows, cols, fill=0xFF):
    """Values and scales as wire rows, with something between them."""
    at, more = -(-cols // 32) * 16, -(-cols // 512) * 16 + 16
    wire = torch.full((rows, at + more), fill, dtype=torch.uint8, device="cuda")
    return wire, wire[:, :-(-cols // 2)].view(E2M1), wire[:, at:at - (-cols // 32)].view(E8M0)


def codes_of(q, cols):
    b = q.view(torch.uint8)
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)[..., :cols]


def decode(q, scales, cols):
    """What packed rows stand for, in 64 bits."""
    c = codes_of(q, cols)
    v = MAGNITUDES.cuda()[(c & 7).long()] * torch.where(c >= 8, -1.0, 1.0)
    s = scales.view(torch.uint8).double()
    s = torch.where(s == 255, NAN, torch.exp2(s - 127))
    return v * s.repeat_interleave(32, -1)[..., :cols]


def quantise_reference(x):
    """The numbers of the magnitudes (with 8 for a sign) and the scales' bytes."""
    x = x.double().cpu()
    rows, cols = x.shape
    blocks = torch.nn.functional.pad(x, (0, -cols % 32)).view(rows, -1, 32)
    broken = ~blocks.isfinite().all(2)
    most = torch.where(broken, 1.0, blocks.abs().amax(2))
    mant, e = torch.frexp(most)
    byte = torch.where(most == 0, 0, (e - 1 - 2 + 127).clamp(min=0))
    v = blocks / torch.exp2(byte.double() - 127)[..., None]
    mids = (MAGNITUDES[1:] + MAGNITUDES[:-1]) / 2
    below, above = torch.searchsorted(mids, v.abs().contiguous()), torch.searchsorted(mids, v.abs().contiguous(), right=True)
    number = torch.where(below % 2 == 0, below, above) + 8 * torch.signbit(v).long()
    number = torch.where(broken[..., None], 0, number)
    return number.view(rows, -1)[:, :cols], torch.where(broken, 255, byte)


QUANTISED_COLS = [1, 2, 3, 31, 32, 33, 63, 64, 100, 255, 520, 2043, 7168, 16384, 20001]


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("cols", QUANTISED_COLS)
def test_quantise(uccl, dtype, cols):
    t, rows, g = T[dtype], 6, gen(cols)
    x = normal(g, rows, cols, t, pad=1)
    x.mul_(torch.exp2(torch.randint(-12, 12, (rows, 1), device="cuda", generator=g).to(t)))
    x[1] = 0.0
    x[2].mul_(-0.0)
    if cols > 40:
        x[3, 33:] = 0.0
        x[4, 7], x[4, 35], x[4, 70 % cols] = NAN, INF, -INF
    wire, q, scales = mx4_rows(rows, cols)
    before, values = wire.clone(), aligned(rows, cols, t, 1)
    around = margin(values)
    uccl.uccl_quantise_rows(q, scales, x, values=values)
    number, byte = quantise_reference(x)
    assert torch.equal(scales.view(torch.uint8).cpu().long(), byte)
    assert torch.equal(codes_of(q, cols).cpu().long(), number)
    if cols % 2:
        assert bool((q.view(torch.uint8)[:, -1] >> 4 == 0).all())
    n, at = -(-cols // 2), -(-cols // 32) * 16
    assert torch.equal(wire[:, n:at], before[:, n:at]) and torch.equal(wire[:, at - (-cols // 32):], before[:, at - (-cols // 32):])
    want = decode(q, scales, cols)
    assert torch.equal(values.double().nan_to_num(nan=1e300), want.nan_to_num(nan=1e300)) and torch.equal(margin(values), around)
    _, again, s = mx4_rows(rows, cols)
    uccl.uccl_quantise_rows(again, s, x)
    assert torch.equal(again.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s.view(torch.uint8), scales.view(torch.uint8))
    uccl.uccl_quantise_rows(again, s, x, values=x)                           # in place
    assert torch.equal(x.view(torch.uint8), values.contiguous().view(torch.uint8) if x.is_contiguous() else values.view(torch.uint8))


def test_quantise_of_every_middle_and_its_neighbours(uccl):
    m = torch.cat([MAGNITUDES, (MAGNITUDES[1:] + MAGNITUDES[:-1]) / 2, torch.tensor([6.5, 7.0, 7.5])]).float()
    v = torch.cat([m, torch.nextafter(m, torch.tensor(9.0)), torch.nextafter(m, torch.tensor(0.0))])
    v = torch.cat([v, -v])
    for e in (-149, -130, -127, -126, -100, -3, 0, 5, 100, 124):
        x = aligned(v.numel(), 32, torch.float32, fill=0.0)
        x[:] = 0.0
        x[:, 0] = torch.ldexp(torch.tensor(4.0), torch.tensor(e)).item() if e > -149 else 0.0
        x[:, 1] = torch.ldexp(v.double(), torch.tensor(e)).float().cuda()
        _, q, s = mx4_rows(v.numel(), 32)
        uccl.uccl_quantise_rows(q, s, x)
        number, byte = quantise_reference(x)
        assert torch.equal(s.view(torch.uint8).cpu().long(), byte) and torch.equal(codes_of(q, 32).cpu().long(), number), e


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_quantise_of_every_16_bit_value(uccl, dtype):
    """Beside a greatest element of every exponent: all values up to twice that."""
    t = T[dtype]
    every = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(t).cuda()
    every = every[every.isfinite()]
    for e in [None] + list(range(-130, 128, 3) if dtype == "bf16" else range(-24, 16)):
        most = torch.tensor(0.0 if e is None else 2.0 ** e, device="cuda").to(t)
        v = every[every.abs() < 2 * most] if e is not None else every
        x = torch.zeros(v.numel(), 32, dtype=t, device="cuda")
        x[:, 31], x[:, 3] = most, v
        _, q, s = mx4_rows(v.numel(), 32)
        values = torch.zeros_like(x)
        uccl.uccl_quantise_rows(q, s, x, values=values)
        number, byte = quantise_reference(x)
        assert torch.equal(s.view(torch.uint8).cpu().long(), byte) and torch.equal(codes_of(q, 32).cpu().long(), number), e
        assert torch.equal(values.double(), decode(q, s, 32)), e


def test_quantise_many_rows_and_few_columns(uccl):
    for rows, cols in ((5000, 33), (70000, 1), (3, 40000), (4000, 999), (300, 7171), (9, 32)):
        x = normal(gen(rows), rows, cols, torch.bfloat16)
        _, q, s = mx4_rows(rows, cols)
        uccl.uccl_quantise_rows(q, s, x)
        number, byte = quantise_reference(x)
        assert torch.equal(s.view(torch.uint8).cpu().long(), byte) and torch.equal(codes_of(q, cols).cpu().long(), number)


# ---- products of weights in 4 bits ----------------------------------------------------------------


def random_mx4(g, rows, cols, low=117, high=128):
    """Any codes, scales of these bytes; what is behind the values and scales of a row would be seen."""
    _, q, s = mx4_rows(rows, cols)
    q.view(torch.uint8).copy_(torch.randint(0, 256, q.shape, device="cuda", generator=g))
    s.view(torch.uint8).copy_(torch.randint(low, high, s.shape, device="cuda", generator=g))
    return q, s


def product_reference(x, w, index, ends):
    y, mag = torch.zeros(ends[-1], w.shape[1], dtype=torch.float64, device="cuda"), torch.zeros(ends[-1], w.shape[1], dtype=torch.float64, device="cuda")
    rows = x if index is None else torch.where(((index >= 0) & (index < len(x)))[:, None], x[index.clamp(0, len(x) - 1).long()], 0.0)
    for k, (b, e) in enumerate(zip(ends, ends[1:])):
        if e > b:
            y[b:e], mag[b:e] = rows[b:e] @ w[k].T.contiguous(), rows[b:e].abs() @ w[k].abs().T.contiguous()
    return y, mag


def ends_of(rows, groups, seed):
    r = np.random.default_rng(seed)
    return [0] + sorted(r.integers(0, rows + 1, groups - 1).tolist()) + [rows]


KINDS = ["mx4", "bf16", "f16"]
PRODUCTS = [(1, 1, 16, 32), (1, 3, 5, 1), (7, 2, 33, 31), (16, 8, 64, 33), (5, 1, 100, 127), (3, 2, 17, 128), (40, 5, 130, 129), (20, 70, 40, 200), (33, 4, 257, 255), (129, 3, 128, 256), (200, 2, 300, 511),
            (64, 1, 512, 1000), (300, 6, 129, 520), (17, 4, 1003, 2043), (600, 3, 700, 300), (1, 1, 2048, 7168), (257, 1, 513, 1024), (1030, 5, 260, 640), (2100, 2, 300, 776)]


def make_x(g, kind, rows, cols):
    if kind == "mx4":
        q, s = random_mx4(g, rows, cols)
        return q, s, decode(q, s, cols)
    x = normal(g, rows, cols, T[kind], pad=1)
    return x, None, x.double()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,groups,wide,cols", PRODUCTS)
def test_product(uccl, kind, rows, groups, wide, cols):
    if kind == "mx4" and cols % 2:
        cols += 1                                                          # packed rows on both sides have whole bytes here
    g = gen(rows + cols)
    w, ws = random_mx4(g, groups * wide, cols)
    dw = decode(w, ws, cols).view(groups, wide, cols)
    w, ws = w.view(torch.uint8).unflatten(0, (groups, wide)).view(E2M1), ws.view(torch.uint8).unflatten(0, (groups, wide)).view(E8M0)
    ends = ends_of(rows, groups, rows)
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    x, xs, dx = make_x(g, kind, max(rows, 9), cols)
    index = torch.randint(0, len(dx), (rows,), dtype=torch.int32, device="cuda", generator=g)
    index[0] = -1 if rows > 1 else 0
    if rows > 3:
        index[2] = len(dx)
    for i, out in ((None, torch.bfloat16), (index, torch.float16), (index, torch.float32)):
        y = aligned(rows + 2, wide, out, 1)
        around, end = margin(y), y[rows:].clone()
        uccl.uccl_group_product(y[:rows], x[:rows] if i is None and kind != "mx4" else x, w, offsets, index=i, x_scales=xs, w_scales=ws)
        want, mag = product_reference(dx, dw, i, ends)
        close(y[:rows], want, mag, cols, f"{kind} to {out}")
        assert torch.equal(margin(y), around) and torch.equal(y[rows:].view(torch.uint8), end.view(torch.uint8))


# sums long enough for every kernel's steady state, by every kernel (tests/test_experts_abi.py has which): rows, groups, columns, depth
DEEP = [(1500, 2, 1030, 4000), (700, 5, 520, 2600), (4500, 3, 2060, 1300), (90, 3, 200, 5000), (1300, 1, 4100, 1500), (400, 1, 1900, 3000), (6000, 1, 4200, 900), (4300, 2, 2040, 1000)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,groups,wide,cols", DEEP)
def test_product_of_long_sums(uccl, kind, rows, groups, wide, cols):
    g = gen(rows + wide)
    w, ws = random_mx4(g, groups * wide, cols)
    dw = decode(w, ws, cols).view(groups, wide, cols)
    w, ws = w.view(torch.uint8).unflatten(0, (groups, wide)).view(E2M1), ws.view(torch.uint8).unflatten(0, (groups, wide)).view(E8M0)
    x, xs, dx = make_x(g, kind, rows, cols)
    index = torch.randperm(rows, device="cuda", generator=g).to(torch.int32)
    index[::17] = -1
    ends = ends_of(rows, groups, rows)
    offsets, y, again = torch.tensor(ends, dtype=torch.int32, device="cuda"), aligned(rows, wide, torch.float32), aligned(rows, wide, torch.float32)
    for out in (y, again):
        uccl.uccl_group_product(out, x, w, offsets, index=index, x_scales=xs, w_scales=ws)
    want, mag = product_reference(dx, dw, index, ends)
    close(y, want, mag, cols, kind)
    assert torch.equal(y, again)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,groups,wide", [(500, 1, 520), (1500, 2, 1030), (150, 8, 1000)])
@pytest.mark.parametrize("cols", [32, 96, 250, 300, 514, 600, 900, 1100, 1358, 1410, 2600])
def test_product_by_small_tiles_of_short_sums(uccl, kind, rows, groups, wide, cols):
    """Of one stage of a ring, two, three and so on, whole ones and not."""
    test_product_of_long_sums(uccl, kind, rows, groups, wide, cols)


@pytest.mark.parametrize("kind", KINDS)
def test_product_of_an_odd_number_of_columns_by_the_struct(uccl, kind):
    """The half byte behind the last element holds anything."""
    import ctypes as C
    g, rows, wide, cols = gen(4), 20, 40, 165
    w, ws = random_mx4(g, wide, cols)
    x, xs, dx = make_x(g, kind, rows, cols)
    y, offsets = aligned(rows, wide, torch.float32), torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    rows_of = lambda t, s, n: C.byref(uccl.uccl_rows(t.data_ptr(), t.stride(0) * t.element_size(), s.data_ptr(), s.stride(0), n, cols, uccl.UCCL_MX4, 0))  # noqa: E731
    xr = rows_of(x, xs, rows) if kind == "mx4" else C.byref(uccl.uccl_rows(x.data_ptr(), x.stride(0) * 2, None, 0, rows, cols, uccl.UCCL_BF16 if kind == "bf16" else uccl.UCCL_F16, 0))
    yr = C.byref(uccl.uccl_rows(y.data_ptr(), y.stride(0) * 4, None, 0, rows, wide, uccl.UCCL_F32, 0))
    assert uccl.load().uccl_group_product(yr, xr, None, rows_of(w, ws, wide), offsets.data_ptr(), 1, torch.cuda.current_stream().cuda_stream) == 0
    want, mag = product_reference(dx, decode(w, ws, cols)[None], None, [0, rows])
    close(y, want, mag, cols, kind)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [3, 100, 700])
def test_product_of_no_columns_and_of_no_rows(uccl, kind, rows):
    """Empty sums; and rows that an index takes from nothing."""
    import ctypes as C
    wide, offsets, index = 300, torch.tensor([0, rows - 1], dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    some = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda").data_ptr()
    code = {"mx4": uccl.UCCL_MX4, "bf16": uccl.UCCL_BF16, "f16": uccl.UCCL_F16}[kind]
    for x_rows, cols, take in ((rows, 0, None), (0, 256, index)):
        y = torch.full((rows, wide), 7.0, device="cuda")
        yr = C.byref(uccl.uccl_rows(y.data_ptr(), wide * 4, None, 0, rows, wide, uccl.UCCL_F32, 0))
        xr = C.byref(uccl.uccl_rows(some, 512, some if kind == "mx4" else None, 8, x_rows, cols, code, 0))
        wr = C.byref(uccl.uccl_rows(some, 128, some, 8, wide, cols, uccl.UCCL_MX4, 0))
        assert uccl.load().uccl_group_product(yr, xr, None if take is None else take.data_ptr(), wr, offsets.data_ptr(), 1, torch.cuda.current_stream().cuda_stream) == 0
        assert bool((y[:rows - 1] == 0).all()) and bool((y[rows - 1:] == 7).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [3, 100, 700])
def test_product_of_scales_far_apart_and_values_that_are_not_finite(uccl, kind, rows):
    g, wide, cols = gen(rows), 300, 640
    w, ws = random_mx4(g, wide, cols, 60, 195)
    b = ws.view(torch.uint8)
    b[5, 3], b[6, 0], b[7, :] = 255, 0, 0
    x, xs, dx = make_x(g, kind, rows, cols)
    if kind == "mx4":
        xs.view(torch.uint8)[1, 2], xs.view(torch.uint8)[2, :] = 255, 0
    else:
        x[1, 70], x[2, 5], x[2, 6] = NAN, INF, 65504.0 if kind == "f16" else 3e38
        x[0, :], x[0, ::3] = 2.0 ** -24, 2.0 ** -14 * (1 + 1 / 512)
    dx, dw = (decode(x, xs, cols) if kind == "mx4" else x.double()), decode(w, ws, cols)
    y, offsets = aligned(rows, wide, torch.float32), torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    uccl.uccl_group_product(y, x, w.view(torch.uint8)[None].view(E2M1), offsets, x_scales=xs, w_scales=ws.view(torch.uint8)[None].view(E8M0))
    clean = torch.ones(rows, dtype=torch.bool, device="cuda")
    clean[1] = False
    if kind != "mx4":
        clean[2] = False
    cols_clean = torch.ones(wide, dtype=torch.bool, device="cuda")
    cols_clean[5] = False
    want, mag = product_reference(torch.where(clean[:, None], dx, 0.0), torch.where(cols_clean[:, None], dw, 0.0)[None], None, [0, rows])
    close(y[clean][:, cols_clean], want[clean][:, cols_clean], mag[clean][:, cols_clean], cols, kind)
    assert bool(y[:, 5].isnan().all()) and bool(y[1].isnan().all())
    if kind != "mx4":
        assert bool((~y[2].isfinite()).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [2, 90, 600])
def test_product_adds_small_terms_beside_large_ones_that_cancel(uccl, kind, rows):
    """Large terms and their opposites in one block, small ones in others: exact, for the large ones' sum is."""
    wide, cols = 64, 768
    g = gen(rows)
    w, ws = random_mx4(g, wide, cols)
    wc, wb = w.view(torch.uint8), ws.view(torch.uint8)
    wc[:], wb[:] = 0, 127 - 10                                              # small: 2^-10 times 1
    wc[:, 0] = 7 | 15 << 4                                                 # 6, -6 with the scale 2^10
    wb[:, 0] = 137
    wc[:, 40], wc[:, 200], wc[:, 300] = 2, 2 << 4, 2                         # ones in the small blocks
    if kind == "mx4":
        x, xs = random_mx4(g, rows, cols)
        x.view(torch.uint8)[:], xs.view(torch.uint8)[:] = 2 | 2 << 4, 127     # ones
    else:
        x, xs = aligned(rows, cols, T[kind]), None
        x[:] = 1.0
    y, offsets = aligned(rows, wide, torch.float32), torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    uccl.uccl_group_product(y, x, wc[None].view(E2M1), offsets, x_scales=xs, w_scales=wb[None].view(E8M0))
    assert bool((y == 3 * 2.0 ** -10).all())


@pytest.mark.parametrize("kind", KINDS)
def test_product_of_offsets_that_say_something_else(uccl, kind):
    """Descending, negative, past the rows: as documented.  Rows of no group are left."""
    g, rows, groups, wide, cols = gen(8), 50, 5, 48, 96
    w, ws = random_mx4(g, groups * wide, cols)
    dw = decode(w, ws, cols).view(groups, wide, cols)
    x, xs, dx = make_x(g, kind, rows, cols)
    for given, used in (([-5, 10, 4, 30, 99, 7], [0, 10, 10, 30, 50, 50]), ([3, 3, 9, 9, 20, 41], [3, 3, 9, 9, 20, 41]), ([60] * 6, [50] * 6)):
        y = torch.full((rows, wide), 7.0, device="cuda")
        uccl.uccl_group_product(y, x, w.view(torch.uint8).unflatten(0, (groups, wide)).view(E2M1), torch.tensor(given, dtype=torch.int32, device="cuda"), x_scales=xs,
                                w_scales=ws.view(torch.uint8).unflatten(0, (groups, wide)).view(E8M0))
        want, mag = torch.full((rows, wide), 7.0, dtype=torch.float64, device="cuda"), torch.zeros(rows, wide, dtype=torch.float64, device="cuda")
        for k in range(groups):
            b, e = used[k], used[k + 1]
            want[b:e], mag[b:e] = dx[b:e] @ dw[k].T.contiguous(), dx[b:e].abs() @ dw[k].abs().T.contiguous()
        close(y, want, mag, cols, kind)


# ---- clipping -------------------------------------------------------------------------------------


def gradients(sizes, seed, dtypes=("f32", "bf16", "f16"), std=1.0):
    g = gen(seed)
    return [(torch.randn(*s, device="cuda", generator=g) * std).to(T[dtypes[i % len(dtypes)]]) for i, s in enumerate(sizes)]


def norm_of(uccl, grads):
    norm = f32(1)
    uccl.uccl_gradient_norm(norm, grads, bytes_(uccl.uccl_gradient_norm_scratch(len(grads))))
    return norm


SIZES = [[(1,)], [(5,), (7, 3), (2, 3, 4)], [(1000003,)], [(1 + 37 * i,) for i in range(64)], [(3, 5)] * 65, [(i % 9, 16) for i in range(200)], [(4100, 2048), (8,), (17,)], [(300, 1003), (129, 2043)]]


@pytest.mark.parametrize("sizes", SIZES, ids=[str(i) for i in range(len(SIZES))])
def test_gradient_norm_and_clip(uccl, sizes):
    for dtypes in (("f32",), ("bf16",), ("f32", "bf16", "f16")):
        grads = gradients(sizes, len(sizes), dtypes)
        want = torch.sqrt(sum((t.double() ** 2).sum() for t in grads))[None]
        norm = norm_of(uccl, grads)
        close(norm, want, want, 0, "norm")
        for most in (float(want) * 0.37, float(want) * 1.5, 1e-6):
            by = torch.clamp(torch.tensor(most, device="cuda") / norm, max=1.0)
            out = [torch.full_like(t, 9.0) for t in grads]
            uccl.uccl_gradient_clip(out, grads, norm, most)
            for o, t in zip(out, grads):
                assert torch.equal(o, (t.float() * by).to(t.dtype))
            same = [t.clone() for t in grads]
            uccl.uccl_gradient_clip(same, same, norm, most)                 # in place
            assert all(torch.equal(o, s) for o, s in zip(out, same))


def test_gradient_norm_and_clip_of_rows_with_gaps(uccl):
    wide = [normal(gen(1), 37, 100, torch.float32, pad=3), normal(gen(2), 1000, 1001, torch.bfloat16, pad=1), torch.randn(6, 8, 64, device="cuda")[:, :, :16]]
    grads = [wide[0], wide[1], wide[2][:, :1], torch.randn(3, 40, 64, device="cuda")[:1, :, :17]]
    want = torch.sqrt(sum((t.double() ** 2).sum() for t in grads))[None]
    norm = norm_of(uccl, grads)
    close(norm, want, want, 0, "norm")
    out = [aligned(37, 100, torch.float32), aligned(1000, 1001, torch.bfloat16, 2), torch.zeros(6, 4, 32, device="cuda")[:, :1, :16], torch.zeros(1, 40, 20, device="cuda")[:, :, :17]]
    around = margin(out[0]), margin(out[1])
    uccl.uccl_gradient_clip(out, grads, norm, 0.5)
    by = torch.tensor(0.5, device="cuda") / norm
    assert all(torch.equal(o, (t.float() * by).to(t.dtype)) for o, t in zip(out, grads))
    assert torch.equal(margin(out[0]), around[0]) and torch.equal(margin(out[1]), around[1])


def test_gradient_norm_of_huge_tiny_and_broken_values(uccl):
    for value, n in ((3e38, 1), (1e38, 9), (1e-40, 1000), (1e-30, 12345), (0.0, 100)):
        grads = [torch.full((n,), value, device="cuda"), torch.zeros(3, device="cuda")]
        want = (grads[0].double() ** 2).sum().sqrt()[None]
        close(norm_of(uccl, grads), want, want, 0, str(value))
    assert norm_of(uccl, [torch.full((9,), 3e38, device="cuda")]).item() == INF      # past binary32
    assert norm_of(uccl, [torch.tensor([1.0, INF], device="cuda")]).item() == INF
    assert norm_of(uccl, [torch.tensor([1.0, NAN, INF], device="cuda")]).isnan().item()
    assert norm_of(uccl, []).item() == 0.0 and norm_of(uccl, [torch.zeros(0, device="cuda")]).item() == 0.0
    g = [torch.tensor([1.0, -2.0, INF], device="cuda")]
    uccl.uccl_gradient_clip(g, g, torch.tensor([INF], device="cuda"), 1.0)
    assert g[0][:2].tolist() == [0.0, -0.0] and g[0][2].isnan()
    g = [torch.tensor([1.0, 0.0], device="cuda")]
    uccl.uccl_gradient_clip(g, g, torch.tensor([NAN], device="cuda"), 1.0)
    assert g[0].isnan().all()
    g = [torch.tensor([1.0, 0.5], device="cuda")]
    uccl.uccl_gradient_clip(g, g, torch.tensor([0.0], device="cuda"), 1.0)
    assert g[0].tolist() == [1.0, 0.5]


# ---- all of them: streams, graphs, the same bits ---------------------------------------------------


def all_calls(uccl, seed):
    """Each operator once on inputs of this seed: a function that makes the calls, and the outputs."""
    g = gen(seed)
    tokens, n, slots, cols, wide = 3000, 40, 4, 320, 200
    scores = normal(g, tokens, n, torch.bfloat16)
    experts, w, counts, sums, loss, ds = i32(tokens, slots), f32(tokens, slots), i32(n), f32(n), f32(1), f32(n)
    index, offsets, pos = i32(tokens * slots), i32(n + 1), i32(tokens, slots)
    dw, dz = torch.randn(tokens, slots, device="cuda", generator=g), aligned(tokens, n, torch.bfloat16)
    x = normal(g, tokens, cols, torch.bfloat16)
    _, q, qs = mx4_rows(tokens, cols, 0)
    values = aligned(tokens, cols, torch.bfloat16, fill=0.0)
    b, bs = random_mx4(g, n * wide, cols)
    b, bs = b.view(torch.uint8).unflatten(0, (n, wide)).view(E2M1), bs.view(torch.uint8).unflatten(0, (n, wide)).view(E8M0)
    y, z = torch.zeros(tokens * slots, wide, dtype=torch.bfloat16, device="cuda"), torch.zeros(tokens * slots, wide, device="cuda")
    grads = gradients([(100, 100), (77,), (3000, 333)], seed)
    norm, out = f32(1), [torch.zeros_like(t) for t in grads]
    scratch = [bytes_(k) for k in (uccl.uccl_route_rows_scratch(tokens, n), uccl.uccl_plan_rows_scratch(tokens * slots, n), uccl.uccl_gradient_norm_scratch(3))]

    def run(stream=None):
        uccl.uccl_route_rows(experts, w, scores, normalise=True, counts=counts, sums=sums, scratch=scratch[0], stream=stream)
        uccl.uccl_plan_rows(index, offsets, pos, experts, scratch[1], stream=stream)
        uccl.uccl_balance_loss(loss, ds, counts, sums, tokens, slots, 0.1, stream=stream)
        uccl.uccl_route_rows_grad(dz, scores, experts, dw, dsums=ds, normalise=True, stream=stream)
        uccl.uccl_quantise_rows(q, qs, x, values=values, stream=stream)
        uccl.uccl_group_product(y, q, b, offsets, index=index, x_scales=qs, w_scales=bs, stream=stream)
        uccl.uccl_group_product(z, x, b, offsets, index=index, w_scales=bs, stream=stream)
        uccl.uccl_gradient_norm(norm, grads, scratch[2], stream=stream)
        uccl.uccl_gradient_clip(out, grads, norm, 1.0, stream=stream)
    results = [experts, w, counts, sums, loss, ds, index, offsets, pos, dz, q.view(torch.uint8), qs.view(torch.uint8), values, y, z, norm, *out]
    return run, results, scores


def test_results_are_the_same_on_another_stream_and_in_a_graph(uccl):
    run, results, scores = all_calls(uccl, 3)
    run()
    torch.cuda.synchronize()
    first = [r.clone() for r in results]
    assert not any(bool(r.isnan().any()) for r in first if r.is_floating_point())

    def wipe():
        for r in results:
            r.zero_()
        torch.cuda.synchronize()
    side = torch.cuda.Stream()
    wipe()
    run(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, results))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for k in range(4):
        wipe()
        if k == 2:                                                        # other inputs, and the first ones again
            scores.neg_()
        graph.replay()
        torch.cuda.synchronize()
        if k == 2:
            eager = [r.clone() for r in results]
            run()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, results)) and not torch.equal(eager[0], first[0])
            scores.neg_()
        else:
            assert all(torch.equal(a, b) for a, b in zip(first, results))
    other, theirs, _ = all_calls(uccl, 4)                                   # two graphs with scratch of their own, on two streams at once
    other()
    torch.cuda.synchronize()
    kept, second = [r.clone() for r in theirs], torch.cuda.CUDAGraph()
    with torch.cuda.graph(second):
        other()
    wipe()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(a):
            graph.replay()
        with torch.cuda.stream(b):
            second.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, r) for p, r in zip(first, results)) and all(torch.equal(p, r) for p, r in zip(kept, theirs))


def test_prepared_calls(uccl):
    run, results, scores = all_calls(uccl, 6)
    experts, w = i32(3000, 4), f32(3000, 4)
    call = uccl.uccl_prepare(uccl.uccl_route_rows, experts, w, scores, normalise=True, scale=1.0)
    grads = gradients([(100,), (5, 5)], 1)
    norm, scratch = f32(1), bytes_(uccl.uccl_gradient_norm_scratch(2))
    of_norm, of_clip = uccl.uccl_prepare(uccl.uccl_gradient_norm, norm, grads, scratch), uccl.uccl_prepare(uccl.uccl_gradient_clip, grads, grads, norm, 1.0)
    run()
    for _ in range(2):
        experts.zero_()
        call()
        assert torch.equal(experts, results[0]) and torch.equal(w, results[1])
    want = torch.sqrt(sum((t.double() ** 2).sum() for t in grads))[None]
    of_norm()
    close(norm, want, want, 0, "norm")
    of_clip()
    of_norm()
    assert abs(norm.item() - 1.0) < 2.0 ** -8
