"""The row operators on the GPU against plain implementations in 64 bits.

Tolerances.  A result is computed in binary32 from inputs as they are and rounded once to its type, so it may be off by half a step of
its type, `eps / 2` of the result, and by what binary32 sums accumulate: at most (n + 4) 2^-24 of the sum of the terms' magnitudes for n
terms, however they are ordered.  Both are counted, term by term, in `close`; bounds of sums are worst cases, so nothing here goes
by luck.  (Matrix instructions add a few products at a time before they round; that is another order of the same sum.)
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E8 = torch.float8_e4m3fn
U = 2.0 ** -24


@pytest.fixture(scope="module")
def uccl(gpu_lib):
    return gpu_lib


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def aligned(rows, cols, dtype, pad=0, fill=float("nan")):
    """Rows on 16-byte boundaries in a buffer whose other elements are `fill` (by bytes for 8 bits: NaN too)."""
    per = 16 // dtype.itemsize
    wide = (-(-cols // per) + pad) * per
    if dtype == E8:
        return torch.full((rows, wide), 0x7F, dtype=torch.uint8, device="cuda").view(E8)[:, :cols]
    return torch.full((rows, wide), fill, dtype=dtype, device="cuda")[:, :cols]


def normal(g, rows, cols, dtype, std=1.0, pad=0):
    t = aligned(rows, cols, dtype, pad)
    t.copy_(torch.randn(rows, cols, device="cuda", generator=g) * std)
    return t


def whole(t):
    """The buffer that a view by rows lies in."""
    return t._base if t._base is not None else t


def margin(t):
    """What lies between the rows of a view: nobody may write there."""
    base = whole(t)
    base = base if base.dim() == 2 else base.view(t.shape[0], -1)
    return base[:, t.shape[-1] * t.element_size() // base.element_size():].clone().view(torch.uint8)


def close(got, want, sum_of_magnitudes, n, what=""):
    """`got` is `want` but for its own rounding and n binary32 operations on terms of these magnitudes."""
    info = torch.finfo(got.dtype)
    bound = want.abs() * (info.eps / 2) + sum_of_magnitudes * ((n + 4) * U * (1 + info.eps)) + info.smallest_normal * info.eps
    d = (got.double() - want).abs()
    ok = (d <= bound) | (want.isnan() & got.isnan()) | (got.double() == want)
    bad = torch.nonzero(~ok)
    assert not len(bad), f"{what}: {len(bad)} of {ok.numel()} off, first at {bad[0].tolist()}: {got[tuple(bad[0])].item()} for {want[tuple(bad[0])].item()}, bound {bound[tuple(bad[0])].item()}"


# ---- norm -----------------------------------------------------------------------------------------

NORM_COLS = [1, 2, 7, 8, 9, 63, 255, 512, 513, 1024, 2043, 2048, 4095, 4100, 7168, 8192, 8200, 16385]


def norm_reference(x, r, w, eps):
    h = x.double() + (r.double() if r is not None else 0.0)
    s = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return h, s, h * s * w.double()


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("cols", NORM_COLS)
def test_norm(uccl, dtype, cols):
    t, g, rows, eps = T[dtype], gen(cols), 5, 1e-6
    x, r, w = normal(g, rows, cols, t), normal(g, rows, cols, t, 3.0, pad=2), normal(g, 1, cols, t)[0].contiguous()
    for res in (None, r):
        y, h, rstd = aligned(rows, cols, t, 1), aligned(rows, cols, t), torch.full((rows,), -1.0, device="cuda")
        around = margin(y), margin(h)
        uccl.uccl_norm_rows(y, x, w, eps, residual=res, h=h, rstd=rstd)
        eh, es, ey = norm_reference(x, res, w, eps)
        # s has a relative error of half that of the mean square, cols operations, and a few more; y three more
        close(h, eh, eh.abs(), 0, "h")
        close(rstd[:, None], es, es, cols / 2 + 6, "rstd")
        close(y, ey, ey.abs(), cols / 2 + 10, "y")
        assert torch.equal(margin(y), around[0]) and torch.equal(margin(h), around[1])


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("cols", NORM_COLS)
def test_norm_to_8_bits(uccl, dtype, cols):
    """Values and scales, as wire rows: scale behind the values, the next row behind the scale."""
    t, g, rows = T[dtype], gen(cols + 1), 4
    x, w = normal(g, rows, cols, t), normal(g, 1, cols, t)[0].contiguous()
    at = -(-cols // 16) * 16
    wire = torch.full((rows, at + 16), 0xAB, dtype=torch.uint8, device="cuda")
    y, scales = wire[:, :cols].view(E8), wire[:, at:at + 4].view(torch.float32)
    uccl.uccl_norm_rows(y, x, w, 0.0, scales=scales)
    _, _, ey = norm_reference(x, None, w, 0.0)
    es = ey.abs().amax(1, keepdim=True) / 448.0
    close(scales, es, es, cols / 2 + 12, "scales")
    # an element is off by half a step of its own size, or of the subnormals, and what binary32 was off before that
    got = y.float().double() * scales.double()
    bound = torch.maximum(ey.abs() * 2.0 ** -4, es * 2.0 ** -10) * (1 + 1e-6) + ey.abs() * (cols + 32) * U
    assert bool(((got - ey).abs() <= bound).all())
    assert bool((y.float().abs().amax(1) == 448.0).all())
    assert bool((wire[:, cols:at] == 0xAB).all()) and bool((wire[:, at + 4:] == 0xAB).all())


def test_norm_in_8_bits_is_the_nearest_value(uccl):
    """Rows whose norm is exact: every e4m3 value, halves between neighbours (ties to even) and values next to them."""
    vals = torch.arange(0, 127, device="cuda", dtype=torch.uint8).view(E8).double()
    mids = (vals[1:] + vals[:-1]) / 2
    v = torch.cat([vals, mids, mids * (1 + 2.0 ** -20), mids * (1 - 2.0 ** -20)])
    v = torch.cat([v, -v])
    # x holds v, the weight undoes the norm up to a power of two: mean square 2^2k exactly is arranged by one more column
    n = v.numel() + 1
    total = 2.0 ** 18 * n
    extra = torch.sqrt(torch.tensor(total, dtype=torch.float64, device="cuda") - (v.float().double() ** 2).sum())
    x = aligned(1, n, torch.float32)
    x[0] = torch.cat([v.float(), extra.float()[None]])
    w = torch.ones(n, device="cuda")
    w[-1] = 0.0
    y, s = aligned(1, n, E8), torch.zeros(1, 1, device="cuda")
    rstd = torch.zeros(1, device="cuda")
    uccl.uccl_norm_rows(y, x, w, 0.0, rstd=rstd, scales=s)
    e = x.double()[0] * rstd.double() * w.double()
    q = (e.float() * (1.0 / s[0, 0])).cpu().numpy().astype(np.float64)
    mant, exp = np.frexp(np.abs(q))
    step = np.exp2(np.maximum(exp - 1, -6) - 3.0)
    want = np.round(q / step) * step
    assert np.array_equal(y.float().cpu().numpy()[0].astype(np.float64), want)


@pytest.mark.parametrize("out", ["same", "e4m3"])
@pytest.mark.parametrize("cols", [64, 1000, 20000])
def test_norm_of_rows_that_are_zero_tiny_huge_or_not_finite(uccl, cols, out):
    x = aligned(6, cols, torch.float32)
    x.copy_(torch.randn(6, cols, device="cuda", generator=gen(3)))
    x[0] = 0.0
    x[1] *= 2.0 ** -70          # its square is below binary32's range: eps decides
    x[2] *= 2.0 ** 60           # its square still is in range
    x[3, 5] = float("nan")
    x[4, 7] = float("inf")
    w = torch.ones(cols, device="cuda")
    y = aligned(6, cols, E8 if out == "e4m3" else torch.float32)
    s = torch.zeros(6, 1, device="cuda") if out == "e4m3" else None
    rstd = torch.zeros(6, device="cuda")
    uccl.uccl_norm_rows(y, x, w, 1e-6, rstd=rstd, scales=s)
    got = y.float().double() * (s.double() if s is not None else 1.0)
    _, _, want = norm_reference(x, None, w, 1e-6)
    assert bool((got[0] == 0).all())
    for i in (1, 2, 5):
        assert bool(((got[i] - want[i]).abs() <= want[i].abs().amax() * (2.0 ** -4 if s is not None else 1e-4)).all())
    assert bool(got[3].isnan().all())
    assert bool(got[4, 7].isnan()) and bool((got[4, :7] == 0).all()) and bool((got[4, 8:] == 0).all())


def test_norm_in_place_and_strided(uccl):
    """y and h may be the input and the residual; rows far apart; one row with any stride; a weight of its own."""
    for cols in (96, 1000, 9000, 40000):
        g = gen(cols)
        x, r, w = normal(g, 3, cols, torch.bfloat16, pad=5), normal(g, 3, cols, torch.bfloat16), normal(g, 1, cols, torch.bfloat16)[0].contiguous()
        y, h = aligned(3, cols, torch.bfloat16), aligned(3, cols, torch.bfloat16)
        uccl.uccl_norm_rows(y, x, w, 1e-5, residual=r, h=h)
        around = margin(x)
        uccl.uccl_norm_rows(x, x, w, 1e-5, residual=r, h=r)
        assert torch.equal(x, y) and torch.equal(r, h) and torch.equal(margin(x), around)


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 255), (5, 256), (700, 640), (9, 2043), (600, 4096), (3, 7168), (2, 8200), (530, 8208), (4, 16390)])
def test_norm_grad(uccl, dtype, rows, cols):
    t, g = T[dtype], gen(rows + cols)
    h, dy, dh = normal(g, rows, cols, t, 2.0), normal(g, rows, cols, t, pad=1), normal(g, rows, cols, t)
    w = normal(g, 1, cols, t)[0].contiguous()
    rstd = torch.rsqrt(h.double().square().mean(1) + 1e-6).float()
    scratch = torch.full((uccl.uccl_norm_rows_scratch(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda")
    n, d = h.double() * rstd.double()[:, None], dy.double()
    gw = d * w.double()
    along, along_mag = (gw * n).mean(1, keepdim=True), (gw * n).abs().mean(1, keepdim=True)
    for carry in (None, dh):
        dx, dw = aligned(rows, cols, t, 3), torch.full((cols,), float("nan"), device="cuda")
        around = margin(dx)
        uccl.uccl_norm_rows_grad(dx, dw, dy, h, rstd, w, scratch, dh=carry)
        c = carry.double() if carry is not None else torch.zeros_like(n)
        s = rstd.double()[:, None]
        # the mean's own error, cols operations on its terms, then a handful on the three terms of the sum
        mag = (s * (gw.abs() + n.abs() * along_mag * (cols + 8) / 8) + c.abs())
        close(dx, c + s * (gw - n * along), mag, 8, "dx")
        close(dw, (d * n).sum(0), (d * n).abs().sum(0), rows + 4, "dweight")
        assert torch.equal(margin(dx), around)
    uccl.uccl_norm_rows_grad(dy, dw, dy, h, rstd, w, scratch, dh=dh)      # in place of what it reads
    assert torch.equal(dy, dx)


def test_norm_grad_of_no_rows_is_zero(uccl):
    e = torch.empty(0, 64, device="cuda")
    dw = torch.full((64,), 5.0, device="cuda")
    uccl.uccl_norm_rows_grad(e, dw, e, e, torch.empty(0, device="cuda"), torch.ones(64, device="cuda"), None)
    assert bool((dw == 0).all())


def test_norm_grad_is_the_derivative(uccl):
    """Against differences of the forward formula in 64 bits."""
    g, rows, cols, eps = gen(11), 3, 40, 1e-3
    x, dy, w = (torch.randn(rows, cols, device="cuda", generator=g) for _ in range(3))
    w = w[0].contiguous()
    h, rstd, y = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty_like(x)
    uccl.uccl_norm_rows(y, x, w, eps, h=h, rstd=rstd)
    dx, dw = torch.empty_like(x), torch.empty(cols, device="cuda")
    uccl.uccl_norm_rows_grad(dx, dw, dy, h, rstd, w, torch.empty(uccl.uccl_norm_rows_scratch(rows, cols), dtype=torch.uint8, device="cuda"))
    f = lambda x, w: float((norm_reference(x, None, w, eps)[2] * dy.double()).sum())  # noqa: E731
    step = 1e-6
    for r, c in ((0, 0), (1, 17), (2, 39)):
        e = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
        e[r, c] = step
        # differences of a smooth function: error of order step^2, and 1e-16 / step of rounding
        assert abs((f(x.double() + e, w) - f(x.double() - e, w)) / (2 * step) - float(dx[r, c])) < 1e-5
        assert abs((f(x, w.double() + e[r]) - f(x, w.double() - e[r])) / (2 * step) - float(dw[c])) < 1e-5


# ---- products -------------------------------------------------------------------------------------


def offsets_of(sizes, first=0):
    return torch.tensor(np.cumsum([first] + list(sizes)), dtype=torch.int32, device="cuda")


def quantised(g, rows, cols, std=1.0):
    v = torch.randn(rows, cols, device="cuda", generator=g) * std
    s = torch.exp2(torch.randint(-4, 4, (rows, 1), device="cuda", generator=g).float()) * 1.25
    t = aligned(rows, cols, E8)
    t.view(torch.uint8).copy_((v * 100).to(E8).view(torch.uint8))
    return t, s


SIZES = {
    "one": [1], "empty": [0, 0], "few": [0, 3, 0, 1, 2, 0], "edge": [63, 64, 65, 0, 1], "ragged": [17, 130, 0, 300, 1, 77],
    "large": [513, 256, 255, 40], "many": [1] * 70 + [0] * 60 + [2] * 70, "single": [700],
}
SHAPES = [(64, 64), (7, 5), (72, 24), (2043, 33), (256, 1003), (640, 257), (33, 64), (1, 1), (129, 512)]   # k, n


def product_inputs(g, dtype, rows, k, n, groups, spare):
    """x (with `spare` rows more, and NaN around), w, and their values in 64 bits."""
    if dtype == "e4m3":
        (x, xs), (w, ws) = quantised(g, rows + spare, k), quantised(g, groups * n, k)
        return x, xs, w.unflatten(0, (groups, n)), ws, x.double() * xs.double(), (w.double() * ws.double()).view(groups, n, k)
    x, w = normal(g, rows + spare, k, T[dtype]), normal(g, max(1, groups * n), k, T[dtype])[:groups * n]
    return x, None, w.unflatten(0, (groups, n)), None, x.double(), w.double().view(groups, n, k)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("sizes", list(SIZES))
@pytest.mark.parametrize("k,n", SHAPES)
def test_group_product(uccl, dtype, sizes, k, n):
    counts = SIZES[sizes]
    g, rows, groups = gen(k * n), sum(counts), len(counts)
    t = T["bf16" if dtype == "e4m3" else dtype]
    x, xs, w, ws, ex, ew = product_inputs(g, dtype, rows, k, n, groups, 3)
    index = torch.randint(0, rows + 3, (rows,), device="cuda", generator=g).to(torch.int32)
    if rows > 2:
        index[1], index[2] = -1, rows + 3     # rows of zeros
    for idx, out in ((None, t), (index, torch.float32)):
        y = aligned(rows, n, out, 1, fill=7.0)
        around = margin(y)
        uccl.uccl_group_product(y, x, w, offsets_of(counts), index=idx, x_scales=xs, w_scales=ws)
        rows_x = ex[:rows]
        if idx is not None:
            i = idx.long()
            there = (i >= 0) & (i < rows + 3)
            rows_x = torch.where(there[:, None], ex[i.clamp(0, rows + 2)], 0.0)
        at = 0
        for e, c in enumerate(counts):
            a = rows_x[at:at + c]
            close(y[at:at + c], a @ ew[e].T, a.abs() @ ew[e].abs().T, k + 4, f"group {e}")
            at += c
        assert torch.equal(margin(y), around)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("sizes", list(SIZES))
@pytest.mark.parametrize("k,n", SHAPES)
def test_group_product_gradients(uccl, dtype, sizes, k, n):
    counts = SIZES[sizes]
    g, rows, groups, t = gen(k + n), sum(counts), len(counts), T[dtype]
    x, _, w, _, ex, ew = product_inputs(g, dtype, rows, k, n, groups, 2)
    dy = normal(g, rows, n, t)
    index = torch.randint(0, rows + 2, (rows,), device="cuda", generator=g).to(torch.int32)
    if rows > 2:
        index[0], index[2] = rows + 2, -7
    off = offsets_of(counts)
    dx = aligned(rows, k, t, 1, fill=7.0)
    around = margin(dx)
    uccl.uccl_group_product_grad_x(dx, dy, w, off)
    assert torch.equal(margin(dx), around)
    for idx, out in ((None, torch.float32), (index, t)):
        dw = aligned(groups * n, k, out, 2, fill=7.0)
        around = margin(dw)
        uccl.uccl_group_product_grad_w(dw.unflatten(0, (groups, n)), dy, x, off, index=idx)
        assert torch.equal(margin(dw), around)
        rows_x = ex[:rows]
        if idx is not None:
            i = idx.long()
            rows_x = torch.where(((i >= 0) & (i < rows + 2))[:, None], ex[i.clamp(0, rows + 1)], 0.0)
        at = 0
        for e, c in enumerate(counts):
            d, a = dy[at:at + c].double(), rows_x[at:at + c]
            if idx is None:
                close(dx[at:at + c], d @ ew[e], d.abs() @ ew[e].abs(), n + 4, f"dx, group {e}")
            close(dw.view(groups, n, k)[e] if dw.is_contiguous() else dw.unflatten(0, (groups, n))[e], d.T @ a, d.abs().T @ a.abs(), c + 4, f"dw, group {e}")
            at += c


# rows by group and columns that take tiles of 256 x 256, of 128 x 256 and (over several rounds of the machine) of 128 x 128
LARGE = {"256x256": ([1100, 0, 1901], 4100), "128x256": ([1299], 4103), "128x128": ([257, 300, 0, 90], 2050), "64 groups": ([41 + g % 7 for g in range(67)], 777)}


def in_pieces(f, n, step=1024):
    """Of long columns, a piece at a time: 64-bit references of large outputs."""
    for at in range(0, n, step):
        f(slice(at, min(n, at + step)))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("shape", list(LARGE))
@pytest.mark.parametrize("k", [40, 64, 200, 521, 1003])
def test_group_product_of_many_tiles(uccl, dtype, shape, k):
    counts, n = LARGE[shape]
    g, rows, groups = gen(k + n), sum(counts), len(counts)
    t = T["bf16" if dtype == "e4m3" else dtype]
    x, xs, w, ws, ex, ew = product_inputs(g, dtype, rows, k, n, groups, 2)
    index = torch.randint(0, rows + 2, (rows,), device="cuda", generator=g).to(torch.int32)
    index[7] = -1
    there = index >= 0
    for idx, out in ((None, torch.float32), (index, t)):
        y = aligned(rows, n, out, 1, fill=7.0)
        around = margin(y)
        uccl.uccl_group_product(y, x, w, offsets_of(counts), index=idx, x_scales=xs, w_scales=ws)
        a_all = ex[:rows] if idx is None else torch.where(there[:, None], ex[index.long().clamp(min=0)], 0.0)
        at = 0
        for e, c in enumerate(counts):
            a = a_all[at:at + c]
            in_pieces(lambda s: close(y[at:at + c, s], a @ ew[e, s].T, a.abs() @ ew[e, s].abs().T, k + 4, f"group {e}"), n)
            at += c
        assert torch.equal(margin(y), around)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", list(LARGE))
@pytest.mark.parametrize("n", [40, 333])
def test_group_product_gradients_of_many_tiles(uccl, dtype, shape, n):
    counts, k = LARGE[shape]
    g, rows, groups, t = gen(k + n), sum(counts), len(counts), T[dtype]
    x, _, w, _, ex, ew = product_inputs(g, dtype, rows, k, n, groups, 2)
    dy = normal(g, rows, n, t)
    index = torch.randperm(rows, device="cuda", generator=g).to(torch.int32)
    index[5] = rows + 2
    dx, dw = aligned(rows, k, t, 1, fill=7.0), aligned(groups * n, k, torch.float32, 1, fill=7.0)
    around = margin(dx), margin(dw)
    uccl.uccl_group_product_grad_x(dx, dy, w, offsets_of(counts))
    uccl.uccl_group_product_grad_w(dw.unflatten(0, (groups, n)), dy, x, offsets_of(counts), index=index)
    assert torch.equal(margin(dx), around[0]) and torch.equal(margin(dw), around[1])
    rows_x = torch.where((index < rows + 2)[:, None], ex[index.long().clamp(max=rows + 1)], 0.0)
    at = 0
    for e, c in enumerate(counts):
        d, a = dy[at:at + c].double(), rows_x[at:at + c]
        in_pieces(lambda s: close(dx[at:at + c, s], d @ ew[e][:, s], d.abs() @ ew[e][:, s].abs(), n + 4, f"dx, group {e}"), k)
        in_pieces(lambda s: close(dw.unflatten(0, (groups, n))[e][:, s], d.T @ a[:, s], d.abs().T @ a[:, s].abs(), c + 4, f"dw, group {e}"), k)
        at += c


@pytest.mark.parametrize("n,k", [(2900, 2300), (630, 4100)])
def test_gradient_of_the_weights_in_large_tiles(uccl, n, k):
    counts = [70, 0, 129]
    g, rows, t = gen(n), sum(counts), torch.bfloat16
    x, dy = normal(g, rows, k, t), normal(g, rows, n, t)
    dw = aligned(3 * n, k, torch.bfloat16, fill=7.0)
    uccl.uccl_group_product_grad_w(dw.unflatten(0, (3, n)), dy, x, offsets_of(counts))
    at = 0
    for e, c in enumerate(counts):
        d, a = dy[at:at + c].double(), x[at:at + c].double()
        in_pieces(lambda s: close(dw[e * n:(e + 1) * n, s], d.T @ a[:, s], d.abs().T @ a[:, s].abs(), c + 4, f"dw, group {e}"), k)
        at += c


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_what_is_beside_the_rows_changes_nothing(uccl, dtype):
    """NaN in rows of other groups, in rows that no index names, in the pieces behind a row's end and in w of other groups."""
    k, n, counts = 100, 70, [40, 0, 90]
    g, rows = gen(5), 130
    x, xs, w, ws, ex, ew = product_inputs(g, dtype, rows, k, n, 3, 0)
    t = T["bf16"]
    nan = torch.full((), 0x7F, dtype=torch.uint8, device="cuda") if dtype == "e4m3" else None

    def poison(v):
        if dtype == "e4m3":
            v.view(torch.uint8).copy_(nan.expand(v.shape))
        else:
            v.fill_(float("nan"))
    poison(x[40:])                      # the second group's rows; the last group's are poisoned
    poison(w[1])                        # a group without rows
    y = aligned(rows, n, torch.float32)
    uccl.uccl_group_product(y, x, w, offsets_of(counts), x_scales=xs, w_scales=ws)
    close(y[:40], ex[:40] @ ew[0].T, ex[:40].abs() @ ew[0].abs().T, k + 4)
    assert bool(y[40:].isnan().all())
    if dtype == "bf16":
        dy = normal(g, rows, n, t)
        dy[40:] = float("nan")
        dx, dw = aligned(rows, k, torch.float32), aligned(3 * n, k, torch.float32)
        uccl.uccl_group_product_grad_x(dx, dy, w, offsets_of(counts))
        uccl.uccl_group_product_grad_w(dw.unflatten(0, (3, n)), dy, x, offsets_of(counts))
        d, a = dy[:40].double(), ex[:40]
        close(dx[:40], d @ ew[0], d.abs() @ ew[0].abs(), n + 4)
        close(dw[:n], d.T @ a, d.abs().T @ a.abs(), 44)
        assert bool((dw[n:2 * n] == 0).all()) and bool(dw[2 * n:].isnan().all()) and bool(dx[40:].isnan().all())


@pytest.mark.parametrize("offsets,begin_end", [
    ([0, 5, 3, 8], [(0, 5), (5, 5), (5, 8)]),           # descending: no row twice
    ([-4, 2, 2, 100], [(0, 2), (2, 2), (2, 9)]),        # outside the rows
    ([3, 4, 6, 7], [(3, 4), (4, 6), (6, 7)]),           # rows of no group on both sides
    ([50, 60, 70, 80], [(9, 9), (9, 9), (9, 9)]),
])
def test_offsets_are_taken_as_they_can_be_used(uccl, offsets, begin_end):
    k, n, rows, t = 40, 24, 9, torch.bfloat16
    g = gen(1)
    x, _, w, _, ex, ew = product_inputs(g, "bf16", rows, k, n, 3, 0)
    dy = normal(g, rows, n, t)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    y, dx, dw = aligned(rows, n, t, fill=9.0), aligned(rows, k, t, fill=9.0), aligned(3 * n, k, torch.float32)
    uccl.uccl_group_product(y, x, w, off)
    uccl.uccl_group_product_grad_x(dx, dy, w, off)
    uccl.uccl_group_product_grad_w(dw.unflatten(0, (3, n)), dy, x, off)
    mine = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for e, (b, f) in enumerate(begin_end):
        mine[b:f] = True
        a, d = ex[b:f], dy[b:f].double()
        close(y[b:f], a @ ew[e].T, a.abs() @ ew[e].abs().T, k + 4)
        close(dx[b:f], d @ ew[e], d.abs() @ ew[e].abs(), n + 4)
        close(dw.unflatten(0, (3, n))[e], d.T @ a, d.abs().T @ a.abs(), rows + 4)
    assert bool((y[~mine] == 9.0).all()) and bool((dx[~mine] == 9.0).all())


def test_products_of_no_depth_are_zero(uccl):
    """No columns to sum over, or no rows: zeros, not what was there."""
    y = torch.full((5, 8), 3.0, dtype=torch.bfloat16, device="cuda")
    off = offsets_of([2, 3])
    uccl.uccl_group_product(y, torch.empty(5, 0, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 8, 0, dtype=torch.bfloat16, device="cuda"), off)
    assert bool((y == 0).all())
    dx = torch.full((5, 16), 3.0, dtype=torch.bfloat16, device="cuda")
    uccl.uccl_group_product_grad_x(dx, torch.empty(5, 0, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 0, 16, dtype=torch.bfloat16, device="cuda"), off)
    assert bool((dx == 0).all())
    dw = torch.full((2, 8, 16), 3.0, device="cuda")
    e = lambda c: torch.empty(0, c, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    uccl.uccl_group_product_grad_w(dw, e(8), e(16), offsets_of([0, 0]))
    assert bool((dw == 0).all())


def test_products_beyond_4_gib(uccl):
    """Rows, weights and outputs whose offsets need more than 32 bits."""
    k, n, rows = 64, 16, 40
    stride = 160 << 20                     # bytes: 40 rows of it are 6.25 GiB
    buf = torch.empty(rows * stride // 2, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, k), (stride // 2, 1))
    y = buf.as_strided((rows, n), (stride // 2, 1), 4096)
    g = gen(8)
    x.copy_(torch.randn(rows, k, device="cuda", generator=g))
    w = torch.randn(2, n, k, device="cuda", generator=g).to(torch.bfloat16)
    off = offsets_of([1, 39])
    uccl.uccl_group_product(y, x, w, off)
    e = torch.cat([x[:1].double() @ w[0].double().T, x[1:].double() @ w[1].double().T])
    m = torch.cat([x[:1].double().abs() @ w[0].double().abs().T, x[1:].double().abs() @ w[1].double().abs().T])
    close(y, e, m, k + 4)
    dx, dw = buf.as_strided((rows, k), (stride // 2, 1), 8192), torch.empty(2, n, k, device="cuda")
    dy = buf.as_strided((rows, n), (stride // 2, 1), 16384)
    dy.copy_(torch.randn(rows, n, device="cuda", generator=g))
    uccl.uccl_group_product_grad_x(dx, dy, w, off)
    uccl.uccl_group_product_grad_w(dw, dy, x, off)
    d = dy.double()
    close(dx[1:], d[1:] @ w[1].double(), d[1:].abs() @ w[1].double().abs(), n + 4)
    close(dw[1], d[1:].T @ x[1:].double(), d[1:].abs().T @ x[1:].double().abs(), 44)
    wide = buf.as_strided((2, n, k), (n * (stride // 2), stride // 2, 1), 32768)
    wide.copy_(w)
    y2 = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    uccl.uccl_group_product(y2, x, wide, off)
    assert torch.equal(y2, y)


# ---- combination ----------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("tokens,slots,cols", [(1, 1, 1), (3, 8, 7), (5, 2, 64), (4, 9, 1003), (33, 8, 7168), (2, 17, 4096), (70, 4, 20), (3, 3, 9000), (6, 0, 40)])
def test_combine_and_its_gradient(uccl, dtype, tokens, slots, cols):
    t, g = T[dtype], gen(tokens * 100 + slots)
    there = torch.rand(tokens, slots, device="cuda", generator=g) < 0.7
    there[0] = False                                   # a token whose slots are all empty
    n = max(1, int(there.sum()))
    pos = torch.full((tokens, slots), -1, dtype=torch.int32, device="cuda")
    pos[there] = torch.randperm(int(there.sum()), device="cuda", generator=g).to(torch.int32)
    if slots > 1:
        pos[0, 0], pos[0, 1] = n, -2 ** 31             # rows that y does not have
    y, r, w = normal(g, n, cols, t), normal(g, tokens, cols, t, 2.0), torch.randn(tokens, slots, device="cuda", generator=g)
    dout = normal(g, tokens, cols, t)
    at = pos.long().clamp(0, n - 1)
    ey = torch.where(there[..., None], y.double()[at], 0.0)
    for weights, res in ((w, r), (None, None)):
        ew = weights.double() if weights is not None else torch.ones(tokens, slots, dtype=torch.float64, device="cuda")
        er = res.double() if res is not None else torch.zeros(tokens, cols, dtype=torch.float64, device="cuda")
        out = aligned(tokens, cols, t, 1)
        around = margin(out)
        uccl.uccl_combine_rows(out, y, pos, weights=weights, residual=res)
        terms = ey * ew[..., None]
        close(out, terms.sum(1) + er, terms.abs().sum(1) + er.abs(), slots, "out")
        assert torch.equal(margin(out), around)
        dy, dw = aligned(n, cols, t, 1, fill=5.0), torch.full((tokens, slots), float("nan"), device="cuda")
        around = margin(dy)
        uccl.uccl_combine_rows_grad(dy, dw, dout, y, pos, weights=weights)
        want = torch.full((n, cols), 5.0, dtype=torch.float64, device="cuda")
        want[pos[there].long()] = (ew[..., None] * dout.double()[:, None])[there]
        close(dy, want, want.abs(), 1, "dy")
        dots = ey * dout.double()[:, None]
        close(dw, dots.sum(2), dots.abs().sum(2), cols, "dweights")
        assert torch.equal(margin(dy), around)
        again = aligned(n, cols, t, 1, fill=5.0)
        uccl.uccl_combine_rows_grad(again, None, dout, y, pos, weights=weights)
        assert torch.equal(again, dy)
    uccl.uccl_combine_rows(r, y, pos, weights=w, residual=r)        # onto the residual
    ref = aligned(tokens, cols, t, 1)
    assert not bool(r.isnan().any())


def test_rows_that_no_slot_names_do_not_count(uccl):
    """NaN in them, and in the weights of empty slots."""
    y = torch.full((4, 64), float("nan"), device="cuda")
    y[2] = 1.0
    pos = torch.tensor([[2, -1], [-1, 9]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[0.5, float("nan")], [float("inf"), 1.0]], device="cuda")
    out, dw = torch.empty(2, 64, device="cuda"), torch.empty(2, 2, device="cuda")
    uccl.uccl_combine_rows(out, y, pos, weights=w)
    assert bool((out[0] == 0.5).all()) and bool((out[1] == 0).all())
    uccl.uccl_combine_rows_grad(torch.empty_like(y), dw, torch.ones(2, 64, device="cuda"), y, pos, weights=w)
    assert dw.tolist() == [[64.0, 0.0], [0.0, 0.0]]


# ---- all of them ----------------------------------------------------------------------------------


def one_of_each(uccl, seed):
    """Calls of every operator on inputs of their own: (calls to make, outputs)."""
    g, t, k, n, groups = gen(seed), torch.bfloat16, 640, 264, 5
    counts = [70, 0, 31, 1, 26]
    rows = sum(counts)
    x, r, w = normal(g, rows, k, t), normal(g, rows, k, t), normal(g, 1, k, t)[0].contiguous()
    y8, s8, h, rstd = aligned(rows, k, E8), torch.zeros(rows, 1, device="cuda"), aligned(rows, k, t), torch.zeros(rows, device="cuda")
    (w8, ws), wt = quantised(g, groups * n, k), normal(g, groups * n, k, t).unflatten(0, (groups, n))
    off, index = offsets_of(counts), torch.randperm(rows, device="cuda", generator=g).to(torch.int32)
    p8, p16, dy = aligned(rows, n, t), aligned(rows, n, t), normal(g, rows, n, t)
    dx, dw = aligned(rows, k, t), torch.zeros(groups, n, k, device="cuda")
    pos = torch.randperm(rows, device="cuda", generator=g).to(torch.int32).view(-1, 2)
    weights, out = torch.rand(rows // 2, 2, device="cuda", generator=g), aligned(rows // 2, k, t)
    dyc, dwc = aligned(rows, k, t), torch.zeros(rows // 2, 2, device="cuda")
    dxn, dwn = aligned(rows, k, t), torch.zeros(k, device="cuda")
    scratch = torch.empty(uccl.uccl_norm_rows_scratch(rows, k), dtype=torch.uint8, device="cuda")

    def calls():
        uccl.uccl_norm_rows(y8, x, w, 1e-6, residual=r, h=h, rstd=rstd, scales=s8)
        uccl.uccl_group_product(p8, y8, w8.unflatten(0, (groups, n)), off, index=index, x_scales=s8, w_scales=ws)
        uccl.uccl_group_product(p16, x, wt, off)
        uccl.uccl_group_product_grad_x(dx, dy, wt, off)
        uccl.uccl_group_product_grad_w(dw, dy, x, off, index=index)
        uccl.uccl_combine_rows(out, dx, pos, weights=weights, residual=x[:rows // 2])
        uccl.uccl_combine_rows_grad(dyc, dwc, out, dx, pos, weights=weights)
        uccl.uccl_norm_rows_grad(dxn, dwn, dyc, h, rstd, w, scratch, dh=dx)
    return calls, [y8.view(torch.uint8), s8, h, rstd, p8, p16, dx, dw, out, dyc, dwc, dxn, dwn], (x, r, dy)


def same_bits(a, b):
    """Of all outputs, NaN among them."""
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


def test_the_same_bits_every_time_on_any_stream_and_from_a_graph(uccl):
    calls, outs, inputs = one_of_each(uccl, 1)
    calls()
    torch.cuda.synchronize()
    first = [o.clone() for o in outs]

    def wipe():
        for o in outs:
            o.zero_()
    side = torch.cuda.Stream()
    wipe()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    assert same_bits(first, outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for turn in range(3):
        wipe()
        if turn == 2:                        # other inputs in the same buffers: nothing is kept from before
            for t in inputs:
                t.mul_(-0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        wipe()
        calls()
        torch.cuda.synchronize()
        assert same_bits(got, outs)
        assert (turn == 2) != same_bits(first, outs)


def test_a_refusal_raises(uccl):
    t = torch.bfloat16
    with pytest.raises(uccl.UcclError) as e:
        uccl.uccl_norm_rows(torch.empty(3, 9, dtype=t, device="cuda"), torch.empty(3, 9, dtype=t, device="cuda"), torch.ones(9, dtype=t, device="cuda"), 1e-6)
    assert e.value.code == uccl.UCCL_EALIGN
    with pytest.raises(uccl.UcclError) as e:
        uccl.uccl_group_product(torch.empty(3, 8, dtype=t, device="cuda"), torch.empty(3, 16, device="cuda"), torch.empty(2, 8, 16, device="cuda"),
                                torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert e.value.code == uccl.UCCL_EINVAL
