"""Row operators at the sizes that take the kernels of large calls: many rows, outputs above 32 MiB that are stored past the caches, more than 64 groups in the order by group,
and outputs that lie where an input does.  tests/test_rows_launches.py has which kernel each of these shapes is launched as; tolerances are those of tests/test_gpu_rows.py."""
import pytest
import torch

from test_gpu_rows import E8, T, aligned, close, gen, in_pieces, margin, norm_reference, normal, offsets_of, product_inputs
from test_gpu_rows_exact import elements

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def uccl(gpu_lib):
    return gpu_lib


# rows, columns: two pieces a thread below and above 32 MiB, ragged; one piece a thread of one wavefront and of several, above; four pieces
NORMS = {"bf16": [(600, 7168), (2500, 7168), (2500, 7171), (40000, 500), (9000, 2043), (4500, 4093), (1100, 16381)],
         "f32": [(600, 4093), (2100, 4093), (1300, 7168), (40000, 250), (9000, 1021), (4500, 2043)]}
NORMS = [(d, r, c) for d in T for r, c in NORMS["f32" if d == "f32" else "bf16"]]


@pytest.mark.parametrize("dtype,rows,cols", NORMS)
def test_norm_of_many_rows(uccl, dtype, rows, cols):
    t, g, eps = T[dtype], gen(rows), 1e-6
    x, r, w = normal(g, rows, cols, t), normal(g, rows, cols, t, 3.0, pad=1), normal(g, 1, cols, t)[0].contiguous()
    y, h, rstd = aligned(rows, cols, t, 1), aligned(rows, cols, t), torch.full((rows,), -1.0, device="cuda")
    around = margin(y), margin(h)
    uccl.uccl_norm_rows(y, x, w, eps, residual=r, h=h, rstd=rstd)
    eh, es, ey = norm_reference(x, r, w, eps)
    close(rstd[:, None], es, es, cols / 2 + 6, "rstd")
    close(h, eh, eh.abs(), 0, "h")
    close(y, ey, ey.abs(), cols / 2 + 10, "y")
    assert torch.equal(margin(y), around[0]) and torch.equal(margin(h), around[1])
    del eh, ey
    # in 8 bits, with h, and in place
    h8, s, rstd8 = aligned(rows, cols, t, 2), torch.zeros(rows, 1, device="cuda"), torch.zeros(rows, device="cuda")
    y8 = aligned(rows, cols, E8, 1)
    around = margin(y8), margin(h8)
    uccl.uccl_norm_rows(y8, x, w, eps, residual=r, h=h8, rstd=rstd8, scales=s)
    assert torch.equal(h8, h) and torch.equal(rstd8, rstd) and torch.equal(margin(y8), around[0]) and torch.equal(margin(h8), around[1])
    v = (x.float() + r.float()) * rstd[:, None] * w.float()
    assert torch.equal(s, (v.abs().amax(1, keepdim=True).double() / 448.0).float())
    assert torch.equal(y8.view(torch.uint8), elements(v, s))
    around = margin(r)
    uccl.uccl_norm_rows(x, x, w, eps, residual=r, h=r)
    assert torch.equal(x, y) and torch.equal(r, h) and torch.equal(margin(r), around)


NORM_GRADS = {"bf16": [(600, 7168), (2500, 7168), (2500, 7171), (9000, 2043), (4500, 4093), (530, 8208), (1100, 16381), (5, 16381), (300, 20000)],
              "f32": [(600, 4093), (2100, 4093), (1300, 7168), (9000, 1021), (4500, 2043), (1100, 8188), (5, 8188), (300, 9000)]}
NORM_GRADS = [(d, r, c) for d in T for r, c in NORM_GRADS["f32" if d == "f32" else "bf16"]]


@pytest.mark.parametrize("dtype,rows,cols", NORM_GRADS)
def test_norm_grad_of_many_rows_and_in_place(uccl, dtype, rows, cols):
    """Against the formula; then dx where dy is, and where dh is."""
    t, g = T[dtype], gen(rows + cols)
    h, dy, dh = normal(g, rows, cols, t, 2.0), normal(g, rows, cols, t, pad=1), normal(g, rows, cols, t, pad=2)
    w = normal(g, 1, cols, t)[0].contiguous()
    rstd = torch.rsqrt(h.double().square().mean(1) + 1e-6).float()
    scratch = torch.full((uccl.uccl_norm_rows_scratch(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda")
    dx, dw = aligned(rows, cols, t, 3), torch.full((cols,), float("nan"), device="cuda")
    around = margin(dx)
    uccl.uccl_norm_rows_grad(dx, dw, dy, h, rstd, w, scratch, dh=dh)
    n, d, s = h.double() * rstd.double()[:, None], dy.double(), rstd.double()[:, None]
    gw = d * w.double()
    along, along_mag = (gw * n).mean(1, keepdim=True), (gw * n).abs().mean(1, keepdim=True)
    mag = s * (gw.abs() + n.abs() * along_mag * (cols + 8) / 8) + dh.double().abs()
    close(dx, dh.double() + s * (gw - n * along), mag, 8, "dx")
    close(dw, (d * n).sum(0), (d * n).abs().sum(0), rows + 4, "dweight")
    assert torch.equal(margin(dx), around)
    del n, d, gw, mag
    for which in (dy, dh):
        kept, around, dw2 = which.clone(), margin(which), torch.full_like(dw, float("nan"))
        uccl.uccl_norm_rows_grad(which, dw2, dy, h, rstd, w, scratch, dh=dh)
        assert torch.equal(which, dx) and torch.equal(dw2, dw) and torch.equal(margin(which), around)
        which.copy_(kept)


# tokens, slots, columns
COMBINES = {"bf16": [(2500, 2, 7168), (2500, 3, 7171), (700, 9, 7171), (70, 4, 20)], "f32": [(1300, 2, 7168), (1300, 3, 7171), (400, 9, 7171), (70, 4, 20)]}
COMBINES = [(d, *s) for d in T for s in COMBINES["f32" if d == "f32" else "bf16"]]


@pytest.mark.parametrize("dtype,tokens,slots,cols", COMBINES)
def test_combine_of_many_rows_and_onto_the_residual(uccl, dtype, tokens, slots, cols):
    """`out` above 32 MiB, or (with 9 slots) the rows' gradient; one slot in eight has no row."""
    t, g = T[dtype], gen(tokens + slots)
    there = torch.rand(tokens, slots, device="cuda", generator=g) < 0.875
    n = int(there.sum())
    pos = torch.full((tokens, slots), -1, dtype=torch.int32, device="cuda")
    pos[there] = torch.randperm(n, device="cuda", generator=g).to(torch.int32)
    y, r, dout = normal(g, n, cols, t), normal(g, tokens, cols, t, 2.0, pad=2), normal(g, tokens, cols, t)
    w = torch.randn(tokens, slots, device="cuda", generator=g)
    out = aligned(tokens, cols, t, 1)
    around = margin(out)
    uccl.uccl_combine_rows(out, y, pos, weights=w, residual=r)
    want, mag, dots, dot_mag = r.double(), r.double().abs(), [], []
    for j in range(slots):
        row = torch.where(there[:, j, None], y[pos[:, j].long().clamp(min=0)].double(), 0.0)
        want, mag = want + row * w[:, j, None].double(), mag + (row * w[:, j, None].double()).abs()
        dots.append((row * dout.double()).sum(1)), dot_mag.append((row * dout.double()).abs().sum(1))
    close(out, want, mag, slots, "out")
    assert torch.equal(margin(out), around)
    around = margin(r)
    uccl.uccl_combine_rows(r, y, pos, weights=w, residual=r)
    assert torch.equal(r, out) and torch.equal(margin(r), around)
    del want, mag
    dy, dw = aligned(n, cols, t, 1, fill=5.0), torch.full((tokens, slots), float("nan"), device="cuda")
    around = margin(dy)
    uccl.uccl_combine_rows_grad(dy, dw, dout, y, pos, weights=w)
    for j in range(slots):
        m = there[:, j]
        e = w[m, j, None].double() * dout[m].double()
        close(dy[pos[m, j].long()], e, e.abs(), 1, "dy")
    close(dw, torch.stack(dots, 1), torch.stack(dot_mag, 1), cols, "dweights")
    assert torch.equal(margin(dy), around)


# more than 64 and more than 128 groups, all of a group's tiles together: rows by group, columns, depth; by 16 rows, and by tiles
MANY_GROUPS = {"few rows": ([(5 * i) % 17 for i in range(150)], 1280, 72), "tiles": ([(29 * i) % 81 for i in range(70)], 14336, 40)}


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape", list(MANY_GROUPS))
def test_more_than_64_groups_by_group(uccl, shape, dtype):
    counts, n, k = MANY_GROUPS[shape]
    g, rows, groups, t = gen(n), sum(counts), len(counts), torch.bfloat16
    x, xs, w, ws, ex, ew = product_inputs(g, dtype, rows, k, n, groups, 0)
    index = torch.randperm(rows, device="cuda", generator=g).to(torch.int32)
    y = aligned(rows, n, t, 1, fill=7.0)
    around = margin(y)
    uccl.uccl_group_product(y, x, w, offsets_of(counts), index=index, x_scales=xs, w_scales=ws)
    at = 0
    for e, c in enumerate(counts):
        a = ex[index[at:at + c].long()]
        in_pieces(lambda s: close(y[at:at + c, s], a @ ew[e, s].T, a.abs() @ ew[e, s].abs().T, k + 4, f"group {e}"), n, 4096)
        at += c
    assert torch.equal(margin(y), around)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_gradient_of_the_rows_of_more_than_64_groups_by_group(uccl, dtype):
    counts, k, n = MANY_GROUPS["tiles"]
    g, rows, groups, t = gen(n), sum(counts), len(counts), T[dtype]
    dy, w = normal(g, rows, n, t), normal(g, groups * n, k, t)
    dx = aligned(rows, k, t, 1, fill=7.0)
    around = margin(dx)
    uccl.uccl_group_product_grad_x(dx, dy, w.unflatten(0, (groups, n)), offsets_of(counts))
    at = 0
    for e, c in enumerate(counts):
        d, v = dy[at:at + c].double(), w[e * n:(e + 1) * n].double()
        close(dx[at:at + c], d @ v, d.abs() @ v.abs(), n + 4, f"dx, group {e}")
        at += c
    assert torch.equal(margin(dx), around)
