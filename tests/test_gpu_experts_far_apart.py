"""Rows so far apart that their offsets pass 32 bits, and matrices of more than 4 GiB: the same results as of rows that lie together, bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu
E2M1, E8M0 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
SPAN = (5 << 30) + (1 << 28)   # bytes from the first row to behind the last


@pytest.fixture(scope="module")
def uccl(gpu_lib):
    yield gpu_lib
    torch.cuda.empty_cache()


def apart(t, per=16):
    """A copy of a tensor of bytes or numbers, [..., cols], whose rows are SPAN / rows bytes apart, rounded to `per`."""
    raw = t.view(torch.uint8)
    rows, width = raw.numel() // raw.shape[-1], raw.shape[-1]
    step = SPAN // rows // per * per
    assert step >= width and (rows - 1) * step > 1 << 32
    room = torch.empty(SPAN, dtype=torch.uint8, device="cuda")
    strides = [step]
    for n in reversed(raw.shape[1:-1]):
        strides.insert(0, strides[0] * n)
    out = room.as_strided(raw.shape, (*strides, 1))
    out.copy_(raw)
    return out.view(t.dtype)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def in_4_bits(uccl, rows, cols, seed):
    q = torch.zeros(rows, cols // 2, dtype=torch.uint8, device="cuda").view(E2M1)
    s = torch.zeros(rows, -(-cols // 128) * 4, dtype=torch.uint8, device="cuda").view(E8M0)[:, :-(-cols // 32)]
    x = torch.randn(rows, cols, device="cuda", generator=gen(seed))
    uccl.uccl_quantise_rows(q, s, x)
    return q, s


@pytest.mark.parametrize("rows", [6, 300, 700, 4000])
@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
def test_product(uccl, kind, rows):
    groups, cols, out = 2, 384, 1280
    w, ws = in_4_bits(uccl, groups * out, cols, 1)
    w, ws = w.view(torch.uint8).unflatten(0, (groups, out)).view(E2M1), ws.view(torch.uint8).unflatten(0, (groups, out)).view(E8M0)
    first = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")
    index = torch.randperm(rows, device="cuda", generator=gen(2)).to(torch.int32)
    if kind == "mx4":
        x, xs = in_4_bits(uccl, rows, cols, 3)
    else:
        x, xs = torch.randn(rows, cols, device="cuda", generator=gen(3)).to(torch.bfloat16 if kind == "bf16" else torch.float16), None
    t = torch.float16 if kind == "f16" else torch.bfloat16
    y = torch.zeros(rows, out, dtype=t, device="cuda")
    uccl.uccl_group_product(y, x, w, first, index=index, x_scales=xs, w_scales=ws)
    assert bool(y.any())
    far = apart(torch.zeros_like(y))
    uccl.uccl_group_product(far, apart(x), apart(w), first, index=index, x_scales=None if xs is None else apart(xs, 4), w_scales=apart(ws, 4))
    assert torch.equal(far, y)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", [(6, 2048), (900, 96)])
def test_rows_to_4_bits(uccl, dtype, rows, cols):
    x = torch.randn(rows, cols, device="cuda", generator=gen(4)).to(dtype)
    q, s, v = torch.zeros(rows, cols // 2, dtype=torch.uint8, device="cuda").view(E2M1), torch.zeros(rows, cols // 32, dtype=torch.uint8, device="cuda").view(E8M0), torch.zeros_like(x)
    if cols // 32 % 4:
        s = torch.zeros(rows, 4, dtype=torch.uint8, device="cuda").view(E8M0)[:, :cols // 32]
    uccl.uccl_quantise_rows(q, s, x, values=v)
    far = [apart(torch.zeros_like(q.view(torch.uint8))), apart(torch.zeros_like(s.view(torch.uint8)), 4), apart(torch.zeros_like(x))]
    uccl.uccl_quantise_rows(far[0].view(E2M1), far[1].view(E8M0), apart(x), values=far[2])
    assert torch.equal(far[0], q.view(torch.uint8)) and torch.equal(far[1], s.view(torch.uint8)) and torch.equal(far[2], v)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,n", [(7, 256), (5000, 64)])
def test_route_and_its_gradient(uccl, dtype, tokens, n):
    slots = 4
    scores = torch.randn(tokens, n, device="cuda", generator=gen(5)).to(dtype)
    scratch = torch.zeros(uccl.uccl_route_rows_scratch(tokens, n) + 16, dtype=torch.uint8, device="cuda")
    d, ds = torch.randn(tokens, slots, device="cuda", generator=gen(6)), torch.randn(n, device="cuda", generator=gen(7))

    def of(z, dz):
        e, w = torch.zeros(tokens, slots, dtype=torch.int32, device="cuda"), torch.zeros(tokens, slots, device="cuda")
        counts, sums = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
        uccl.uccl_route_rows(e, w, z, counts=counts, sums=sums, scratch=scratch)
        uccl.uccl_route_rows_grad(dz, z, e, d, dsums=ds)
        return e, w, counts, sums, dz
    for a, b in zip(of(scores, torch.zeros_like(scores)), of(apart(scores), apart(torch.zeros_like(scores)))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_and_clipping_of_rows_far_apart(uccl, dtype):
    g = torch.randn(600, 333, device="cuda", generator=gen(8)).to(dtype)
    per = 16 // g.element_size()
    wide = torch.zeros(600, -(-333 // per) * per, dtype=dtype, device="cuda")
    wide[:, :333] = g
    near, far = wide[:, :333], apart(wide)[:, :333]
    norms, outs = torch.zeros(2, device="cuda"), [torch.zeros_like(wide)[:, :333], apart(torch.zeros_like(wide))[:, :333]]
    scratch = torch.zeros(uccl.uccl_gradient_norm_scratch(1), dtype=torch.uint8, device="cuda")
    for i, (m, out) in enumerate(zip((near, far), outs)):
        uccl.uccl_gradient_norm(norms[i:i + 1], [m], scratch)
        uccl.uccl_gradient_clip([out], [m], norms[i:i + 1], 1.0)
    want = g.double().norm()
    assert abs(float(norms[0]) - float(want)) <= 2 ** -23 * float(want) and torch.equal(norms[0], norms[1])
    assert torch.equal(outs[0], outs[1]) and bool(outs[0].any())


def test_norm_and_clipping_of_more_than_four_gib(uccl):
    n = (1 << 31) + (1 << 20) + 5                                          # bf16: two rows of 2^30 and one of what is left
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    at = [0, 1, (1 << 30) - 1, 1 << 30, (1 << 31) - 1, 1 << 31, n - 1]
    g[at] = torch.tensor([1.0, 2.0, 3.0, 4.0, 5.0, 6.0, 7.0], dtype=torch.bfloat16, device="cuda")
    norm, out = torch.zeros(1, device="cuda"), torch.ones_like(g)
    scratch = torch.zeros(uccl.uccl_gradient_norm_scratch(3), dtype=torch.uint8, device="cuda")
    uccl.uccl_gradient_norm(norm, [g], scratch)
    want = 140.0 ** 0.5                                                    # 1 + 4 + 9 + 16 + 25 + 36 + 49
    assert abs(float(norm) - want) <= 2 ** -23 * want
    uccl.uccl_gradient_clip([out], [g], norm, 0.5)
    by = torch.tensor(0.5, device="cuda") / norm
    assert torch.equal(out[at], (g[at].float() * by).to(torch.bfloat16))
    out[at] = 0
    assert not any(bool(piece.any()) for piece in out.split(1 << 28))
