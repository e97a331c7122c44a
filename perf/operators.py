"""The row operators around an all-to-all dispatch, as cases that can be timed and compared.

A rank of an expert-parallel layer normalises its tokens' rows and sends them (in 8 bits with a scale beside each
row), multiplies the rows that it received with the weights of its own experts, and adds what comes back to its
tokens.  The kinds:

  norm          residual's addition, root-mean-square norm, output in the input's type or in e4m3 with a scale a row
  norm_grad     gradients of the same to its input and its weight
  product       products grouped by expert: ragged groups, rows taken through an index, 16 or 8 bits
  product_grad  gradients of the same to its rows and to the experts' weights
  combine       every token's weighted sum of its experts' rows, and the residual
  combine_grad  gradients of the same to the rows and to the weights

Where ``own`` is false, run() computes them with elementary operations in 32 bits; where it is true it makes the
calls of this library.
"""
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
EPS = 1e-6


def listed():
    return [
        # serving: one token's row before its dispatch, all latency
        {"name": "norm-1-e4m3", "kind": "norm", "rows": 1, "cols": 7168, "dtype": "bf16", "out": "e4m3", "residual": True},
        # the rows of a full dispatch (7 peers, at most 16 MiB of rows each: 4096 on average), as 8-bit wire rows
        {"name": "norm-4096-e4m3", "kind": "norm", "rows": 4096, "cols": 7168, "dtype": "bf16", "out": "e4m3", "residual": True},
        # odd sizes: a norm inside an expert, rows that end inside a load
        {"name": "norm-odd-f16", "kind": "norm", "rows": 1777, "cols": 2043, "dtype": "f16", "out": "same", "residual": False},
        # training: the gradient of the dispatch's norm, with what arrives along the residual
        {"name": "norm-grad-4096", "kind": "norm_grad", "rows": 4096, "cols": 7168, "dtype": "bf16", "carry": True},
        # serving: 16 rows that went to 8 of 32 experts, in 16 bits: the experts' weights are what is read
        {"name": "product-few-bf16", "kind": "product", "rows": 16, "cols": 7168, "out": 2048, "groups": 32, "spread": "few",
         "dtype": "bf16", "gather": True},
        # serving: 128 rows over all of 32 experts, in 8 bits
        {"name": "product-128-e4m3", "kind": "product", "rows": 128, "cols": 7168, "out": 2048, "groups": 32, "spread": "ragged",
         "dtype": "e4m3", "gather": True},
        # the rows of an average dispatch in 8 bits, read where the scatter placed them
        {"name": "product-4096-e4m3", "kind": "product", "rows": 4096, "cols": 7168, "out": 2048, "groups": 16, "spread": "ragged",
         "dtype": "e4m3", "gather": True},
        # the second product of an expert for the fullest dispatch (7 x 1170 rows), 16 bits
        {"name": "product-8190-bf16", "kind": "product", "rows": 8190, "cols": 2048, "out": 7168, "groups": 16, "spread": "ragged",
         "dtype": "bf16", "gather": False},
        # odd sizes everywhere, some experts without a row
        {"name": "product-odd-f16", "kind": "product", "rows": 2999, "cols": 2043, "out": 1003, "groups": 24, "spread": "skewed",
         "dtype": "f16", "gather": True},
        # training: both gradients for an average dispatch
        {"name": "product-grad-4096", "kind": "product_grad", "rows": 4096, "cols": 7168, "out": 2048, "groups": 16,
         "spread": "ragged", "dtype": "bf16", "gather": True},
        # 4096 tokens' sums over eight experts each, one in eight of them on no rank that answered
        {"name": "combine-4096", "kind": "combine", "tokens": 4096, "slots": 8, "cols": 7168, "dtype": "bf16", "residual": True,
         "missing": 0.125},
        # training: the gradient of a smaller one, without holes
        {"name": "combine-grad-1024", "kind": "combine_grad", "tokens": 1024, "slots": 8, "cols": 7168, "dtype": "bf16",
         "missing": 0.0},
    ]


def _log(rng, lo, hi):
    return lo * (hi / lo) ** rng.random()


def _cols(rng, lo, hi):
    """A row's length: a multiple of 56 (7168 = 128 x 56) or, one time in three, an odd number."""
    n = _log(rng, lo, hi)
    return int(n) | 1 if rng.random() < 1 / 3 else max(1, round(n / 56)) * 56


def _count(rng, lo, hi):
    n = int(_log(rng, lo, hi))
    return n + 1 if n % 1024 == 0 else n


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "product", "product", "product_grad", "combine", "combine_grad"])
    if kind in ("norm", "norm_grad"):
        c = {"kind": kind, "rows": _count(rng, 1, 4096), "cols": _cols(rng, 256, 7168), "dtype": rng.choice(["bf16", "f16", "f32"])}
        if kind == "norm":
            return {**c, "out": rng.choice(["same", "e4m3"]), "residual": rng.random() < 0.5}
        return {**c, "carry": rng.random() < 0.5}
    if kind in ("product", "product_grad"):
        few = kind == "product" and rng.random() < 0.4   # serving
        return {"kind": kind, "rows": _count(rng, 1, 128) if few else _count(rng, 128, 4096), "cols": _cols(rng, 512, 7168),
                "out": _cols(rng, 512, 2048), "groups": int(_log(rng, 1, 32)), "spread": rng.choice(["even", "ragged", "skewed", "few"]),
                "dtype": rng.choice(["bf16", "f16"] if kind == "product_grad" else ["bf16", "f16", "e4m3", "e4m3"]),
                "gather": rng.random() < 0.5}
    c = {"kind": kind, "tokens": _count(rng, 1, 2048), "slots": rng.choice([1, 2, 4, 6, 8]), "cols": _cols(rng, 256, 7168),
         "dtype": rng.choice(["bf16", "f16", "f32"]), "missing": rng.choice([0.0, 0.125, 0.5])}
    return {**c, "residual": rng.random() < 0.5} if kind == "combine" else c


# ---- inputs ---------------------------------------------------------------------------------------


def _rows(rows, cols, dtype):
    """Rows of `cols` elements whose starts are 16-byte aligned, as the library takes them: a view of a wider buffer."""
    per = 16 // dtype.itemsize
    return torch.zeros(rows, -(-cols // per) * per, dtype=dtype, device="cuda")[:, :cols]


def _normal(gen, rows, cols, dtype, std=1.0):
    t = _rows(rows, cols, dtype)
    t.copy_(torch.randn(rows, cols, device="cuda", generator=gen).mul_(std))
    return t


def _wire_rows(rows, cols):
    """8-bit rows as they are dispatched: the values, then the row's scale on the next 16-byte boundary."""
    at = -(-cols // 16) * 16
    wire = torch.zeros(rows, at + 16, dtype=torch.uint8, device="cuda")
    return wire[:, :cols].view(E4M3), wire[:, at:at + 4].view(torch.float32)


def _quantised(gen, rows, cols, std=1.0, wire=True):
    """8-bit rows and their scales: as wire rows, or (weights) each on its own."""
    if wire:
        q, scales = _wire_rows(rows, cols)
    else:
        q, scales = _rows(rows, cols, E4M3), torch.zeros(rows, 1, device="cuda")
    for at in range(0, rows, 8192):   # in pieces, for the largest weights
        t = torch.randn(min(8192, rows - at), cols, device="cuda", generator=gen).mul_(std)
        s = t.abs().amax(1, keepdim=True) / E4M3_MAX
        scales[at:at + 8192] = s
        q[at:at + 8192] = (t / s).to(E4M3)
    return q, scales


def group_sizes(rows, groups, spread, seed):
    """How many rows each expert has."""
    r = random.Random(seed)
    share = [{"even": 1.0, "ragged": u, "skewed": u ** 4, "few": u}[spread] for u in (r.random() + 1e-9 for _ in range(groups))]
    if spread == "few":
        for g in r.sample(range(groups), groups - max(1, groups // 4)):
            share[g] = 0.0
    if spread == "skewed" and groups > 1:
        share[r.randrange(groups)] = 0.0
    total, run_, ends = sum(share) or 1.0, 0.0, []
    for s in share:
        run_ += s
        ends.append(round(rows * run_ / total))
    last = max(g for g in range(groups) if share[g]) if sum(share) else groups - 1
    ends[last:] = [rows] * (groups - last)
    return [b - a for a, b in zip([0] + ends, ends)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    s = dict(case)
    if kind in ("norm", "norm_grad"):
        rows, cols, t = case["rows"], case["cols"], DTYPES[case["dtype"]]
        s["weight"] = _normal(gen, 1, cols, t, 0.1).add_(1.0)[0]
        if kind == "norm":
            s["x"] = _normal(gen, rows, cols, t)
            s["r"] = _normal(gen, rows, cols, t, 3.0) if case["residual"] else None
            s["h"] = _rows(rows, cols, t) if case["residual"] else None
            s["y"], s["scales"] = _wire_rows(rows, cols) if case["out"] == "e4m3" else (_rows(rows, cols, t), None)
            s["rstd"] = torch.zeros(rows, device="cuda")
        else:
            s["h"], s["dy"] = _normal(gen, rows, cols, t, 3.0), _normal(gen, rows, cols, t)
            s["dh"] = _normal(gen, rows, cols, t) if case["carry"] else None
            s["rstd"] = torch.rsqrt(s["h"].double().square().mean(1) + EPS).float()
            s["dx"], s["dweight"] = _rows(rows, cols, t), torch.zeros(cols, device="cuda")
            s["scratch"] = None   # made by the library's own callers, on the first pass
    elif kind in ("product", "product_grad"):
        rows, cols, out, groups = case["rows"], case["cols"], case["out"], case["groups"]
        s["sizes"] = group_sizes(rows, groups, case["spread"], seed)
        s["offsets"] = torch.tensor([sum(s["sizes"][:g]) for g in range(groups + 1)], dtype=torch.int32).cuda()
        s["index"] = torch.randperm(rows, device="cuda", generator=gen).to(torch.int32) if case["gather"] else None
        s["xs"] = s["ws"] = None
        if case["dtype"] == "e4m3":
            t = torch.bfloat16
            s["x"], s["xs"] = _quantised(gen, rows, cols)
            w, ws = _quantised(gen, groups * out, cols, cols ** -0.5, wire=False)
            s["w"], s["ws"] = w.unflatten(0, (groups, out)), ws.unflatten(0, (groups, out))
        else:
            t = DTYPES[case["dtype"]]
            s["x"] = _normal(gen, rows, cols, t)
            s["w"] = _normal(gen, groups * out, cols, t, cols ** -0.5).unflatten(0, (groups, out))
        if kind == "product":
            s["y"] = _rows(rows, out, t)
        else:
            s["dy"] = _normal(gen, rows, out, t)
            s["dx"] = _rows(rows, cols, t)
            s["dw"] = _rows(groups * out, cols, torch.float32).unflatten(0, (groups, out))
    else:
        tokens, slots, cols, t = case["tokens"], case["slots"], case["cols"], DTYPES[case["dtype"]]
        there = torch.rand(tokens * slots, device="cuda", generator=gen) >= case["missing"]
        n = int(there.sum())
        s["pos"] = torch.full((tokens * slots,), -1, dtype=torch.int32, device="cuda")
        s["pos"][there] = torch.randperm(n, device="cuda", generator=gen).to(torch.int32)
        s["pos"] = s["pos"].view(tokens, slots)
        s["w"] = torch.softmax(torch.randn(tokens, slots, device="cuda", generator=gen), 1)
        s["y"] = _normal(gen, max(1, n), cols, t)
        if kind == "combine":
            s["r"] = _normal(gen, tokens, cols, t, 3.0) if case["residual"] else None
            s["out"] = _rows(tokens, cols, t)
        else:
            s["dout"], s["dy"] = _normal(gen, tokens, cols, t), _rows(max(1, n), cols, t)
            s["dw"] = torch.zeros(tokens, slots, device="cuda")
    return s


# ---- one pass -------------------------------------------------------------------------------------


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2504_17307_amd as uccl
    kind = s["kind"]
    if kind == "norm":
        uccl.uccl_norm_rows(s["y"], s["x"], s["weight"], EPS, residual=s["r"], h=s["h"], rstd=s["rstd"], scales=s["scales"])
        return {"y": s["y"], "h": s["h"], "scales": s["scales"], "rstd": s["rstd"]}
    if kind == "norm_grad":
        if s["scratch"] is None:
            s["scratch"] = torch.empty(uccl.uccl_norm_rows_scratch(s["rows"], s["cols"]), dtype=torch.uint8, device="cuda")
        uccl.uccl_norm_rows_grad(s["dx"], s["dweight"], s["dy"], s["h"], s["rstd"], s["weight"], s["scratch"], dh=s["dh"])
        return {"dx": s["dx"], "dweight": s["dweight"]}
    if kind == "product":
        uccl.uccl_group_product(s["y"], s["x"], s["w"], s["offsets"], index=s["index"], x_scales=s["xs"], w_scales=s["ws"])
        return {"y": s["y"]}
    if kind == "product_grad":
        uccl.uccl_group_product_grad_x(s["dx"], s["dy"], s["w"], s["offsets"])
        uccl.uccl_group_product_grad_w(s["dw"], s["dy"], s["x"], s["offsets"], index=s["index"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if kind == "combine":
        uccl.uccl_combine_rows(s["out"], s["y"], s["pos"], weights=s["w"], residual=s["r"])
        return {"out": s["out"]}
    uccl.uccl_combine_rows_grad(s["dy"], s["dw"], s["dout"], s["y"], s["pos"], weights=s["w"])
    return {"dy": s["dy"], "dw": s["dw"]}


def _products(a, b, sizes):
    """a's rows of each group times that group's b."""
    return torch.cat([part @ b[g].float() for g, part in enumerate(a.split(sizes)) if part.shape[0]])


def _run_plain(s):
    kind = s["kind"]
    if kind == "norm":
        t, h = s["x"].dtype, s["x"].float()
        if s["r"] is not None:
            h = h + s["r"].float()
        rstd = torch.rsqrt(h.square().mean(1) + EPS)
        y = h * rstd[:, None] * s["weight"].float()
        scales = None
        if s["scales"] is not None:
            scales = y.abs().amax(1, keepdim=True) / E4M3_MAX
            y = y / scales
        return {"y": y.to(s["y"].dtype), "h": None if s["h"] is None else h.to(t), "scales": scales, "rstd": rstd}
    if kind == "norm_grad":
        h, dy, rstd = s["h"].float(), s["dy"].float(), s["rstd"][:, None]
        n, g = h * rstd, dy * s["weight"].float()
        dx = rstd * (g - n * (g * n).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(s["dx"].dtype), "dweight": (dy * n).sum(0)}
    if kind in ("product", "product_grad"):
        x = s["x"] if s["index"] is None else s["x"].view(torch.uint8 if s["xs"] is not None else s["x"].dtype)[s["index"].long()].view(s["x"].dtype)
        x, w, sizes = x.float(), s["w"], s["sizes"]
        if kind == "product":
            if s["xs"] is not None:
                x = x * (s["xs"] if s["index"] is None else s["xs"][s["index"].long()])
                w = w.float() * s["ws"]
            return {"y": _products(x, w.transpose(1, 2), sizes).to(s["y"].dtype)}
        dy = s["dy"].float()
        dw = torch.stack([a.t() @ b for a, b in zip(dy.split(sizes), x.split(sizes))])
        return {"dx": _products(dy, w, sizes).to(s["dx"].dtype), "dw": dw}
    pos, there = s["pos"].long().clamp(min=0), (s["pos"] >= 0)[..., None]
    y = torch.where(there, s["y"][pos].float(), 0.0)
    if kind == "combine":
        out = (y * s["w"][..., None]).sum(1)
        return {"out": (out if s["r"] is None else out + s["r"].float()).to(s["out"].dtype)}
    dout = s["dout"].float()
    dy = torch.zeros_like(s["y"])
    dy[s["pos"][there[..., 0]].long()] = (s["w"][..., None] * dout[:, None])[there[..., 0]].to(dy.dtype)
    return {"dy": dy, "dw": (y * dout[:, None]).sum(2)}


# ---- the definition in 64 bits --------------------------------------------------------------------


def _e4m3_nearest(v):
    """The e4m3 value nearest to each of v (|v| <= 448), ties to even: 3 bits after the leading one, steps of 2^-9 below 2^-6."""
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(v.abs(), min=2.0 ** -20))), min=-6.0) - 3.0)
    return torch.round(v / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    d = lambda name: s[name].double()  # noqa: E731
    if kind == "norm":
        h = d("x") + (d("r") if s["r"] is not None else 0.0)
        mean = (h * h).sum(1) / h.shape[1]
        rstd = 1.0 / torch.sqrt(mean + EPS)
        y = rstd[:, None] * h * d("weight")
        scales = None
        if s["scales"] is not None:
            scales = torch.amax(torch.abs(y), dim=1, keepdim=True) / E4M3_MAX
            y = _e4m3_nearest(y / scales)
        return {"y": y, "h": h if s["h"] is not None else None, "scales": scales, "rstd": rstd}
    if kind == "norm_grad":
        h, dy, w, r = d("h"), d("dy"), d("weight"), d("rstd")
        along = torch.einsum("rc,rc,c->r", dy, h, w) / h.shape[1]
        dx = r[:, None] * dy * w - (r ** 3 * along)[:, None] * h
        return {"dx": dx + d("dh") if s["dh"] is not None else dx, "dweight": torch.einsum("rc,rc,r->c", dy, h, r)}
    if kind in ("product", "product_grad"):
        rows = torch.arange(case["rows"], device="cuda") if s["index"] is None else s["index"].long()
        group = torch.repeat_interleave(torch.arange(case["groups"], device="cuda"), torch.tensor(s["sizes"], device="cuda"))
        x = s["x"].double()[rows]
        if s["xs"] is not None:
            x = x * s["xs"].double()[rows]
        if kind == "product":
            y = torch.zeros(case["rows"], case["out"], dtype=torch.float64, device="cuda")
        else:
            dx, dw, dy = torch.zeros_like(x), torch.zeros(s["dw"].shape, dtype=torch.float64, device="cuda"), d("dy")
        for g in range(case["groups"]):
            mine = torch.nonzero(group == g)[:, 0]
            w = s["w"][g].double() * (s["ws"][g].double() if s["ws"] is not None else 1.0)
            if kind == "product":
                y[mine] = torch.matmul(w, x[mine].t()).t()
            else:
                dx[mine] = torch.matmul(w.t(), dy[mine].t()).t()
                dw[g] = torch.matmul(x[mine].t(), dy[mine]).t()
        return {"y": y} if kind == "product" else {"dx": dx, "dw": dw}
    tokens, slots, cols = case["tokens"], case["slots"], case["cols"]
    if kind == "combine":
        out = d("r") if s["r"] is not None else torch.zeros(tokens, cols, dtype=torch.float64, device="cuda")
    else:
        dout = d("dout")
        dy, dw = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda"), torch.zeros(tokens, slots, dtype=torch.float64, device="cuda")
    for j in range(slots):
        t = torch.nonzero(s["pos"][:, j] >= 0)[:, 0]
        p = s["pos"][t, j].long()
        if kind == "combine":
            out[t] += s["w"][t, j, None].double() * s["y"][p].double()
        else:
            dy[p] = s["w"][t, j, None].double() * dout[t]
            dw[t, j] = torch.einsum("tc,tc->t", s["y"][p].double(), dout[t])
    return {"out": out} if kind == "combine" else {"dy": dy, "dw": dw}


# ---- what one pass cannot do without --------------------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        n, e = case["rows"] * case["cols"], DTYPES[case["dtype"]].itemsize
        if kind == "norm":
            moved = n * (e * (3 if case["residual"] else 1) + (1 if case["out"] == "e4m3" else e))
            return {"bytes": moved + case["cols"] * e + 8 * case["rows"], "flops": 6 * n}
        return {"bytes": n * e * (4 if case["carry"] else 3) + case["cols"] * (e + 4) + 4 * case["rows"], "flops": 10 * n}
    if kind in ("product", "product_grad"):
        rows, cols, out, groups = case["rows"], case["cols"], case["out"], case["groups"]
        e = 1 if case["dtype"] == "e4m3" else 2
        # the weights of the groups that have rows; "few" leaves a quarter of them
        with_rows = max(1, groups // 4) if case["spread"] == "few" else groups
        used = min(rows, with_rows) * out * cols
        if kind == "product":
            return {"bytes": e * (rows * cols + used) + 2 * rows * out, "flops": 2 * rows * cols * out}
        return {"bytes": 2 * (rows * cols + used + rows * out + rows * cols) + 4 * groups * out * cols, "flops": 4 * rows * cols * out}
    e = DTYPES[case["dtype"]].itemsize
    there = int(case["tokens"] * case["slots"] * (1 - case["missing"])) * case["cols"]
    n = case["tokens"] * case["cols"]
    if kind == "combine":
        return {"bytes": e * (there + n * (2 if case["residual"] else 1)) + 8 * case["tokens"] * case["slots"], "flops": 2 * there}
    return {"bytes": e * (2 * there + n) + 12 * case["tokens"] * case["slots"], "flops": 3 * there}
