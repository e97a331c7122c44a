"""Routing of tokens to experts, experts in 4 bits, and the norm that gradients are clipped to, as cases that can be timed and
compared.

They are what an expert-parallel layer does beside the row operators: a router's scores become every token's experts and weights, and
these the order of the rows that the grouped products read; the experts' weights lie in microscaled 4 bits (e2m1 values, two a byte, and
a power of two as the scale of every 32 of a row); and the gradients of all that is learned are clipped together.  The kinds:

  route        scores to experts and weights, and these to the rows' order: what a token costs before its dispatch
  route_train  the same with the experts' counts and probabilities, the balance loss of them, and the gradient of the scores
  quantise     rows in 16 or 32 bits to microscaled 4 bits, and the values that these stand for
  product      products grouped by expert with weights in microscaled 4 bits, of rows in 16 bits or of rows that are quantised first
  clip         the norm of many gradients together, and the gradients clipped to it

Where ``own`` is false, run() computes them with elementary operations in 32 bits; where it is true it makes the calls of this library.
"""
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E2M1, E8M0 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
BLOCK = 32
COEF = 0.01        # of the balance loss
SCALE = 2.5        # of the weights of a token's experts


def listed():
    return [
        # serving: one token, 32 experts on each of 8 ranks, eight of them for the token: all latency
        {"name": "route-1", "kind": "route", "tokens": 1, "experts": 256, "slots": 8, "dtype": "bf16", "bias": True, "normalise": True, "masked": 0.0},
        # the tokens of an average dispatch
        {"name": "route-4096", "kind": "route", "tokens": 4096, "experts": 256, "slots": 8, "dtype": "bf16", "bias": True, "normalise": True, "masked": 0.0},
        # odd sizes, experts that are not there for some tokens, and tokens that have none at all
        {"name": "route-train-odd", "kind": "route_train", "tokens": 1777, "experts": 61, "slots": 6, "dtype": "f16", "bias": False, "normalise": False, "masked": 0.25},
        # training: a rank's tokens in one step, scores in 32 bits
        {"name": "route-train-32768", "kind": "route_train", "tokens": 32768, "experts": 256, "slots": 8, "dtype": "f32", "bias": True, "normalise": True, "masked": 0.0},
        # rows of an average dispatch
        {"name": "quantise-4096", "kind": "quantise", "rows": 4096, "cols": 7168, "dtype": "bf16"},
        # odd sizes: rows that end inside a block and inside a byte
        {"name": "quantise-odd-f32", "kind": "quantise", "rows": 999, "cols": 2043, "dtype": "f32"},
        # serving: 16 rows that went to 8 of 32 experts, the rows in 16 bits: the experts' weights are what is read
        {"name": "product-few-bf16", "kind": "product", "rows": 16, "cols": 7168, "out": 2048, "groups": 32, "spread": "few", "dtype": "bf16", "gather": True},
        # serving: 128 rows over all of 32 experts, quantised before the product
        {"name": "product-128-mx4", "kind": "product", "rows": 128, "cols": 7168, "out": 2048, "groups": 32, "spread": "ragged", "dtype": "mx4", "gather": True},
        # the rows of an average dispatch
        {"name": "product-4096-mx4", "kind": "product", "rows": 4096, "cols": 7168, "out": 2048, "groups": 16, "spread": "ragged", "dtype": "mx4", "gather": True},
        # odd sizes everywhere, rows in 16 bits, some experts without a row
        {"name": "product-odd-f16", "kind": "product", "rows": 2999, "cols": 2043, "out": 1003, "groups": 24, "spread": "skewed", "dtype": "f16", "gather": True},
        # training: the gradients of 16 experts' two matrices in 32 bits, and of the norm before them
        {"name": "clip-experts", "kind": "clip", "tensors": 3, "largest": 16 * 2048 * 7168, "dtype": "f32", "even": True},
        # many gradients of all sizes, from a few elements on
        {"name": "clip-many", "kind": "clip", "tensors": 300, "largest": 400000, "dtype": "bf16", "even": False},
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
    kind = rng.choice(["route", "route_train", "quantise", "product", "product", "clip"])
    if kind in ("route", "route_train"):
        experts = int(_log(rng, 8, 256))
        return {"kind": kind, "tokens": _count(rng, 1, 4096 if kind == "route" else 16384), "experts": experts, "slots": min(experts, rng.choice([1, 2, 4, 6, 8])),
                "dtype": rng.choice(["bf16", "f16", "f32"]), "bias": rng.random() < 0.5, "normalise": rng.random() < 0.5, "masked": rng.choice([0.0, 0.0, 0.125, 0.5])}
    if kind == "quantise":
        return {"kind": kind, "rows": _count(rng, 1, 4096), "cols": _cols(rng, 32, 7168), "dtype": rng.choice(["bf16", "f16"] * 2 + ["f32"])}
    if kind == "product":
        few = rng.random() < 0.5   # serving
        return {"kind": kind, "rows": _count(rng, 1, 128) if few else _count(rng, 128, 4096), "cols": _cols(rng, 512, 7168),
                "out": _cols(rng, 512, 2048), "groups": int(_log(rng, 1, 16)), "spread": rng.choice(["even", "ragged", "skewed", "few"]),
                "dtype": rng.choice(["bf16", "f16", "mx4", "mx4"]), "gather": rng.random() < 0.5}
    return {"kind": kind, "tensors": int(_log(rng, 1, 300)), "largest": _count(rng, 1000, 4000000), "dtype": rng.choice(["f32", "bf16", "f16"]), "even": False}


# ---- inputs ---------------------------------------------------------------------------------------


def _rows(rows, cols, dtype):
    """Rows of `cols` elements whose starts are 16-byte aligned, as the library takes them: a view of a wider buffer."""
    per = 16 // dtype.itemsize
    return torch.zeros(rows, -(-cols // per) * per, dtype=dtype, device="cuda")[:, :cols]


def _normal(gen, rows, cols, dtype, std=1.0):
    t = _rows(rows, cols, dtype)
    t.copy_(torch.randn(rows, cols, device="cuda", generator=gen).mul_(std))
    return t


def _mx4_rows(rows, cols):
    """Rows of packed values and of their blocks' scales, side by side as they are dispatched."""
    at, more = -(-cols // 32) * 16, -(-cols // (16 * BLOCK)) * 16
    wire = torch.zeros(rows, at + more, dtype=torch.uint8, device="cuda")
    return wire[:, :-(-cols // 2)].view(E2M1), wire[:, at:at - (-cols // BLOCK)].view(E8M0)


def _quantised(gen, rows, cols, std):
    """Rows in microscaled 4 bits."""
    q, scales = _mx4_rows(rows, cols)
    for at in range(0, rows, 8192):   # in pieces, for the largest weights
        codes, e = _to_mx4(torch.randn(min(8192, rows - at), cols, device="cuda", generator=gen).mul_(std))
        codes = torch.nn.functional.pad(codes, (0, -cols % 2))
        q.view(torch.uint8)[at:at + 8192] = codes[:, 0::2] | codes[:, 1::2] << 4
        scales.view(torch.uint8)[at:at + 8192] = (e + 127).to(torch.uint8)
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


def tensor_sizes(case):
    """Elements of every gradient: two of the largest with a small one between them, or spread over the logarithm."""
    if case["even"]:
        return [case["largest"] if i != 1 else 7168 for i in range(case["tensors"])]
    r = random.Random(case["tensors"] * 1000003 + case["largest"])
    return [case["largest"]] + [int(_log(r, 1, case["largest"])) for _ in range(case["tensors"] - 1)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    s = dict(case)
    i32 = dict(dtype=torch.int32, device="cuda")
    if kind in ("route", "route_train"):
        tokens, n, slots = case["tokens"], case["experts"], case["slots"]
        rand = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
        z = rand(tokens, n) * 1.5 + rand(n) * 0.5
        gone = torch.rand(tokens, n, device="cuda", generator=gen) < case["masked"]
        gone |= torch.rand(tokens, 1, device="cuda", generator=gen) < case["masked"] / 4
        s["scores"] = _rows(tokens, n, DTYPES[case["dtype"]])
        s["scores"].copy_(z.masked_fill(gone, float("-inf")))
        s["add"] = rand(n) * 0.1 if case["bias"] else None
        s["chosen"], s["weights"] = torch.zeros(tokens, slots, **i32), torch.zeros(tokens, slots, device="cuda")
        s["scratch"] = None   # made by the library's own callers, on the first pass
        if kind == "route":
            s["index"], s["offsets"], s["pos"] = torch.zeros(tokens * slots, **i32), torch.zeros(n + 1, **i32), torch.zeros(tokens, slots, **i32)
        else:
            s["dweights"] = rand(tokens, slots)
            s["counts"], s["sums"], s["dsums"] = torch.zeros(n, **i32), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
            s["loss"], s["dscores"] = torch.zeros(1, device="cuda"), _rows(tokens, n, DTYPES[case["dtype"]])
    elif kind == "quantise":
        rows, cols = case["rows"], case["cols"]
        # rows of different magnitudes, as activations have them
        s["x"] = _rows(rows, cols, DTYPES[case["dtype"]])
        s["x"].copy_(torch.randn(rows, cols, device="cuda", generator=gen) * torch.exp(torch.randn(rows, 1, device="cuda", generator=gen)))
        s["q"], s["scales"] = _mx4_rows(rows, cols)
        s["values"] = _rows(rows, cols, DTYPES[case["dtype"]])
    elif kind == "product":
        rows, cols, out, groups = case["rows"], case["cols"], case["out"], case["groups"]
        t = DTYPES.get(case["dtype"], torch.bfloat16)
        s["sizes"] = group_sizes(rows, groups, case["spread"], seed)
        s["first"] = torch.tensor([sum(s["sizes"][:g]) for g in range(groups + 1)], dtype=torch.int32).cuda()
        s["take"] = torch.randperm(rows, device="cuda", generator=gen).to(torch.int32) if case["gather"] else None
        s["x"] = _normal(gen, rows, cols, t)
        s["xq"], s["xs"] = _mx4_rows(rows, cols) if case["dtype"] == "mx4" else (None, None)
        w, ws = _quantised(gen, groups * out, cols, cols ** -0.5)
        s["w"], s["ws"] = w.view(torch.uint8).unflatten(0, (groups, out)).view(E2M1), ws.view(torch.uint8).unflatten(0, (groups, out)).view(E8M0)
        s["y"] = _rows(rows, out, t)
    else:
        t = DTYPES[case["dtype"]]
        sizes, per = tensor_sizes(case), 16 // t.itemsize
        starts = [0]
        for n in sizes:
            starts.append(starts[-1] + -(-n // per) * per)
        s["grads"], s["clipped"] = torch.zeros(starts[-1], dtype=t, device="cuda"), torch.zeros(starts[-1], dtype=t, device="cuda")
        s["from"] = [s["grads"][b:b + n] for b, n in zip(starts, sizes)]
        s["to"] = [s["clipped"][b:b + n] for b, n in zip(starts, sizes)]
        for g in s["from"]:
            g.copy_(torch.randn(g.shape, device="cuda", generator=gen).mul_(0.01))
        s["norm"], s["scratch"] = torch.zeros(1, device="cuda"), None
    return s


# ---- one pass -------------------------------------------------------------------------------------


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2504_17307_amd as uccl
    kind = s["kind"]
    if kind == "route":
        if s["scratch"] is None:
            s["scratch"] = torch.empty(uccl.uccl_plan_rows_scratch(s["tokens"] * s["slots"], s["experts"]), dtype=torch.uint8, device="cuda")
        uccl.uccl_route_rows(s["chosen"], s["weights"], s["scores"], bias=s["add"], normalise=s["normalise"], scale=SCALE)
        uccl.uccl_plan_rows(s["index"], s["offsets"], s["pos"], s["chosen"], s["scratch"])
        return {k: s[k] for k in ("chosen", "weights", "index", "offsets", "pos")}
    if kind == "route_train":
        if s["scratch"] is None:
            s["scratch"] = torch.empty(uccl.uccl_route_rows_scratch(s["tokens"], s["experts"]), dtype=torch.uint8, device="cuda")
        how = dict(normalise=s["normalise"], scale=SCALE)
        uccl.uccl_route_rows(s["chosen"], s["weights"], s["scores"], bias=s["add"], counts=s["counts"], sums=s["sums"], scratch=s["scratch"], **how)
        uccl.uccl_balance_loss(s["loss"], s["dsums"], s["counts"], s["sums"], s["tokens"], s["slots"], COEF)
        uccl.uccl_route_rows_grad(s["dscores"], s["scores"], s["chosen"], s["dweights"], dsums=s["dsums"], **how)
        return {k: s[k] for k in ("chosen", "weights", "counts", "sums", "loss", "dsums", "dscores")}
    if kind == "quantise":
        uccl.uccl_quantise_rows(s["q"], s["scales"], s["x"], values=s["values"])
        return {"values": s["values"]}
    if kind == "product":
        x = s["x"]
        if s["xq"] is not None:
            uccl.uccl_quantise_rows(s["xq"], s["xs"], x)
            x = s["xq"]
        uccl.uccl_group_product(s["y"], x, s["w"], s["first"], index=s["take"], x_scales=s["xs"], w_scales=s["ws"])
        return {"y": s["y"]}
    if s["scratch"] is None:
        s["scratch"] = torch.empty(uccl.uccl_gradient_norm_scratch(len(s["from"])), dtype=torch.uint8, device="cuda")
    uccl.uccl_gradient_norm(s["norm"], s["from"], s["scratch"])
    uccl.uccl_gradient_clip(s["to"], s["from"], s["norm"], 1.0)
    return {"norm": s["norm"], "clipped": s["clipped"]}


def _to_mx4(x):
    """The codes of x's elements (sign, then the number of the magnitude) and the exponents of its blocks' scales."""
    cols = x.shape[1]
    blocks = torch.nn.functional.pad(x, (0, -cols % BLOCK)).unflatten(1, (-1, BLOCK))
    most = blocks.abs().amax(2)
    e = torch.where(most > 0, torch.frexp(most)[1] - 3, -127).clamp(min=-127)   # of the greatest power of two in the block, less that of 4
    v = torch.ldexp(blocks, -e[..., None]).abs().clamp(max=6.0)
    fine = (torch.frexp(v)[1] - 1).clamp(min=0)                                 # steps of a half below 2, of 1 below 4, then of 2
    halves = torch.ldexp(torch.round(torch.ldexp(v, 1 - fine)), fine).to(torch.uint8)   # the magnitude in halves, ties to even
    number = torch.where(halves <= 4, halves, torch.where(halves <= 8, halves // 2 + 2, 7))
    return (number | (torch.signbit(blocks).to(torch.uint8) << 3)).flatten(1)[:, :cols], e


def _from_mx4(q, scales, cols):
    """The values that packed rows stand for."""
    lut = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device="cuda")
    packed = q.view(torch.uint8)
    v = lut[torch.stack([packed & 15, packed >> 4], -1).flatten(-2).int()][..., :cols]
    return v * torch.exp2(scales.view(torch.uint8).float() - 127.0).repeat_interleave(BLOCK, -1)[..., :cols]


def _routed(s):
    """Scores in 32 bits, probabilities, every token's experts in the order of their keys, and which of them are there."""
    z = s["scores"].float()
    most = z.amax(1, keepdim=True)
    p = torch.exp(z - torch.where(most > float("-inf"), most, 0.0))
    p = p / p.sum(1, keepdim=True).clamp(min=1e-30)
    key, order = torch.sort(z if s["add"] is None else z + s["add"], dim=1, descending=True, stable=True)
    return p, order[:, :s["slots"]], key[:, :s["slots"]] > float("-inf")


def _run_plain(s):
    kind = s["kind"]
    if kind in ("route", "route_train"):
        n, slots, tokens = s["experts"], s["slots"], s["tokens"]
        p, order, there = _routed(s)
        mine = torch.where(there, p.gather(1, order), 0.0)
        total = mine.sum(1, keepdim=True).clamp(min=1e-30)
        w = SCALE * (mine / total if s["normalise"] else mine)
        chosen = torch.where(there, order, -1).to(torch.int32)
        flat = chosen.reshape(-1).long()
        if kind == "route":
            key = torch.where(flat < 0, n, flat)
            by = torch.argsort(key, stable=True)
            offsets = torch.searchsorted(key[by], torch.arange(n + 1, device="cuda"))
            place = torch.empty_like(flat)
            place[by] = torch.arange(len(flat), device="cuda")
            index = torch.where(key[by] < n, by // slots, -1)
            return {"chosen": chosen, "weights": w, "index": index.to(torch.int32), "offsets": offsets.to(torch.int32),
                    "pos": torch.where(flat < 0, -1, place).to(torch.int32).view(tokens, slots)}
        counts = torch.bincount(torch.where(flat < 0, n, flat), minlength=n + 1)[:n].to(torch.int32)
        sums = p.sum(0)
        dsums = COEF * n / (slots * float(tokens) * tokens) * counts.float()
        loss = (dsums * sums).sum(0, keepdim=True)
        d = torch.where(there, s["dweights"], 0.0)
        if s["normalise"]:
            mine = mine / total
            dz = torch.zeros_like(p).scatter_add_(1, order, SCALE * mine * (d - (d * mine).sum(1, keepdim=True)))
        else:
            dz = torch.zeros_like(p).scatter_add_(1, order, SCALE * mine * d) - p * (SCALE * mine * d).sum(1, keepdim=True)
        dz = dz + p * (dsums - (p * dsums).sum(1, keepdim=True))
        return {"chosen": chosen, "weights": w, "counts": counts, "sums": sums, "loss": loss, "dsums": dsums, "dscores": dz.to(s["dscores"].dtype)}
    if kind == "quantise":
        x = s["x"].float()
        codes, e = _to_mx4(x)
        lut = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device="cuda")
        v = lut[codes.int()] * torch.exp2(e.float()).repeat_interleave(BLOCK, 1)[:, :x.shape[1]]
        return {"values": v.to(s["values"].dtype)}
    if kind == "product":
        cols = s["cols"]
        x = s["x"].float()
        if s["xq"] is not None:
            codes, e = _to_mx4(x)
            lut = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device="cuda")
            x = lut[codes.int()] * torch.exp2(e.float()).repeat_interleave(BLOCK, 1)[:, :cols]
        if s["take"] is not None:
            x = x[s["take"].long()]
        parts = x.split(s["sizes"])
        y = torch.cat([part @ _from_mx4(s["w"][g], s["ws"][g], cols).t() for g, part in enumerate(parts) if part.shape[0]])
        return {"y": y.to(s["y"].dtype)}
    squares = torch.stack([g.float().square().sum() for g in s["from"]])
    norm = squares.double().sum().sqrt().float().reshape(1)
    return {"norm": norm, "clipped": (s["grads"].float() * torch.clamp(1.0 / norm, max=1.0)).to(s["clipped"].dtype)}


# ---- the definition in 64 bits --------------------------------------------------------------------

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _mx4_nearest(x):
    """What every element of x becomes: the nearest of the values there are, of two that are as near the one with an even number."""
    x = x.double()
    out = torch.empty_like(x)
    mids = torch.tensor([(a + b) / 2 for a, b in zip(MAGNITUDES, MAGNITUDES[1:])], dtype=torch.float64, device="cuda")
    values = torch.tensor(MAGNITUDES, dtype=torch.float64, device="cuda")
    for at in range(0, x.shape[1], BLOCK):
        part = x[:, at:at + BLOCK]
        most = part.abs().amax(1, keepdim=True)
        scale = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(most, min=2.0 ** -140))) - 2, min=-127))
        v = part.abs() / scale
        below, above = torch.searchsorted(mids, v.contiguous()), torch.searchsorted(mids, v.contiguous(), right=True)
        number = torch.where(below % 2 == 0, below, above)   # they differ at a middle only
        out[:, at:at + BLOCK] = values[number] * scale * torch.sign(part)
    return out


def _mx4_values(q, scales, cols):
    bits = q.view(torch.uint8).long()
    v = torch.zeros(q.shape[0], cols, dtype=torch.float64, device="cuda")
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float64, device="cuda")
    v[:, 0::2], v[:, 1::2] = table[bits % 16], table[bits // 16][:, :cols // 2]
    power = torch.pow(2.0, scales.view(torch.uint8).double() - 127.0)
    return v * power[:, torch.arange(cols, device="cuda") // BLOCK]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("route", "route_train"):
        tokens, n, slots = case["tokens"], case["experts"], case["slots"]
        z = s["scores"].double()
        p = torch.nan_to_num(torch.exp(z - torch.logsumexp(z, 1, keepdim=True)))
        key = s["scores"].float() + (s["add"] if s["add"] is not None else 0.0)   # binary32, as the choice is defined
        at = torch.arange(n, device="cuda")
        chosen = torch.full((tokens, slots), -1, dtype=torch.int64, device="cuda")
        for j in range(slots):
            most = key.amax(1, keepdim=True)
            first = torch.where(key == most, at, n).amin(1)
            some = most[:, 0] > float("-inf")
            chosen[:, j] = torch.where(some, first, -1)
            key[torch.arange(tokens, device="cuda"), first] = float("-inf")
        t, j = torch.nonzero(chosen >= 0, as_tuple=True)
        e = chosen[t, j]
        share = p[t, e]
        if case["normalise"]:
            share = share / torch.zeros(tokens, dtype=torch.float64, device="cuda").index_add_(0, t, share)[t]
        w = torch.zeros(tokens, slots, dtype=torch.float64, device="cuda")
        w[t, j] = SCALE * share
        counts = (e[None] == at[:, None]).sum(1) if len(e) * n < 1 << 28 else torch.bincount(e, minlength=n)
        if kind == "route":
            ends = torch.cumsum(counts, 0)
            index, pos = torch.full((tokens * slots,), -1, dtype=torch.int64, device="cuda"), torch.full((tokens, slots), -1, dtype=torch.int64, device="cuda")
            for x in range(n):
                mine = torch.nonzero(chosen.reshape(-1) == x)[:, 0]
                begin = int(ends[x]) - len(mine)
                index[begin:begin + len(mine)] = mine // slots
                pos.view(-1)[mine] = begin + torch.arange(len(mine), device="cuda")
            offsets = torch.cat([torch.zeros_like(ends[:1]), ends])
            return {"chosen": chosen, "weights": w, "index": index, "offsets": offsets, "pos": pos}
        sums = torch.einsum("te->e", p)
        dsums = counts.double() * COEF * n / slots / tokens / tokens
        g = torch.zeros_like(p)   # what arrives at every probability, or at the weights themselves where these add up to SCALE
        g[t, e] = s["dweights"].double()[t, j] * SCALE
        if case["normalise"]:
            q = torch.zeros_like(p)
            q[t, e] = share
            dz = q * g - q * torch.einsum("te,te->t", q, g)[:, None]
        else:
            dz = p * g - p * torch.einsum("te,te->t", p, g)[:, None]
        dz = dz + p * (dsums[None] - torch.mv(p, dsums)[:, None])
        return {"chosen": chosen, "weights": w, "counts": counts, "sums": sums, "loss": torch.dot(dsums, sums)[None], "dsums": dsums, "dscores": dz}
    if kind == "quantise":
        return {"values": _mx4_nearest(s["x"])}
    if kind == "product":
        x = s["x"].double() if s["xq"] is None else _mx4_nearest(s["x"])
        if s["take"] is not None:
            x = torch.index_select(x, 0, s["take"].long())
        y = torch.zeros(case["rows"], case["out"], dtype=torch.float64, device="cuda")
        for g, (a, b) in enumerate(zip(s["first"].tolist(), s["first"].tolist()[1:])):
            if b > a:
                y[a:b] = torch.matmul(_mx4_values(s["w"][g], s["ws"][g], case["cols"]), x[a:b].t()).t()
        return {"y": y}
    g = s["grads"].double()
    norm = torch.linalg.vector_norm(g)
    return {"norm": norm[None], "clipped": g * min(1.0, 1.0 / float(norm))}


# ---- what one pass cannot do without --------------------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind in ("route", "route_train"):
        tokens, n, slots, e = case["tokens"], case["experts"], case["slots"], DTYPES[case["dtype"]].itemsize
        bias = 4 * n if case["bias"] else 0
        if kind == "route":
            return {"bytes": tokens * (n * e + slots * 16) + bias + 4 * (n + 1), "flops": tokens * n * 5}
        return {"bytes": tokens * (n * 2 * e + slots * 12) + bias + 12 * n, "flops": tokens * n * 12}
    if kind == "quantise":
        n, e = case["rows"] * case["cols"], DTYPES[case["dtype"]].itemsize
        return {"bytes": int(n * (2 * e + 17 / 32)), "flops": 4 * n}
    if kind == "product":
        rows, cols, out, groups = case["rows"], case["cols"], case["out"], case["groups"]
        # the weights of the groups that have rows; "few" leaves a quarter of them
        with_rows = max(1, groups // 4) if case["spread"] == "few" else groups
        used = min(rows, with_rows) * out * cols
        return {"bytes": int(2 * rows * cols + used * 17 / 32 + 2 * rows * out), "flops": 2 * rows * cols * out}
    n = sum(tensor_sizes(case))
    return {"bytes": 2 * n * DTYPES[case["dtype"]].itemsize + 4, "flops": 3 * n}
