"""An expert-parallel layer on one GPU: the row operators around a dispatch through the chunk path.

    out[t] = x[t] + sum over the token's experts e of weight[t, e] down_e(silu(up_e(norm(x[t]))))

`dispatch` is what lies between a sender's rows and a receiver's: staged chunks, arrivals in any order and some of them twice, deduplication
and placement.  `serve` sends rows of 8 bits with their scales and multiplies them as they arrived; `train` sends 16-bit rows and
returns the gradients too.  Which row goes where is planned on the GPU, and nothing here reads it back; the records of what arrived come from
the host, as a receiver's control path has them.

A `Router` chooses the experts from scores of the normalised rows.  `serve_in_4_bits` goes by one and sends rows of microscaled 4 bits to experts whose
weights lie in them too; `train_routed` trains it with the experts, with a loss that keeps them evenly used, and clips all gradients together.

    python examples/expert_layer.py
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2504_17307_amd as uccl  # noqa: E402
from synth.layout import DESC, NO_FORWARD, bitmap_words  # noqa: E402

E4M3, E2M1, E8M0 = torch.float8_e4m3fn, torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
EPS = 1e-6


def plan(experts, n_experts):
    """``experts``: tokens x slots, the expert of every slot, -1: none.  Returns what the operators go by: the token of every
    row in order of experts (-1 behind the last), the experts' first rows, and every slot's row (-1: none)."""
    experts = experts.to(torch.int32).contiguous()
    new = lambda *shape: torch.empty(*shape, dtype=torch.int32, device=experts.device)  # noqa: E731
    index, offsets, pos = new(experts.numel()), new(n_experts + 1), new(*experts.shape)
    scratch = torch.empty(uccl.uccl_plan_rows_scratch(experts.numel(), n_experts), dtype=torch.uint8, device=experts.device)
    uccl.uccl_plan_rows(index, offsets, pos, experts, scratch)
    return index, offsets, pos


def wire_rows(rows, cols, device="cuda"):
    """Rows of 8 bits as they are sent: values, then the row's scale on the next 16-byte boundary."""
    at = -(-cols // 16) * 16
    wire = torch.zeros(rows, at + 16, dtype=torch.uint8, device=device)
    return wire, wire[:, :cols].view(E4M3), wire[:, at:at + 4].view(torch.float32)


def dispatch(rows, arrival_order, chunk_rows=1):
    """``rows`` (contiguous, each a multiple of 16 bytes) through staging, the network and placement: a new tensor with the same
    rows.  ``arrival_order`` names the chunks as they arrive, each at least once."""
    total = rows.numel() * rows.element_size()
    chunk = chunk_rows * rows.shape[1] * rows.element_size()
    n = -(-total // chunk)
    staged, placed = torch.empty(n * chunk, dtype=torch.uint8, device=rows.device), torch.zeros_like(rows)
    uccl.uccl_chunk_segment(staged, rows, 0, total, chunk)
    # what the receiver's control path writes: here a slot of the sender's staging is the slot of every arrival of its chunk
    d = np.zeros(len(arrival_order), dtype=DESC)
    d["seq"] = arrival_order
    d["src_off"] = d["dst_off"] = d["seq"].astype(np.uint64) * chunk
    d["out_off"] = NO_FORWARD
    d["len"] = np.minimum(chunk, total - d["dst_off"].astype(np.int64))
    records = torch.from_numpy(d.view(np.uint8)).to(rows.device)
    seen = torch.empty(bitmap_words(n), dtype=torch.int32, device=rows.device)
    uccl.uccl_dedup_reset(seen, n)
    uccl.uccl_chunk_scatter(placed, staged, records, len(d), seen)
    return placed


def serve(x, norm_weight, up, up_scales, down, experts, weights, arrival_order):
    """The layer's output.  ``up``: experts x hidden x cols in 8 bits with a scale for every row, ``down``: experts x cols x hidden
    in x's type."""
    (tokens, cols), (n_experts, hidden, _) = x.shape, up.shape
    index, offsets, pos = plan(experts, n_experts)
    rows = index.numel()
    wire, y, scales = wire_rows(tokens, cols, x.device)
    uccl.uccl_norm_rows(y, x, norm_weight, EPS, scales=scales)
    at = wire.shape[1] - 16
    wire = dispatch(wire, arrival_order)
    y, scales = wire[:, :cols].view(E4M3), wire[:, at:at + 4].view(torch.float32)
    u = torch.empty(rows, hidden, dtype=x.dtype, device=x.device)
    uccl.uccl_group_product(u, y, up, offsets, index=index, x_scales=scales, w_scales=up_scales)
    a = torch.nn.functional.silu(u)
    z = torch.empty(rows, cols, dtype=x.dtype, device=x.device)
    uccl.uccl_group_product(z, a, down, offsets)
    out = torch.empty_like(x)
    uccl.uccl_combine_rows(out, z, pos, weights=weights, residual=x)
    return {"y": y, "scales": scales, "u": u, "a": a, "z": z, "pos": pos, "out": out}


def train(x, norm_weight, up, down, experts, weights, dout, arrival_order, router=None):
    """The layer's output and, for the gradient ``dout`` of it, the gradients of all that is learned and of x; all in 16 bits.  A ``router``
    chooses the experts and their weights from the normalised rows, and has its own gradient then."""
    (tokens, cols), (n_experts, hidden, _) = x.shape, up.shape
    like = dict(dtype=x.dtype, device=x.device)
    f32 = dict(dtype=torch.float32, device=x.device)
    y, rstd = torch.empty_like(x), torch.empty(tokens, **f32)
    uccl.uccl_norm_rows(y, x, norm_weight, EPS, rstd=rstd)
    if router is not None:
        experts, weights = router.forward(y)
    index, offsets, pos = plan(experts, n_experts)
    rows = index.numel()
    y = dispatch(y, arrival_order)
    u, z, out = torch.empty(rows, hidden, **like), torch.empty(rows, cols, **like), torch.empty_like(x)
    uccl.uccl_group_product(u, y, up, offsets, index=index)
    a = torch.nn.functional.silu(u)
    uccl.uccl_group_product(z, a, down, offsets)
    uccl.uccl_combine_rows(out, z, pos, weights=weights, residual=x)

    dz, dweights = torch.empty_like(z), torch.empty_like(weights)
    uccl.uccl_combine_rows_grad(dz, dweights, dout, z, pos, weights=weights)
    da, ddown = torch.empty_like(a), torch.empty(down.shape, **f32)
    uccl.uccl_group_product_grad_x(da, dz, down, offsets)
    uccl.uccl_group_product_grad_w(ddown, dz, a, offsets)
    du = torch.ops.aten.silu_backward(da, u)
    dr, dup = torch.empty(rows, cols, **like), torch.empty(up.shape, **f32)
    uccl.uccl_group_product_grad_x(dr, du, up, offsets)
    uccl.uccl_group_product_grad_w(dup, du, y, offsets, index=index)
    dy = torch.empty_like(x)                       # a token's row went to several experts: the sum of theirs
    uccl.uccl_combine_rows(dy, dr, pos, residual=None if router is None else router.backward(dweights))
    dx, dnorm = torch.empty_like(x), torch.empty(cols, **f32)
    scratch = torch.empty(uccl.uccl_norm_rows_scratch(tokens, cols), dtype=torch.uint8, device=x.device)
    uccl.uccl_norm_rows_grad(dx, dnorm, dy, x, rstd, norm_weight, scratch, dh=dout)
    return {"y": y, "rstd": rstd, "u": u, "a": a, "z": z, "pos": pos, "out": out, "dz": dz, "dweights": dweights, "da": da, "ddown": ddown,
            "du": du, "dr": dr, "dup": dup, "dy": dy, "dx": dx, "dnorm": dnorm}


class Router:
    """Experts of rows by a linear layer: ``weight``, n_experts x cols, in the rows' type; ``bias``: float32, one an expert, for the choice only."""

    def __init__(self, weight, bias, slots, coef=0.01):
        self.weight, self.bias, self.slots, self.coef = weight, bias, slots, coef

    def forward(self, y):
        """The experts and weights of the rows; counts, sums, loss and all that backward() needs stay here."""
        n, device = self.weight.shape[0], y.device
        f32 = dict(dtype=torch.float32, device=device)
        self.y, self.all = y, torch.tensor([0, y.shape[0]], dtype=torch.int32).to(device, non_blocking=True)   # one group: every row
        self.scores = self._rows(torch.float32)
        uccl.uccl_group_product(self.scores, y, self.weight[None], self.all)
        self.experts, weights = torch.empty(y.shape[0], self.slots, dtype=torch.int32, device=device), torch.empty(y.shape[0], self.slots, **f32)
        self.counts, self.sums = torch.empty(n, dtype=torch.int32, device=device), torch.empty(n, **f32)
        scratch = torch.empty(uccl.uccl_route_rows_scratch(y.shape[0], n), dtype=torch.uint8, device=device)
        uccl.uccl_route_rows(self.experts, weights, self.scores, bias=self.bias, normalise=True, counts=self.counts, sums=self.sums, scratch=scratch)
        self.loss, self.dsums = torch.empty(1, **f32), torch.empty(n, **f32)
        uccl.uccl_balance_loss(self.loss, self.dsums, self.counts, self.sums, y.shape[0], self.slots, self.coef)
        return self.experts, weights

    def _rows(self, dtype):
        """One number for every row and expert, rows on 16-byte boundaries."""
        n, per = self.weight.shape[0], 16 // dtype.itemsize
        return torch.empty(self.y.shape[0], -(-n // per) * per, dtype=dtype, device=self.y.device)[:, :n]

    def backward(self, dweights):
        """The gradient of the rows, for ``dweights`` of the weights and the balance loss; the weight's stays here."""
        dscores = self._rows(torch.float32)
        uccl.uccl_route_rows_grad(dscores, self.scores, self.experts, dweights, dsums=self.dsums, normalise=True)
        if self.y.dtype == torch.bfloat16:
            dy, self.dweight = self._products(self._rows(torch.bfloat16).copy_(dscores), torch.bfloat16)   # products are of 16 bits
            return dy
        # f16 has nothing below 2^-24, which the balance loss's part of a score is below already with some thousand tokens: the greatest is brought to 1 by a power of two,
        # and what the first 11 bits leave, 2^24 times as large, is multiplied by itself
        by = torch.exp2(-torch.frexp(dscores.abs().amax())[1].clamp(min=-100).float())
        dscores *= by
        first = self._rows(torch.float16).copy_(dscores)
        (dy, dweight), (dy2, dweight2) = self._products(first, torch.float32), self._products(self._rows(torch.float16).copy_((dscores - first) * 2.0 ** 24), torch.float32)
        self.dweight = (dweight + dweight2 * 2.0 ** -24) / by
        return ((dy + dy2 * 2.0 ** -24) / by).to(torch.float16)

    def _products(self, dscores, dtype):
        """The gradients of the rows, in that type, and of the weight."""
        dy, dweight = torch.empty(self.y.shape, dtype=dtype, device=self.y.device), torch.empty(self.weight.shape, dtype=torch.float32, device=self.y.device)
        uccl.uccl_group_product_grad_x(dy, dscores, self.weight[None], self.all)
        uccl.uccl_group_product_grad_w(dweight[None], dscores, self.y, self.all)
        return dy, dweight


def serve_in_4_bits(x, norm_weight, router, up, up_scales, down, down_scales, arrival_order):
    """The layer's output.  ``up``: experts x hidden x cols, ``down``: experts x cols x hidden, both in microscaled 4 bits.  Rows are sent in 4 bits; what is
    between the products stays in x's type."""
    (tokens, cols), (n_experts, hidden, _) = x.shape, up.shape
    like = dict(dtype=x.dtype, device=x.device)
    n = torch.empty_like(x)
    uccl.uccl_norm_rows(n, x, norm_weight, EPS)
    experts, weights = router.forward(n)
    index, offsets, pos = plan(experts, n_experts)
    at, more = -(-cols // 32) * 16, -(-cols // 512) * 16
    wire = torch.zeros(tokens, at + more, dtype=torch.uint8, device=x.device)   # values, then the blocks' scales
    split = lambda w: (w[:, :-(-cols // 2)].view(E2M1), w[:, at:at - (-cols // 32)].view(E8M0))  # noqa: E731
    uccl.uccl_quantise_rows(*split(wire), n)
    y, scales = split(dispatch(wire, arrival_order))
    u = torch.empty(index.numel(), hidden, **like)
    uccl.uccl_group_product(u, y, up, offsets, index=index, x_scales=scales, w_scales=up_scales)
    a = torch.nn.functional.silu(u)
    z = torch.empty(index.numel(), cols, **like)
    uccl.uccl_group_product(z, a, down, offsets, w_scales=down_scales)
    out = torch.empty_like(x)
    uccl.uccl_combine_rows(out, z, pos, weights=weights, residual=x)
    return {"n": n, "y": y, "scales": scales, "experts": experts, "weights": weights, "u": u, "a": a, "z": z, "pos": pos, "out": out}


def train_routed(x, norm_weight, router, up, down, dout, arrival_order, most=1.0):
    """`train` with a router, and the gradients of all that is learned, clipped to a norm of ``most`` together."""
    got = train(x, norm_weight, up, down, None, None, dout, arrival_order, router=router)
    grads = [got["dnorm"], router.dweight, got["dup"], got["ddown"]]
    norm = torch.empty(1, dtype=torch.float32, device=x.device)
    uccl.uccl_gradient_norm(norm, grads, torch.empty(uccl.uccl_gradient_norm_scratch(len(grads)), dtype=torch.uint8, device=x.device))
    clipped = [torch.empty_like(g) for g in grads]
    uccl.uccl_gradient_clip(clipped, grads, norm, most)
    return dict(got, drouter=router.dweight, loss=router.loss, norm=norm, clipped=dict(zip(("dnorm", "drouter", "dup", "ddown"), clipped)))


def inputs(tokens, slots, cols, hidden, n_experts, dtype=torch.bfloat16, seed=0, missing=0.125):
    """Random ones: x, the norm's weight, up, down, experts, weights, dout and an order of arrival with every 50th chunk twice."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    experts = torch.argsort(torch.rand(tokens, n_experts, device="cuda", generator=g), 1)[:, :slots]
    experts = torch.where(torch.rand(tokens, slots, device="cuda", generator=g) < missing, -1, experts)
    r = np.random.default_rng(seed)
    arrivals = r.permutation(np.concatenate([np.arange(tokens), np.arange(0, tokens, 50)])).astype(np.uint32)
    return dict(x=normal(tokens, cols).to(dtype), norm_weight=(1 + 0.1 * normal(cols)).to(dtype),
                up=(normal(n_experts, hidden, cols) * cols ** -0.5).to(dtype), down=(normal(n_experts, cols, hidden) * hidden ** -0.5).to(dtype),
                experts=experts, weights=torch.softmax(normal(tokens, slots), 1), dout=normal(tokens, cols).to(dtype), arrival_order=arrivals)


def in_8_bits(w):
    """Weights in 8 bits with a scale for every row."""
    scales = w.float().abs().amax(-1, keepdim=True).clamp(min=2.0 ** -126) / 448.0
    return (w.float() / scales).to(E4M3), scales


def in_4_bits(w):
    """Weights in microscaled 4 bits: experts x rows x pairs, and experts x rows x blocks of scales.  Rows are multiples of 32 elements."""
    n, rows, cols = w.shape
    q, scales = torch.empty(n, rows, cols // 2, dtype=torch.uint8, device=w.device), torch.empty(n, rows, -(-cols // 128) * 4, dtype=torch.uint8, device=w.device)[..., :cols // 32]
    uccl.uccl_quantise_rows(q.view(E2M1), scales.view(E8M0), w)
    return q.view(E2M1), scales.view(E8M0)


def main():
    given = inputs(tokens=512, slots=8, cols=7168, hidden=2048, n_experts=32)
    up8, up_scales = in_8_bits(given["up"])
    serving = dict(given, up=up8, up_scales=up_scales)
    del serving["dout"]
    n_experts, cols = up8.shape[0], up8.shape[2]
    router = Router(torch.randn(n_experts, cols, device="cuda").mul_(cols ** -0.5).to(torch.bfloat16), torch.zeros(n_experts, device="cuda"), 8)
    common = dict(x=given["x"], norm_weight=given["norm_weight"], router=router, arrival_order=given["arrival_order"])
    (up4, up4_scales), (down4, down4_scales) = in_4_bits(given["up"]), in_4_bits(given["down"])
    for name, step in (("serve", lambda: serve(**serving)), ("serve in 4 bits", lambda: serve_in_4_bits(up=up4, up_scales=up4_scales, down=down4, down_scales=down4_scales, **common)),
                       ("train", lambda: train(**given)), ("train, routed", lambda: train_routed(up=given["up"], down=given["down"], dout=given["dout"], **common))):
        step()
        start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        for _ in range(10):
            result = step()
        stop.record()
        torch.cuda.synchronize()
        print(f"{name}: {start.elapsed_time(stop) / 10:.2f} ms a step, {tuple(result['out'].shape)} of {result['out'].dtype}")


if __name__ == "__main__":
    main()
