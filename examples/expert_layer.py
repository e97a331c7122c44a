"""An expert-parallel layer on one GPU: the row operators around a dispatch through the chunk path.

    out[t] = x[t] + sum over the token's experts e of weight[t, e] down_e(silu(up_e(norm(x[t]))))

`dispatch` is what lies between a sender's rows and a receiver's: staged chunks, arrivals in any order and some of them twice, deduplication
and placement.  `serve` sends rows of 8 bits with their scales and multiplies them as they arrived; `train` sends 16-bit rows and
returns the gradients too.  Which row goes where is planned on the GPU, and nothing here reads it back; the records of what arrived come from
the host, as a receiver's control path has them.

    python examples/expert_layer.py
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2504_17307_amd as uccl  # noqa: E402
from synth.layout import DESC, NO_FORWARD, bitmap_words  # noqa: E402

E4M3 = torch.float8_e4m3fn
EPS = 1e-6


def plan(experts, n_experts):
    """``experts``: tokens x slots, the expert of every slot, -1: none.  Returns what the operators go by: the token of every
    row in order of experts, the experts' first rows, and every slot's row (-1: none).  Slots without an expert come last, behind
    the last group: their rows are nobody's."""
    flat = experts.reshape(-1)
    key = torch.where(flat < 0, n_experts, flat)
    order = torch.argsort(key, stable=True)
    offsets = torch.searchsorted(key[order], torch.arange(n_experts + 1, device=key.device, dtype=key.dtype)).to(torch.int32)
    pos = torch.empty_like(flat, dtype=torch.int32)
    pos[order] = torch.arange(len(flat), device=flat.device, dtype=torch.int32)
    pos = torch.where(flat < 0, -1, pos).view(experts.shape)
    return (order // experts.shape[1]).to(torch.int32), offsets, pos


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


def train(x, norm_weight, up, down, experts, weights, dout, arrival_order):
    """The layer's output and, for the gradient ``dout`` of it, the gradients of all that is learned and of x; all in 16 bits."""
    (tokens, cols), (n_experts, hidden, _) = x.shape, up.shape
    like = dict(dtype=x.dtype, device=x.device)
    f32 = dict(dtype=torch.float32, device=x.device)
    index, offsets, pos = plan(experts, n_experts)
    rows = index.numel()
    y, rstd = torch.empty_like(x), torch.empty(tokens, **f32)
    uccl.uccl_norm_rows(y, x, norm_weight, EPS, rstd=rstd)
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
    uccl.uccl_combine_rows(dy, dr, pos)
    dx, dnorm = torch.empty_like(x), torch.empty(cols, **f32)
    scratch = torch.empty(uccl.uccl_norm_rows_scratch(tokens, cols), dtype=torch.uint8, device=x.device)
    uccl.uccl_norm_rows_grad(dx, dnorm, dy, x, rstd, norm_weight, scratch, dh=dout)
    return {"y": y, "rstd": rstd, "u": u, "a": a, "z": z, "pos": pos, "out": out, "dz": dz, "dweights": dweights, "da": da, "ddown": ddown,
            "du": du, "dr": dr, "dup": dup, "dy": dy, "dx": dx, "dnorm": dnorm}


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


def main():
    given = inputs(tokens=512, slots=8, cols=7168, hidden=2048, n_experts=32)
    up8, up_scales = in_8_bits(given["up"])
    serving = dict(given, up=up8, up_scales=up_scales)
    del serving["dout"]
    for name, step in (("serve", lambda: serve(**serving)), ("train", lambda: train(**given))):
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
