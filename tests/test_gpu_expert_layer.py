"""The example of an expert-parallel layer, stage by stage against formulas in 64 bits that go by the slots' experts, not by the plan.

Every stage is computed from the stage before it as that was rounded, so a result may be off by half a step of its type, and by (n + 8) 2^-24 of the sum of
its n terms' magnitudes.
"""
import os
import re
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def layer(gpu_lib):
    import expert_layer
    return expert_layer


def close(got, want, magnitude, n, what):
    info = torch.finfo(got.dtype)
    bound = want.abs() * (info.eps / 2) + magnitude * ((n + 8) * 2.0 ** -24 * (1 + info.eps)) + info.smallest_normal * info.eps
    over = (got.double() - want).abs() - bound
    assert bool((over <= 0).all()), f"{what}: {int((over > 0).sum())} of {over.numel()} off, by {float(over.max())} at most"


def slots_of(experts):
    """Token, slot and expert of every slot that has one."""
    t, j = torch.nonzero(experts >= 0, as_tuple=True)
    return t, j, experts[t, j]


def product_of_rows(a, w):
    """a[i] . w[i]^T by rows, with the sum of the terms' magnitudes."""
    return torch.bmm(w, a[..., None])[..., 0], torch.bmm(w.abs(), a.abs()[..., None])[..., 0]


def check_silu(a, u):
    """Between the products: an exponential, whose argument is off by its own size, a sum and a quotient."""
    want = u.double() * torch.sigmoid(u.double())
    close(a, want, want.abs() * (1 + u.double().abs()), 8, "a")


CASES = [(5, 2, 64, 32, 3, 0.125), (33, 4, 200, 72, 6, 0.0), (70, 8, 130, 44, 12, 0.5), (4, 3, 64, 16, 4, 1.0)]   # tokens, slots, cols, hidden, experts, missing


@pytest.mark.parametrize("tokens,slots,cols,hidden,n_experts,missing", CASES)
def test_training_step(layer, tokens, slots, cols, hidden, n_experts, missing):
    dtype = torch.float16
    cols, hidden = cols // 8 * 8, hidden // 8 * 8           # contiguous rows start on 16-byte boundaries
    given = layer.inputs(tokens, slots, cols, hidden, n_experts, dtype, seed=tokens, missing=missing)
    got = layer.train(**given)
    d = lambda v: v.double()  # noqa: E731
    x, nw, up, down, dout, weights = (d(given[k]) for k in ("x", "norm_weight", "up", "down", "dout", "weights"))
    t, j, e = slots_of(given["experts"])
    row = got["pos"][t, j].long()                           # where the slot's row is
    assert len(set(row.tolist())) == len(row) and bool((got["pos"][given["experts"] < 0] == -1).all())
    n = x * d(got["rstd"])[:, None]
    close(got["rstd"][:, None], 1 / torch.sqrt((x * x).mean(1, keepdim=True) + layer.EPS), d(got["rstd"])[:, None], cols, "rstd")
    close(got["y"], n * nw, (n * nw).abs(), 4, "y")
    want, mag = product_of_rows(d(got["y"])[t], up[e])
    close(got["u"][row], want, mag, cols, "u")
    check_silu(got["a"][row], got["u"][row])
    want, mag = product_of_rows(d(got["a"])[row], down[e])
    close(got["z"][row], want, mag, hidden, "z")
    terms = weights[t, j, None] * d(got["z"])[row]
    total = lambda v, over, like: torch.zeros_like(like).index_add_(0, over, v)  # noqa: E731
    close(got["out"], x + total(terms, t, x), x.abs() + total(terms.abs(), t, x), slots, "out")

    want = weights[t, j, None] * dout[t]
    close(got["dz"][row], want, want.abs(), 1, "dz")
    dot = dout[t] * d(got["z"])[row]
    close(got["dweights"][t, j], dot.sum(1), dot.abs().sum(1), cols, "dweights")
    assert bool((got["dweights"][given["experts"] < 0] == 0).all())
    want, mag = product_of_rows(d(got["dz"])[row], down[e].transpose(1, 2).contiguous())
    close(got["da"][row], want, mag, cols, "da")
    u, s = d(got["u"])[row], torch.sigmoid(d(got["u"])[row])
    want = d(got["da"])[row] * s * (1 + u * (1 - s))
    close(got["du"][row], want, d(got["da"])[row].abs() * (1 + u.abs()), 8, "du")
    want, mag = product_of_rows(d(got["du"])[row], up[e].transpose(1, 2).contiguous())
    close(got["dr"][row], want, mag, hidden, "dr")
    for name, left, right, like in (("ddown", d(got["dz"])[row], d(got["a"])[row], down), ("dup", d(got["du"])[row], d(got["y"])[t], up)):
        outer = left[:, :, None] * right[:, None]
        close(got[name], total(outer, e, like), total(outer.abs(), e, like), len(row), name)
    dr = d(got["dr"])[row]
    close(got["dy"], total(dr, t, x), total(dr.abs(), t, x), slots, "dy")
    dy, r = d(got["dy"]), d(got["rstd"])[:, None]
    g = dy * nw
    close(got["dnorm"], (dy * n).sum(0), (dy * n).abs().sum(0), tokens, "dnorm")
    mag = dout.abs() + r * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True) * (cols + 8) / 8)
    close(got["dx"], dout + r * (g - n * (g * n).mean(1, keepdim=True)), mag, 8, "dx")


def test_gradients_are_the_derivative_of_the_layer(layer):
    """Of the whole layer: the change of sum(out dout) along a direction, from the layer in 64 bits, against the gradients."""
    given = layer.inputs(24, 3, 64, 32, 5, torch.bfloat16, seed=9)
    got = layer.train(**given)
    names = {"x": "dx", "norm_weight": "dnorm", "up": "dup", "down": "ddown", "weights": "dweights"}
    t, j, e = slots_of(given["experts"])

    def value(p):
        y = p["x"] / torch.sqrt((p["x"] ** 2).mean(1, keepdim=True) + layer.EPS) * p["norm_weight"]
        u = torch.bmm(p["up"][e], y[t][..., None])[..., 0]
        z = torch.bmm(p["down"][e], (u * torch.sigmoid(u))[..., None])[..., 0]
        return float(((p["x"].index_add(0, t, p["weights"][t, j, None] * z)) * given["dout"].double()).sum())
    at = {k: given[k].double() for k in names}
    for k, grad in names.items():
        # along the gradient itself, where the change is the square of its length; on the way to it some ten values were rounded to
        # 8 bits, each off by 2^-8 of itself at most
        way = got[grad].double()
        way = way / way.norm()
        step = 1e-5
        there, back = dict(at, **{k: at[k] + step * way}), dict(at, **{k: at[k] - step * way})
        slope = (value(there) - value(back)) / (2 * step)
        assert abs(slope - float((got[grad].double() * way).sum())) <= 10 * 2.0 ** -8 * abs(slope), k


@pytest.mark.parametrize("tokens,slots,cols,hidden,n_experts,missing", CASES + [(1, 2, 256, 64, 32, 0.0)])
def test_serving_step(layer, tokens, slots, cols, hidden, n_experts, missing):
    dtype = torch.bfloat16
    cols, hidden = -(-cols // 16) * 16, -(-hidden // 16) * 16
    given = layer.inputs(tokens, slots, cols, hidden, n_experts, dtype, seed=tokens, missing=missing)
    del given["dout"]
    given["up"], given["up_scales"] = layer.in_8_bits(given["up"])
    got = layer.serve(**given)
    x, nw, down, weights = (given[k].double() for k in ("x", "norm_weight", "down", "weights"))
    up = given["up"].double() * given["up_scales"].double()
    t, j, e = slots_of(given["experts"])
    row = got["pos"][t, j].long()
    y = x / torch.sqrt((x * x).mean(1, keepdim=True) + layer.EPS) * nw
    scale = y.abs().amax(1, keepdim=True) / 448.0
    close(got["scales"], scale, scale, cols, "scales")
    sent = got["y"].double() * got["scales"].double()
    # half a step of the element's own size or of the subnormals, and what binary32 was off before
    assert bool(((sent - y).abs() <= torch.maximum(y.abs() * 2.0 ** -4, scale * 2.0 ** -10) * (1 + 1e-6) + y.abs() * (cols + 32) * 2.0 ** -24).all())
    want, mag = product_of_rows(sent[t], up[e])
    close(got["u"][row], want, mag, cols + 4, "u")
    check_silu(got["a"][row], got["u"][row])
    want, mag = product_of_rows(got["a"][row].double(), down[e])
    close(got["z"][row], want, mag, hidden, "z")
    terms = weights[t, j, None] * got["z"][row].double()
    total = lambda v: torch.zeros_like(x).index_add_(0, t, v)  # noqa: E731
    close(got["out"], x + total(terms), x.abs() + total(terms.abs()), slots, "out")


def test_what_arrives_is_what_was_sent(layer):
    """Whatever the order, with chunks that come twice and a last chunk that is short."""
    g = torch.Generator(device="cuda").manual_seed(2)
    rows = torch.randint(0, 256, (37, 96), dtype=torch.uint8, device="cuda", generator=g)
    for chunk_rows, n in ((1, 37), (4, 10), (64, 1)):
        order = torch.randperm(n).tolist() + [0, n - 1]
        assert torch.equal(layer.dispatch(rows, order, chunk_rows), rows)


def test_readme_example_of_a_product_runs(gpu_lib):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    code = re.findall(r"```python\n(.*?)```", text, re.S)[1]
    ns = {"torch": torch, "uccl": gpu_lib}
    exec(compile(code, "README.md", "exec"), ns)
    first = ns["first"].tolist()
    for e, (b, f) in enumerate(zip(first, first[1:])):
        x, w = ns["x"][b:f].double(), ns["w"][e].double()
        close(ns["y"][b:f], x @ w.T, x.abs() @ w.abs().T, ns["cols"], f"expert {e}")
