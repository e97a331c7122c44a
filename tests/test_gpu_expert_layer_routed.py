"""The example's layer with a router: served in microscaled 4 bits stage by stage, trained with balance loss and clipping, against formulas in 64 bits.

Tolerances as in tests/test_gpu_expert_layer.py: every stage is computed from the stage before it as that was rounded.
"""
import os
import re
import sys

import pytest
import torch

from test_gpu_expert_layer import check_silu, close, product_of_rows, slots_of
from test_gpu_experts import choice, decode, quantise_reference, weights_of

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def layer(gpu_lib):
    import expert_layer
    return expert_layer


def router_of(layer, given, slots, seed=1, coef=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, _, cols = given["up"].shape
    return layer.Router((torch.randn(n, cols, device="cuda", generator=g) * 2 * cols ** -0.5).to(given["x"].dtype), torch.randn(n, device="cuda", generator=g) * 0.1, slots, coef)


CASES = [(5, 2, 64, 32, 3), (33, 4, 192, 96, 6), (70, 8, 128, 64, 12), (1, 2, 256, 64, 32), (300, 6, 512, 160, 60)]   # tokens, slots, cols, hidden, experts


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,slots,cols,hidden,n_experts", CASES)
def test_serving_step_in_4_bits(layer, tokens, slots, cols, hidden, n_experts, dtype):
    given = layer.inputs(tokens, slots, cols, hidden, n_experts, dtype, seed=tokens)
    router = router_of(layer, given, slots)
    (up, us), (down, ds) = layer.in_4_bits(given["up"]), layer.in_4_bits(given["down"])
    got = layer.serve_in_4_bits(given["x"], given["norm_weight"], router, up, us, down, ds, given["arrival_order"])
    x, nw = given["x"].double(), given["norm_weight"].double()
    n = x / torch.sqrt((x * x).mean(1, keepdim=True) + layer.EPS) * nw
    close(got["n"], n, n.abs(), cols / 2 + 10, "n")
    rows, w = got["n"].double(), router.weight.double()
    close(router.scores, rows @ w.T, rows.abs() @ w.abs().T, cols, "scores")
    assert torch.equal(got["experts"].long(), choice(router.scores, router.bias, slots))
    want = weights_of(router.scores, got["experts"].long(), True, 1.0)
    close(got["weights"], want, want * (2 + float(router.scores.amax() - router.scores.amin())), n_experts + 8, "weights")
    number, byte = quantise_reference(got["n"])
    y = decode(got["y"], got["scales"], cols)
    assert torch.equal(got["scales"].view(torch.uint8).cpu().long(), byte)
    t, j, e = slots_of(got["experts"])
    row = got["pos"][t, j].long()
    assert sorted(row.tolist()) == list(range(tokens * slots))
    uw, dw = decode(up.flatten(0, 1), us.flatten(0, 1), cols).view(n_experts, hidden, cols), decode(down.flatten(0, 1), ds.flatten(0, 1), hidden).view(n_experts, cols, hidden)
    want, mag = product_of_rows(y[t], uw[e])
    close(got["u"][row], want, mag, cols, "u")
    check_silu(got["a"][row], got["u"][row])
    want, mag = product_of_rows(got["a"][row].double(), dw[e])
    close(got["z"][row], want, mag, hidden, "z")
    terms = got["weights"][t, j, None].double() * got["z"][row].double()
    total = lambda v: torch.zeros_like(x).index_add_(0, t, v)  # noqa: E731
    close(got["out"], x + total(terms), x.abs() + total(terms.abs()), slots, "out")


def test_gradients_of_the_routed_layer_are_its_derivative(layer):
    """Of sum(out dout) and the balance loss together, with the choice held, along each gradient: the change is the square of its length.  On the way some twelve values
    were rounded to 11 bits, each off by 2^-11 of itself at most, and gradients add up several of them."""
    given = layer.inputs(40, 3, 64, 32, 6, torch.float16, seed=9)
    router = router_of(layer, given, 3)
    got = layer.train_routed(given["x"], given["norm_weight"], router, given["up"], given["down"], given["dout"], given["arrival_order"], most=0.5)
    t, j, e = slots_of(got_experts := router.experts)
    tokens, n = given["x"].shape[0], router.weight.shape[0]

    def value(p):
        y = p["x"] / torch.sqrt((p["x"] ** 2).mean(1, keepdim=True) + layer.EPS) * p["norm_weight"]
        probs = torch.softmax(y @ p["router"].T, 1)
        w = probs.gather(1, got_experts.long())
        w = w / w.sum(1, keepdim=True)
        u = torch.bmm(p["up"][e], y[t][..., None])[..., 0]
        z = torch.bmm(p["down"][e], (u * torch.sigmoid(u))[..., None])[..., 0]
        balance = router.coef * n / (router.slots * tokens ** 2) * (router.counts.double() * probs.sum(0)).sum()
        return float((p["x"].index_add(0, t, w[t, j, None] * z) * given["dout"].double()).sum() + balance)
    at = {"x": given["x"].double(), "norm_weight": given["norm_weight"].double(), "router": router.weight.double(), "up": given["up"].double(), "down": given["down"].double()}
    names = {"x": "dx", "norm_weight": "dnorm", "router": "drouter", "up": "dup", "down": "ddown"}
    for k, grad in names.items():
        way = got[grad].double()
        way = way / way.norm()
        step = 1e-5
        there, back = dict(at, **{k: at[k] + step * way}), dict(at, **{k: at[k] - step * way})
        slope = (value(there) - value(back)) / (2 * step)
        assert abs(slope - float((got[grad].double() * way).sum())) <= 12 * 2.0 ** -11 * abs(slope), k
    balance = router.coef * n / (3 * tokens ** 2) * (router.counts.double() * torch.softmax(router.scores.double(), 1).sum(0)).sum()
    assert abs(got["loss"].item() - float(balance)) <= 1e-5 * float(balance) and int(router.counts.sum()) == tokens * 3
    grads = [got[k] for k in ("dnorm", "drouter", "dup", "ddown")]
    norm = torch.sqrt(sum((g.double() ** 2).sum() for g in grads))
    assert abs(got["norm"].item() - float(norm)) <= 2.0 ** -24 * float(norm)
    by = torch.tensor(0.5, device="cuda") / got["norm"]
    assert all(torch.equal(c, g * by) for c, g in zip(got["clipped"].values(), grads))
    assert abs(float(torch.sqrt(sum((g.double() ** 2).sum() for g in got["clipped"].values()))) - 0.5) <= 1e-6


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", [0.0, 1e-6, 1.0, 300.0])
def test_gradient_of_the_router_has_the_balance_loss_of_many_tokens(layer, dtype, size):
    """Whose part of a score is about 1e-7, beside gradients of the weights of any size.  Each score's gradient is rounded to bf16, half of finfo.eps of itself (2^-8), or to two f16: the first is off
    by 2^-11 of itself at most, and the second by 2^-11 of that, or, where it is subnormal, by half of 2^-24 by 2^-24 where the greatest is 1/2 or more: 2^-48 of it.
    Products as elsewhere."""
    import paper_2504_17307_amd as uccl
    tokens, cols, n, slots = 4096, 64, 32, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    given = {"up": torch.empty(n, 1, cols), "x": torch.empty(1, cols, dtype=dtype)}
    router, y = router_of(layer, given, slots, coef=0.01), torch.randn(tokens, cols, device="cuda", generator=g).to(dtype)
    _, weights = router.forward(y)
    dweights = size * torch.randn(tokens, slots, device="cuda", generator=g)
    dy = router.backward(dweights)
    dscores = torch.empty(tokens, n, device="cuda")
    uccl.uccl_route_rows_grad(dscores, router.scores, router.experts, dweights, dsums=router.dsums, normalise=True)
    d, yd, wd = dscores.double(), y.double(), router.weight.double()
    off = d.abs() * 2.0 ** -8 if dtype == torch.bfloat16 else d.abs() * 2.0 ** -22 + d.abs().amax() * 2.0 ** -48
    want, mag = d.T @ yd, d.abs().T @ yd.abs()
    sums = (tokens + 8) * 2.0 ** -24
    assert bool(((router.dweight.double() - want).abs() <= off.T @ yd.abs() + mag * sums).all())
    assert bool((router.dweight != 0).all())
    want, mag = d @ wd, d.abs() @ wd.abs()
    info = torch.finfo(dtype)
    assert bool(((dy.double() - want).abs() <= want.abs() * info.eps / 2 + info.smallest_normal * info.eps + off @ wd.abs() * (1 + info.eps) + mag * (n + 8) * 2.0 ** -24).all())


def test_readme_example_of_routing_and_4_bits_runs(gpu_lib):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    ns = {"torch": torch, "uccl": gpu_lib}
    for code in re.findall(r"```python\n(.*?)```", text, re.S)[1:]:
        exec(compile(code, "README.md", "exec"), ns)
    chosen = choice(ns["scores"], None, 2)
    assert torch.equal(ns["chosen"].long(), chosen)
    assert bool(((ns["weight"].sum(1) - 1).abs() <= 4 * torch.finfo(torch.float32).eps).all())
    first = ns["first"].tolist()
    for e, (b, f) in enumerate(zip(first, first[1:])):
        take = ns["index"][b:f].long()
        assert torch.equal(take, (chosen == e).nonzero()[:, 0])
        x, w = ns["x"][take].double(), decode(ns["w4"][e], ns["s4"][e], ns["cols"])
        close(ns["y"][b:f], x @ w.T, x.abs() @ w.abs().T, ns["cols"], f"expert {e}")
