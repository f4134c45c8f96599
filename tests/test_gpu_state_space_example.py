"""The state-space layers together, as the example uses them: gradients of a whole layer, packed against alone, prompts and steps."""
import importlib.util
import os

import pytest
import torch

import layer_util as L
import state_space_util as S

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "packed_state_space.py")
    spec = importlib.util.spec_from_file_location("packed_state_space", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("video", [False, True])
def test_the_example_runs_and_every_parameter_has_a_gradient(video):
    model, losses, apart = example().main(steps=3, video=video, quiet=True)
    assert all(map(lambda x: x == x and x < float("inf"), losses))
    for name, p in model.named_parameters():
        assert p.grad is not None and bool(torch.isfinite(p.grad).all()) and bool(p.grad.any()), name
    # a step's activations are rounded where the whole sequence's are; differences in 32 bits turn a few of these roundings (2^-8)
    assert apart is None or apart < 4 * 2.0 ** -8


def chain(e, x, dt, z, b, c, pos, w):
    """norm, convolution and scan in 32 bits through the example's functions"""
    n = e.Norm.apply(x, pos, w["norm_weight"], w["norm_bias"])
    u = e.Conv.apply(n, pos, w["conv_weight"], w["conv_bias"])
    return e.Scan.apply(u, dt, z, b, c, w["a"], w["d"], w["dt_bias"], pos)


def definition(blocks, x, dt, z, b, c, w):
    """the same in 64 bits by torch, one sequence at a time"""
    out = []
    for q, s0, s1 in S.spans(blocks):
        X = x[q, s0:s1]
        n = torch.nn.functional.layer_norm(X, X.shape[-1:], w["norm_weight"], w["norm_bias"])
        k = w["conv_weight"].shape[1]
        wide = torch.cat((torch.zeros_like(n[:1]).expand(k - 1, -1), n))
        u = torch.nn.functional.silu(sum(w["conv_weight"][:, i] * wide[i:i + n.shape[0]] for i in range(k)) + w["conv_bias"])
        delta = torch.nn.functional.softplus(dt[q, s0:s1] + w["dt_bias"])
        h, ys = torch.zeros_like(w["a"]), []
        for s in range(s1 - s0):
            h = torch.exp(delta[s][:, None] * w["a"]) * h + (delta[s] * u[s])[:, None] * b[q, s0 + s]
            ys.append((h * c[q, s0 + s]).sum(-1))
        y = (torch.stack(ys) + w["d"] * u) * torch.nn.functional.silu(z[q, s0:s1])
        out.append(y)
    return out


def test_gradients_of_the_layers_together():
    e = example()
    blocks, t, ch, n = [[40, 1, 23], [-3, 61]], 64, 24, 16
    pos = L.positions(t, blocks)
    i = S.scan_inputs(2, t, ch, n, torch.float32, 5)
    w = {"norm_weight": L.normal((ch,), torch.float32, 1, 1.0, 0.2), "norm_bias": L.normal((ch,), torch.float32, 2), "a": i["a"], "d": i["d"],
         "conv_weight": L.normal((ch, 4), torch.float32, 3), "conv_bias": L.normal((ch,), torch.float32, 4), "dt_bias": i["dt_bias"]}
    names = ("x", "dt", "z", "b", "c")
    mine = [i[k].clone().requires_grad_() for k in names]
    w32 = {k: v.clone().requires_grad_() for k, v in w.items()}
    y = chain(e, *mine, pos, w32)
    got = torch.autograd.grad(y, mine + list(w32.values()), i["dy"])
    wide = [i[k].double().requires_grad_() for k in names]
    w64 = {k: v.double().requires_grad_() for k, v in w.items()}
    ys = definition(blocks, *wide, w64)
    loss = sum((v * i["dy"][q, s0:s1].double()).sum() for v, (q, s0, s1) in zip(ys, S.spans(blocks)))
    want = torch.autograd.grad(loss, wide + list(w64.values()))
    for v, (q, s0, s1) in zip(ys, S.spans(blocks)):
        assert float((y[q, s0:s1].double() - v).detach().norm()) <= 2.0 ** -15 * float(v.detach().norm())
    # three operators in 32 bits, each within some tens of roundings of what it gets: far below 2^-13 of the whole
    for name, a, b in zip(names + tuple(w), got, want):
        assert float((a.double() - b).norm()) <= 2.0 ** -13 * float(b.norm()), name


@pytest.mark.parametrize("name", ["norm", "conv", "scan", "rotary_axes"])
def test_a_second_derivative_is_refused(name):
    e = example()
    pos = L.positions(40, [[25, 15]])
    i = S.scan_inputs(1, 40, 16, 4, torch.float32, 2)
    w = [torch.ones(16, device=L.DEV), torch.zeros(16, device=L.DEV)]
    x = i["x"].clone().requires_grad_()
    heads = L.normal((1, 40, 2, 32), torch.float32, 3).requires_grad_()
    run, of = {"norm": (lambda: e.Norm.apply(x, pos, *w), x), "conv": (lambda: e.Conv.apply(x, pos, torch.ones((16, 4), device=L.DEV), w[1]), x),
               "scan": (lambda: e.Scan.apply(x, i["dt"], i["z"], i["b"], i["c"], i["a"], i["d"], i["dt_bias"], pos), x),
               "rotary_axes": (lambda: e.RotaryAxes.apply(heads, pos, torch.stack((pos, pos)), torch.zeros(16, dtype=torch.int32, device=L.DEV),
                                                          torch.ones(16, device=L.DEV)), heads)}[name]
    y = run()
    first, = torch.autograd.grad(y, of, torch.ones_like(y).requires_grad_(), create_graph=True)
    assert bool(torch.isfinite(first).all())
    with pytest.raises(RuntimeError, match="once_differentiable"):
        first.square().sum().backward()


def test_a_backward_pass_is_captured_into_a_graph():
    e = example()
    blocks, t, ch, n = [[40, 24], [64]], 64, 24, 16
    pos = L.positions(t, blocks)
    i = S.scan_inputs(2, t, ch, n, torch.bfloat16, 5)
    w = {"norm_weight": torch.ones(ch, device=L.DEV), "norm_bias": torch.zeros(ch, device=L.DEV), "a": i["a"], "d": i["d"],
         "conv_weight": L.normal((ch, 4), torch.float32, 3), "conv_bias": torch.zeros(ch, device=L.DEV), "dt_bias": i["dt_bias"]}

    def run():
        leaves = [i[k].detach().requires_grad_() for k in ("x", "dt", "z", "b", "c")]
        weights = {k: v.detach().requires_grad_() for k, v in w.items()}
        y = chain(e, *leaves, pos, weights)
        return (y, *torch.autograd.grad(y, leaves + list(weights.values()), i["dy"]))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [v.clone() for v in run()]
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    g.replay()
    g.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
