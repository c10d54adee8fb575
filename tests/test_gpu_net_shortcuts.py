"""Gradients of networks whose blocks read their input twice: through a layer norm or a pooling, and through a projection
shortcut that is added behind the block.  Against a 64-bit pass over the same ternary weights.

Every activation and every gradient on the way is rounded to bf16, 2^-8 of its value at most, in a dozen places forward and a dozen
back; the bars are those of the networks with identity shortcuts (10 forward, 22 for a gradient), which have longer ways.
"""
import pytest
import torch

from paper_1605_04711_b200 import datagen as dg
from paper_1605_04711_b200 import nets
from test_gpu_net_norm_muon import _near, _weights

pytestmark = pytest.mark.gpu

C, B = 64, 24


def _layer(name, src, cin, cout, H=4, **kw):
    return ("layer", nets.Layer(name, cin, cout, H=H, W=H, src=src, **{"relu": False, **kw}))


def _tail(src, c=C, H=4):
    return [("layernorm", "last", src), ("avgpool", "gap", "last"), _layer("fc", "gap", c, 16, H=1, out_f32=True)]


def _norm_block(order):
    """x -> layer norm -> up -> down, with proj(x) added; the projection before or behind the branch in the list."""
    branch = [("layernorm", "n", "x"), _layer("up", "n", C, 128, relu=True)]
    proj = [_layer("proj", "x", C, C)]
    return [_layer("x0", "input", 64, C, relu=True), _layer("x", "x0", C, C), *(proj + branch if order else branch + proj),
            _layer("down", "up", 128, C, residual="proj"), *_tail("down")]


def _pool_block():
    return [_layer("x0", "input", 64, C, relu=True), _layer("x", "x0", C, C, relu=True), ("maxpool", "p", "x", 2, 2, 0), _layer("up", "p", C, 128, H=2, relu=True),
            _layer("proj", "x", C, C, stride=2), _layer("down", "up", 128, C, H=2, residual="proj"), *_tail("down")]


def _two_projections():
    """Two blocks read x, each with a projection of x of its own."""
    return [_layer("x0", "input", 64, C, relu=True), _layer("x", "x0", C, C), ("layernorm", "n", "x"), _layer("up", "n", C, 128, relu=True), _layer("p1", "x", C, C),
            _layer("down", "up", 128, C, residual="p1"), _layer("up2", "down", C, 128, relu=True), _layer("p2", "x", C, C),
            _layer("down2", "up2", 128, C, residual="p2"), *_tail("down2")]


def _projection_alone():
    """The projection is all that reads x; the branch comes from further up."""
    return [_layer("x0", "input", 64, C, relu=True), _layer("x", "x0", C, C), ("layernorm", "n", "x0"), _layer("up", "n", C, 128, relu=True), _layer("proj", "x", C, C),
            _layer("down", "up", 128, C, residual="proj"), *_tail("down")]


def _layers_before():
    """The list of a usual block, its projection before its first layer."""
    return [_layer("x0", "input", 64, C, relu=True), _layer("x", "x0", C, C, relu=True), _layer("proj", "x", C, C), _layer("up", "x", C, 128, relu=True),
            _layer("down", "up", 128, C, residual="proj"), *_tail("down")]


def _wide_source():
    """A norm of a layer whose output is kept in fp32."""
    return [_layer("x0", "input", 64, C, relu=True), _layer("x", "x0", C, C, out_f32=True), ("layernorm", "n", "x"), _layer("up", "n", C, C, relu=True), *_tail("up")]


def _flat_wide_source():
    return [_layer("x0", "input", 64, C, relu=True), _layer("x", "x0", C, 8, out_f32=True), ("flatten", "f", "x"), ("layernorm", "n", "f"),
            _layer("fc", "n", 128, 16, H=1, out_f32=True)]


NETS = {"norm": _norm_block(False), "norm, projection first": _norm_block(True), "pool": _pool_block(), "two projections": _two_projections(),
        "projection alone": _projection_alone(), "layers, projection first": _layers_before(), "fp32 source": _wide_source(), "fp32 source, flat": _flat_wide_source()}


def reference(net, x, T, norm, dlogits):
    T = {k: v.clone().requires_grad_() for k, v in T.items()}
    norm = {k: v.double().clone().requires_grad_() for k, v in norm.items() if k.endswith((".gamma", ".beta"))}
    act = {"input": x.double()}
    for op in net.ops:
        if op[0] == "layer":
            L = op[1]
            y = act[L.src][:, ::L.stride, ::L.stride] @ T[L.name].T
            if L.residual:
                y = y + act[L.residual]
            act[L.name] = torch.relu(y) if L.relu else y
        elif op[0] == "layernorm":
            v = act[op[2]]
            v = (v - v.mean(-1, keepdim=True)) / (v.var(-1, unbiased=False, keepdim=True) + net.norm_eps).sqrt()
            act[op[1]] = v * norm[op[1] + ".gamma"] + norm[op[1] + ".beta"]
        elif op[0] == "maxpool":
            # the largest of what the network itself compared: its rounding decides which one it is
            v, n = act[op[2]], net.act[op[2]].double()
            split = lambda t: t.unfold(1, 2, 2).unfold(2, 2, 2).flatten(4)  # noqa: E731
            act[op[1]] = split(v).gather(4, split(n).argmax(4, keepdim=True)).squeeze(4)
        elif op[0] == "flatten":
            act[op[1]] = act[op[2]].flatten(1)[:, None, None]
        else:
            act[op[1]] = act[op[2]].mean((1, 2), keepdim=True)
    y = act[net.ops[-1][1].name]
    (y * dlogits.double().view(y.shape)).sum().backward()
    return y.detach(), {k: v.grad for k, v in T.items()}, {k: v.grad for k, v in norm.items()}


@pytest.mark.parametrize("which", list(NETS))
def test_every_gradient_is_that_of_64_bits(which):
    net = nets.TernaryNet("shortcuts", B, (4, 4, 64), NETS[which], seed=3, train=True)
    norms = [op[1] for op in net.ops if op[0] == "layernorm"]
    for i, name in enumerate(norms):
        net.norm[name + ".gamma"].copy_(torch.from_numpy(1 + dg.draw(5, f"g{i}", net.norm[name + ".gamma"].numel(), "normal", 0.0, 0.2)).cuda())
    net.set_input(dg.draw_bf16(7, "x", B * 16 * 64, "normal"))
    dlogits = torch.from_numpy(dg.draw(9, "dl", B * 16, "normal")).cuda().view(B, 16).to(torch.bfloat16)
    for _ in range(2):
        net.train_step(dlogits)
    torch.cuda.synchronize()
    net.check_status()
    y, dT, dn = reference(net, net.act["input"], _weights(net), net.norm, dlogits)
    _near(net.act["fc"], y, 10 * 2.0 ** -8)
    for name, L in net.layers.items():
        _near(L.extra["dW"], dT[name], 22 * 2.0 ** -8)
    for name in norms:
        for k in ("gamma", "beta"):
            _near(net.norm[f"{name}.d{k}"], dn[f"{name}.{k}"], 22 * 2.0 ** -8)


def test_a_relu_of_an_fp32_output_is_not_trained_through():
    """The gate of a ReLU is read from bf16."""
    ops = [_layer("x", "input", 64, C, out_f32=True, relu=True), ("layernorm", "n", "x"), *_tail("n")]
    flat = [_layer("x", "input", 64, 8, out_f32=True, relu=True), ("flatten", "f", "x"), ("layernorm", "n", "f"), _layer("fc", "n", 128, 16, H=1, out_f32=True)]
    for o in (ops, flat):
        with pytest.raises(NotImplementedError):
            nets.TernaryNet("gate", B, (4, 4, 64), o, train=True)
        nets.TernaryNet("gate", B, (4, 4, 64), o)


@pytest.mark.parametrize("rule", ["sgd", "muon"])
def test_the_norms_parameters_are_the_caller_s(rule):
    """An update moves the weights; gamma and beta stay, with their gradients beside them."""
    net = nets.TernaryNet("kept", B, (4, 4, 64), _norm_block(False), seed=3, train=True, optimizer={"rule": rule, "lr": 0.02, "momentum": 0.9, "weight_decay": 0.0})
    net.set_input(dg.draw_bf16(7, "x", B * 16 * 64, "normal"))
    dlogits = torch.from_numpy(dg.draw(9, "dl", B * 16, "normal")).cuda().view(B, 16).to(torch.bfloat16)
    net.train_step(dlogits)
    torch.cuda.synchronize()
    for name in ("n", "last"):
        assert bool((net.norm[name + ".gamma"] == 1).all()) and bool((net.norm[name + ".beta"] == 0).all())
        assert float(net.norm[name + ".dgamma"].abs().max()) > 0 and float(net.norm[name + ".dbeta"].abs().max()) > 0
