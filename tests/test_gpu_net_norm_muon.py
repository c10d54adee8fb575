"""A network whose blocks begin with a layer norm and go around themselves by a shortcut, and whose weights are updated with
orthogonalised momentum: the operators in a row, as a training step uses them."""
import numpy as np
import pytest
import torch

from paper_1605_04711_b200 import datagen as dg
from paper_1605_04711_b200 import nets, twn
from _gpu_util import workspace

pytestmark = pytest.mark.gpu

MUON = {"rule": "muon", "lr": 0.02, "momentum": 0.95, "weight_decay": 0.01}


def _ops(blocks=2, C=128, hidden=256, classes=16):
    H = W = 4
    ops = [("layer", nets.Layer("embed", 64, C, H=H, W=W, relu=False, src="input"))]
    src = "embed"
    for b in range(blocks):
        ops.append(("layernorm", f"n{b}", src))
        ops.append(("layer", nets.Layer(f"up{b}", C, hidden, H=H, W=W, src=f"n{b}")))
        ops.append(("layer", nets.Layer(f"down{b}", hidden, C, H=H, W=W, relu=False, residual=src, src=f"up{b}")))
        src = f"down{b}"
    ops += [("layernorm", "last", src), ("avgpool", "gap", "last"), ("layer", nets.Layer("fc", C, classes, relu=False, src="gap", out_f32=True))]
    return ops


def _net(batch=24, optimizer=MUON, train=True):
    net = nets.TernaryNet("blocks", batch, (4, 4, 64), _ops(), seed=3, train=train, optimizer=optimizer)
    for i, name in enumerate(("n0", "n1", "last")):
        net.norm[name + ".gamma"].copy_(torch.from_numpy(1 + dg.draw(5, f"g{i}", 128, "normal", 0.0, 0.2)).cuda())
        net.norm[name + ".beta"].copy_(torch.from_numpy(dg.draw(5, f"b{i}", 128, "normal", 0.0, 0.2)).cuda())
    net.set_input(dg.draw_bf16(7, "x", batch * 4 * 4 * 64, "normal"))
    return net


def _weights(net):
    """alpha * codes of every layer, in 64 bits."""
    out = {}
    for name, L in net.layers.items():
        codes = torch.empty(L.Cout, L.K, dtype=torch.int8, device="cuda")
        twn.unpack(L.extra["packed"], L.Cout, L.K, L.extra["ld"], codes)
        out[name] = codes.double() * twn.stats_to_host(L.extra["stats"])["alpha"]
    return out


def _reference(net, x, T, norm, dlogits):
    """Forward and backward in 64 bits; the gradients of the weights and of the norms' parameters."""
    T = {k: v.clone().requires_grad_() for k, v in T.items()}
    norm = {k: v.double().clone().requires_grad_() for k, v in norm.items() if k.endswith((".gamma", ".beta"))}
    act = {"input": x.double()}
    for op in net.ops:
        if op[0] == "layer":
            L = op[1]
            y = act[L.src].reshape(*act[L.src].shape[:-1], L.K) @ T[L.name].T
            if L.residual:
                y = y + act[L.residual]
            act[L.name] = torch.relu(y) if L.relu else y
        elif op[0] == "layernorm":
            v = act[op[2]]
            v = (v - v.mean(-1, keepdim=True)) / (v.var(-1, unbiased=False, keepdim=True) + net.norm_eps).sqrt()
            act[op[1]] = v * norm[op[1] + ".gamma"] + norm[op[1] + ".beta"]
        else:
            act[op[1]] = act[op[2]].mean((1, 2), keepdim=True)
    y = act[net.ops[-1][1].name]
    (y * dlogits.double().view(y.shape)).sum().backward()
    return y.detach(), {k: v.grad for k, v in T.items()}, {k: v.grad for k, v in norm.items()}


def _near(a, b, bar):
    assert float((a.double() - b).norm()) <= bar * float(b.norm())


def test_a_step_is_that_of_64_bits():
    """Every activation and every gradient on the way is rounded to bf16, 2^-8 of its value at most; the longest way has eight of
    them forward and ten back, in which a norm (by 1 / deviation of what it got rounded) repeats one."""
    net = _net(optimizer=None)
    dlogits = torch.from_numpy(dg.draw(9, "dl", 24 * 16, "normal")).cuda().view(24, 16).to(torch.bfloat16)
    net.train_step(dlogits)
    torch.cuda.synchronize()
    net.check_status()
    y, dT, dn = _reference(net, net.act["input"], _weights(net), net.norm, dlogits)
    _near(net.act["fc"], y, 10 * 2.0 ** -8)
    for name, L in net.layers.items():
        _near(L.extra["dW"], dT[name], 22 * 2.0 ** -8)
    for name in ("n0", "n1", "last"):
        for k in ("gamma", "beta"):
            _near(net.norm[f"{name}.d{k}"], dn[f"{name}.{k}"], 22 * 2.0 ** -8)


def test_a_block_around_the_input():
    """The shortcut of the first block leaves a gradient at the input, which nobody asks for."""
    H = W = 4
    ops = [("layernorm", "n0", "input"), ("layer", nets.Layer("up", 64, 128, H=H, W=W, src="n0")),
           ("layer", nets.Layer("down", 128, 64, H=H, W=W, relu=False, residual="input", src="up")),
           ("layernorm", "last", "down"), ("avgpool", "gap", "last"), ("layer", nets.Layer("fc", 64, 16, relu=False, src="gap", out_f32=True))]
    net = nets.TernaryNet("first", 24, (H, W, 64), ops, seed=3, train=True)
    net.set_input(dg.draw_bf16(7, "x", 24 * H * W * 64, "normal"))
    dlogits = torch.from_numpy(dg.draw(9, "dl", 24 * 16, "normal")).cuda().view(24, 16).to(torch.bfloat16)
    net.train_step(dlogits)
    torch.cuda.synchronize()
    net.check_status()
    y, dT, dn = _reference(net, net.act["input"], _weights(net), net.norm, dlogits)
    # fewer roundings on the way than in the step above
    _near(net.act["fc"], y, 10 * 2.0 ** -8)
    for name, L in net.layers.items():
        _near(L.extra["dW"], dT[name], 22 * 2.0 ** -8)
    for name in ("n0", "last"):
        for k in ("gamma", "beta"):
            _near(net.norm[f"{name}.d{k}"], dn[f"{name}.{k}"], 22 * 2.0 ** -8)


def test_steps_with_muon_update_every_weight_as_the_call_alone_does():
    net = _net()
    dlogits = torch.from_numpy(dg.draw(9, "dl", 24 * 16, "normal")).cuda().view(24, 16).to(torch.bfloat16)
    layers = list(net.layers.values())
    ws = workspace(twn.muon_workspace_bytes([(L.Cout, L.K) for L in layers]))
    for _ in range(3):
        before = [(L.extra["W"].clone(), L.extra["V"].clone()) for L in layers]
        net.train_step(dlogits)
        dW = [L.extra["dW"].clone() for L in layers]
        stats = [twn.new_stats() for _ in layers]
        twn.muon_update_batch([(w, d, v, L.Cout, L.K, st) for (w, v), d, L, st in zip(before, dW, layers, stats)], 0.02, 0.95, 0.01, True, 5, 1e-7,
                              net.delta_factor, ws)
        torch.cuda.synchronize()
        for (w, v), L in zip(before, layers):
            assert torch.equal(w, L.extra["W"]) and torch.equal(v, L.extra["V"]) and bool(w.isfinite().all())
    net.check_status()


def test_a_captured_step_gives_the_bits_of_a_direct_one():
    dlogits = torch.from_numpy(dg.draw(9, "dl", 24 * 16, "normal")).cuda().view(24, 16).to(torch.bfloat16)
    direct, graphed = _net(), _net()
    for _ in range(4):
        direct.train_step(dlogits)
    graphed.train_step(dlogits)              # the second step has its thresholds from the first
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.train_step(dlogits)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(direct.layers.values(), graphed.layers.values()):
        assert torch.equal(a.extra["W"], b.extra["W"]) and torch.equal(a.extra["packed"], b.extra["packed"])


@pytest.mark.parametrize("key", ["gamma", "beta", "mean", "rstd", "dgamma", "dbeta", "ws"])
def test_a_norm_s_buffer_may_be_replaced_between_passes(key):
    dlogits = torch.from_numpy(dg.draw(9, "dl", 24 * 16, "normal")).cuda().view(24, 16).to(torch.bfloat16)

    def results(net):
        net.train_step(dlogits)
        torch.cuda.synchronize()
        return [net.act["fc"].clone()] + [L.extra["dW"].clone() for L in net.layers.values()] + [net.norm[f"{n}.d{k}"].clone()
                                                                                                 for n in ("n0", "n1", "last") for k in ("gamma", "beta")]

    net = _net(optimizer=None)
    want = results(net)
    old = net.norm["n1." + key]
    net.norm["n1." + key] = old.clone()
    old.view(torch.uint8).fill_(255)
    for a, b in zip(want, results(net)):
        assert torch.equal(a, b)
    assert bool((old.view(torch.uint8) == 255).all())


def test_inference_and_an_unknown_rule():
    a, b = _net(train=False, optimizer=None), _net(train=True, optimizer=None)
    for net in (a, b):
        net.ternarize_all()
        net.forward()
    torch.cuda.synchronize()
    # the training pass sums in order, inference as the batch suggests: a rounding of bf16 on every activation
    _near(a.act["fc"], b.act["fc"].double(), 10 * 2.0 ** -8)
    with pytest.raises(ValueError):
        _net(optimizer={"rule": "other", "lr": 0.1, "momentum": 0.9, "weight_decay": 0.0})


def test_a_net_of_images_takes_the_rule():
    net = nets.resnet18(2, image=64, classes=40, optimizer=MUON)
    net.set_input(dg.draw_bf16(1, "img", 2 * 64 * 64 * 3, "normal"))
    dlogits = torch.from_numpy(dg.draw(1, "dl", 2 * 40, "normal")).cuda().view(2, 40).to(torch.bfloat16)
    before = {n: L.extra["W"].clone() for n, L in net.layers.items()}
    for _ in range(2):
        net.train_step(dlogits)
    torch.cuda.synchronize()
    net.check_status()
    for n, L in net.layers.items():
        step = (L.extra["W"] - before[n]).double()
        # two steps of 0.02 s O and a decay of 2e-4: O's singular values are at most 1.21
        bar = 2 * 0.02 * max(1.0, L.Cout / L.K) ** 0.5 * 1.25 * min(L.Cout, L.K) ** 0.5 + 5e-4 * float(before[n].double().norm())
        assert 0.0 < float(step.norm()) <= bar
