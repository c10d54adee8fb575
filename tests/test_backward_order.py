"""The order of a network's backward pass: what reads an activation comes before what made it, whatever its kind, and projection
shortcuts come behind the first convolution of their block."""
import pytest

from paper_1605_04711_b200 import nets


def _layer(name, src, **kw):
    return ("layer", nets.Layer(name, 16, 16, src=src, **kw))


def _proj(name, src):
    return _layer(name, src, relu=False)


def _is_shortcut(ops):
    residuals = [op[1].residual for op in ops if op[0] == "layer"]
    return lambda L: not L.relu and not L.residual and L.src != "input" and residuals.count(L.name) == 1


def _name(op):
    return op[1].name if op[0] == "layer" else op[1]


def _order(ops):
    return [_name(op) for op in nets.backward_order(ops, _is_shortcut(ops))]


X = _layer("x", "input")
HEAD = [_layer("fc", "down")]
DOWN = _layer("down", "up", residual="proj")
NETS = {
    "layer norm": [X, ("layernorm", "n", "x"), _layer("up", "n"), _proj("proj", "x"), DOWN, *HEAD],
    "layer norm, projection first": [X, _proj("proj", "x"), ("layernorm", "n", "x"), _layer("up", "n"), DOWN, *HEAD],
    "pooling": [X, ("maxpool", "p", "x", 2, 2, 0), _layer("up", "p"), _proj("proj", "x"), DOWN, *HEAD],
    "mean": [X, _proj("proj", "x"), ("avgpool", "p", "x"), _layer("up", "p"), DOWN, *HEAD],
    "layer": [X, _layer("up", "x"), _proj("proj", "x"), DOWN, *HEAD],
    "layer, projection first": [X, _proj("proj", "x"), _layer("up", "x"), DOWN, *HEAD],
    "layer and norm": [X, ("layernorm", "n", "x"), _layer("side", "n"), _layer("up", "x", residual="side"), _proj("proj", "x"), DOWN, *HEAD],
    "two": [X, ("layernorm", "n", "x"), _layer("up1", "n"), _proj("p1", "x"), _proj("p2", "x"), _layer("mid", "up1", residual="p1"), _layer("up", "mid"),
            _layer("down", "up", residual="p2"), *HEAD],
    "alone": [X, _layer("y", "x"), ("layernorm", "n", "x"), _layer("up", "n"), _proj("proj", "y"), DOWN, *HEAD],
    "identity beside it": [X, _layer("up", "x"), _layer("mid", "up", residual="x"), _proj("proj", "x"), _layer("down", "mid", residual="proj"), *HEAD],
}


@pytest.mark.parametrize("which", list(NETS))
def test_readers_come_before_what_made_their_input(which):
    ops, order = NETS[which], _order(NETS[which])
    assert sorted(order) == sorted(_name(op) for op in ops)
    at = {n: i for i, n in enumerate(order)}
    for op in ops:
        for src in ([op[1].src, op[1].residual] if op[0] == "layer" else [op[2]]):
            if src in at:
                assert at[_name(op)] < at[src]


def test_the_place_of_a_shortcut():
    assert _order(NETS["layer"]) == ["fc", "down", "up", "proj", "x"]
    assert _order(NETS["layer norm"]) == ["fc", "down", "up", "n", "proj", "x"]
    assert _order(NETS["layer and norm"]) == ["fc", "down", "up", "proj", "side", "n", "x"]
    # the networks of images: every projection right behind the first convolution of its block
    ops = nets.resnet18_ops()
    order = _order(ops)
    assert [n for n in order if n.endswith(".down")] == ["l4.b0.down", "l3.b0.down", "l2.b0.down"]
    for n in order:
        if n.endswith(".down"):
            assert order[order.index(n) - 1] == n.replace("down", "conv1")
