"""Orthogonalised updates of the longest and the largest matrices, where sums are long and offsets pass 32 bits.

Bar.  The header's: 1e-3 of the result's norm for independent elements (4e-3 for a handful of rows); a result in bf16 is off by half a
step more.  Rows that agree, of mean 1 or all the same, are the ones whose sums only grow: what a sum that is cut off at every addition
loses adds up there.

Equal rows: all elements of A off its diagonal are one number, which rounds to fp16 one way, and so are those of B = b A + c A^2.  With
u = 2^-11, X of one singular value t, A = t^2 and l = b A + c A^2, a step is off by at most u t (|b + 2 c A| A for A's rounding, |l| for B's,
|l| / sqrt(3) for the upper halves of X's elements, which differ along a row).  From t = 1 the five t are 1, 0.701, 1.114, 0.721, 1.090 and the
result 0.696; the steps are off by 2.46, 1.47, 2.58, 1.56, 2.38 thousandths, times the slopes of the polynomial in the steps behind
(-1.14, 1.30, -1.26, 0.755 from the second on): 3.47 + 1.81 + 2.45 + 1.18 + 2.38 = 11.3 thousandths of 0.696, 1.62e-2.
"""
import pytest
import torch

from paper_1605_04711_b200 import twn
from _gpu_util import workspace
from test_gpu_orthogonalize import NS, _exact, _run

pytestmark = pytest.mark.gpu

F, B = torch.float32, torch.bfloat16


def _matrix(kind, rows, cols, dtype=F):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    G = torch.randn(rows, cols, generator=g, device="cuda", dtype=dtype)
    if kind == "mean":
        G += 1.0
    elif kind == "equal":
        G[:] = G[:1].clone() if rows < cols else G[:, :1].clone()
    return G


def _error(G, O):
    want = _exact(G)
    total = float(want.norm())
    want -= O
    return float(want.norm()) / total


# a block's share of a reduction: 128 blocks of 64 columns and fewer in one sum, one column more, several, and uneven ones
@pytest.mark.parametrize("rows,cols", [(2, 32768), (2, 32769), (129, 32768), (129, 32832), (300, 40000), (2, 1 << 20), (3, (1 << 22) + 5), (2, 1 << 24), (1 << 20, 5), (129, 1 << 20), (700, 1 << 17),
                                       (1500, 8192), (1500, 8256), (2000, 20001), (2700, 1 << 17), (2700, (1 << 17) + 1)])
@pytest.mark.parametrize("kind", ["any", "mean", "equal"])
def test_long_rows(rows, cols, kind):
    G = _matrix(kind, rows, cols)
    assert _error(G, _run([G])[0]) <= (4e-3 if min(rows, cols) < 64 else 1.63e-2 if kind == "equal" else 1e-3)


def test_long_and_short_ones_in_one_call_have_the_bits_of_their_own():
    Gs = [_matrix("mean", r, c) for r, c in ((129, 700), (2, 1 << 20), (300, 40000), (1000, 513), (200, 8192))]
    many = _run(Gs)
    for G, O, again in zip(Gs, many, _run(Gs)):
        assert torch.equal(O, again) and torch.equal(_run([G])[0], O)


@pytest.mark.parametrize("rows,cols", [(129, 1 << 24), (1 << 24, 130)])
def test_more_elements_than_32_bits_count(rows, cols):
    G = _matrix("mean", rows, cols, B)
    assert G.numel() > 1 << 31
    O = torch.empty_like(G)
    ws = workspace(twn.orthogonalize_workspace_bytes([(rows, cols)]))
    twn.orthogonalize_batch([(G, rows, cols, O)], 5, 1e-7, ws)
    del ws
    assert _error(G, O) <= 1e-3 + 2.0 ** -8


def test_the_largest_square():
    """A Kronecker product of two matrices of known singular vectors has theirs, and the products of their singular values."""
    n, k = 2048, 16
    g = torch.Generator(device="cuda").manual_seed(1)
    basis = lambda m: torch.linalg.qr(torch.randn(m, m, generator=g, device="cuda", dtype=torch.float64))[0]  # noqa: E731
    us, vs, ur, vr = basis(n), basis(n), basis(k), basis(k)
    s, t = (0.2 + 0.8 * torch.rand(m, generator=g, device="cuda", dtype=torch.float64) for m in (n, k))
    S, R = (us * s) @ vs.T, (ur * t) @ vr.T
    S, R = (S / S.norm()), (R / R.norm())
    G = torch.empty(n, k, n, k, device="cuda")
    for i in range(k):
        for j in range(k):
            G[:, i, :, j] = (S * R[i, j]).float()
    G = G.view(n * k, n * k)
    O = torch.empty_like(G)
    ws = workspace(twn.orthogonalize_workspace_bytes([tuple(G.shape)]))
    twn.orthogonalize_batch([(G, n * k, n * k, O)], 5, 1e-7, ws)
    del ws
    value = (s / s.norm())[:, None] * (t / t.norm())
    for _ in range(5):
        value = NS[0] * value + NS[1] * value ** 3 + NS[2] * value ** 5
    parts = [(us * value[:, b]) @ vs.T for b in range(k)]
    total = float(value.norm())
    O, lost = O.view(n, k, n, k), 0.0
    for i in range(k):
        for j in range(k):
            want = sum(ur[i, b] * vr[j, b] * parts[b] for b in range(k))
            # rounding of G to fp32, 2^-24, times 485 at most: far below the bar
            d = float((O[:, i, :, j].double() - want).norm())
            assert d <= 8 * 1e-3 * total / k
            lost += d * d
    assert lost ** 0.5 <= 1e-3 * total


def test_small_ones_have_the_same_bits_beside_any_larger_one():
    """Not those that they have in a call of small matrices alone, which goes another way."""
    small = [_matrix("any", r, c) for r, c in ((64, 576), (1, 33), (300, 4), (128, 8192))]
    first = _run(small + [_matrix("any", 300, 300)])
    for other in ([_matrix("any", 1000, 513)], [_matrix("any", 129, 40000), _matrix("any", 2820, 2900)]):
        for O, want in zip(_run(small + other), first[:4]):
            assert torch.equal(O, want)
