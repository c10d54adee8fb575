"""GPU parity: twn_layer_norm_fwd and twn_layer_norm_bwd against the formulas in 64 bits.

Tolerances, with u = 2^-24 (half a step of fp32) and k the most additions that a value goes through (up to 32 in a thread, ten
levels of a tree, a few single operations; more where a row is walked): a sum of n terms is off by at most k u sum|terms|.  An
output that is rounded to bf16 is off by half a step more, 2^-8 of its value.
"""
import numpy as np
import pytest
import torch

from paper_1605_04711_b200 import twn
from _gpu_util import workspace

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
F, B = torch.float32, torch.bfloat16
SHAPES = [(1, 1), (1, 7), (3, 2), (5, 31), (4, 32), (9, 33), (64, 64), (130, 256), (17, 257), (300, 264), (33, 1000), (7, 1001), (1, 1024), (20, 4096),
          (3, 4104), (3, 8192), (2, 8200), (3, 16384), (2, 16385), (2, 32768), (2, 32776), (1, 50001)]


# a million elements and more, where rows go through shared memory, and the sizes about them
LARGE = [(4100, 260), (2100, 512), (2047, 516), (1100, 1024), (1050, 1004), (1100, 1001), (600, 2048), (300, 4096), (131, 8192), (130, 8200), (70, 16384), (64, 16392),
         (40, 32768), (9000, 1001), (1100, 8191)]


def _normal(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32)).cuda()


def _depth(C):
    return 48 + C // 1024


def _rows(seed, M, C, ld, dtype, offset=0):
    """A view [M, C] into a buffer of pitch ld that starts `offset` elements after an aligned address, and the buffer."""
    buf = torch.full((offset + M * ld,), -7.0, dtype=dtype, device="cuda")
    view = buf[offset:].view(M, ld)[:, :C]
    view.copy_(_normal(seed, M, C) * 1.5 + 0.5 * _normal(seed + 1, M, 1))
    return view, buf[offset:]


def _fwd_reference(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / ((x - mean).square().mean(1, keepdim=True) + eps).sqrt()
    xh = (x - mean) * rstd
    y = xh * (gamma.double() if gamma is not None else 1.0) + (beta.double() if beta is not None else 0.0)
    return xh, mean, rstd, y


def _fwd_bound(x, gamma, beta, xh, mean, rstd, y, half):
    k = _depth(x.shape[1])
    e_mean = k * U * x.double().abs().mean(1, keepdim=True)
    e_diff = e_mean + U * (x.double() - mean).abs()          # of x - mean, before the product with rstd
    # the variance: k u of itself, and the square of the mean's error; with eps the same relative error at most, halved by the root
    rel = (k + 4) * U + (e_mean * rstd) ** 2
    e_xh = e_diff * rstd + xh.abs() * rel
    g = gamma.double().abs() if gamma is not None else 1.0
    b = beta.double().abs() if beta is not None else 0.0
    e = e_xh * g + 3 * U * (xh.abs() * g + b)
    return e + half * (y.abs() + e), e_mean + U * mean.abs(), rel * rstd


def _check_fwd(M, C, xt, yt, ldx, ldy, gamma=True, beta=True, offset=0, seed=1, x_from=None):
    x, xbuf = _rows(seed, M, C, ldx, xt, offset)
    if x_from is not None:
        x.copy_(x_from)
    ga = 1 + 0.3 * _normal(seed + 2, C) if gamma else None
    be = 0.3 * _normal(seed + 3, C) if beta else None
    ybuf = torch.full((offset + M * ldy,), 5.0, dtype=yt, device="cuda")[offset:]
    mean, rstd = torch.full((M,), 9.0, device="cuda"), torch.full((M,), 9.0, device="cuda")
    twn.layer_norm_fwd(xbuf, ldx, M, C, ga, be, EPS, ybuf, ldy, mean, rstd)
    y = ybuf.view(M, ldy)
    xh, rm, rr, ry = _fwd_reference(x, ga, be, EPS)
    ty, tm, tr = _fwd_bound(x, ga, be, xh, rm, rr, ry, HALF[yt])
    assert bool(((y[:, :C].double() - ry).abs() <= ty).all())
    assert bool(((mean.double()[:, None] - rm).abs() <= tm).all())
    assert bool(((rstd.double()[:, None] - rr).abs() <= tr).all())
    assert bool((y[:, C:] == 5.0).all())
    return x, y


@pytest.mark.parametrize("M,C", SHAPES)
@pytest.mark.parametrize("xt,yt", [(F, F), (B, B), (F, B), (B, F)])
def test_forward(M, C, xt, yt):
    _check_fwd(M, C, xt, yt, C, C)


@pytest.mark.parametrize("M,C", LARGE)
@pytest.mark.parametrize("xt,yt", [(F, F), (B, B), (F, B), (B, F)])
def test_forward_large(M, C, xt, yt):
    _check_fwd(M, C, xt, yt, C, C + 24, gamma=C % 3 > 0, beta=C % 5 > 0)


@pytest.mark.parametrize("M,C", [(148, 1001), (149, 1001), (296, 4001), (297, 4001), (2368, 1001), (2369, 1024), (1184, 2048), (1185, 2048), (4736, 512), (4737, 512),
                                 (149, 8192), (297, 8192), (148, 16384), (149, 16384), (296, 16383), (5000, 33), (4737, 500), (200, 40), (19000, 60)])
@pytest.mark.parametrize("xt,yt", [(F, F), (B, B), (F, B)])
def test_forward_where_the_blocks_change(M, C, xt, yt):
    """The most rows that one launch of a block an SM takes, for its teams' sizes, and one more."""
    _check_fwd(M, C, xt, yt, C, C)


@pytest.mark.parametrize("ldx,ldy,offset", [(1008, 1024, 0), (1001, 1000, 0), (1000, 1000, 1), (1000, 1003, 8), (1024, 1024, 0)])
@pytest.mark.parametrize("xt,yt", [(F, F), (B, B), (F, B), (B, F)])
def test_forward_pitches_and_offsets(ldx, ldy, offset, xt, yt):
    _check_fwd(37, 1000, xt, yt, ldx, ldy, offset=offset)


@pytest.mark.parametrize("gamma,beta", [(False, False), (True, False), (False, True)])
def test_forward_without_parameters(gamma, beta):
    for C in (24, 515, 4096):
        _check_fwd(11, C, B, B, C, C, gamma, beta)


def test_forward_rows_far_from_zero_and_rows_of_equal_values():
    x = 1000.0 + _normal(5, 16, 768)
    _check_fwd(16, 768, F, F, 768, 768, x_from=x)
    x[3] = 2.5
    x[4] = 0.0
    _, y = _check_fwd(16, 768, F, F, 768, 768, gamma=False, beta=False, x_from=x)
    assert bool((y[3:5] == 0.0).all())


def test_forward_nonfinite_rows_stay_alone():
    x, y = _normal(6, 8, 200), torch.empty(8, 200, device="cuda")
    clean = torch.empty_like(y)
    twn.layer_norm_fwd(x, 200, 8, 200, None, None, EPS, clean, 200)
    x[2, 5], x[5, 199], x[7, 0] = float("nan"), float("inf"), float("-inf")
    twn.layer_norm_fwd(x, 200, 8, 200, None, None, EPS, y, 200)
    for r in range(8):
        assert bool(y[r].isnan().all()) if r in (2, 5, 7) else torch.equal(y[r], clean[r])


@pytest.mark.parametrize("C,dtype", [(96, B), (1001, F), (4096, B), (32768, F), (33000, B), (60000, F)])
def test_forward_in_place_gives_the_same_bits(C, dtype):
    x, buf = _rows(7, 21, C, C, dtype)
    y = torch.empty(21, C, dtype=dtype, device="cuda")
    twn.layer_norm_fwd(buf, C, 21, C, None, None, EPS, y, C)
    twn.layer_norm_fwd(buf, C, 21, C, None, None, EPS, buf, C)
    assert torch.equal(buf.view(21, C), y)


def test_a_row_has_the_same_bits_at_every_place_and_in_every_call():
    for M, C in ((600, 64), (600, 1000), (600, 4096), (3, 4096), (600, 1001), (30, 40000)):
        x = _normal(8, M, C).to(B)
        x[M - 1] = x[M // 2] = x[0]
        y, again = torch.empty_like(x), torch.empty_like(x)
        twn.layer_norm_fwd(x, C, M, C, None, None, EPS, y, C)
        twn.layer_norm_fwd(x, C, M, C, None, None, EPS, again, C)
        assert torch.equal(y, again) and torch.equal(y[0], y[M - 1]) and torch.equal(y[0], y[M // 2])


def _bwd_reference(dy, x, gamma, mean, rstd):
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    dy = dy.double()
    g = dy * (gamma.double() if gamma is not None else 1.0)
    c0, c1 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    return xh, g, (g - c0 - xh * c1) * rstd.double()[:, None], (dy * xh).sum(0), dy.sum(0)


def _check_bwd(M, C, dt, xt, ot, lddy, ldx, lddx, gamma=True, offset=0, seed=11, sums=True, data=True, in_place=None, residual=None, shift=0.0):
    x, xbuf = _rows(seed, M, C, ldx, xt, offset)
    if shift:
        x.add_(shift)
    dy, dbuf = _rows(seed + 5, M, C, lddy, dt, offset)
    ga = 1 + 0.3 * _normal(seed + 2, C) if gamma else None
    _, m, r, _ = _fwd_reference(x, None, None, EPS)
    mean, rstd = m.float().flatten(), r.float().flatten()
    xh, g, rdx, rdg, rdb = _bwd_reference(dy, x, ga, mean, rstd)
    ady = dy.double().abs()
    obuf = {"dY": dbuf, "X": xbuf, None: torch.full((offset + M * lddx,), 5.0, dtype=ot, device="cuda")[offset:]}[in_place]
    rbuf = None
    if residual:                             # "apart", or "in place": dX itself
        rbuf = obuf if residual == "in place" else torch.empty_like(obuf)
        rbuf.copy_(_normal(seed + 9, 1, rbuf.numel()).flatten())
        rdx = rdx + rbuf.view(M, lddx)[:, :C].double()
    keep = obuf.view(M, lddx)[:, C:].clone()
    dg, db = (torch.full((C,), 9.0, device="cuda") for _ in range(2))
    ws = workspace(twn.layer_norm_bwd_workspace_bytes(M, C))
    ws.fill_(255)                            # NaNs: nothing of it may be read before it is written
    twn.layer_norm_bwd(dbuf, lddy, xbuf, ldx, M, C, ga, mean, rstd, obuf if data else None, lddx, dg if sums else None, db if sums else None, ws, rbuf)
    k = _depth(C)
    # xh: two roundings of a difference (u of |x|, |mean| counted in it) and a product
    e_xh = 2 * U * xh.abs() + U * (x.double().abs() + m.abs()) * r
    if data:
        size = g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True)
        spread = e_xh * (g * xh).abs().mean(1, keepdim=True) + xh.abs() * (g.abs() * e_xh).mean(1, keepdim=True)
        e = r * (k * U * size + 2 * spread) + U * rdx.abs()
        dx = obuf.view(M, lddx)
        assert bool(((dx[:, :C].double() - rdx).abs() <= e + HALF[ot] * (rdx.abs() + e)).all())
        assert torch.equal(dx[:, C:], keep)
    if sums:
        # a thread adds the rows of its part, a tree and eight runs join them
        depth = M + 64
        assert bool(((dg.double() - rdg).abs() <= depth * U * (ady * xh.abs()).sum(0) + (ady * e_xh).sum(0)).all())
        assert bool(((db.double() - rdb).abs() <= depth * U * ady.sum(0)).all())


@pytest.mark.parametrize("M,C", SHAPES + [(1000, 64), (5000, 24), (700, 1024), (333, 4096), (150, 9000), (0, 40), (0, 9000)])
@pytest.mark.parametrize("dt,xt,ot", [(F, F, F), (B, B, B), (B, F, F), (F, B, B)])
def test_backward(M, C, dt, xt, ot):
    _check_bwd(M, C, dt, xt, ot, C, C, C)


@pytest.mark.parametrize("M,C", LARGE)
@pytest.mark.parametrize("dt,xt,ot", [(F, F, F), (B, B, B), (B, F, B), (F, B, F)])
def test_backward_large(M, C, dt, xt, ot):
    _check_bwd(M, C, dt, xt, ot, C, C + 8, C + 24, gamma=C % 3 > 0)


@pytest.mark.parametrize("M,C", [(200, 12004), (90, 12004), (300, 8188), (5000, 212), (70, 16384), (40, 32768)])
@pytest.mark.parametrize("dt,xt,ot", [(F, F, F), (B, B, B), (B, F, B), (F, B, F)])
def test_backward_rows_of_eight_bytes(M, C, dt, xt, ot):
    """C % 8 == 4: rows of bf16 lie on 8-byte boundaries, those of fp32 on 16; and rows beside them that fill their threads."""
    _check_bwd(M, C, dt, xt, ot, C, C + 4, C + 12)


@pytest.mark.parametrize("dt,xt,ot", [(F, F, F), (B, F, F)])
@pytest.mark.parametrize("M,C", [(700, 1001), (700, 1024), (80, 16384)])
def test_backward_rows_far_from_zero(M, C, dt, xt, ot):
    """Rows at 300 with a deviation of 1.5: X - mean is off by what the fp32 mean is off, which the bound counts."""
    _check_bwd(M, C, dt, xt, ot, C, C, C, shift=300.0)


@pytest.mark.parametrize("M,C", [(3, 20), (50, 1000), (41, 1001), (300, 4096), (70, 16384), (9000, 1001), (20, 20000), (30, 9001)])
@pytest.mark.parametrize("residual", ["apart", "in place"])
@pytest.mark.parametrize("dt,xt,ot", [(F, F, F), (B, B, B), (B, F, F), (F, F, B)])
def test_backward_with_a_residual(M, C, residual, dt, xt, ot):
    _check_bwd(M, C, dt, xt, ot, C, C, C + 8, residual=residual)


@pytest.mark.parametrize("lddy,ldx,lddx,offset", [(1008, 1024, 1000, 0), (1001, 1000, 1000, 0), (1000, 1000, 1003, 0), (1000, 1000, 1000, 1)])
@pytest.mark.parametrize("dt,xt,ot", [(F, F, B), (B, B, F), (B, F, B), (F, B, F), (B, B, B)])
def test_backward_pitches_and_offsets(lddy, ldx, lddx, offset, dt, xt, ot):
    _check_bwd(41, 1000, dt, xt, ot, lddy, ldx, lddx, offset=offset)


@pytest.mark.parametrize("C", [40, 1000, 4096, 9001, 20000])
def test_backward_parts(C):
    _check_bwd(50, C, B, B, B, C, C, C, gamma=False)
    _check_bwd(50, C, B, B, B, C, C, C, sums=False)
    _check_bwd(50, C, B, B, B, C, C, C, data=False)
    _check_bwd(50, C, B, B, B, C, C, C, in_place="dY")
    _check_bwd(50, C, F, F, F, C, C, C, in_place="X")


def test_backward_against_differences():
    """The gradients of sum(dY * Y) against central differences of the forward formula in 64 bits."""
    M, C, h = 3, 24, 1e-6
    x, ga, be, dy = _normal(20, M, C), 1 + 0.3 * _normal(21, C), 0.3 * _normal(22, C), _normal(23, M, C)
    _, m, r, _ = _fwd_reference(x, ga, be, EPS)
    dx, dg, db = torch.empty_like(x), torch.empty_like(ga), torch.empty_like(be)
    ws = workspace(twn.layer_norm_bwd_workspace_bytes(M, C))
    twn.layer_norm_bwd(dy, C, x, C, M, C, ga, m.float().flatten(), r.float().flatten(), dx, C, dg, db, ws)

    def loss(x, ga, be):
        return float((dy.double() * _fwd_reference(x, ga, be, EPS)[3]).sum())

    args = [x.double(), ga.double(), be.double()]
    for at, got in enumerate((dx, dg, db)):
        flat = args[at].view(-1)
        for i in range(flat.numel()):
            keep = float(flat[i])
            flat[i] = keep + h
            up = loss(*args)
            flat[i] = keep - h
            down = loss(*args)
            flat[i] = keep
            # the difference: h^2 of a third derivative, and 1e-16 of a loss of some 10, over 2 h; the kernel: fp32
            assert abs((up - down) / (2 * h) - float(got.view(-1)[i])) <= 2e-5 * (1 + abs(float(got.view(-1)[i])))


def test_offsets_beyond_32_bits():
    C, ld = 520, (1 << 32) + 8
    buf = torch.empty(ld + C, dtype=B, device="cuda")
    x = _normal(30, 2, C).to(B)
    buf[:C], buf[ld:] = x[0], x[1]
    y, near = torch.empty(2, C, dtype=B, device="cuda"), torch.empty(2, C, dtype=B, device="cuda")
    mean, rstd = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    twn.layer_norm_fwd(buf, ld, 2, C, None, None, EPS, y, C, mean, rstd)
    twn.layer_norm_fwd(x, C, 2, C, None, None, EPS, near, C)
    assert torch.equal(y, near)
    dx, dg, db = torch.empty_like(y), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    dx2, dg2, db2 = torch.empty_like(y), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = workspace(twn.layer_norm_bwd_workspace_bytes(2, C))
    twn.layer_norm_bwd(y, C, buf, ld, 2, C, None, mean, rstd, dx, C, dg, db, ws)
    twn.layer_norm_bwd(y, C, x, C, 2, C, None, mean, rstd, dx2, C, dg2, db2, ws)
    assert torch.equal(dx, dx2) and torch.equal(dg, dg2) and torch.equal(db, db2)


def test_streams_graphs_and_repeated_calls():
    M, C = 500, 1536
    x, dy = _normal(31, M, C).to(B), _normal(32, M, C).to(B)
    ga, be = 1 + 0.1 * _normal(33, C), _normal(34, C)

    def buffers():
        return (torch.empty_like(x), torch.empty(M, device="cuda"), torch.empty(M, device="cuda"), torch.empty_like(x), torch.empty(C, device="cuda"),
                torch.empty(C, device="cuda"), workspace(twn.layer_norm_bwd_workspace_bytes(M, C)))

    def call(b, stream=None):
        y, mean, rstd, dx, dg, db, ws = b
        twn.layer_norm_fwd(x, C, M, C, ga, be, EPS, y, C, mean, rstd, stream=stream)
        twn.layer_norm_bwd(dy, C, x, C, M, C, ga, mean, rstd, dx, C, dg, db, ws, stream=stream)

    want, sides, graphed = buffers(), [buffers(), buffers()], buffers()
    call(want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for b, st in zip(sides, streams):
            call(b, st)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(graphed)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for b in (*sides, graphed):
        for p, q in zip(want[:-1], b[:-1]):
            assert torch.equal(p, q)


def test_binding_refuses_tensors_that_are_too_small_or_of_another_type():
    x, y = torch.zeros(4, 64, device="cuda"), torch.zeros(4, 64, device="cuda")
    with pytest.raises(AssertionError):
        twn.layer_norm_fwd(x, 64, 5, 64, None, None, EPS, y, 64)
    with pytest.raises(AssertionError):
        twn.layer_norm_fwd(x, 64, 4, 64, torch.zeros(63, device="cuda"), None, EPS, y, 64)
    with pytest.raises(TypeError):
        twn.layer_norm_fwd(x.half(), 64, 4, 64, None, None, EPS, y, 64)
    with pytest.raises(TypeError):
        twn.layer_norm_fwd(x, 64, 4, 64, torch.zeros(64, device="cuda", dtype=torch.bfloat16), None, EPS, y, 64)
    with pytest.raises(twn.TwnError):
        twn.layer_norm_fwd(x, 63, 4, 64, None, None, EPS, y, 64)
