"""GPU parity: twn_orthogonalize_batch and twn_muon_update_batch against Newton-Schulz steps in 64 bits.

Bar.  The header's: the 2-norm of the error relative to the result is within 4e-3 for five steps, within 1e-3 for matrices of
independent elements (the roundings of the kernels, carried out in 64 bits on the CPU, gave 2.3e-3 for rank one, 1e-3 for rank 32
and 5e-4 to 8e-4 for full spectra); a result in bf16 is off by half a step more, 2^-8.  No 64 x 64 block may be off by more than eight
times its share.  Where the steps act on one singular value with power-of-two scales, the result is that of fp32 arithmetic.
"""
import numpy as np
import pytest
import torch

from paper_1605_04711_b200 import twn
from _gpu_util import workspace

pytestmark = pytest.mark.gpu

NS = (3.4445, -4.7750, 2.0315)
F, B = torch.float32, torch.bfloat16
SHAPES = [(1, 1), (1, 7), (7, 1), (2, 3), (63, 65), (64, 64), (65, 63), (64, 576), (128, 128), (129, 300), (300, 129), (255, 257), (256, 1000),
          (1000, 512), (513, 511), (640, 640), (1024, 2048), (2047, 1111), (1, 5000), (130, 10000), (768, 6912), (1500, 2700), (2560, 2304), (2309, 2701), (2817, 2900), (3100, 2820)]


def _normal(seed, rows, cols):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal((rows, cols)).astype(np.float32)).cuda()


def _exact(G, steps=5, eps=1e-7):
    a, b, c = NS
    x = G.double()
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / max(float(x.norm()), eps)
    for _ in range(steps):
        s = x @ x.T
        x = a * x + (b * s + c * s @ s) @ x
    return x.T if tall else x


def _run(Gs, types=F, steps=5, eps=1e-7, status=None):
    types = types if isinstance(types, list) else [types] * len(Gs)
    Os = [torch.full(G.shape, 7.0, dtype=t, device="cuda") for G, t in zip(Gs, types)]
    ws = workspace(twn.orthogonalize_workspace_bytes([tuple(G.shape) for G in Gs]))
    ws.fill_(255)                            # NaNs: nothing of it may be read before it is written
    twn.orthogonalize_batch([(G, G.shape[0], G.shape[1], O) for G, O in zip(Gs, Os)], steps, eps, ws, status)
    return Os


def _check(G, O, bar, steps=5):
    want = _exact(G, steps)
    bar = bar + (2.0 ** -8 if O.dtype == B else 0.0)
    d = O.double() - want
    total = float(want.norm())
    assert float(d.norm()) <= bar * total
    rows, cols = G.shape
    share = total / (rows * cols) ** 0.5
    wide = 64 if rows * cols < 1 << 20 else 512
    for r in range(0, rows, 64):
        for c in range(0, cols, wide):
            part = d[r:r + 64, c:c + wide]
            assert float(part.norm()) <= 8 * bar * share * part.numel() ** 0.5 + bar * total * (min(rows, cols) < 64)


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("gt,ot", [(F, F), (B, B)])
def test_independent_elements(rows, cols, gt, ot):
    G = (0.01 * _normal(rows + cols, rows, cols)).to(gt)
    # few rows: the error is that of a handful of sums, not an average over them
    _check(G, _run([G], ot)[0], 1e-3 if min(rows, cols) >= 64 else 4e-3)


@pytest.mark.parametrize("rows,cols", [(256, 384), (384, 256), (520, 1000)])
@pytest.mark.parametrize("kind", ["rank1", "rank32", "power1", "power2", "identity"])
def test_spectra(rows, cols, kind):
    m = min(rows, cols)
    if kind == "identity":
        G = torch.eye(rows, cols, device="cuda")
    elif kind.startswith("rank"):
        k = int(kind[4:])
        G = _normal(3, rows, k) @ _normal(4, k, cols)
    else:
        u, _ = torch.linalg.qr(_normal(5, rows, m).double())
        v, _ = torch.linalg.qr(_normal(6, cols, m).double())
        G = ((u * torch.arange(1, m + 1, device="cuda").double() ** -int(kind[5:])) @ v.T).float()
    O = _run([G])[0]
    assert float((O.double() - _exact(G)).norm()) <= 4e-3 * float(_exact(G).norm())


@pytest.mark.parametrize("rows,cols", [(1, 1), (4, 9), (16, 16), (64, 70), (70, 64), (256, 256), (300, 256), (256, 1025), (1024, 1300)])
@pytest.mark.parametrize("steps", [1, 2, 5])
def test_permutations_are_served_to_fp32_and_land_where_they_belong(rows, cols, steps):
    """m = 4^k ones, one in every row (or column): every singular value is 2^-k, and X, A and B have one element a row.  A step is one
    polynomial of one number; the upper half of X is rounded to fp16 (2^-11) only where it is multiplied, in A, beside 22 bits of a X."""
    m, n = min(rows, cols), max(rows, cols)
    at = torch.from_numpy(np.random.default_rng(rows + cols).permutation(n)[:m].copy()).cuda()
    G = torch.zeros(m, n, device="cuda")
    G[torch.arange(m, device="cuda"), at] = 3.0
    G = G.T.contiguous() if rows > cols else G
    O = _run([G], steps=steps)[0]
    t = m ** -0.5
    for _ in range(steps):
        t = NS[0] * t + NS[1] * t ** 3 + NS[2] * t ** 5
    got = O.T if rows > cols else O
    values = got[torch.arange(m, device="cuda"), at].double()
    # the first step's fp16 half is exact (3 / (3 2^k), a power of two)
    bar = 4e-6 if steps == 1 else 4e-3
    assert float((values - t).abs().max()) <= bar * abs(t)
    assert int((O != 0).sum()) == m


def test_scales():
    G = _normal(9, 200, 300)
    want = _run([G])[0]
    for scale in (2.0 ** -60, 2.0 ** 60, 2.0 ** 120):
        # powers of two change no digit of G, and the norm's square root and quotient round as before
        assert float((_run([G * scale], eps=1e-30)[0] - want).norm()) <= 1e-6 * float(want.norm())
    # below eps the norm is taken as eps
    tiny = G * (1e-9 / float(G.norm()))
    O = _run([tiny], steps=1, eps=1e-7)[0]
    assert float((O.double() - NS[0] * 0.01 * G.double() / float(G.norm())).norm()) <= 1e-3 * NS[0] * 0.01
    assert bool((_run([torch.zeros(70, 90, device="cuda")])[0] == 0).all())


@pytest.mark.parametrize("shapes", [[(64, 576), (512, 64), (1, 1), (100, 128), (128, 128), (128, 8192), (5, 2000), (8192, 3)] * 4,
                                    [(300, 300), (129, 131), (1000, 512), (256, 2304), (1500, 2700), (7000, 200)] * 3])
def test_a_batch_gives_the_bits_of_single_calls_and_repeats_them(shapes):
    Gs = [_normal(40 + i, r, c).to(B if i % 3 == 0 else F) for i, (r, c) in enumerate(shapes)]
    types = [B if i % 2 else F for i in range(len(Gs))]
    many, again = _run(Gs, types), _run(Gs, types)
    for G, t, O, O2 in zip(Gs, types, many, again):
        assert torch.equal(O, O2) and torch.equal(_run([G], t)[0], O)


@pytest.mark.parametrize("gt,ot", [(F, F), (B, B)])
def test_small_matrices_among_larger_ones(gt, ot):
    shapes = [s for s in SHAPES if min(s) <= 128] + [(150, 200)]
    Gs = [(0.01 * _normal(sum(s), *s)).to(gt) for s in shapes]
    for G, O in zip(Gs, _run(Gs, ot)):
        _check(G, O, 1e-3 if min(G.shape) >= 64 else 4e-3)


SMALL = [(1, 1), (1, 8192), (8192, 1), (3, 5), (31, 33), (64, 64), (64, 147), (147, 64), (100, 1000), (999, 101), (127, 129), (128, 128), (128, 8192), (8192, 128), (128, 8193), (129, 700)]


@pytest.mark.parametrize("rows,cols", SMALL)
@pytest.mark.parametrize("gt,ot", [(F, F), (B, B), (F, B), (B, F)])
@pytest.mark.parametrize("steps", [1, 2, 5, 6])
def test_small_matrices(rows, cols, gt, ot, steps):
    G = (0.01 * _normal(rows + cols, rows, cols)).to(gt)
    # one launch of its own: 1e-3 for any of them
    _check(G, _run([G], ot, steps=steps)[0], 1e-3 if max(rows, cols) <= 8192 and min(rows, cols) in range(2, 129) and steps <= 5 else 4e-3, steps)


@pytest.mark.parametrize("rows,cols", [(96, 700), (700, 96), (128, 128), (40, 3000)])
@pytest.mark.parametrize("kind", ["rank1", "rank4", "rank32", "power1", "power2", "power3", "identity", "ones", "blocks"])
def test_spectra_of_small_matrices(rows, cols, kind):
    m = min(rows, cols)
    if kind == "identity":
        G = torch.eye(rows, cols, device="cuda")
    elif kind == "ones":
        G = torch.ones(rows, cols, device="cuda")
    elif kind == "blocks":
        G = torch.zeros(rows, cols, device="cuda")
        G.view(-1)[::cols + 1] = 1.0
        G = G[:rows // 4, :cols // 4].repeat_interleave(4, 0).repeat_interleave(4, 1).contiguous()
    elif kind.startswith("rank"):
        k = int(kind[4:])
        G = _normal(3, rows, k) @ _normal(4, k, cols)
    else:
        u, _ = torch.linalg.qr(_normal(5, rows, m).double())
        v, _ = torch.linalg.qr(_normal(6, cols, m).double())
        G = ((u * torch.arange(1, m + 1, device="cuda").double() ** -int(kind[5:])) @ v.T).float()
    O = _run([G])[0]
    # Elements of A = X X^T are off by 2^-22 of their value (its two fp16 parts), so its eigenvalues s^2 by 2^-22 of the trace, 1, at most.
    # The result for s is s times a product of a + b t + c t^2 over t = s^2, 11.9 s^2, ...; for s = 2e-3, the least that five steps bring to
    # about 1, t is off by 6 % and reaches 0.08 in the last factor, which changes by 4.775 * 0.08 / 3.06 * 6 % = 0.75 %.  Larger s are off
    # by less (the shift is the same, and t stops growing), smaller ones come out as 485 s, with a smaller share of t.  A spectrum that falls off
    # has less than a quarter of its result (in squares) there: 0.75 % / 2 = 3.8e-3.  Rank one, equal elements and the identity have
    # singular values 1 and 0 alone.
    assert float((O.double() - _exact(G)).norm()) <= (4e-3 if kind.startswith("power") else 1e-3) * float(_exact(G).norm())


def test_scales_of_small_matrices():
    G = _normal(9, 60, 300)
    want = _run([G])[0]
    for scale in (2.0 ** -60, 2.0 ** 60, 2.0 ** 120, 2.0 ** -100):
        assert float((_run([G * scale], eps=1e-30)[0] - want).norm()) <= 1e-5 * float(want.norm())
    for scale in (2.0 ** -60, 2.0 ** 100):
        assert float((_run([(G * scale).to(B)], eps=1e-30)[0] - _run([G.to(B)])[0]).norm()) <= 1e-5 * float(want.norm())
    tiny = G * (1e-9 / float(G.norm()))
    O = _run([tiny], steps=1, eps=1e-7)[0]
    assert float((O.double() - NS[0] * 0.01 * G.double() / float(G.norm())).norm()) <= 1e-3 * NS[0] * 0.01
    assert bool((_run([torch.zeros(70, 90, device="cuda")])[0] == 0).all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_nonfinite_small_matrices(bad):
    Gs = [_normal(60 + i, r, c) for i, (r, c) in enumerate([(70, 300), (300, 70), (128, 128)])]
    clean = _run(Gs)
    Gs[1][299, 3] = bad
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    Os = _run(Gs, status=status)
    assert twn.read_status(status) == -4 and bool(Os[1].isnan().all())
    assert torch.equal(Os[0], clean[0]) and torch.equal(Os[2], clean[2])


def test_small_matrices_in_place_unaligned_and_on_streams():
    for r, c in ((100, 333), (333, 100)):
        G = _normal(51, r, c)
        want = _run([G])[0]
        buf = torch.empty(r * c + 1, device="cuda")[1:].view(r, c)
        buf.copy_(G)
        ws = [workspace(twn.orthogonalize_workspace_bytes([(r, c)])) for _ in range(3)]
        twn.orthogonalize_batch([(buf, r, c, buf)], 5, 1e-7, ws[0])
        assert torch.equal(buf, want)
        outs, streams = [torch.empty_like(G) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(4):
            for O, w, st in zip(outs, ws[1:], streams):
                twn.orthogonalize_batch([(G, r, c, O)], 5, 1e-7, w, stream=st)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_empty_matrices_are_skipped_and_output_may_be_the_input():
    G = _normal(50, 100, 130)
    want = _run([G])[0]
    e = torch.empty(0, 5, device="cuda")
    ws = workspace(twn.orthogonalize_workspace_bytes([(0, 5), (100, 130)]))
    twn.orthogonalize_batch([(e, 0, 5, e), (G, 100, 130, G)], 5, 1e-7, ws)
    assert torch.equal(G, want)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_nonfinite_matrices_are_told_and_stay_alone(bad):
    Gs = [_normal(60 + i, r, c) for i, (r, c) in enumerate([(70, 300), (300, 70), (128, 128)])]
    clean = _run(Gs)
    Gs[1][299, 3] = bad
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    Os = _run(Gs, status=status)
    assert twn.read_status(status) == -4 and bool(Os[1].isnan().all())
    assert torch.equal(Os[0], clean[0]) and torch.equal(Os[2], clean[2])


def test_unaligned_tensors():
    buf, out = _normal(70, 1, 200 * 301 + 1).flatten(), torch.zeros(200 * 301 + 1, device="cuda", dtype=B)
    G, O = buf[1:].view(200, 301), out[1:].view(200, 301)
    ws = workspace(twn.orthogonalize_workspace_bytes([(200, 301)]))
    twn.orthogonalize_batch([(G, 200, 301, O)], 5, 1e-7, ws)
    _check(G, O, 1e-3)
    assert float(out[0]) == 0.0


def test_streams_and_graphs():
    Gs = [_normal(80, 320, 500), _normal(81, 900, 250)]
    want = _run(Gs)
    shapes = [tuple(G.shape) for G in Gs]
    sets = [([torch.empty_like(G) for G in Gs], workspace(twn.orthogonalize_workspace_bytes(shapes))) for _ in range(3)]

    def call(s, stream=None):
        twn.orthogonalize_batch([(G, *G.shape, O) for G, O in zip(Gs, s[0])], 5, 1e-7, s[1], stream=stream)

    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s, st in zip(sets, streams):
            call(s, st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(sets[2])
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for s in sets:
        for O, w in zip(s[0], want):
            assert torch.equal(O, w)


def _f32(a, b, c):
    """a + b * c, each operation rounded to fp32."""
    return (a + (b * c).float()).float()


@pytest.mark.parametrize("look", [False, True])
@pytest.mark.parametrize("shapes", [[(64, 576)], [(64, 147), (300, 64), (1, 33), (128, 1152)], [(10, 1024), (512, 64), (300, 300), (1, 33), (1000, 512)]])
def test_muon_steps(look, shapes):
    lr, mu, wd = (float(np.float32(v)) for v in (0.02, 0.95, 0.1))
    W = [0.05 * _normal(90 + i, r, c) for i, (r, c) in enumerate(shapes)]
    V = [0.01 * _normal(190 + i, r, c) for i, (r, c) in enumerate(shapes)]
    stats = [twn.new_stats() for _ in shapes]
    ws = workspace(twn.muon_workspace_bytes(shapes))
    ws.fill_(255)
    t = lambda v: torch.tensor(v, dtype=F, device="cuda")  # noqa: E731
    for step in range(3):
        dW = [0.01 * _normal(290 + 10 * step + i, r, c) for i, (r, c) in enumerate(shapes)]
        V2 = [_f32(d, t(mu), v) for d, v in zip(dW, V)]
        U = [_f32(d, t(mu), v) if look else v for d, v in zip(dW, V2)]
        W2 = []
        for w, O in zip(W, _run(U)):
            s = t(float(np.float32((O.shape[0] / O.shape[1]) ** 0.5)) if O.shape[0] > O.shape[1] else 1.0)
            W2.append((w - t(lr) * _f32(O * s, t(wd), w)).float())
        keep = [d.clone() for d in dW]
        twn.muon_update_batch([(w, d, v, *w.shape, st) for w, d, v, st in zip(W, dW, V, stats)], lr, mu, wd, look, 5, 1e-7, 0.7, ws)
        for w, v, d, w2, v2, k, st in zip(W, V, dW, W2, V2, keep, stats):
            assert torch.equal(v, v2) and torch.equal(w, w2) and torch.equal(d, k)
            h = twn.stats_to_host(st)
            total = float(w.double().abs().sum())
            assert h["status"] == 0 and abs(h["sum_abs"] - total) <= 1e-12 * total and abs(h["delta"] - 0.7 * total / w.numel()) <= 1e-12


def test_muon_then_codes():
    r, c = 192, 1000
    W, dW, V, stats, other = _normal(1, r, c), _normal(2, r, c), torch.zeros(r, c, device="cuda"), twn.new_stats(), twn.new_stats()
    twn.muon_update_batch([(W, dW, V, r, c, stats)], 0.02, 0.95, 0.0, True, 5, 1e-7, 0.7, workspace(twn.muon_workspace_bytes([(r, c)])))
    ld = twn.ld_for(c)
    codes = [torch.empty(r, ld // 16, dtype=torch.int32, device="cuda") for _ in range(2)]
    ws = workspace(twn.ternarize_workspace_bytes())
    twn.ternarize_codes(W, r, c, stats, codes[0], ld, None, ws)
    twn.ternarize(W, 0.7, other, codes[1], ld, None, ws)
    assert torch.equal(*codes)


def test_muon_tells_of_nonfinite_gradients():
    W, dW, V, stats = _normal(1, 64, 80), _normal(2, 64, 80), torch.zeros(64, 80, device="cuda"), twn.new_stats()
    dW[3, 4] = float("inf")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    twn.muon_update_batch([(W, dW, V, 64, 80, stats)], 0.02, 0.95, 0.0, False, 5, 1e-7, 0.7, workspace(twn.muon_workspace_bytes([(64, 80)])), status)
    assert twn.read_status(status) == -4 and twn.stats_to_host(stats)["status"] == -4


def test_binding_refuses_tensors_that_are_too_small_or_of_another_type():
    x, ws = torch.zeros(4, 4, device="cuda"), workspace(1 << 20)
    with pytest.raises(AssertionError):
        twn.orthogonalize_batch([(x, 4, 5, x)], 5, 1e-7, ws)
    with pytest.raises(TypeError):
        twn.orthogonalize_batch([(x, 4, 4, x.half())], 5, 1e-7, ws)
    with pytest.raises(AssertionError):
        twn.muon_update_batch([(x, x, x, 4, 5, None)], 0.1, 0.9, 0.0, True, 5, 1e-7, 0.7, ws)
    with pytest.raises(TypeError):
        twn.muon_update_batch([(x, x.to(B), x, 4, 4, None)], 0.1, 0.9, 0.0, True, 5, 1e-7, 0.7, ws)
    with pytest.raises(twn.TwnError):
        twn.orthogonalize_batch([(x, 4, 4, x)], 0, 1e-7, ws)
