"""GPU tests of the text operators at the ends of their ranges: gains and streams near fp32's largest and least numbers, quotients
among the least 8-bit values, tensors at any address, and gradients that are differentiated again.

Bounds as in test_text_ops_gpu.py: E = 2^-24 for each fp32 operation, u half a step of a result's format."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import text_ops as ops
from tests.test_text_ops_gpu import BF, E, FP, HF, U, _linear_check, _norm_check, _rows8_check, f64, randn, within

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------- 8 bits
@pytest.mark.parametrize("h_size,w_size", [(100.0, 2e37), (1e10, 1e30), (1e15, 1e25)])
@pytest.mark.parametrize("M,D", [(5, 64), (9, 256), (3, 768), (600, 768), (2, 4096), (2, 8208)])
def test_rows_in_8_bits_products_past_fp32(h_size, w_size, M, D):
    """h w lies beyond fp32's largest number, y = h rstd w does not; every other row's products are ordinary ones."""
    import torch
    from paper_2309_16669_amd import autograd as ag
    w = w_size * (1 + 0.1 * randn(1, (D,), FP))
    r = h_size * randn(2, (M, D), FP)
    r[1::2] *= 1e-12
    x = torch.zeros((M, D), dtype=torch.bfloat16, device="cuda")
    y, h = ag.add_rms_norm(x, r, w, 1e-20)
    assert torch.equal(h, r) and y.isfinite().all()
    q, s, h = ag.add_rms_norm_fp8(x, r, w, 1e-20)
    assert torch.equal(h, r)
    _rows8_check(ops.rms_fwd(f64(r), f64(w), 1e-20)[0], q, s, (D / 2 + 20) * E)
    if h_size < 1e4:    # the same without a residual, and with ordinary gains on the same rows
        q, s = ag.rms_norm_fp8(r.to(torch.bfloat16), w, 1e-20)
        _rows8_check(ops.rms_fwd(f64(r.to(torch.bfloat16)), f64(w), 1e-20)[0], q, s, (D / 2 + 20) * E)
    q, s, h = ag.add_rms_norm_fp8(x, r, w / w_size, 1e-20)
    _rows8_check(ops.rms_fwd(f64(r), f64(w / w_size), 1e-20)[0], q, s, (D / 2 + 20) * E)


def _small_ties():
    """(big, value) of 8-bit significands, value / big * 448 exactly in the middle of two of the least 8-bit values (steps of
    2^-9), and the even one of the two."""
    out = []
    for m in range(128, 256):
        for a in range(128, 256):
            for e in range(-22, -12):
                v = Fraction(a, m) * 448 * Fraction(2) ** e * 1024      # in half steps
                if v.denominator == 1 and v.numerator % 2 and v < 16:
                    k = (v.numerator - 1) // 2
                    out.append((m / 64.0, a * 2.0 ** (e - 6), (k + k % 2) * 2.0 ** -9))
    return out


@pytest.mark.parametrize("D", [16, 256, 768, 4096, 8208])
def test_norm_in_8_bits_exact_middles_of_the_least_values(D):
    import torch
    from paper_2309_16669_amd import autograd as ag
    ties = _small_ties()
    assert len(ties) > 10 and any(abs(b - 2.109375) < 1e-9 for b, _, _ in ties)
    x = torch.zeros((len(ties), D), dtype=torch.float64)
    want = torch.zeros((len(ties), D))
    for i, (big, value, q) in enumerate(ties):
        at = 1 + (7 * i) % (D - 1)
        x[i, 0], x[i, at] = big, -value if i % 2 else value
        want[i, 0], want[i, at] = 448.0, -q if i % 2 else q
    xb = x.to(torch.bfloat16)
    assert torch.equal(xb.double(), x)
    q, _ = ag.rms_norm_fp8(xb.cuda(), torch.ones(D, device="cuda"))
    assert torch.equal(q.float().cpu(), want)
    q, _ = ag.quantize_rows(xb.cuda())
    assert torch.equal(q.float().cpu(), want)


@pytest.mark.parametrize("M,D", [(6000, 128), (4000, 240), (5000, 768), (400, 768), (700, 4096), (200, 8208)])
@pytest.mark.parametrize("fmt,stream", [(BF, BF), (HF, FP), (BF, None)])
def test_norm_in_8_bits_is_the_nearest_of_the_least_values(M, D, fmt, stream):
    """Of all values, those below 2^-6 among them (all but one of a row here), the nearest 8-bit one, unless the quotient lies within
    2^-38 of the middle between two."""
    import torch
    from paper_2309_16669_amd import autograd as ag
    x, w = randn(M + D, (M, D), fmt, 2.0 ** -11), 1 + 0.1 * randn(2, (D,), FP)
    w[::7] = 1.0
    x[:, 3] = 64.0 * (1 + torch.rand(M, device="cuda")).to(x.dtype)
    if stream is None:
        q, s = ag.rms_norm_fp8(x, w)
        h = x
    else:
        q, s, h = ag.add_rms_norm_fp8(x, randn(3, (M, D), stream, 2.0 ** -11), w)
    p = h.double() * w.double()
    v = (p / p.abs().amax(1, keepdim=True) * 448.0).abs()
    assert float((v < 2.0 ** -6).double().mean()) > 0.5
    e = torch.floor(torch.log2(v.clamp_min(2.0 ** -6)))
    steps = v * torch.exp2(3 - e)
    open_side = (steps - torch.floor(steps) - 0.5).abs() <= steps * 2.0 ** -38
    near = torch.round(steps) * torch.exp2(e - 3)
    off = (q.double().abs() != near) & ~open_side
    assert not off.any(), (int(off.sum()), v[off][:4], q.double().abs()[off][:4])


# narrow and short y with many tiles: half a tile of 256 x 256 and less, 64 columns
@pytest.mark.parametrize("M,N,K", [(36001, 64, 80), (36865, 72, 144), (40001, 128, 96), (40001, 136, 48), (33, 40000, 64), (128, 40000, 80), (129, 40000, 48)])
@pytest.mark.parametrize("fmt,bias", [(BF, True), (HF, False)])
def test_linear_narrow_and_short(M, N, K, fmt, bias):
    _linear_check(M, N, K, fmt, bias, seed=M + N)


# up to 32 rows, around the width from which tiles take them
@pytest.mark.parametrize("M,N,K", [(17, 4096, 2064), (32, 4096, 4096), (32, 4104, 2048), (17, 4104, 272), (24, 6144, 1040), (32, 33000, 48)])
@pytest.mark.parametrize("fmt,bias", [(BF, True), (HF, False)])
def test_linear_few_rows(M, N, K, fmt, bias):
    _linear_check(M, N, K, fmt, bias, seed=M + K)


# --------------------------------------------------------------------------------------------- RMS normalisation
def test_norm_of_rows_near_the_least_numbers():
    """A mean of squares (with eps) below fp32's least normal number, 2^-126: rows of zeros under such an eps stay zeros, and rows
    whose squares fp32 holds as multiples of 2^-149 have a norm of size 1."""
    import torch
    from paper_2309_16669_amd import autograd as ag
    for D in (64, 256, 768, 4096):
        w = 1 + 0.1 * randn(1, (D,), FP)
        zeros = torch.zeros((5, D), dtype=torch.bfloat16, device="cuda")
        for eps in (1e-38, 1e-40, 1e-44):
            assert not ag.rms_norm(zeros, w, eps).any()
            q, s = ag.rms_norm_fp8(zeros, w, eps)
            assert not q.float().any() and abs(float(s[0]) - 2.0 ** -96 / 448) <= 2 * E * 2.0 ** -96 / 448
            x = zeros.clone().requires_grad_()
            (dx,) = torch.autograd.grad(ag.rms_norm(x, w, eps), x, torch.zeros_like(x))
            assert not dx.any()
        r = 1e-20 * randn(2, (5, D), FP)
        y, h = ag.add_rms_norm(zeros, r, w, 0.0)
        ref, rstd = ops.rms_fwd(f64(r), f64(w), 0.0)
        # each addition to the sum, and the mean, is off by half of 2^-149 at most; half of that relative error is rstd's
        lost = (D + D) * 2.0 ** -150 / (2 * D) * rstd[:, None] ** 2
        assert lost.max() < 1e-4
        within("y", y, ref, (U[BF] + (D / 2 + 12) * E + lost) * np.abs(ref))
        q, s, h = ag.add_rms_norm_fp8(zeros, r, w, 0.0)
        _rows8_check(ref, q, s, (D / 2 + 20) * E + float(lost.max()))


# the gains' gradient in the same launch, and in one of its own
@pytest.mark.parametrize("M", [639, 640, 641])
@pytest.mark.parametrize("D", [64, 136, 768, 2056, 8200])
def test_norm_around_one_launch(M, D):
    _norm_check(M, D, BF, FP, seed=M + D)


def test_norm_of_the_widest_rows_in_one_launch():
    _norm_check(600, 16384, HF, HF, seed=5)


# ---------------------------------------------------------------------------------------------------- addresses
def odd(t):
    """The same values in memory whose address is a multiple of the element's size only."""
    import torch
    room = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    out = room[1:].view(t.shape)
    out.copy_(t.detach())
    assert out.is_contiguous() and out.data_ptr() % 16 != 0
    return out


def _both_ways(monkeypatch):
    """The native calls, then the classes."""
    from types import SimpleNamespace
    from paper_2309_16669_amd import autograd as ag
    names = ("embedding", "rms_norm", "add_rms_norm", "rms_norm_fp8", "add_rms_norm_fp8", "quantize_rows", "linear_fp8")
    ag.native_calls()
    yield "native"
    with monkeypatch.context() as m:
        m.setattr(ag, "_native", SimpleNamespace(**{n: lambda *args: None for n in names}))
        yield "classes"


def test_tensors_at_any_address(monkeypatch):
    import torch
    from paper_2309_16669_amd import autograd as ag
    M, D = 37, 144
    t = torch.arange(2 * M, device="cuda").view(2, M) % 50
    table, x, r, w = randn(1, (50, D), BF), randn(2, (M, D), BF), randn(3, (M, D), FP), 1 + 0.1 * randn(4, (D,), FP)
    dy2, dy, dh = randn(5, (2, M, D), BF), randn(6, (M, D), BF), randn(7, (M, D), FP)
    calls = [(lambda a: ag.embedding(t, a, 2.0), [table], [dy2]), (ag.rms_norm, [x, w], [dy]), (ag.add_rms_norm, [x, r, w], [dy, dh]),
             (ag.add_rms_norm, [x, r.bfloat16(), w], [dy, dh.bfloat16()])]
    x8, xs = ag.quantize_rows(x)
    w8, ws = ag.quantize_rows(randn(8, (64, D), BF))
    b = randn(9, (64,), FP)
    plain = [(ag.rms_norm_fp8, [x, w]), (ag.add_rms_norm_fp8, [x, r, w]), (ag.quantize_rows, [x]), (ag.linear_fp8, [x8, xs, w8, ws, b])]
    for way in _both_ways(monkeypatch):
        for call, args, grads in calls:
            got = []
            for place_args, place_grads in ((torch.clone, torch.clone), (odd, torch.clone), (torch.clone, odd), (odd, odd)):
                leaves = [place_args(a).requires_grad_() for a in args]
                out = call(*leaves)
                out = out if isinstance(out, tuple) else (out,)
                g = torch.autograd.grad(out, leaves, [place_grads(d) for d in grads])
                got.append([*out, *g])
            for other in got[1:]:
                assert all(torch.equal(a, c) for a, c in zip(got[0], other)), way
        for call, args in plain:
            with torch.no_grad():
                a, c = call(*args), call(*[odd(v) for v in args])
            for u, v in zip(a if isinstance(a, tuple) else (a,), c if isinstance(c, tuple) else (c,)):
                assert torch.equal(u.float(), v.float()), way


def test_gradients_from_behind_an_odd_part(monkeypatch):
    # what a concatenation hands back: a contiguous piece that begins at an odd element
    import torch
    from paper_2309_16669_amd import autograd as ag
    x, w = randn(1, (9, 64), BF), 1 + 0.1 * randn(2, (64,), FP)
    t, table, a = torch.arange(9, device="cuda"), randn(3, (9, 64), BF), randn(4, (3,), BF)
    for way in _both_ways(monkeypatch):
        for call, leaf in ((lambda v: ag.rms_norm(v, w), x), (lambda v: ag.add_rms_norm(v, x, w)[0], x),
                           (lambda v: ag.add_rms_norm(x, v, w)[1], x), (lambda v: ag.embedding(t, v), table)):
            p, q = leaf.clone().requires_grad_(), leaf.clone().requires_grad_()
            torch.cat([a, call(p).flatten()]).float().square().sum().backward()
            call(q).float().square().sum().backward()
            assert torch.equal(p.grad, q.grad), way


# ---------------------------------------------------------------------------------------------- differentiated again
def test_second_derivatives_raise(monkeypatch):
    import torch
    from paper_2309_16669_amd import autograd as ag
    t, table, w = torch.arange(9, device="cuda") % 4, randn(1, (5, 64), BF), 1 + 0.1 * randn(2, (64,), FP)
    x, r = randn(3, (9, 64), BF), randn(4, (9, 64), FP)
    columns = randn(5, (64, 9), BF).t()
    square = lambda y: y.float().square().sum()
    cases = [(lambda a: square(ag.embedding(t, a)), [table]),
             (lambda a, b: ag.rms_norm(a, b).float().sum(), [x, w]),          # dy depends on nothing: the norm's own curvature
             (lambda a: ag.rms_norm(a, w).float().sum(), [columns]),          # an input that is laid out anew
             (lambda b: square(ag.rms_norm(x, b)), [w]),
             (lambda a, b, c: ag.add_rms_norm(a, b, c)[0].float().sum(), [x, r, w]),
             (lambda a: ag.add_rms_norm(a, r, w)[0].float().sum(), [x]),
             (lambda b: ag.add_rms_norm(x, b, w)[0].float().sum(), [r]),
             (lambda a, b: ag.add_rms_norm(a, b, w)[0].float().sum(), [x, x]),
             (lambda a: square(ag.add_rms_norm(a, r, w)[1]), [x])]
    for way in _both_ways(monkeypatch):
        for f, args in cases:
            leaves = [a.clone(memory_format=torch.preserve_format).requires_grad_() for a in args]
            first = torch.autograd.grad(f(*leaves), leaves)
            g = torch.autograd.grad(f(*leaves), leaves, create_graph=True)
            assert all(torch.equal(a, b) for a, b in zip(first, g)), way    # the first derivative alone is served
            penalty = sum(square(v) for v in g) + sum(v.float().sum() for v in leaves)
            with pytest.raises(RuntimeError, match="second derivative"):
                torch.autograd.grad(penalty, leaves, retain_graph=True)
            with pytest.raises(RuntimeError, match="second derivative"):
                penalty.backward()


def test_gradients_that_depend_on_nothing_carry_no_node(monkeypatch):
    import torch
    from paper_2309_16669_amd import autograd as ag
    t, table, w = torch.arange(9, device="cuda") % 4, randn(1, (5, 64), BF).requires_grad_(), (1 + 0.1 * randn(2, (64,), FP)).requires_grad_()
    x = randn(3, (9, 64), BF)
    for way in _both_ways(monkeypatch):
        # linear in the table, and in the gains
        for y, leaf in ((ag.embedding(t, table), table), (ag.rms_norm(x, w), w), (ag.add_rms_norm(x, x, w)[0], w)):
            (g,) = torch.autograd.grad(y, leaf, torch.ones_like(y), create_graph=True)
            assert not g.requires_grad, way
