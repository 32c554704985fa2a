"""Pins of oracle/text_ops.py to things other than itself: hand-worked rows, central differences of every input coordinate,
torch's conversion to e4m3 and a dense library computation.  Runs on the CPU."""
import numpy as np
import pytest

from oracle import text_ops as ops


def test_embedding_by_hand():
    W = np.array([[1.0, 2.0], [3.0, 5.0], [-1.0, 0.5]])
    t = np.array([2, 0, 2, -1, 3, 2])
    assert np.array_equal(ops.embedding_fwd(t, W, 2.0), [[-2, 1], [2, 4], [-2, 1], [0, 0], [0, 0], [-2, 1]])
    dy = np.arange(12.0).reshape(6, 2)
    dw, mag = ops.embedding_bwd(t, dy, 3, 2.0)
    assert np.array_equal(dw, [[4, 6], [0, 0], [28, 34]]) and np.array_equal(mag, np.abs(dw))


def test_embedding_gradient_is_the_derivative():
    rng = np.random.default_rng(3)
    W, t, dy = rng.normal(size=(5, 3)), rng.integers(-1, 6, size=11), rng.normal(size=(11, 3))
    dw, _ = ops.embedding_bwd(t, dy, 5, 1.7)
    for v in range(5):
        for c in range(3):
            d = np.zeros_like(W)
            d[v, c] = 0.5
            num = ((ops.embedding_fwd(t, W + d, 1.7) - ops.embedding_fwd(t, W - d, 1.7)) * dy).sum()
            assert abs(num - dw[v, c]) < 1e-12   # linear: differences are exact


def test_norm_by_hand():
    # mean(h^2) = (9 + 16) / 2 = 12.5, eps 3.5: rstd 1/4; g = dy w = (2, -3), xhat = (3/4, 1): mean(g xhat) = -3/4
    y, r = ops.rms_fwd([[3.0, 4.0]], [2.0, 3.0], 3.5)
    assert np.allclose(r, 0.25, rtol=1e-15) and np.allclose(y, [[1.5, 3.0]], rtol=1e-15)
    d, dw = ops.rms_bwd([[3.0, 4.0]], [2.0, 3.0], [[1.0, -1.0]], [[10.0, 20.0]], 3.5)
    assert np.allclose(d, [[10 + (2 + 9 / 16) / 4, 20 + (-3 + 3 / 4) / 4]], rtol=1e-15)
    assert np.allclose(dw, [0.75, -1.0], rtol=1e-15)


@pytest.mark.parametrize("M,D", [(1, 1), (3, 5), (2, 16)])
def test_norm_gradient_is_the_derivative(M, D):
    rng = np.random.default_rng(M * 10 + D)
    h, w, dy, dh = rng.normal(size=(M, D)), 1 + 0.1 * rng.normal(size=D), rng.normal(size=(M, D)), rng.normal(size=(M, D))
    loss = lambda h_, w_: (ops.rms_fwd(h_, w_, 1e-3)[0] * dy + h_ * dh).sum()
    d, dw = ops.rms_bwd(h, w, dy, dh, 1e-3)
    e, eps = 1e-5, 1e-3
    for m in range(M):
        # a central difference is off by e^2 / 6 of the third derivative at most: along one coordinate, with s = h_c / sqrt(D)
        # and a = eps + the rest of the mean square, y_c is sqrt(D) s / (s^2 + a)^(1/2) and the others h_d (s^2 + a)^(-1/2)
        # with |h_d| <= sqrt(D a); the third derivatives of u / (u^2 + 1)^(1/2) and of (u^2 + 1)^(-1/2) stay within 3, so
        # with h_c = sqrt(D) s each is within 3 a^(-3/2) / D <= 3 eps^(-3/2)
        off = 1e-8 + e ** 2 / 2 * eps ** -1.5 * np.abs(dy[m] * w).sum()
        for c in range(D):
            p = np.zeros_like(h)
            p[m, c] = e
            assert abs((loss(h + p, w) - loss(h - p, w)) / (2 * e) - d[m, c]) < off
    for c in range(D):
        p = np.zeros_like(w)
        p[c] = e
        assert abs((loss(h, w + p) - loss(h, w - p)) / (2 * e) - dw[c]) < 1e-8


def test_e4m3_is_the_library_format():
    import torch
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(every[:0x7f], ops.e4m3_values()) and np.isnan(every[0x7f]) and np.array_equal(every[0x80:0xff], -every[:0x7f])
    rng = np.random.default_rng(5)
    v = np.concatenate([rng.normal(size=20000) * 2.0 ** rng.integers(-12, 8, size=20000), every[:0x7f],
                        (every[:0x7e] + every[1:0x7f]) / 2, [447.9, 448.0, 463.9]]).astype(np.float32)
    v = v[np.abs(v) < 464]
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ops.e4m3(v.astype(np.float64)), want)
    assert np.all(np.abs(want - v) <= ops.e4m3_half_step(v))


def test_rows8_and_product():
    q, s = ops.rows8([[0.0, 0.0], [-3.5, 1.75], [1e-40, 0.0]])
    assert np.array_equal(s, [2.0 ** -96 / 448, 3.5 / 448, 2.0 ** -96 / 448])
    assert np.array_equal(q, [[0, 0], [-448, 224], [0, 0]])
    import torch
    rng = np.random.default_rng(6)
    x, w, b = rng.normal(size=(5, 7)), rng.normal(size=(3, 7)), rng.normal(size=3)
    sx, sw = rng.uniform(size=5), rng.uniform(size=3)
    y, mag = ops.linear(x, sx, w, sw, b)
    want = torch.nn.functional.linear(torch.from_numpy(x * sx[:, None]), torch.from_numpy(w * sw[:, None]), torch.from_numpy(b))
    assert np.allclose(y, want.numpy(), atol=1e-13) and np.all(mag >= np.abs(y - b) - 1e-13)
