"""The training operators' oracle against differences and by hand."""
import numpy as np
import pytest

from oracle import train as OT


def _slope(f, x, d, h=1e-6):
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


@pytest.mark.parametrize("kind,gated", [(0, False), (1, False), (2, False), (3, True), (2, True)])
def test_grouped_gradients_are_differences(kind, gated):
    """Through X = f(Z), Y = X W_e^T: the gradient to Z and to W along random directions."""
    rng = np.random.default_rng(3)
    ends, K, N = [3, 3, 8], 4, 6
    Z = rng.standard_normal((8, 2 * K if gated else K))
    W, dY = rng.standard_normal((3, N, K)), rng.standard_normal((8, N))
    eye = np.broadcast_to(np.eye(Z.shape[1]), (3, Z.shape[1], Z.shape[1]))
    inner = lambda z: OT.grouped(z, eye, ends, kind, gated)[0]  # noqa: E731
    loss = lambda z, w: float((OT.grouped(inner(z), w, ends, 0)[0] * dY).sum())  # noqa: E731
    dZ, _, _ = OT.grouped_grad(dY, W, ends, kind, gated, Z if (kind or gated) else None)
    d = rng.standard_normal(Z.shape)
    assert abs(_slope(lambda z: loss(z, W), Z, d) - (dZ * d).sum()) < 1e-6 * np.abs(dZ).sum()
    dW, _ = OT.grouped_wgrad(dY, inner(Z), ends)
    d = rng.standard_normal(W.shape)
    assert abs(_slope(lambda w: loss(Z, w), W, d) - (dW * d).sum()) < 1e-6 * np.abs(dW).sum()
    assert (dW[1] == 0).all()


def test_cross_entropy_gradients_are_differences():
    rng = np.random.default_rng(4)
    X, W, t = rng.standard_normal((5, 6)), rng.standard_normal((9, 6)), np.array([0, 8, -100, 9, 4])
    g = rng.random(5) + 0.5
    total = lambda x, w: float((OT.cross_entropy(x, w, t, 0.7)[0] * g).sum())  # noqa: E731
    loss, lse, z, P = OT.cross_entropy(X, W, t, 0.7, g)
    assert loss[2] == loss[3] == 0 and (P[[2, 3]] == 0).all()
    d = rng.standard_normal(X.shape)
    assert abs(_slope(lambda x: total(x, W), X, d) - ((P @ W) * d).sum()) < 1e-6
    d = rng.standard_normal(W.shape)
    assert abs(_slope(lambda w: total(X, w), W, d) - ((P.T @ X) * d).sum()) < 1e-6


@pytest.mark.parametrize("bits", [4, 5])
def test_moment_formats(bits):
    values = OT.moment_values(bits)
    positive = values[:128 if bits == 4 else 256]
    positive = positive[np.isfinite(positive)]
    assert (np.diff(positive) > 0).all() and positive[0] == 0
    # a block whose largest value sets the scale: every value up to it comes back as itself
    biggest = 1.5 * 2.0 ** OT.REACH[bits]
    values = positive[positive <= biggest]
    for i in range(0, len(values), 127):
        block = np.concatenate([[biggest], values[i:i + 127]])
        got, scale = OT.moment_encode(block, np.zeros(len(block), np.int64), bits)
        assert np.array_equal(OT.moment_decode(got, scale, bits), block)


@pytest.mark.parametrize("bits", [4, 5])
def test_random_rounding_is_fair(bits):
    """A value's codes are its two neighbours, as often as their distance asks: a mean of n draws of one of two values a
    step s apart is within 4 s / (2 sqrt n) of it (4 standard deviations)."""
    n = 128 * 512
    x = np.full(n, 0.3)
    x[::128] = 1.0
    got = OT.moment_decode(*OT.moment_encode(x, OT.chances(n, 7) & 0xFFFF, bits), bits)
    body = got.reshape(-1, 128)[:, 1:].reshape(-1)
    step = 2.0 ** -2 / 8
    assert set(np.unique(body)) == {0.28125, 0.3125}
    assert abs(body.mean() - 0.3) < 2 * step / np.sqrt(len(body))


def test_v_taken():
    """Only a v of 0 under a live m is another code, its smallest."""
    m, v = np.meshgrid(np.arange(256, dtype=np.uint8), np.arange(256, dtype=np.uint8))
    got = OT.v_taken(m.ravel(), v.ravel()).reshape(m.shape)
    live = (m != 0) & (m != 128)
    assert (got[(v == 0) & live] == 1).all() and np.array_equal(got[(v > 0) | ~live], v[(v > 0) | ~live])
