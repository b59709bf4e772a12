"""The FFN operators' oracle against differences, torch's autograd in float64
and hand-made cases (CPU)."""
import numpy as np
import pytest
import torch

from oracle import ffn as OF

KINDS = [OF.NONE, OF.RELU, OF.GELU, OF.SILU]


@pytest.mark.parametrize("kind", KINDS)
def test_activation_gradient_against_differences(kind):
    z = np.concatenate([np.linspace(-9, 9, 4001), [-60.0, 60.0]]) + 1e-3 * np.sqrt(2)
    h = 1e-5
    diff = (OF.act(z + h, kind) - OF.act(z - h, kind)) / (2 * h)
    # central differences: h^2 / 6 of the third derivative (below 2) and the
    # rounding of the values over 2 h
    assert np.abs(diff - OF.act_grad(z, kind)).max() < 2 * h * h + 60 * 2.3e-16 / h + 1e-10


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("gated", [False, True])
def test_linear_grad_against_differences(kind, gated):
    """Loss sum(W * C(Z)) with D = W: its differences in Z are dZ."""
    rng = np.random.default_rng(3)
    M, N = 5, 64
    Z = rng.standard_normal((M, N))
    W = rng.standard_normal((M, N // 2 if gated else N))
    eye = np.eye(W.shape[1])

    def loss(z):
        if gated:
            g, u = OF.split_gated(z)
            return (W * OF.act(g, kind) * u).sum()
        return (W * OF.act(z, kind)).sum()

    dZ, dbias = OF.linear_grad(W, eye, Z, kind, gated)
    h = 1e-5
    for i, j in [(0, 0), (1, 15), (2, 16), (3, 31), (4, 63), (2, 40)]:
        E = np.zeros_like(Z)
        E[i, j] = h
        assert abs((loss(Z + E) - loss(Z - E)) / (2 * h) - dZ[i, j]) < 1e-8
    assert np.allclose(dbias, dZ.sum(0), rtol=0, atol=1e-13)


def test_activations_equal_torch():
    z = torch.linspace(-8, 8, 1001, dtype=torch.float64)
    n = z.numpy()
    assert np.allclose(OF.act(n, OF.GELU), torch.nn.functional.gelu(z, approximate="tanh").numpy(), atol=1e-14)
    assert np.allclose(OF.act(n, OF.SILU), torch.nn.functional.silu(z).numpy(), atol=1e-14)


def test_gated_columns_round_trip():
    z = np.arange(3 * 96, dtype=np.float64).reshape(3, 96)
    g, u = OF.split_gated(z)
    assert np.array_equal(g[0, :17], list(range(16)) + [32])
    assert np.array_equal(u[0, :17], list(range(16, 32)) + [48])
    assert np.array_equal(OF.join_gated(g, u), z)


def test_route_ties_and_masks():
    inf = np.inf
    ids, probs = OF.route(np.array([[1.0, 2.0, 2.0, 0.0], [-inf, 3.0, -inf, np.nan], [-inf] * 4, [0.0] * 4]), 2, True)
    assert ids.tolist() == [[1, 2], [1, -1], [-1, -1], [0, 1]]
    assert np.allclose(probs, [[0.5, 0.5], [1, 0], [0, 0], [0.5, 0.5]])
    _, probs = OF.route(np.zeros((1, 4)), 2, False)
    assert np.allclose(probs, 0.25)


def test_orthogonalize_brings_singular_values_near_one():
    rng = np.random.default_rng(5)
    for shape in ((40, 70), (70, 40), (32, 32)):
        s = np.linalg.svd(OF.orthogonalize(rng.standard_normal(shape)), compute_uv=False)
        assert s.max() < 1.25 and np.median(s) > 0.65
    assert not OF.orthogonalize(np.zeros((3, 5))).any()
