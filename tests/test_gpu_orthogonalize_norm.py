"""ccl_orthogonalize on matrices whose norm, or its inverse, leaves fp32's
range: bounds as in test_gpu_orthogonalize, whose float64 simulation does not
depend on G's scale (X is the same but for the norm)."""
import numpy as np
import pytest
import torch

from oracle import ffn as OF
from paper_2606_11718_amd import ccl
from tests.test_gpu_orthogonalize import BF16, FP32, _close, _gradients, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("steps", [0, 5])
@pytest.mark.parametrize("g_type", [BF16, FP32])
def test_zeros_without_eps(g_type, steps):
    got, _ = _run(torch.zeros(2, 40, 70), g_type, eps=0.0, steps=steps)
    assert not got.any()


def test_one_zero_matrix_of_a_batch():
    G = _gradients(3, 3, 60, 90)
    G[1] = 0
    got, seen = _run(G, FP32, eps=0.0)
    assert not got[1].any()
    for i in (0, 2):
        _close(got[i], OF.orthogonalize(seen[i], eps=0.0))


@pytest.mark.parametrize("rows,cols", [(80, 120), (120, 80)])
@pytest.mark.parametrize("scale", [1e-36, 1e-38, 1e-40])
def test_tiny_norms_without_eps(scale, rows, cols):
    """The inverse of the norm past fp32's largest; at 1e-40 every element of G is
    a subnormal, which the oracle sees as the library does."""
    G = (_gradients(4, 1, rows, cols, 1.0).double() * scale).float()
    assert G.any()
    got, seen = _run(G, FP32, eps=0.0)
    _close(got[0], OF.orthogonalize(seen[0], eps=0.0))


def test_largest_norm():
    """Elements near fp32's largest, whose norm is past it."""
    G = _gradients(5, 1, 300, 700, 1.0)
    G = (G.double() * (3e38 / G.abs().max().item())).float()
    got, seen = _run(G, FP32, eps=0.0)
    _close(got[0], OF.orthogonalize(seen[0], eps=0.0))


def test_the_same_bits_at_every_scale():
    """Powers of two scale G without rounding: X, and so the result, is the same."""
    G = _gradients(6, 1, 130, 200, 1.0)
    got = [_run(G * 2.0 ** e, FP32, eps=0.0)[0] for e in (0, -100, 100)]
    assert all(np.array_equal(got[0], g) for g in got[1:])
