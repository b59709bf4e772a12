"""Rows of a ragged call's operands past the valid ones: what they hold reaches
no gradient and no weight (the bits of a call on zeros)."""
import pytest
import torch

from paper_2606_11718_amd import ffn

pytestmark = pytest.mark.gpu

M, D, F = 512, 256, 384


def _operands(rows, fill):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(M, D, generator=gen, device="cuda").bfloat16()
    dy = torch.randn(M, D, generator=gen, device="cuda").mul_(0.01).bfloat16()
    target = torch.randn(M, D, generator=gen, device="cuda").bfloat16()
    for t in (x, dy, target):
        t[rows:] = fill
    return x, dy, target


@pytest.mark.parametrize("fill", [float("nan"), float("inf")])
@pytest.mark.parametrize("rows", [0, 1, 389])
def test_gradients(rows, fill):
    got = []
    for f in (0.0, fill):
        net = ffn.GatedFFN(M, D, F)
        x, dy, _ = _operands(rows, f)
        y, h, z = net.forward(x, rows)
        got.append(net.backward(x, h, z, dy, rows))
        assert x[rows:].isnan().any() or f == f            # the caller's x is as it was
    assert all(torch.equal(a, b) and a.isfinite().all() for a, b in zip(*got))


def test_step():
    got = []
    for f in (0.0, float("nan")):
        net = ffn.GatedFFN(M, D, F)
        x, _, target = _operands(300, f)
        loss = net.step(x, target, 0.02, rows=300)
        got.append((loss, net.w_up, net.w_down))
    assert got[0][0] == got[1][0]
    assert torch.equal(got[0][1], got[1][1]) and torch.equal(got[0][2], got[1][2])
