"""The operators together, as paper_2606_11718_amd.ffn runs them: a training step's
gradients against float64 autograd, the loss going down, and decoding."""
import pytest
import torch

from oracle import ffn as OF
from paper_2606_11718_amd import ccl, ffn

pytestmark = pytest.mark.gpu


def _reference(net, x, dy):
    """dW_up, dW_down of sum(dy * Y) in float64 from the same bf16 weights."""
    wu = net.w_up16.double().cpu().requires_grad_()
    wd = net.w_down16.double().cpu().requires_grad_()
    z = x.double().cpu() @ wu
    g = z.view(z.shape[0], -1, 2, ffn.GROUP)
    gate, up = g[:, :, 0].reshape(z.shape[0], -1), g[:, :, 1].reshape(z.shape[0], -1)
    h = torch.nn.functional.silu(gate) * up
    y = x.double().cpu() + h @ wd
    (y * dy.double().cpu()).sum().backward()
    return y.detach(), wu.grad, wd.grad


@pytest.mark.parametrize("rows", [512, 389])
def test_gradients_of_a_step(rows):
    torch.manual_seed(0)
    net = ffn.GatedFFN(512, 256, 384)
    x = torch.randn(512, 256, device="cuda").bfloat16()
    dy = torch.randn(512, 256, device="cuda").mul_(0.01).bfloat16()
    dy[rows:] = 0
    y, h, z = net.forward(x, rows)
    gu, gd = net.backward(x, h, z, dy, rows)
    yw, guw, gdw = _reference(net, x, dy)
    assert not y[rows:].any() and not h[rows:].any()
    # bf16 results (1.7e-3 in the 2-norm each) of one rounding of h (y, dW_down),
    # z and dz (dW_up): at most three of them add up
    for got, want, bound in ((y[:rows], yw[:rows], 4e-3), (gd, gdw, 4e-3), (gu, guw, 6e-3)):
        off = (got.double().cpu() - want).norm() / want.norm()
        assert off <= bound, off


def test_training_goes_down():
    torch.manual_seed(1)
    x = torch.randn(256, 256, device="cuda").bfloat16()
    target = x + 0.5 * torch.tanh(x.roll(3, 1))
    net = ffn.GatedFFN(256, 256, 512)
    losses = [net.step(x, target, 0.02, rows=200) for _ in range(12)]
    assert losses[-1] < 0.6 * losses[0], losses


def test_decode():
    layer = ffn.MoELayer(256, 64, 16, 4)
    x = torch.randn(7, 256, device="cuda").bfloat16()
    y, ids, probs = layer.decode(x)
    d = lambda t: t.double().cpu().numpy()  # noqa: E731
    logits = (x.float() @ layer.router).cpu().numpy()
    want, iw, pw = OF.moe(d(x), logits, d(layer.gate_up), d(layer.down), 4, ccl.CCL_ACT_SILU, True)
    assert (ids.cpu().numpy() == iw).all()
    got = d(y)
    assert ((got - want) ** 2).sum() ** 0.5 <= 2.0 ** -8 * (want ** 2).sum() ** 0.5
