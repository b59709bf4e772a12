"""The vocabulary loss and its gradients with logits of -inf, and with rows that hold
NaN, in small launches and where 256x256 tiles and smaller ones behind them share the
vocabulary (tests/train_forms.py). Tolerances as in test_gpu_cross_entropy, over the
columns that are not masked.
"""
import numpy as np
import pytest
import torch

from oracle import train as OT
from paper_2606_11718_amd import ccl
from tests import test_gpu_cross_entropy as TC
from tests import train_forms as F

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
LARGE = F.LOGITS_REST[64][0]
# (tokens, hidden, vocab, masked columns): whole tiles of each launch, and parts of tiles
CASES = [(70, 64, 700, [*range(256), *range(300, 310)]),
         (*LARGE, [*range(256, 512), *range(1000, 1010), *range(16384, 16512), *range(16690, 16701)])]


def _call(x, w, t, weights):
    (tokens, D), V = x.shape, w.shape[0]
    head = ccl.ccl_vocab(hidden=D, vocab=V)
    ws = torch.empty(ccl.ccl_cross_entropy_workspace(head, tokens, grad=True), dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty(V, D, device="cuda")
    ccl.ccl_cross_entropy_grad(head, tokens, x, w, t, loss, dx, dw, lse=lse, dloss=weights, workspace=ws, workspace_bytes=ws.numel())
    return loss, lse, dx, dw


def _f64(t):
    return t.double().cpu().numpy()


def _inputs(tokens, D, V, masked, at_x, at_w):
    """x[:, 0] = at_x and w[masked, 0] = at_w, whose product is -inf; w[:, 0] is 0 elsewhere. Some tokens do not count."""
    gen = torch.Generator(device="cuda").manual_seed(31)
    x = torch.randn(tokens, D, generator=gen, device="cuda").to(BF)
    w = (torch.randn(V, D, generator=gen, device="cuda") * 0.05).to(BF)
    x[:, 0], w[:, 0] = at_x, 0.0
    w[masked, 0] = at_w
    live = np.setdiff1d(np.arange(V), masked)
    t = torch.from_numpy(live).cuda()[torch.randint(0, len(live), (tokens,), generator=gen, device="cuda")]
    t[3::7] = -100
    weights = (torch.rand(tokens, generator=gen, device="cuda") + 0.5) / tokens
    return x, w, t, weights, live


def _check(x, w, t, weights, live, out, columns):
    loss, lse, dx, dw = out
    V, D = w.shape
    tokens = x.shape[0]
    xv, wv, g = _f64(x), _f64(w)[live], _f64(weights)
    t = t.cpu().numpy()
    counts = t >= 0
    lw, sw, z, P = OT.cross_entropy(xv, wv, np.where(counts, np.searchsorted(live, t), -100), 1.0, g)
    dz = (D * TC.F32 * (np.abs(xv) @ np.abs(wv).T) + TC.F32 * np.abs(z)).max(axis=1)
    dlse = dz + TC.F32 * (100 + np.abs(sw))
    assert (np.abs(_f64(lse) - sw) <= dlse).all() and (np.abs(_f64(loss) - lw) <= 2 * dlse).all()
    assert (_f64(loss)[~counts] == 0).all()
    err = (2 * TC.B16 + 2.0 ** -15 + dz + dlse)[:, None] * np.abs(P)
    rows = np.flatnonzero(counts)
    err[rows, np.searchsorted(live, t[rows])] += (dz + dlse)[rows] * g[rows]
    got, want = _f64(dx)[:, columns], (P @ wv)[:, columns]
    tol = (err @ np.abs(wv) + V * TC.F32 * (np.abs(P) @ np.abs(wv)))[:, columns]
    assert (np.abs(got - want) <= tol * 1.01 + TC.B16 * np.abs(want) + 1e-38).all()
    assert (got[~counts] == 0).all()
    got, want = _f64(dw), P.T @ xv
    tol = err.T @ np.abs(xv) + tokens * TC.F32 * (np.abs(P).T @ np.abs(xv))
    assert (np.abs(got[live] - want) <= tol * 1.01).all()
    assert (np.delete(got, live, axis=0) == 0).all()


@pytest.mark.parametrize("tokens,D,V,masked", CASES, ids=["small", "large"])
def test_gradients_of_logits_that_overflow(tokens, D, V, masked):
    """-2^200 from finite operands: -inf in fp32. Such columns are terms of 0, in both gradients too."""
    x, w, t, weights, live = _inputs(tokens, D, V, masked, 2.0 ** 100, -2.0 ** 100)
    _check(x, w, t, weights, live, _call(x, w, t, weights), np.arange(D))


@pytest.mark.parametrize("tokens,D,V,masked", CASES, ids=["small", "large"])
def test_weights_of_minus_infinity(tokens, D, V, masked):
    """Loss, dW and the other columns of dX are what they are without the masked rows; the column of dX that sums
    0 * -inf is NaN in every row."""
    x, w, t, weights, live = _inputs(tokens, D, V, masked, 1.0, float("-inf"))
    out = _call(x, w, t, weights)
    assert bool(torch.isnan(out[2][:, 0]).all())
    _check(x, w, t, weights, live, out, np.arange(1, D))


def test_a_bad_row_stays_its_own():
    tokens, D, V = LARGE
    t = np.arange(tokens, dtype=np.int64) * 16
    t[7] = -1

    def bad(x, w):
        x[5] = float("nan")
    clean = TC.run(tokens, D, V, grad=True, targets=t)
    loss, lse, dx, dw = TC.run(tokens, D, V, grad=True, targets=t, mutate=bad)
    others = [i for i in range(tokens) if i != 5]
    assert bool(torch.isnan(loss[5])) and bool(torch.isnan(lse[5])) and bool(torch.isnan(dx[5]).all())
    for a, b in zip((loss[:tokens], lse[:tokens], dx), (clean[0][:tokens], clean[1][:tokens], clean[2][:tokens, :D])):
        assert torch.equal(a[others], b[others])
    assert bool(torch.isnan(dw).all())


@pytest.mark.parametrize("fill", [float("nan"), float("inf")])
def test_padding_tokens_reach_no_gradient(fill):
    tokens, D, V = LARGE
    t = np.arange(tokens, dtype=np.int64) * 16
    off = [3, 64, 300, 511, 768, tokens - 1]
    t[off] = -100

    def bad(x, w):
        x[off] = fill
    clean = TC.run(tokens, D, V, grad=True, targets=t)
    loss, _, dx, dw = TC.run(tokens, D, V, grad=True, targets=t, mutate=bad)
    assert torch.equal(loss, clean[0]) and torch.equal(dx, clean[2][:tokens, :D]) and torch.equal(dw, clean[3][:V, :D])
