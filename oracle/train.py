"""Oracle of the training operators around the FFN products: numpy, float64,
straight from the definitions. Shares nothing with the kernels.

  grouped        Z = X W_e^T on rows sorted by expert, Y = act(Z) or
                 act(Zg) Zu of Z's two halves
  grouped_grad   D = dY W_e; dX = D, or dZ of X = act(Z), act(Zg) Zu
  grouped_wgrad  dW_e = dY_e^T X_e
"""
from __future__ import annotations

import numpy as np

from oracle.ffn import act, act_grad


def expert_ranges(ends):
    """[(expert, first row, past the last)] of the experts that have rows."""
    first, out = 0, []
    for e, end in enumerate(ends):
        if end > first:
            out.append((e, first, int(end)))
        first = int(end)
    return out


def grouped(X, W, ends, kind, gated=False):
    """(Y, Z, sum |x w|) of the rows up to the last end."""
    used = int(ends[-1])
    Z, mag = np.zeros((used, W.shape[1])), np.zeros((used, W.shape[1]))
    for e, a, b in expert_ranges(ends):
        Z[a:b] = X[a:b] @ W[e].T
        mag[a:b] = np.abs(X[a:b]) @ np.abs(W[e]).T
    half = W.shape[1] // 2
    Y = act(Z[:, :half], kind) * Z[:, half:] if gated else act(Z, kind)
    return Y, Z, mag


def grouped_grad(dY, W, ends, kind, gated=False, Z=None):
    """(dX or dZ, D, sum |dy w|) of the rows up to the last end."""
    used = int(ends[-1])
    D, mag = np.zeros((used, W.shape[2])), np.zeros((used, W.shape[2]))
    for e, a, b in expert_ranges(ends):
        D[a:b] = dY[a:b] @ W[e]
        mag[a:b] = np.abs(dY[a:b]) @ np.abs(W[e])
    if gated:
        g, u = Z[:used, :W.shape[2]], Z[:used, W.shape[2]:]
        return np.concatenate([D * u * act_grad(g, kind), D * act(g, kind)], axis=1), D, mag
    return (D * act_grad(Z[:used], kind) if Z is not None else D), D, mag


def grouped_wgrad(dY, X, ends):
    """(dW, sum |dy x|)."""
    E = len(ends)
    dW, mag = np.zeros((E, dY.shape[1], X.shape[1])), np.zeros((E, dY.shape[1], X.shape[1]))
    for e, a, b in expert_ranges(ends):
        dW[e] = dY[a:b].T @ X[a:b]
        mag[e] = np.abs(dY[a:b]).T @ np.abs(X[a:b])
    return dW, mag
