"""Oracle of the FFN operators around the GEMM: numpy, float64, straight from
the definitions. Shares nothing with the kernels.

  linear       Z = alpha A B + bias; C = act(Z) + beta R, or gated
               C = act(Zg) Zu + beta R with gate and up columns alternating in
               groups of 16
  linear_grad  dZ = (alpha A B) act'(Z), gated dZg = D Zu act'(Zg),
               dZu = D act(Zg); and its column sums
  route, moe   softmax routing with the lowest expert first among equals, and
               the weighted sum of the chosen experts' gated FFNs
  orthogonalize  Newton-Schulz steps X <- a X + (b S + c S S) X, S = X X^T
"""
from __future__ import annotations

import numpy as np

NONE, RELU, GELU, SILU = 0, 1, 2, 3
GROUP = 16
QUINTIC = (3.4445, -4.7750, 2.0315)


def act(z, kind: int):
    z = np.asarray(z, np.float64)
    if kind == RELU:
        return np.where(z < 0, 0.0, z)
    if kind == GELU:
        return 0.5 * z * (1 + np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)))
    if kind == SILU:
        return z * (0.5 * (1 + np.tanh(0.5 * z)))
    return z.copy()


def act_grad(z, kind: int):
    z = np.asarray(z, np.float64)
    if kind == RELU:
        return np.where(z > 0, 1.0, 0.0)
    if kind == GELU:
        k = np.sqrt(2 / np.pi)
        t = np.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    if kind == SILU:
        s = 0.5 * (1 + np.tanh(0.5 * z))
        return s + z * s * (1 - s)
    return np.ones_like(z)


def split_gated(z):
    """Gate and up columns of an interleaved matrix."""
    g = z.reshape(z.shape[0], -1, 2, GROUP)
    return g[:, :, 0].reshape(z.shape[0], -1), g[:, :, 1].reshape(z.shape[0], -1)


def join_gated(gate, up):
    """The interleaved matrix of gate and up columns."""
    m = gate.shape[0]
    return np.stack([gate.reshape(m, -1, GROUP), up.reshape(m, -1, GROUP)], axis=2).reshape(m, -1)


def linear(A, B, kind, gated=False, bias=None, residual=None, beta=1.0, alpha=1.0, rows=None):
    """(C, Z), rows at and past `rows` zero."""
    Z = alpha * (A @ B)
    if bias is not None:
        Z = Z + bias
    if gated:
        g, u = split_gated(Z)
        C = act(g, kind) * u
    else:
        C = act(Z, kind)
    if residual is not None:
        C = C + beta * residual
    if rows is not None:
        Z, C = Z.copy(), C.copy()
        Z[rows:] = 0
        C[rows:] = 0
    return C, Z


def linear_grad(A, B, Z, kind, gated=False, alpha=1.0, rows=None):
    """(dZ, its column sums)."""
    D = alpha * (A @ B)
    if gated:
        g, u = split_gated(Z)
        dZ = join_gated(D * u * act_grad(g, kind), D * act(g, kind))
    else:
        dZ = D * act_grad(Z, kind)
    if rows is not None:
        dZ = dZ.copy()
        dZ[rows:] = 0
    return dZ, dZ.sum(0)


def route(logits, top_k, normalize):
    """(ids, probs) of each token: the top_k largest logits, the lowest expert
    first among equals. Logits of -inf and NaN are never chosen: id -1, probability 0."""
    logits = np.asarray(logits, np.float64)
    T, E = logits.shape
    ids = np.full((T, top_k), -1, np.int32)
    probs = np.zeros((T, top_k))
    for t in range(T):
        ok = [e for e in range(E) if not np.isnan(logits[t, e]) and logits[t, e] != -np.inf]
        order = sorted(ok, key=lambda e: (-logits[t, e], e))[:top_k]
        if not order:
            continue
        top = logits[t, order[0]]
        # equal to the largest, infinite or not: weight 1
        w = np.array([1.0 if logits[t, e] == top else np.exp(logits[t, e] - top) for e in (order if normalize else ok)])
        chosen = w if normalize else np.array([1.0 if logits[t, e] == top else np.exp(logits[t, e] - top) for e in order])
        ids[t, :len(order)] = order
        probs[t, :len(order)] = chosen / w.sum()
    return ids, probs


def moe(x, logits, gate_up, down, top_k, kind, normalize, gate_up_scale=None, down_scale=None):
    """(y, ids, probs). gate_up: (E, 2F, D), gate rows first; down: (E, D, F)."""
    ids, probs = route(logits, top_k, normalize)
    F = down.shape[2]
    y = np.zeros((x.shape[0], down.shape[1]))
    for t in range(x.shape[0]):
        for e, p in zip(ids[t], probs[t]):
            if e < 0:
                continue
            z = gate_up[e] @ x[t]
            if gate_up_scale is not None:
                z = z * gate_up_scale[e]
            v = down[e] @ (act(z[:F], kind) * z[F:])
            if down_scale is not None:
                v = v * down_scale[e]
            y[t] += p * v
    return y, ids, probs


def orthogonalize(G, steps=5, coeffs=QUINTIC, eps=1e-7):
    a, b, c = coeffs
    X = np.asarray(G, np.float64)
    X = X / (np.sqrt((X * X).sum()) + eps)
    tall = X.shape[0] > X.shape[1]
    if tall:
        X = X.T
    for _ in range(steps):
        S = X @ X.T
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.T if tall else X
