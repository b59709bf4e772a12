"""Oracle of the training operators around the FFN products: numpy, float64,
straight from the definitions. Shares nothing with the kernels.

  grouped        Z = X W_e^T on rows sorted by expert, Y = act(Z) or
                 act(Zg) Zu of Z's two halves
  grouped_grad   D = dY W_e; dX = D, or dZ of X = act(Z), act(Zg) Zu
  grouped_wgrad  dW_e = dY_e^T X_e
  cross_entropy  lse, loss and P = g scale (softmax(scale X W^T) - one-hot)
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


def cross_entropy(X, W, targets, scale=1.0, g=None):
    """(loss, lse, z, P) of rows X against the rows of W; P is None without token weights g."""
    z = scale * (X @ W.T)
    top = z.max(axis=1, keepdims=True)
    lse = (top + np.log(np.exp(z - top).sum(axis=1, keepdims=True)))[:, 0]
    live = (targets >= 0) & (targets < W.shape[0])
    rows = np.arange(len(targets))
    t = np.where(live, targets, 0)
    loss = np.where(live, lse - z[rows, t], 0.0)
    if g is None:
        return loss, lse, z, None
    P = np.exp(z - lse[:, None])
    P[rows, t] = np.expm1(z[rows, t] - lse)
    return loss, lse, z, P * (np.where(live, g, 0.0) * scale)[:, None]


# ---- AdamW ----

BLOCK = 128
REACH, BIAS = {4: 7, 5: 14}, {4: 7, 5: 16}     # of moments with 4 (and a sign) and 5 exponent bits


def adamw(p, g, m, v, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=1.0):
    """(p, m, v) after one step."""
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    hat = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p - lr * weight_decay * p - lr * hat, m, v


def moment_values(exponent_bits):
    """What the 256 codes stand for, before their block's scale."""
    out = np.empty(256)
    for c in range(256):
        field, part = (c & 127 if exponent_bits == 4 else c) >> 3, c & 7
        bias = BIAS[exponent_bits]
        out[c] = (8 + part) * 2.0 ** (field - bias - 3) if field else part * 2.0 ** (-bias - 2)
        if exponent_bits == 4 and c & 128:
            out[c] = -out[c]
    for c in ([0x7F, 0xFF] if exponent_bits == 4 else [0xFF]):
        out[c] = np.nan
    return out


def moment_decode(codes, scales, exponent_bits):
    top = np.maximum(scales.astype(np.int64), REACH[exponent_bits] + 1)
    factor = np.exp2((top - 127 - REACH[exponent_bits]).astype(np.float64))
    return moment_values(exponent_bits)[codes] * np.repeat(factor, BLOCK)[:len(codes)]


def v_taken(m_codes, v_codes):
    """v's codes as they are read beside m's: no 0 under an m that is not."""
    return np.where((v_codes == 0) & ((m_codes & 0x7F) != 0), 1, v_codes).astype(np.uint8)


def chances(n, step):
    """32 bits an element, of its place and the step."""
    i = np.arange(n, dtype=np.uint64)
    mask = np.uint64(0xFFFFFFFF)
    h = (i + ((i >> np.uint64(32)) << np.uint64(7))) & mask
    h = (h * np.uint64(0x9E3779B1) + np.uint64(step * 0x3C6EF373 & 0xFFFFFFFF)) & mask
    h ^= h >> np.uint64(16)
    h = (h * np.uint64(0x6A09E667)) & mask
    h ^= h >> np.uint64(13)
    h = (h * np.uint64(0xBB67AE85)) & mask
    return (h ^ (h >> np.uint64(16))).astype(np.int64)


def moment_encode(x, chance, exponent_bits):
    """(codes, scales) of fp32 values, rounded up where the fraction of a step and chance / 65536 reach 1."""
    n = len(x)
    x = np.concatenate([x, np.zeros(-n % BLOCK)]).astype(np.float64)
    chance = np.concatenate([chance, np.zeros(-n % BLOCK, np.int64)])
    finite = np.isfinite(x)
    a = np.where(finite, np.abs(x), 0.0).reshape(-1, BLOCK)
    reach, bias = REACH[exponent_bits], BIAS[exponent_bits]
    big = a.max(axis=1)
    # the biased exponent of fp32, 0 below its normal range
    top = np.where(big >= 2.0 ** -126, np.floor(np.log2(np.where(big > 0, big, 1.0))) + 127, 0).astype(np.int64)
    top = np.where((top > 0) & (np.exp2((top - 127).astype(np.float64)) > big), top - 1, top)
    top = np.maximum(top, reach + 1)
    y = a * np.exp2((reach + 127 - top).astype(np.float64))[:, None]
    low = 1 - bias
    e = np.maximum(np.where(y > 0, np.floor(np.log2(np.where(y > 0, y, 1.0))), low), low).astype(np.int64)
    steps = y * np.exp2((3 - e).astype(np.float64))
    assert (steps < 16).all()
    # the sum is fp32's
    k = np.floor((steps.astype(np.float32) + (chance.reshape(-1, BLOCK) / 65536).astype(np.float32))).astype(np.int64)
    code = (k + ((e - low) << 3)).reshape(-1)
    if exponent_bits == 4:
        code = np.where(x < 0, code | 128, code)
        code = np.where(finite, code, 0x7F | np.where(x < 0, 128, 0))
    else:
        code = np.where(finite, code, 0xFF)
    return code[:n].astype(np.uint8), top.astype(np.uint8)
