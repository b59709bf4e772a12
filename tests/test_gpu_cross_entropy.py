"""GPU parity of the vocabulary loss and its gradients with the fp64 oracle.

A logit carries dz = |scale| hidden 2^-23 sum |x w| + 2^-23 |z|. The sum of
exponentials: arguments (z - m) log2 e with two roundings and a 1-ulp
exponential change a term by 2^-23 (|z - m| + 2) of itself, which weighted with p
is at most 2^-23 (log V + 2); a term passes at most 32 + 6 additions in its tile
and V / (128 64) + 6 behind it (2^-24 each). So lse is within dz + 2^-23 (100 +
|lse|) for the sizes here, the loss within twice that.

P is rounded twice (2^-8 each), the target's once, and carries the errors of z
and lse: each gradient is within (2^-7 + 2^-15 + dz + dlse) sum |P| |w| (the
target's P moves by (dz + dlse) |g scale| p_t as well), its sum's n 2^-23 of the
same, and its own rounding. Those bounds count every rounding at its worst and
with one sign; roundings are spread evenly over half a step instead, so that the
2-norm of the error is below sqrt(2 (2^-8 / sqrt 3)^2 + (2^-8 / sqrt 3)^2) = 3.9e-3
of the result where terms do not cancel; 6e-3 is asked for.
"""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import gemm as OG
from oracle import train as OT
from paper_2606_11718_amd import ccl

pytestmark = pytest.mark.gpu

B16, F32 = 2.0 ** -8, 2.0 ** -23
CANARY = 777.0


def _matrix(seed, rows, cols, std, pad=0):
    """(values, bf16 view on the GPU with NaN behind each row)."""
    bits = W.draw_array(seed, rows, cols, "normal", std)
    t = torch.full((rows, cols + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
    t[:, :cols] = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    return OG.decode_bf16(bits), t[:, :cols]


def _targets(rng, tokens, vocab, ignored):
    t = rng.integers(0, vocab, tokens)
    t[rng.random(tokens) < ignored] = -100
    if tokens > 3:
        t[1], t[2], t[3] = vocab - 1, 0, vocab      # the last and first token, and one past them
    return t


def run(tokens, D, V, grad=False, scale=1.0, ignored=0.3, std=0.05, pad=0, dw="bf16", accumulate=False, block=0, weights=True,
        seed=1, only=None, targets=None, mutate=None):
    print(f"cross entropy tokens={tokens} D={D} V={V} grad={grad} scale={scale} pad={pad} dw={dw} accumulate={accumulate} "
          f"block={block} only={only}", flush=True)
    rng = np.random.default_rng(seed)
    xv, x = _matrix(seed, tokens, D, 1.0, pad)
    wv, w = _matrix(seed + 1, V, D, std, pad)
    t = _targets(rng, tokens, V, ignored) if targets is None else targets
    head = ccl.ccl_vocab(hidden=D, vocab=V, scale=scale, w_ld=D + pad, block=block)
    need = ccl.ccl_cross_entropy_workspace(head, tokens, grad=grad)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    loss, lse = (torch.full((tokens + 3,), CANARY, device="cuda") for _ in range(2))
    td = torch.from_numpy(t).cuda()
    common = dict(lse=lse, workspace=ws, workspace_bytes=need)
    if mutate is not None:
        mutate(x, w)
    if not grad:
        ccl.ccl_cross_entropy(head, tokens, x, w, td, loss, **common)
        g = None
    else:
        g = (rng.random(tokens) + 0.5) / tokens if weights else np.full(tokens, 1.0)
        g = g.astype(np.float32).astype(np.float64)
        dx = torch.full((tokens + 1, D + pad), CANARY, dtype=torch.bfloat16, device="cuda")
        dwt = torch.full((V + 1, D + pad), 0.25 if accumulate else CANARY,
                         dtype=torch.bfloat16 if dw == "bf16" else torch.float32, device="cuda")
        ccl.ccl_cross_entropy_grad(head, tokens, x, w, td, loss, None if only == "dW" else dx[:tokens, :D],
                                   None if only == "dX" else dwt[:V, :D],
                                   dloss=torch.from_numpy(g.astype(np.float32)).cuda() if weights else None, dloss_scale=0.5,
                                   accumulate=accumulate, **common)
        g = g * 0.5
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0xFF).all()) and bool((loss[tokens:] == CANARY).all()) and bool((lse[tokens:] == CANARY).all())
    if mutate is not None:
        return (loss, lse, dx[:tokens, :D], dwt[:V, :D]) if grad else (loss, lse)
    lw, sw, z, P = OT.cross_entropy(xv, wv, t, scale, g)
    dz = (abs(scale) * D * F32 * (np.abs(xv) @ np.abs(wv).T) + F32 * np.abs(z)).max(axis=1)
    dlse = dz + F32 * (100 + np.abs(sw))
    got_lse, got_loss = lse[:tokens].double().cpu().numpy(), loss[:tokens].double().cpu().numpy()
    assert (np.abs(got_lse - sw) <= dlse).all(), np.abs(got_lse - sw).max()
    assert (np.abs(got_loss - lw) <= 2 * dlse).all(), np.abs(got_loss - lw).max()
    assert (got_loss[(t < 0) | (t >= V)] == 0).all()
    if not grad:
        return loss, lse
    rel = (2 * B16 + 2.0 ** -15 + dz + dlse)[:, None]
    err = rel * np.abs(P)
    live = np.flatnonzero((t >= 0) & (t < V))
    err[live, t[live]] += (dz + dlse)[live] * np.abs(g * scale)[live]
    for name, out, want, tol, cancel in (
            ("dX", dx[:tokens, :D], P @ wv, err @ np.abs(wv) + V * F32 * (np.abs(P) @ np.abs(wv)), None),
            ("dW", dwt[:V, :D], P.T @ xv, err.T @ np.abs(xv) + tokens * F32 * (np.abs(P).T @ np.abs(xv)), None)):
        if only is not None and only != name:
            assert bool((out == (0.25 if name == "dW" and accumulate else CANARY)).all())
            continue
        got = out.double().cpu().numpy()
        if name == "dW" and accumulate:
            want = want + 0.25
            tol = tol + F32 * (np.abs(want) + 0.25) * 4
        rounding = 0.0 if out.dtype == torch.float32 else B16 * np.abs(want)
        over = np.abs(got - want) - tol * 1.01 - rounding - 1e-38
        assert np.isfinite(got).all() and over.max() <= 0, (name, over.max())
        if np.linalg.norm(want) > 0:
            off = np.linalg.norm(got - want) / np.linalg.norm(want)
            assert off <= 6e-3, (name, off)
    assert bool((dx[tokens:] == CANARY).all()) and bool((dx[:, D:] == CANARY).all())
    keep = 0.25 if accumulate else CANARY
    assert bool((dwt[V:] == keep).all()) and bool((dwt[:, D:] == keep).all())
    return loss, lse, dx, dwt


SHAPES = [(1, 16, 1), (1, 256, 1000), (2, 48, 129), (63, 80, 300), (65, 128, 127), (130, 272, 1001), (257, 64, 513), (300, 336, 2049)]


@pytest.mark.parametrize("tokens,D,V", SHAPES)
def test_loss(tokens, D, V):
    run(tokens, D, V, pad=8)


@pytest.mark.parametrize("dw,accumulate", [("bf16", False), ("fp32", True)])
@pytest.mark.parametrize("tokens,D,V", SHAPES)
def test_gradients(tokens, D, V, dw, accumulate):
    run(tokens, D, V, grad=True, scale=0.5, pad=8, dw=dw, accumulate=accumulate)


@pytest.mark.parametrize("dw,accumulate", [("bf16", False), ("bf16", True), ("fp32", False), ("fp32", True)])
@pytest.mark.parametrize("block", [1, 100, 128, 299])
def test_blocks(block, dw, accumulate):
    run(300, 80, 700, grad=True, block=block, dw=dw, accumulate=accumulate)
    run(300, 80, 700, block=block)


@pytest.mark.parametrize("only", ["dX", "dW"])
def test_one_gradient(only):
    run(140, 96, 500, grad=True, only=only, weights=False)


def test_no_token_counts():
    """Every target outside the vocabulary: zero losses and gradients."""
    t = np.array([-1, 500, -100, 1 << 40, -(1 << 62)] * 20, np.int64)
    _, _, dx, dw = run(100, 64, 500, grad=True, targets=t)
    assert bool((dx[:100, :64] == 0).all()) and bool((dw[:500, :64] == 0).all())


def test_confident_tokens():
    """Logits of a hundred and more: p - 1 of the target keeps its digits where p is near 1 (z - z' is 10 to 30), and
    rows whose other terms vanish have a loss near 0."""
    for std in (0.5, 2.0):
        run(70, 256, 400, grad=True, std=std, ignored=0.0)


def test_target_gradient_near_one():
    """Two tokens of which one leads by 12: P of the target is -g sigmoid(-12), far below bf16's step at 1."""
    D, V = 16, 2
    x = torch.zeros(1, D, dtype=torch.bfloat16, device="cuda")
    x[0, 0] = 1.0
    w = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    w[0, 0] = 12.0
    head = ccl.ccl_vocab(hidden=D, vocab=V)
    ws = torch.empty(ccl.ccl_cross_entropy_workspace(head, 1, grad=True), dtype=torch.uint8, device="cuda")
    loss, dx, dw = torch.empty(1, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    ccl.ccl_cross_entropy_grad(head, 1, x, w, torch.zeros(1, dtype=torch.int64, device="cuda"), loss, dx, dw, workspace=ws,
                               workspace_bytes=ws.numel())
    q = 1 / (1 + np.exp(12.0))
    got = dw.double().cpu().numpy()
    # one rounding of P and one of dW, fp32 within (12 + 100) 2^-23 of 1 in lse; the other token's P is rounded twice
    assert abs(got[0, 0] + q) <= q * 2 * B16 + 112 * F32 and abs(got[1, 0] - q) <= q * 3 * B16 + 112 * F32
    assert abs(float(loss) - np.log1p(np.exp(-12.0))) <= 112 * F32


def test_a_bad_row_stays_its_own():
    """NaN in one token's x: its loss and dX are NaN, the other tokens' values are what they were; a token that does not
    count adds nothing to dW."""
    t = np.arange(40, dtype=np.int64)
    t[7] = -1

    def bad(x, w):
        x[5] = float("nan")
    clean = run(40, 64, 300, grad=True, targets=t)
    loss, lse, dx, dw = run(40, 64, 300, grad=True, targets=t, mutate=bad)
    others = [i for i in range(40) if i != 5]
    assert bool(torch.isnan(loss[5])) and bool(torch.isnan(lse[5])) and bool(torch.isnan(dx[5]).all())
    for a, b in zip((loss[:40], lse[:40], dx), (clean[0][:40], clean[1][:40], clean[2][:40, :64])):
        assert torch.equal(a[others], b[others])
    assert bool(torch.isnan(dw).all())


@pytest.mark.parametrize("fill", [float("nan"), float("inf")])
def test_padding_tokens_reach_no_gradient(fill):
    """Whatever x holds where the target says that the token does not count, or its weight is 0."""
    t = np.arange(70, dtype=np.int64)
    t[[3, 64, 69]] = -100

    def bad(x, w):
        x[[3, 64, 69]] = fill
    clean = run(70, 64, 300, grad=True, targets=t)
    loss, _, dx, dw = run(70, 64, 300, grad=True, targets=t, mutate=bad)
    assert torch.equal(loss, clean[0]) and torch.equal(dx, clean[2][:70, :64]) and torch.equal(dw, clean[3][:300, :64])


def test_no_tokens():
    head = ccl.ccl_vocab(hidden=64, vocab=100)
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(100, 64, dtype=torch.bfloat16, device="cuda")
    t, loss = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    for dt in (torch.bfloat16, torch.float32):
        dw = torch.full((101, 80), 5.0, dtype=dt, device="cuda")
        ccl.ccl_cross_entropy_grad(head, 0, x, w, t, loss, x, dw[:100, :64], accumulate=True)
        assert bool((dw == 5).all())
        ccl.ccl_cross_entropy_grad(head, 0, x, w, t, loss, x, dw[:100, :64])
        assert bool((dw[:100, :64] == 0).all()) and bool((dw[100:] == 5).all()) and bool((dw[:, 64:] == 5).all())
    ccl.ccl_cross_entropy(head, 0, x, w, t, loss)
