"""GPU parity of the experts' products on sorted rows with the fp64 oracle.

A product carries the fp32 error of its K-term sum, at most K 2^-23 sum |a b|,
and the activation 2^-18 of its argument (test_gpu_moe); each output is rounded
to bf16 once (2^-8 relative) unless it is fp32. Through a gate the errors are
multiplied by what the formula multiplies them by.
"""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import gemm as OG
from oracle import train as OT
from paper_2606_11718_amd import ccl

pytestmark = pytest.mark.gpu

NONE, RELU, GELU, SILU = ccl.CCL_ACT_NONE, ccl.CCL_ACT_RELU, ccl.CCL_ACT_GELU, ccl.CCL_ACT_SILU
B16, SUM, ACT = 2.0 ** -8, 2.0 ** -23, 2.0 ** -18
CANARY = 777.0


def _ends(counts):
    return np.cumsum(counts).astype(np.int32)


def _matrix(seed, rows, cols, std, pad=0, live=None):
    """(values, bf16 tensor on the GPU): NaN in `pad` columns behind each row and in rows from `live` on."""
    bits = W.draw_array(seed, max(rows, 1), cols, "normal", std)[:rows]
    t = torch.full((rows, cols + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
    t[:, :cols] = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    if live is not None:
        t[live:] = float("nan")
    return OG.decode_bf16(bits), t[:, :cols]


def _weights(seed, E, N, K, std, pad=False):
    """(values, tensor, w_ld, w_stride), NaN between rows and experts."""
    bits = W.draw_array(seed, E * N, K, "normal", std).reshape(E, N, K)
    ld = K + 8 if pad else K
    stride = N * ld + 16 if pad else N * ld
    flat = torch.full((E * stride,), float("nan"), dtype=torch.bfloat16, device="cuda")
    view = flat.as_strided((E, N, K), (stride, ld, 1))
    view.copy_(torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16))
    return OG.decode_bf16(bits), view, ld, stride


def _out(rows, cols, pad=0, dtype=torch.bfloat16):
    return torch.full((rows, cols + pad), CANARY, dtype=dtype, device="cuda")


def _check(name, got, want, tol):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape, name
    over = np.abs(got - want) - tol
    assert np.isfinite(got).all() and over.max(initial=-1.0) <= 0, (name, over.max(), np.unravel_index(over.argmax(), over.shape))


def _workspace(g, rows, way):
    return torch.full((max(16, ccl.ccl_grouped_gemm_workspace(g, rows, way)),), 0xFF, dtype=torch.uint8, device="cuda")


def run_forward(counts, K, N, act=NONE, gated=False, keep=True, behind=0, pad=0, seed=1, stream=None):
    print(f"grouped forward counts={counts} K={K} N={N} act={act} gated={gated} behind={behind} pad={pad}", flush=True)
    ends = _ends(counts)
    used, rows, E = int(ends[-1]), int(ends[-1]) + behind, len(counts)
    xv, x = _matrix(seed, rows, K, 1.0, pad, used)
    wv, w, ld, stride = _weights(seed + 1, E, N, K, 1 / np.sqrt(K), bool(pad))
    g = ccl.ccl_grouped(in_features=K, out_features=N, experts=E, activation=act, gated=gated, w_ld=ld, w_stride=stride)
    cols = N // 2 if gated else N
    y, z = _out(rows, cols, pad), _out(rows, N, pad) if keep else None
    ws = _workspace(g, rows, ccl.CCL_GROUPED_FORWARD)
    ccl.ccl_grouped_gemm(g, rows, torch.from_numpy(ends).cuda(), x, w, y[:, :cols], preact=z[:, :N] if keep else None,
                         workspace=ws, workspace_bytes=ws.numel(), stream=stream)
    torch.cuda.synchronize()
    yw, zw, mag = OT.grouped(xv, wv, ends, act, gated)
    dz = K * SUM * mag
    if keep:
        _check("Z", z[:used, :N], zw, B16 * np.abs(zw) + dz)
        assert bool((z[used:] == CANARY).all()) and bool((z[:, N:] == CANARY).all())
    if gated:
        h = N // 2
        # |act'| < 1.13
        tol = (1.13 * dz[:, :h] + ACT * np.abs(zw[:, :h])) * np.abs(zw[:, h:]) * (1 + SUM) + (np.abs(zw[:, :h]) + dz[:, :h]) * dz[:, h:]
    else:
        tol = 1.13 * dz + ACT * np.abs(zw)
    _check("Y", y[:used, :cols], yw, B16 * np.abs(yw) + 1.01 * tol)
    assert bool((y[used:] == CANARY).all()) and bool((y[:, cols:] == CANARY).all())
    return y, z


def run_grad(counts, K, N, act=NONE, gated=False, behind=0, pad=0, seed=1, in_place=False):
    print(f"grouped grad counts={counts} K={K} N={N} act={act} gated={gated} behind={behind} pad={pad}", flush=True)
    ends = _ends(counts)
    used, rows, E = int(ends[-1]), int(ends[-1]) + behind, len(counts)
    wide = 2 * K if gated else K
    dv, dy = _matrix(seed, rows, N, 1.0, pad, used)
    wv, w, ld, stride = _weights(seed + 1, E, N, K, 1 / np.sqrt(N), bool(pad))
    through = act != NONE or gated
    zv, z = _matrix(seed + 2, rows, wide, 1.0, pad, used) if through else (None, None)
    g = ccl.ccl_grouped(in_features=K, out_features=N, experts=E, activation=act, gated=gated, w_ld=ld, w_stride=stride)
    full = _out(rows, wide, pad)
    dx = z if in_place else full[:, :wide]
    ws = _workspace(g, rows, ccl.CCL_GROUPED_GRAD)
    ccl.ccl_grouped_gemm_grad(g, rows, torch.from_numpy(ends).cuda(), dy, w, dx, preact=z, workspace=ws,
                              workspace_bytes=ws.numel())
    torch.cuda.synchronize()
    want, d, mag = OT.grouped_grad(dv, wv, ends, act, gated, zv)
    dd = N * SUM * mag
    if gated:
        gate, up = zv[:used, :K], zv[:used, K:]
        # act and act' carry 2^-18 of (1 + |z|), |act'| < 1.13, |act(z)| <= |z|
        tol = np.concatenate([(1.13 * dd + ACT * (1 + np.abs(gate)) * np.abs(d)) * np.abs(up),
                              np.abs(gate) * dd + ACT * (1 + np.abs(gate)) * np.abs(d)], axis=1)
    elif through:
        tol = 1.13 * dd + ACT * (1 + np.abs(zv[:used])) * np.abs(d)
    else:
        tol = dd
    _check("dX", dx[:used], want, B16 * np.abs(want) + 1.01 * tol)
    if not in_place:
        assert bool((full[used:] == CANARY).all()) and bool((full[:, wide:] == CANARY).all())
    return dx


def run_wgrad(counts, K, N, f32=False, accumulate=False, behind=0, pad=0, seed=1):
    print(f"grouped wgrad counts={counts} K={K} N={N} f32={f32} accumulate={accumulate} behind={behind} pad={pad}", flush=True)
    ends = _ends(counts)
    used, rows, E = int(ends[-1]), int(ends[-1]) + behind, len(counts)
    dv, dy = _matrix(seed, rows, N, 1.0, pad, used)
    xv, x = _matrix(seed + 1, rows, K, 1.0, pad, used)
    ld = K + 8 if pad else K
    stride = N * ld + 16 if pad else N * ld
    g = ccl.ccl_grouped(in_features=K, out_features=N, experts=E, w_ld=ld, w_stride=stride)
    flat = torch.full((E * stride,), 3.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    dw = flat.as_strided((E, N, K), (stride, ld, 1))
    ws = _workspace(g, rows, ccl.CCL_GROUPED_WGRAD)
    ccl.ccl_grouped_gemm_wgrad(g, rows, torch.from_numpy(ends).cuda(), dy, x, dw, accumulate=accumulate, workspace=ws,
                               workspace_bytes=ws.numel())
    torch.cuda.synchronize()
    want, mag = OT.grouped_wgrad(dv[:used], xv[:used], ends)
    most = max(counts)
    tol = most * SUM * mag
    if accumulate:
        want = want + 3.0
        tol = tol + SUM * (mag + 3.0)
    _check("dW", dw, want, tol + (0 if f32 else B16 * np.abs(want)))
    touched = torch.zeros_like(flat, dtype=torch.bool)
    touched.as_strided((E, N, K), (stride, ld, 1)).fill_(True)
    assert bool((flat[~touched] == 3.0).all())
    return dw


COUNTS = [[1], [0, 0, 1], [130, 0, 1, 127, 129], [128, 256, 0, 64], [5, 3, 0, 17, 300]]
SIDES = [(16, 32), (48, 96), (144, 288), (256, 128), (320, 544)]


@pytest.mark.parametrize("K,N", SIDES)
@pytest.mark.parametrize("counts", COUNTS, ids=str)
def test_forward(counts, K, N):
    run_forward(counts, K, N, behind=7, pad=8)


@pytest.mark.parametrize("act,gated,keep", [(RELU, False, True), (GELU, False, False), (SILU, True, True), (GELU, True, False),
                                            (NONE, True, True), (RELU, True, True)])
@pytest.mark.parametrize("counts,K,N", [([130, 0, 1, 127], 64, 288), ([40, 300], 272, 64), ([3, 0, 2], 80, 544)], ids=str)
def test_forward_activations(counts, K, N, act, gated, keep):
    run_forward(counts, K, N, act, gated, keep)


@pytest.mark.parametrize("K,N", SIDES)
@pytest.mark.parametrize("counts", COUNTS, ids=str)
def test_grad(counts, K, N):
    run_grad(counts, K, N, behind=7, pad=8)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("act,gated", [(RELU, False), (GELU, False), (SILU, True), (GELU, True), (NONE, True)])
@pytest.mark.parametrize("counts,K,N", [([130, 0, 1, 127], 144, 64), ([40, 300], 272, 272), ([3, 0, 2], 48, 80)], ids=str)
def test_grad_activations(counts, K, N, act, gated, in_place):
    run_grad(counts, K, N, act, gated, in_place=in_place)


@pytest.mark.parametrize("f32,accumulate", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("K,N", SIDES)
@pytest.mark.parametrize("counts", COUNTS, ids=str)
def test_wgrad(counts, K, N, f32, accumulate):
    run_wgrad(counts, K, N, f32, accumulate, behind=7, pad=8)


def test_no_rows():
    g = ccl.ccl_grouped(in_features=64, out_features=64, experts=3)
    ends = torch.zeros(3, dtype=torch.int32, device="cuda")
    x, y = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(3, 64, 64, dtype=torch.bfloat16, device="cuda")
    ccl.ccl_grouped_gemm(g, 0, ends, x, w, y)
    ccl.ccl_grouped_gemm_grad(g, 0, ends, y, w, x)
    ccl.ccl_grouped_gemm_wgrad(g, 0, ends, y, x, w)
    torch.cuda.synchronize()
    assert bool((w == 0).all())


def test_rows_that_no_expert_has():
    """Nothing but zeros in ends: outputs stay, a weight gradient becomes zeros."""
    g = ccl.ccl_grouped(in_features=64, out_features=64, experts=3)
    ends = torch.zeros(3, dtype=torch.int32, device="cuda")
    nan = lambda: torch.full((50, 64), float("nan"), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    y, dw = _out(50, 64), _out(3 * 64, 64).view(3, 64, 64)
    w = torch.ones(3, 64, 64, dtype=torch.bfloat16, device="cuda")
    ccl.ccl_grouped_gemm(g, 50, ends, nan(), w, y)
    ccl.ccl_grouped_gemm_wgrad(g, 50, ends, nan(), nan(), dw)
    torch.cuda.synchronize()
    assert bool((y == CANARY).all()) and bool((dw == 0).all())
