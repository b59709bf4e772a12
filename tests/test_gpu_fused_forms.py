"""The forms of the fused products that shapes of ordinary tests do not reach:
tiles with valid rows over all XCDs, pairs of workgroups, K ranges with whole tiles
that are not valid, the form for operands of 2 GiB and more. Against float64
products on the GPU, within test_gpu_fused's bounds; rows past the valid ones
hold NaNs. tests/test_host_forms.py asserts that these cases reach the forms."""
import pytest
import torch

from paper_2606_11718_amd import ccl
from tests import forms

pytestmark = pytest.mark.gpu

NAN = float("nan")
ROWMAJOR = ccl.CCL_LAYOUT_ROWMAJOR


def _halves(z):
    m, n = z.shape
    g = z.view(m, n // 32, 2, 16)
    return g[:, :, 0].reshape(m, n // 2), g[:, :, 1].reshape(m, n // 2)


def _join(g, u):
    m, n = g.shape
    return torch.stack([g.view(m, n // 16, 16), u.view(m, n // 16, 16)], 2).reshape(m, 2 * n)


def _silu(z):
    """Value and derivative in float64."""
    s = torch.sigmoid(z)
    return z * s, s + z * s * torch.sigmoid(-z)


def _within(got, want, err, rows, what):
    assert not got[rows:].any(), f"{what}: rows past the valid ones"
    g = got[:rows].double()
    bad = ~((g - want).abs() <= 2.0 ** -8 * torch.maximum(g.abs(), want.abs()) + err + 1e-37)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:3].tolist())


@pytest.mark.parametrize("case", forms.FUSED, ids=forms.fused_name)
def test_forms(case, monkeypatch):
    for k, v in case["env"].items():
        monkeypatch.setenv(k, v)
    M, N, K, rows, gated, fp8 = (case[k] for k in ("M", "N", "K", "rows", "gated", "fp8"))
    print(f"fused forms {forms.fused_name(case)} {case['expect']}", flush=True)
    plan = ccl.ccl_plan_typed(M, N, K, case["chiplets"], case["grid_rows"], 4096,
                              ccl.CCL_DT_FP8_E4M3 if fp8 else ccl.CCL_DT_BF16, ccl.CCL_DT_BF16)
    gen = torch.Generator(device="cuda").manual_seed(M + N + K + rows)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
    alpha = 0.03 if fp8 else 1.0
    A, B = rnd(M, K).to(dt), (rnd(K, N) * (1.0 if fp8 else 0.06)).to(dt)
    A[rows:] = NAN
    a, b = A[:rows].double(), B.double()
    d = alpha * torch.mm(a, b)
    ed = alpha * K * 2.0 ** -23 * torch.mm(a.abs(), b.abs())
    if case["grad"]:
        cols = 2 * N if gated else N
        Z = (2.0 * rnd(M, cols)).bfloat16()
        Z[rows:] = NAN
        dZ = torch.full((M, cols), 777.0, device="cuda", dtype=torch.bfloat16)
        db = torch.full((cols,), NAN, device="cuda")
        need = ccl.ccl_gemm_fused_grad_workspace(plan, gated=gated, dbias=True, layout=ROWMAJOR)
        ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
        ccl.ccl_gemm_fused_grad(plan, A, B, Z, dZ, activation=ccl.CCL_ACT_SILU, gated=gated, dbias=db, alpha=alpha,
                                rows=rows, layout=ROWMAJOR, workspace=ws, workspace_bytes=need)
        z = Z[:rows].double()
        e0 = 1.2 * (ed + 2.0 ** -18 * d.abs())
        if gated:
            (g, u) = _halves(z)
            v, dv = _silu(g)
            want, err = _join(d * u * dv, d * v), _join(u.abs() * e0, g.abs() * e0)
        else:
            want, err = d * _silu(z)[1], e0
        _within(dZ, want, err, rows, "dZ")
        tol = err.sum(0) + (M + 8) * 2.0 ** -24 * want.abs().sum(0) + 1e-30
        assert ((db.double() - want.sum(0)).abs() <= tol).all()
    else:
        cols = N // 2 if gated else N
        bias, R = rnd(N), rnd(M, cols).bfloat16()
        R[rows:] = NAN
        C, Z = (torch.full((M, c), 777.0, device="cuda", dtype=torch.bfloat16) for c in (cols, N))
        ranges, need = ccl.ccl_gemm_fused_workspace(plan, case["splits"], layout=ROWMAJOR)
        assert ranges == case["expect"].get("ranges", 1)
        ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
        ccl.ccl_gemm_fused(plan, A, B, C, activation=ccl.CCL_ACT_SILU, gated=gated, bias=bias, residual=R, beta=0.5, preact=Z,
                           alpha=alpha, rows=rows, layout=ROWMAJOR, splits=case["splits"], workspace=ws, workspace_bytes=need)
        z = d + bias.double()
        ez = ed + 2.0 ** -22 * z.abs()
        r = R[:rows].double()
        if gated:
            (g, u), (eg, eu) = _halves(z), _halves(ez)
            want = _silu(g)[0] * u + 0.5 * r
            err = 1.2 * (eg + 2.0 ** -18 * g.abs()) * (u.abs() + eu) + g.abs() * eu + 2.0 ** -22 * (0.5 * r).abs()
        else:
            want = _silu(z)[0] + 0.5 * r
            err = 1.2 * (ez + 2.0 ** -18 * z.abs()) + 2.0 ** -22 * (0.5 * r).abs()
        _within(C, want, err, rows, "C")
        _within(Z, z, ez, rows, "Z")
    assert (ws[need:] == 0xFF).all()                       # nothing past the workspace that was asked for
