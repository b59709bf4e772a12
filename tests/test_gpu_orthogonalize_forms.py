"""Every form of the Newton-Schulz products (tiles of 64, 128 and 256 rows, one
or two workgroups to a CU, K ranges of some or all tiles, edges inside a tile,
transposed results) against the steps in float64. Bounds as in
test_gpu_orthogonalize; tests/test_host_forms.py asserts that these cases reach
the forms."""
import pytest
import torch

from oracle.ffn import QUINTIC
from paper_2606_11718_amd import ccl
from tests import forms

pytestmark = pytest.mark.gpu

BF16, FP32 = ccl.CCL_DT_BF16, ccl.CCL_DT_FP32


def _steps64(G):
    """Five steps on one matrix, plain products of row-major operands."""
    a, b, c = QUINTIC
    X = G / (G.square().sum().sqrt() + 1e-7)
    tall = X.shape[0] > X.shape[1]
    if tall:
        X = X.t().contiguous()
    for _ in range(5):
        S = torch.mm(X, X.t().contiguous())
        X = a * X + torch.mm(b * S + c * torch.mm(S, S), X)
    return X.t() if tall else X


@pytest.mark.parametrize("g_type", [BF16, FP32])
@pytest.mark.parametrize("case", forms.ORTHO, ids=lambda c: "x".join(map(str, c)))
def test_forms(case, g_type):
    batch, rows, cols = case
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    pad = 3 if g_type == BF16 else 8
    flat = torch.full((batch, rows, cols + pad), float("nan"), device="cuda",
                      dtype=torch.bfloat16 if g_type == BF16 else torch.float32)
    G = flat[:, :, :cols]
    for i in range(batch):                     # noise and a few strong directions
        G[i] = 0.01 * (rnd(rows, cols) + torch.mm(rnd(rows, 4), rnd(4, cols)))
    O = torch.full((batch, rows + 1, cols + pad), 777.0, device="cuda", dtype=torch.bfloat16)
    need = ccl.ccl_orthogonalize_workspace(batch, rows, cols)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    print(f"orthogonalize forms {case} type={g_type}", flush=True)
    ccl.ccl_orthogonalize(batch, rows, cols, G, g_type, cols + pad, rows * (cols + pad), O, o_ld=cols + pad,
                          o_stride=(rows + 1) * (cols + pad), workspace=ws, workspace_bytes=need)
    for i in range(batch):
        got, want = O[i, :rows, :cols].double(), _steps64(G[i].double())
        rms, off = want.square().mean().sqrt(), got - want
        rel, worst = off.norm() / want.norm(), ((off.abs() - 2.0 ** -8 * want.abs()).max() / rms)
        assert rel <= 3e-3 and worst <= 1.5e-2, (i, rel.item(), worst.item())
    print(f"last matrix: rel {rel.item():.2e} worst {worst.item():.2e}", flush=True)
    O[:, :rows, :cols] = 777.0
    assert (O == 777.0).all()                  # nothing beside the results was written
