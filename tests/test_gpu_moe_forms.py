"""ccl_moe_decode on wide layers and large batches: up workgroups that stream
several tiles in several chunks of K, the down product's units of weights over
many lines, in ranges and past the last column tile. Against float64 products on
the GPU; the bound is test_gpu_moe's, and tests/test_host_forms.py asserts that
these cases reach the forms."""
import pytest
import torch

from paper_2606_11718_amd import ccl
from tests import forms

pytestmark = pytest.mark.gpu


def _layer64(x, logits, gate_up, down, gs, ds, top_k, ids):
    """(y, its bound, probabilities) in float64, with the experts of ids (checked apart)."""
    T, E = logits.shape
    F = down.shape[2]
    x = x.double()
    top = logits.double().gather(1, ids)
    probs = torch.softmax(top, 1)
    y = torch.zeros(T, down.shape[1], dtype=torch.float64, device=x.device)
    tol = torch.zeros_like(y)
    for e in range(E):
        at, slot = (ids == e).nonzero(as_tuple=True)
        if at.numel() == 0:
            continue
        sg = 1.0 if gs is None else gs[e].double()
        sd = 1.0 if ds is None else ds[e].double()
        w, d = gate_up[e].double().t().contiguous(), down[e].double().t().contiguous()
        z = sg * (x[at] @ w)
        ez = x.shape[1] * 2.0 ** -23 * sg * (x[at].abs() @ w.abs()) + 2.0 ** -18 * z.abs()
        g, u, eg, eu = z[:, :F], z[:, F:], ez[:, :F], ez[:, F:]
        h = g * torch.sigmoid(g) * u
        eh = 1.2 * eg * (u.abs() + eu) + g.abs() * eu + 2.0 ** -16 * h.abs()
        p = probs[at, slot][:, None] * sd
        y.index_add_(0, at, p * (h @ d))
        tol.index_add_(0, at, p * ((eh + (F * 2.0 ** -23 + 2.0 ** -20) * h.abs()) @ d.abs()))
    return y, tol, probs


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case", forms.MOE, ids=lambda c: "x".join(map(str, c)))
def test_forms(case, fp8):
    T, D, F, E, k = case
    print(f"moe forms {case} fp8={fp8}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(sum(case))
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
    gate_up, down = (torch.empty(s, dtype=dt, device="cuda") for s in ((E, 2 * F, D), (E, D, F)))
    for w in (gate_up, down):
        for e in range(E):
            w[e] = (rnd(*w[e].shape) * (1.0 if fp8 else w.shape[2] ** -0.5)).to(dt)
    gs, ds = ((torch.rand(E, generator=gen, device="cuda") + 0.5) / n ** 0.5 for n in (D, F)) if fp8 else (None, None)
    x, logits = rnd(T, D).bfloat16(), 1.5 * rnd(T, E)
    y = torch.full((T, D), 777.0, dtype=torch.bfloat16, device="cuda")
    ids = torch.empty(T, k, dtype=torch.int32, device="cuda")
    probs = torch.empty(T, k, device="cuda")
    moe = ccl.ccl_moe(hidden=D, ffn=F, experts=E, top_k=k, weight_type=ccl.CCL_DT_FP8_E4M3 if fp8 else ccl.CCL_DT_BF16)
    ws = torch.full((ccl.ccl_moe_workspace(moe, T),), 0xFF, dtype=torch.uint8, device="cuda")
    ccl.ccl_moe_decode(moe, T, x, logits, gate_up, down, y, ids=ids, probs=probs, gate_up_scale=gs, down_scale=ds,
                       workspace=ws, workspace_bytes=ws.numel())
    order = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(ids.long(), order)
    want, tol, pw = _layer64(x, logits, gate_up, down, gs, ds, k, order)
    assert ((probs - pw).abs() <= 2.0 ** -20 * pw).all()
    got = y.double()
    off = (got - want).abs() - 2.0 ** -8 * torch.maximum(got.abs(), want.abs()) - 1.01 * tol
    print(f"rel {((got - want).norm() / want.norm()).item():.2e}", flush=True)
    assert (off <= 1e-37).all(), (off > 1e-37).sum()
