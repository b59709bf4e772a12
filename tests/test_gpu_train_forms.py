"""GPU parity of every form of the experts' products and of the loss's products, at
sizes off their grids (tests/train_forms.py; which form a case takes is asserted on the
CPU). Tolerances as in test_gpu_grouped and test_gpu_cross_entropy."""
import pytest

from paper_2606_11718_amd import ccl
from tests import test_gpu_cross_entropy as TC
from tests import test_gpu_grouped as TG
from tests import train_forms as F

pytestmark = pytest.mark.gpu

ACTS = (ccl.CCL_ACT_SILU, ccl.CCL_ACT_GELU)


@pytest.mark.parametrize("form", list(F.GROUPED), ids=str)
def test_grouped(form):
    for i, (way, counts, K, N, gated) in enumerate(F.GROUPED[form]):
        act = ACTS[i % 2] if gated else ccl.CCL_ACT_NONE
        if way == F.FORWARD:
            TG.run_forward(counts, K, N, act, gated, keep=i % 2 == 0, behind=3 if form[0] < 256 else 0, pad=8)
        elif way == F.GRAD:
            TG.run_grad(counts, K, N, act, gated, behind=3 if form[0] < 256 else 0, pad=8)
        else:
            for f32 in (False, True):
                for accumulate in (False, True):
                    TG.run_wgrad(counts, K, N, f32, accumulate, pad=8)


@pytest.mark.parametrize("case", [c for k in ((64, True), (128, True)) for c in F.GROUPED[k] if c[0] == F.GRAD], ids=str)
def test_grouped_ranges_in_place(case):
    way, counts, K, N, gated = case
    TG.run_grad(counts, K, N, ccl.CCL_ACT_SILU, gated, in_place=True)


@pytest.mark.parametrize("tokens,D,V", [c for cases in F.LOGITS.values() for c in cases])
def test_logits(tokens, D, V):
    TC.run(tokens, D, V, pad=8)


@pytest.mark.parametrize("tokens,D,V", F.DX_REST)
def test_dx_of_whole_rounds_and_the_rest(tokens, D, V):
    TC.run(tokens, D, V, grad=True, pad=8, only="dX")


@pytest.mark.parametrize("dw,accumulate", [("bf16", False), ("fp32", True)])
@pytest.mark.parametrize("tokens,D,V", [c for cases in F.LOGITS_REST.values() for c in cases] + F.DW_REST)
def test_whole_rounds_and_the_rest(tokens, D, V, dw, accumulate):
    TC.run(tokens, D, V, grad=True, pad=8, dw=dw, accumulate=accumulate)


@pytest.mark.parametrize("tokens,D,V", [c for cases in F.DX.values() for c in cases])
def test_dx(tokens, D, V):
    TC.run(tokens, D, V, grad=True, pad=8, only="dX")


@pytest.mark.parametrize("dw,accumulate", [("bf16", False), ("fp32", True)])
@pytest.mark.parametrize("tokens,D,V", [c for cases in F.DW.values() for c in cases])
def test_dw(tokens, D, V, dw, accumulate):
    TC.run(tokens, D, V, grad=True, pad=8, only="dW", dw=dw, accumulate=accumulate)


def test_logits_and_gradients_of_large_tiles():
    TC.run(250, 80, 65400, grad=True, pad=8)
