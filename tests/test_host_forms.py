"""The cases of tests/forms.py reach the forms that they are there for."""
import pytest

from tests import forms


def test_orthogonalize():
    reached, tall = set(), set()
    for case in forms.ORTHO:
        f = forms.ortho_forms(*case)
        reached |= f
        if case[1] > case[2]:
            tall |= {x[:4] for x in f if x[0] == "update"}
    assert not forms.ORTHO_FORMS - reached
    assert not forms.ORTHO_TALL - tall


def test_moe():
    for fp8 in (False, True):
        all_forms = [forms.moe_form(case, fp8) for case in forms.MOE]
        has = lambda **want: any(all(f[k] == v for k, v in want.items()) for f in all_forms)  # noqa: E731
        several = [f for f in all_forms if f["up_group"] > 1 and f["chunks"] > 1]
        assert any(f["list"] for f in several) and any(not f["list"] for f in several)
        assert any(f["up_tiles"] % f["up_group"] for f in several)           # a shorter last group
        wide = [f for f in all_forms if f["down_nt"] == 4 and f["lines"] >= 6]
        assert any(f["ranges"] == 1 for f in wide) and any(f["ranges"] > 1 for f in wide)
        assert any(f["clamped"] for f in wide)
        assert has(up_group=1, list=1) or has(up_group=1, list=0)


@pytest.mark.parametrize("case", forms.FUSED, ids=forms.fused_name)
def test_fused(case):
    form = forms.fused_form(case)
    assert {k: form[k] for k in case["expect"]} == case["expect"]
