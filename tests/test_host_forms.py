"""The cases of tests/forms.py reach the forms that they are there for."""
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
