"""One token: the stride between rows is never used, so whatever a tensor says
of it is no reason to refuse the call (the last of the library's checks before the
first device call shows that the others passed)."""
import pytest
import torch

from paper_2606_11718_amd import ccl

D, F, E = 256, 64, 16
BF16 = torch.bfloat16


def _call(x, logits, y):
    moe = ccl.ccl_moe(hidden=D, ffn=F, experts=E, top_k=4)
    with pytest.raises(ccl.CCLError) as e:
        ccl.ccl_moe_decode(moe, 1, x, logits, 1 << 20, 1 << 20, y, workspace=1 << 20, workspace_bytes=1)
    return str(e.value)


@pytest.mark.parametrize("stride", [0, 1, 255, 1 << 23])
def test_row_stride(stride):
    rows = lambda n, dtype: torch.zeros(n, dtype=dtype).as_strided((1, n), (stride, 1))  # noqa: E731
    assert "workspace smaller" in _call(rows(D, BF16), rows(E, torch.float32), rows(D, BF16))


def test_a_column_as_a_row():
    column = lambda n, dtype: torch.zeros(n, 1, dtype=dtype).t()  # noqa: E731
    assert "workspace smaller" in _call(column(D, BF16), column(E, torch.float32), column(D, BF16))


def test_one_row_of_a_narrow_stride_among_several():
    """Rows that overlap are refused where there is more than one."""
    x = torch.zeros(2 * D, dtype=BF16).as_strided((2, D), (1, 1))
    moe = ccl.ccl_moe(hidden=D, ffn=F, experts=E, top_k=4)
    with pytest.raises(ccl.CCLError) as e:
        ccl.ccl_moe_decode(moe, 2, x, torch.zeros(2, E), 1 << 20, 1 << 20, torch.zeros(2, D, dtype=BF16),
                           workspace=1 << 20, workspace_bytes=1)
    assert "leading dimension" in str(e.value)
