"""What GatedFFN refuses: its products take their operands as whole row-major
matrices of the sizes it was made for, and would read past the end of a smaller
one (tensors on the host stand for those on the GPU; the refusal comes before
the first device call)."""
import pytest
import torch

from paper_2606_11718_amd import ffn

M, D, F = 256, 128, 384
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def net():
    return ffn.GatedFFN(M, D, F, device="cpu")


def _bad(rows, cols):
    """Tensors that are not a whole rows x cols matrix in bf16."""
    return [torch.zeros(rows - 1, cols, dtype=BF16), torch.zeros(rows, cols - 16, dtype=BF16), torch.zeros(rows, cols),
            torch.zeros(rows, cols, dtype=torch.float16), torch.zeros(cols, rows, dtype=BF16).t(),
            torch.zeros(rows, cols + 8, dtype=BF16)[:, :cols], torch.zeros(1, cols, dtype=BF16).expand(rows, cols)]


def test_forward(net):
    for x in _bad(M, D):
        with pytest.raises(ValueError, match="x has to be"):
            net.forward(x, 100)
        with pytest.raises(ValueError, match="x has to be"):
            net.step(x, torch.zeros(M, D, dtype=BF16), 0.1)


@pytest.mark.parametrize("name,cols", [("x", D), ("h", F), ("z", 2 * F), ("dy", D)])
def test_backward(net, name, cols):
    good = dict(x=torch.zeros(M, D, dtype=BF16), h=torch.zeros(M, F, dtype=BF16), z=torch.zeros(M, 2 * F, dtype=BF16),
                dy=torch.zeros(M, D, dtype=BF16))
    for t in _bad(M, cols):
        with pytest.raises(ValueError, match=f"{name} has to be"):
            net.backward(**{**good, name: t}, rows=100)
