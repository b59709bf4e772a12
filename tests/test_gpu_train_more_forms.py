"""Forms of the training operators that no other parity test runs: dW of more experts
than are put in order, and bf16 dW over several blocks of tokens in 256x256 tiles.
Tolerances as in test_gpu_grouped and test_gpu_cross_entropy; which form a case takes
is asserted on the CPU.
"""
import pytest

from paper_2606_11718_amd import ccl
from tests import test_gpu_cross_entropy as TC
from tests import test_gpu_grouped as TG
from tests import train_forms as F

COUNTS = [3, 0, 70, 1, 130, 0, 64, 0, 200, 65] * 9     # 90 experts
# (tile rows, in, out)
WGRAD = [(128, 144, 112), (256, 272, 288)]
# (hidden, vocab, block, tokens, tiles behind the whole rounds or not)
BLOCKS = [(1040, 13900, 300, 700, False), (1040, 13900, 520, 1100, True)]


def test_cases():
    for tile, K, N in WGRAD:
        got = F.ask("grouped", F.WGRAD, len(COUNTS), N, K, False, sum(COUNTS))
        assert (got["tile_m"], got["splits"]) == (tile, 1), got
    assert len(COUNTS) > 64
    for D, V, block, tokens, rest in BLOCKS:
        head = ccl.ccl_vocab(hidden=D, vocab=V, block=block)
        assert ccl.ccl_cross_entropy_workspace(head, tokens, grad=True) > 0 and tokens > block
        assert F.ask("dw", D, V, block)["tile_m"] == 256 and (F.ask("dw_rest", D, V, block)["tiles"] > 0) == rest


@pytest.mark.gpu
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("tile,K,N", WGRAD)
def test_wgrad_of_many_experts(tile, K, N, f32, accumulate):
    TG.run_wgrad(COUNTS, K, N, f32, accumulate, pad=8)


@pytest.mark.gpu
@pytest.mark.parametrize("dw,accumulate", [("bf16", False), ("bf16", True), ("fp32", False)])
@pytest.mark.parametrize("D,V,block,tokens,rest", BLOCKS)
def test_blocks_of_large_tiles(D, V, block, tokens, rest, dw, accumulate):
    TC.run(tokens, D, V, grad=True, block=block, pad=8, only="dW", dw=dw, accumulate=accumulate)
