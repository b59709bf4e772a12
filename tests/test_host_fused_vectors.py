"""The bias that ccl_gemm_fused's binding takes the type of, and the bias
gradient that the library writes in fp32: tensors that are read or written past
their end, or wrongly, are refused (tensors on the host stand for those on the
GPU; a missing workspace is the library's last check before the first device
call)."""
import pytest
import torch

from paper_2606_11718_amd import ccl

P = 1 << 20
N = 1024


def _plan():
    return ccl.ccl_plan_typed(512, N, 512, 8, 2, 4096, ccl.CCL_DT_BF16, ccl.CCL_DT_BF16)


def _bias(bias, **more):
    with pytest.raises(ccl.CCLError) as e:
        ccl.ccl_gemm_fused(_plan(), P, P, P, bias=bias, splits=4, **more)
    assert e.value.status_name == "CCL_ERR_INVALID_ARG"
    return str(e.value)


def _dbias(dbias, gated=False):
    with pytest.raises(ccl.CCLError) as e:
        ccl.ccl_gemm_fused_grad(_plan(), P, P, P, P, activation=ccl.CCL_ACT_SILU, gated=gated, dbias=dbias)
    assert e.value.status_name == "CCL_ERR_INVALID_ARG"
    return str(e.value)


@pytest.mark.parametrize("gated", [False, True])
def test_taken(gated):
    for dtype in (torch.float32, torch.bfloat16):
        assert "workspace" in _bias(torch.zeros(N, dtype=dtype), gated=gated)
        assert "workspace" in _bias(torch.zeros(1, N, dtype=dtype), gated=gated)
    assert "workspace" in _bias(torch.zeros(N, dtype=torch.int16), bias_type=ccl.CCL_DT_BF16, gated=gated)
    assert "workspace" in _bias(P, gated=gated)
    assert "workspace" in _dbias(torch.zeros(2 * N if gated else N), gated)
    assert "workspace" in _dbias(P, gated)


@pytest.mark.parametrize("bias", [
    torch.zeros(N - 4), torch.zeros(2 * N)[::2], torch.zeros(1).expand(N), torch.zeros(N, dtype=torch.float16),
    torch.zeros(N, dtype=torch.float64), torch.zeros(N, dtype=torch.int32)],
    ids=["short", "strided", "broadcast", "fp16", "fp64", "int32"])
def test_bias(bias):
    assert "bias" in _bias(bias) and "workspace" not in _bias(bias)


def test_bias_of_a_stated_type():
    for bias, t in ((torch.zeros(N, dtype=torch.bfloat16), ccl.CCL_DT_FP32), (torch.zeros(N), ccl.CCL_DT_BF16),
                    (torch.zeros(N, dtype=torch.int16), ccl.CCL_DT_FP32)):
        assert "bias" in _bias(bias, bias_type=t) and "workspace" not in _bias(bias, bias_type=t)


@pytest.mark.parametrize("dbias", [
    torch.zeros(N, dtype=torch.bfloat16), torch.zeros(N - 4), torch.zeros(2 * N)[::2], torch.zeros(N, dtype=torch.float64)],
    ids=["bf16", "short", "strided", "fp64"])
def test_dbias(dbias):
    assert "dbias" in _dbias(dbias) and "workspace" not in _dbias(dbias)


def test_dbias_of_a_gated_product():
    assert "dbias" in _dbias(torch.zeros(N), gated=True) and "workspace" not in _dbias(torch.zeros(N), gated=True)
