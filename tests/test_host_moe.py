"""What ccl_moe_decode and its query refuse (every refusal comes before the
first device call), and the workspace's monotony."""
import pytest

from paper_2606_11718_amd import ccl

P = 1 << 20
OK = dict(hidden=256, ffn=64, experts=16, top_k=4)


def _refused(status, call, *args, **more):
    with pytest.raises(ccl.CCLError) as e:
        call(*args, **more)
    assert e.value.status_name == status, str(e.value)


@pytest.mark.parametrize("change,status", [
    (dict(hidden=0), "CCL_ERR_INVALID_ARG"),
    (dict(ffn=-16), "CCL_ERR_INVALID_ARG"),
    (dict(hidden=250), "CCL_ERR_UNSUPPORTED"),
    (dict(ffn=72), "CCL_ERR_UNSUPPORTED"),
    (dict(hidden=1 << 25), "CCL_ERR_UNSUPPORTED"),
    (dict(experts=0), "CCL_ERR_INVALID_ARG"),
    (dict(experts=513), "CCL_ERR_INVALID_ARG"),
    (dict(top_k=0), "CCL_ERR_INVALID_ARG"),
    (dict(top_k=17, experts=32), "CCL_ERR_INVALID_ARG"),
    (dict(top_k=5, experts=4), "CCL_ERR_INVALID_ARG"),
    (dict(activation=7), "CCL_ERR_INVALID_ARG"),
    (dict(normalize=2), "CCL_ERR_INVALID_ARG"),
    (dict(weight_type=ccl.CCL_DT_FP32), "CCL_ERR_INVALID_ARG"),
    (dict(gate_up_ld=255), "CCL_ERR_INVALID_ARG"),
    (dict(gate_up_ld=-256), "CCL_ERR_INVALID_ARG"),
    (dict(gate_up_ld=260), "CCL_ERR_MISALIGNED_POINTER"),
    (dict(down_ld=264, weight_type=ccl.CCL_DT_FP8_E4M3), "CCL_ERR_MISALIGNED_POINTER"),
    (dict(gate_up_stride=2 * 64 * 256 - 8), "CCL_ERR_INVALID_ARG"),
    (dict(down_stride=1 << 49), "CCL_ERR_INVALID_ARG"),
])
def test_layer_refusals(change, status):
    moe = ccl.ccl_moe(**{**OK, **change})
    _refused(status, ccl.ccl_moe_workspace, moe, 4)
    _refused(status, ccl.ccl_moe_decode, moe, 4, P, P, P, P, P, workspace=P, workspace_bytes=1 << 40)


@pytest.mark.parametrize("more,status", [
    (dict(workspace=None), "CCL_ERR_INVALID_ARG"),
    (dict(workspace_bytes=8), "CCL_ERR_INVALID_ARG"),
    (dict(workspace=P + 4), "CCL_ERR_MISALIGNED_POINTER"),
    (dict(x_ld=255), "CCL_ERR_INVALID_ARG"),
    (dict(x_ld=260), "CCL_ERR_MISALIGNED_POINTER"),
    (dict(y_ld=200), "CCL_ERR_INVALID_ARG"),
    (dict(logits_ld=15), "CCL_ERR_INVALID_ARG"),
    (dict(ids=P + 2), "CCL_ERR_MISALIGNED_POINTER"),
    (dict(probs=P + 1), "CCL_ERR_MISALIGNED_POINTER"),
    (dict(gate_up_scale=P + 2), "CCL_ERR_MISALIGNED_POINTER"),
])
def test_call_refusals(more, status):
    args = {"workspace": P, "workspace_bytes": 1 << 40, **more}
    _refused(status, ccl.ccl_moe_decode, ccl.ccl_moe(**OK), 4, P, P, P, P, P, **args)


def test_operands_and_tokens():
    moe = ccl.ccl_moe(**OK)
    for i in range(5):
        args = [P] * 5
        args[i] = None
        _refused("CCL_ERR_INVALID_ARG", ccl.ccl_moe_decode, moe, 1, *args, workspace=P, workspace_bytes=1 << 40)
    for i in (0, 2, 3):          # x and the weights
        args = [P] * 5
        args[i] = P + 8
        _refused("CCL_ERR_MISALIGNED_POINTER", ccl.ccl_moe_decode, moe, 1, *args, workspace=P, workspace_bytes=1 << 40)
    for t in (-1, 65):
        _refused("CCL_ERR_INVALID_ARG", ccl.ccl_moe_workspace, moe, t)
    ccl.ccl_moe_decode(moe, 0, None, None, None, None, None)       # no tokens: nothing to do


def test_workspace_serves_fewer_tokens():
    moe = ccl.ccl_moe(hidden=4096, ffn=1024, experts=64, top_k=8)
    sizes = [ccl.ccl_moe_workspace(moe, t) for t in range(65)]
    assert sizes == sorted(sizes) and sizes[1] > 0
