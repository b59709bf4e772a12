"""What ccl_gemm_fused, its gradient and their queries refuse (no GPU needed:
every refusal comes before the first device call), and the workspaces they ask
for."""
import pathlib
import subprocess

import pytest

from paper_2606_11718_amd import ccl

P = 1 << 20     # an aligned address that is never read


def _plan(c=ccl.CCL_DT_BF16, ab=ccl.CCL_DT_BF16):
    return ccl.ccl_plan_typed(512, 1024, 512, 8, 2, 4096, ab, c)


def _refused(status, call, *args, **more):
    with pytest.raises(ccl.CCLError) as e:
        call(*args, **more)
    assert e.value.status_name == status, str(e.value)


@pytest.mark.parametrize("more,status", [
    (dict(activation=4), "CCL_ERR_INVALID_ARG"),
    (dict(activation=-1), "CCL_ERR_INVALID_ARG"),
    (dict(layout=2), "CCL_ERR_INVALID_ARG"),
    (dict(gated=2), "CCL_ERR_INVALID_ARG"),
    (dict(rows=513), "CCL_ERR_INVALID_ARG"),
    (dict(rows=-1), "CCL_ERR_INVALID_ARG"),
    (dict(splits=0), "CCL_ERR_INVALID_ARG"),
    (dict(splits=17), "CCL_ERR_INVALID_ARG"),
    (dict(splits=4), "CCL_ERR_INVALID_ARG"),                                   # no workspace
    (dict(splits=4, workspace=P, workspace_bytes=64), "CCL_ERR_INVALID_ARG"),  # too small
    (dict(splits=4, workspace=P + 8, workspace_bytes=1 << 40), "CCL_ERR_MISALIGNED_POINTER"),
    (dict(bias=P, bias_type=ccl.CCL_DT_FP8_E4M3), "CCL_ERR_INVALID_ARG"),
    (dict(bias=P + 4), "CCL_ERR_MISALIGNED_POINTER"),
    (dict(residual=P + 2), "CCL_ERR_MISALIGNED_POINTER"),
    (dict(preact=P + 8), "CCL_ERR_MISALIGNED_POINTER"),
])
def test_forward_refusals(more, status):
    _refused(status, ccl.ccl_gemm_fused, _plan(), P, P, P, **more)


@pytest.mark.parametrize("more,status", [
    (dict(activation=9), "CCL_ERR_INVALID_ARG"),
    (dict(layout=-1), "CCL_ERR_INVALID_ARG"),
    (dict(gated=3), "CCL_ERR_INVALID_ARG"),
    (dict(rows=1 << 40), "CCL_ERR_INVALID_ARG"),
    (dict(dbias=P), "CCL_ERR_INVALID_ARG"),                                    # no workspace for the sums
    (dict(dbias=P + 4, workspace=P, workspace_bytes=1 << 40), "CCL_ERR_MISALIGNED_POINTER"),
])
def test_grad_refusals(more, status):
    _refused(status, ccl.ccl_gemm_fused_grad, _plan(), P, P, P, P, **more)


def test_null_and_misaligned_operands():
    for args in ((None, P, P), (P, None, P), (P, P, None)):
        _refused("CCL_ERR_INVALID_ARG", ccl.ccl_gemm_fused, _plan(), *args)
    for args in ((P + 8, P, P), (P, P + 2, P), (P, P, P + 4)):
        _refused("CCL_ERR_MISALIGNED_POINTER", ccl.ccl_gemm_fused, _plan(), *args)
    for args in ((None, P, P, P), (P, None, P, P), (P, P, P, None)):
        _refused("CCL_ERR_INVALID_ARG", ccl.ccl_gemm_fused_grad, _plan(), *args)
    # pre-activations may be missing only where no formula needs them
    _refused("CCL_ERR_INVALID_ARG", ccl.ccl_gemm_fused_grad, _plan(), P, P, None, P, activation=ccl.CCL_ACT_SILU)
    _refused("CCL_ERR_INVALID_ARG", ccl.ccl_gemm_fused_grad, _plan(), P, P, None, P, gated=True)
    _refused("CCL_ERR_MISALIGNED_POINTER", ccl.ccl_gemm_fused_grad, _plan(), P, P, P + 8, P)


def test_fp32_results_and_operands_are_refused():
    _refused("CCL_ERR_UNSUPPORTED", ccl.ccl_gemm_fused, _plan(c=ccl.CCL_DT_FP32), P, P, P)
    _refused("CCL_ERR_UNSUPPORTED", ccl.ccl_gemm_fused_grad, _plan(c=ccl.CCL_DT_FP32), P, P, P, P)
    _refused("CCL_ERR_UNSUPPORTED", ccl.ccl_gemm_fused, _plan(ab=ccl.CCL_DT_FP32), P, P, P)


def test_queries():
    plan = _plan()
    chosen = ccl.ccl_gemm_splitk_workspace(plan, 0)[0]
    assert chosen == 2                               # 16 K steps in ranges of 8
    for asked in (0, 2, 4):                          # no more than the CUs have use for
        assert ccl.ccl_gemm_fused_workspace(plan, asked) == ccl.ccl_gemm_splitk_workspace(plan, chosen)
    assert ccl.ccl_gemm_fused_workspace(plan, 1) == (1, 0)
    _refused("CCL_ERR_INVALID_ARG", ccl.ccl_gemm_fused_workspace, plan, 17)
    _refused("CCL_ERR_INVALID_ARG", ccl.ccl_gemm_fused_workspace, plan, -1)
    _refused("CCL_ERR_INVALID_ARG", ccl.ccl_gemm_fused_workspace, plan, 1, layout=5)
    plain = ccl.ccl_gemm_fused_grad_workspace(plan, dbias=False)
    sums = ccl.ccl_gemm_fused_grad_workspace(plan, dbias=True) - plain
    assert sums > 0
    assert ccl.ccl_gemm_fused_grad_workspace(plan, gated=True, dbias=True) == plain + 2 * sums


def test_matrix_layout():
    plan = _plan()
    assert ccl.ccl_plan_matrix_layout(plan, 1024) == ccl.ccl_plan_layout(plan, ccl.CCL_C)
    assert ccl.ccl_plan_matrix_layout(plan, 512) == ccl.ccl_plan_layout(plan, ccl.CCL_A)
    lay = ccl.ccl_plan_matrix_layout(plan, 2048)
    assert (lay.block_rows, lay.block_cols, lay.total_bytes) == (256, 512, 512 * 2048 * 2)
    for cols in (0, -4, 6, 1 << 31):
        _refused("CCL_ERR_INVALID_ARG", ccl.ccl_plan_matrix_layout, plan, cols)


def test_live_map_covers_every_tile_once(tmp_path):
    """The map over the tiles with valid rows, compiled for the host."""
    root = pathlib.Path(__file__).resolve().parent.parent
    exe = tmp_path / "live_map"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", str(root / "paper_2606_11718_amd/csrc/host"),
                    str(root / "tests/c/live_map.cpp"), "-o", str(exe)], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout
