"""The launch rules of the training operators: the parity tests' cases reach the forms
they are there for, and over a spread of sizes every tile has its workgroup and the
ranges their workspace."""
import random

import numpy as np
import pytest

from paper_2606_11718_amd import ccl
from tests import train_forms as F


@pytest.mark.parametrize("form", list(F.GROUPED), ids=str)
def test_grouped_cases(form):
    for way, counts, K, N, gated in F.GROUPED[form]:
        got = F.ask("grouped", way, len(counts), N, K, gated, sum(counts))
        assert (got["tile_m"], got["splits"] > 1) == form, (way, counts[:4], K, N, got)
        g = ccl.ccl_grouped(in_features=K, out_features=N, experts=len(counts), gated=gated)
        assert ccl.ccl_grouped_gemm_workspace(g, sum(counts), way) >= got["bytes"]


def test_loss_cases():
    for tile, cases in F.LOGITS.items():
        for t, D, V in cases:
            assert F.ask("logits", D, V, t)["tile_m"] == tile, (t, D, V)
    # both numbers of stages
    assert {F.ask("logits", D, V, t)["tiles"] <= 256 for t, D, V in F.LOGITS[128]} == {True, False}
    for tile, cases in F.LOGITS_REST.items():
        for t, D, V in cases:
            whole, rest = F.ask("logits", D, V, t), F.ask("logits_rest", D, V, t)
            assert whole["tile_m"] == 256 and whole["tiles"] <= 256 and rest["tiles"] and rest["tile_m"] == tile, (t, D, V, whole, rest)
    for t, D, V in F.DX_REST:
        assert F.ask("dx", D, V, t)["tile_m"] == 256 and F.ask("dx_rest", D, V, t)["tiles"] > 0, (t, D, V)
    for t, D, V in F.DW_REST:
        assert F.ask("dw", D, V, t)["tile_m"] == 256 and F.ask("dw_rest", D, V, t)["tiles"] > 0, (t, D, V)
    for form, cases in F.DX.items():
        for t, D, V in cases:
            got = F.ask("dx", D, V, t)
            assert (got["tile_m"], got["splits"] > 1) == form, (t, D, V, got)
    for tile, cases in F.DW.items():
        for t, D, V in cases:
            assert F.ask("dw", D, V, t)["tile_m"] == tile, (t, D, V)


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _dealt(f):
    """Every tile of a round has its workgroup: the kernels' numbering (dealt_tile), whose
    rounds follow one another, odd ones with the workgroups backwards."""
    block = np.arange(f["workgroups"])
    slot, chunk = block // 8, f["chunk"]
    tile = (slot // chunk * 8 + block % 8) * chunk + slot % chunk
    return np.array_equal(np.sort(tile), block)


def test_launches_over_a_spread_of_sizes():
    rng = random.Random(5)
    cases = [(rng.randint(0, 2), _log(rng, 1, 512), 16 * _log(rng, 1, 2048), 16 * _log(rng, 1, 2048), 0, _log(rng, 1, 1 << 20))
             for _ in range(3000)]
    for (way, E, N, K, gated, rows), f in zip(cases, F.ask_many([("grouped", *c) for c in cases])):
        per_cu = 1 if f["tile_m"] == 256 else 2
        case = (way, E, N, K, rows, f)
        assert f["workgroups"] % 8 == 0 and 8 <= f["workgroups"] <= 256 * per_cu, case
        assert f["workgroups"] == 256 * per_cu or f["workgroups"] >= f["tiles"], case
        assert _dealt(f), case
        assert f["splits"] == 1 or f["tile_m"] < 256, case        # the kernels of 256x256 tiles know no ranges
        assert 1 <= f["splits"] <= 64 and f["bytes"] <= 32 << 20, case
        columns = {0: N, 1: K, 2: K}[way]
        if f["splits"] > 1:
            assert f["bytes"] == 4 * f["splits"] * (E * N * K if way == 2 else rows * columns), case
            assert f["tiles"] <= 512, case
            g = ccl.ccl_grouped(in_features=K, out_features=N, experts=E)
            assert f["bytes"] <= ccl.ccl_grouped_gemm_workspace(g, rows, way), case
        else:
            assert f["bytes"] == 0, case


def test_loss_launches_over_a_spread_of_sizes():
    rng = random.Random(6)
    cases = [(16 * _log(rng, 1, 1024), _log(rng, 1, 1 << 20), _log(rng, 1, 32768)) for _ in range(1000)]
    for kind in ("logits", "logits_rest", "dx", "dx_rest", "dw", "dw_rest"):
        for c, f in zip(cases, F.ask_many([(kind, *c) for c in cases])):
            per_cu = 1 if f["tile_m"] == 256 else 2
            assert f["workgroups"] % 8 == 0 and 8 <= f["workgroups"] <= 256 * per_cu, (kind, c, f)
            assert f["workgroups"] == 256 * per_cu or f["workgroups"] >= f["tiles"], (kind, c, f)
            assert _dealt(f), (kind, c, f)
            assert f["splits"] == 1 or kind[:2] == "dx", (kind, c, f)
            assert f["bytes"] <= 64 << 20, (kind, c, f)
    for (D, V, t), f in zip(cases, F.ask_many([("vocab", *c, 1) for c in cases])):
        assert (f["blocks"] - 1) * f["block"] < t <= f["blocks"] * f["block"], (D, V, t, f)
        assert f["bytes"] == ccl.ccl_cross_entropy_workspace(ccl.ccl_vocab(hidden=D, vocab=V), t, grad=True), (D, V, t, f)
