"""The gfx950 assembly of the FFN operators' kernels, built here from source (no
GPU needed): loads that share an M0 write carry the instruction offsets 0, 1024,
2048, ... in that order with no other M0 write inside the run (see
test_host_isa), and only the kernels on 256x256 tiles, whose accumulators take
half of the registers, use scratch memory."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2606_11718_amd import build as B
from tests.test_host_isa import _lds_offset

SOURCES = ("gemm_fused", "newton_schulz", "moe")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{source: {kernel symbol: its lines}}"""
    if shutil.which(B.HIPCC) is None and not os.path.exists(B.HIPCC):
        pytest.skip("hipcc not available")
    out = tmp_path_factory.mktemp("isa")

    def compile_(name):
        path = out / (name + ".s")
        r = subprocess.run([B.HIPCC] + B.HIP_FLAGS + ["-x", "hip", "--cuda-device-only", "-S",
                                                      os.path.join(B.CSRC, "kernels", name + ".hip"), "-o", str(path)],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        text = path.read_text()
        bodies = {}
        for m in re.finditer(r"^(_ZN\w+):", text, re.M):
            bodies[m.group(1)] = [ln.strip() for ln in text[m.end():text.index(".Lfunc_end", m.end())].splitlines()]
        return name, bodies

    with ThreadPoolExecutor(len(SOURCES)) as pool:
        return dict(pool.map(compile_, SOURCES))


def _runs(body):
    runs = []
    for ln in body:
        if re.match(r"s_\w+\s+m0\b", ln):
            runs.append([])
        elif ln.startswith("buffer_load") and re.search(r"\blds\b", ln):
            assert runs, f"direct-to-LDS load before any M0 write: {ln}"
            runs[-1].append(_lds_offset(ln))
    return [r for r in runs if r]


# symbol pattern: (kernels of that kind, lengths of their load runs)
KINDS = {
    "fused_k64_kernelILi256ELi128": (8, {2, 4}), "fused_k64_kernelILi128ELi256": (8, {2, 4}),
    "fused_k64_kernelILi128ELi128": (8, {2}), "fused_k64_kernelILi128ELi192": (12, {2, 3}),
    "fused_k64_kernelILi128ELi320": (12, {1, 2, 4}), "fused_k32_kernel": (8, {1}), "fused_a2_kernel": (2, {2, 4}),
    "fused_fp8p_kernel": (2, {4}), "fused_fp8s_kernelILi256ELi128": (2, {2, 4}),
    "fused_fp8s_kernelILi128ELi256": (2, {2, 4}), "fused_fp8s_kernelILi128ELi128": (2, {2}),
    "ns_product_kernelILi64ELi64": (1, {1}), "ns_product_kernelILi64ELi128": (1, {1, 2}),
    "ns_product_kernelILi128ELi128": (4, {2}), "ns_product_kernelILi256ELi256": (2, {4}),
}


@pytest.mark.parametrize("kind", list(KINDS))
def test_load_runs(kernels, kind):
    count, lengths = KINDS[kind]
    found = {n: b for bodies in kernels.values() for n, b in bodies.items() if kind in n}
    assert len(found) == count, list(found)
    for name, body in found.items():
        runs = _runs(body)
        assert len(runs) > 5, name
        assert all(r == [1024 * i for i in range(len(r))] for r in runs), name
        assert {len(r) for r in runs} == lengths, name


def test_every_kernel_with_such_loads_is_looked_at(kernels):
    for bodies in kernels.values():
        for name, body in bodies.items():
            assert not _runs(body) or any(kind in name for kind in KINDS), name


def test_scratch(kernels):
    full = ("fused_a2_kernel", "fused_fp8p_kernel", "fused_k32_kernelILi256ELi256", "ns_product_kernelILi256ELi256")
    for bodies in kernels.values():
        for name, body in bodies.items():
            if not any(k in name for k in full):
                assert not [ln for ln in body if ln.startswith("scratch_")][:2], name
