"""The gfx950 assembly of the training operators' kernels, built here from source (no
GPU needed): direct-to-LDS loads that share an M0 write carry the instruction
offsets 0, 1024, ... in that order (see test_host_isa); no packed fp32 arithmetic; and
scratch memory only in the few kernels of 256x256 tiles, whose accumulators take half of the registers, and
there at most what a handful of values take."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2606_11718_amd import build as B
from tests.test_host_isa_operators import _runs

SOURCES = ("grouped", "cross_entropy", "adamw")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{kernel symbol: (its lines, bytes of scratch)}"""
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
        found = {}
        for m in re.finditer(r"^(_ZN\w+):", text, re.M):
            lines = [ln.strip() for ln in text[m.end():text.index(".Lfunc_end", m.end())].splitlines()]
            size = re.search(rf"\.name:\s+{m.group(1)}\n\s+\.private_segment_fixed_size:\s+(\d+)", text)
            if size:
                found[m.group(1)] = (lines, int(size.group(1)))
        return found

    with ThreadPoolExecutor(len(SOURCES)) as pool:
        return {k: v for found in pool.map(compile_, SOURCES) for k, v in found.items()}


# (kernel, tile): (kernels, lengths of their load runs)
KINDS = {
    ("grouped_rows_kernel", "64ELi128"): (4, {1, 2}), ("grouped_rows_kernel", "128ELi128"): (4, {2}),
    ("grouped_rows_kernel", "256ELi256"): (4, {4}), ("grouped_wgrad_kernel", "128ELi128"): (3, {2}),
    ("grouped_wgrad_kernel", "256ELi256"): (3, {4}), ("logits_kernel", "64ELi128"): (1, {1, 2}),
    ("logits_kernel", "128ELi128"): (2, {2}), ("logits_kernel", "256ELi256"): (2, {4}), ("plain_kernel", "64ELi128"): (2, {1, 2}),
    ("plain_kernel", "128ELi128"): (4, {2}), ("plain_kernel", "256ELi256"): (4, {4}),
}


@pytest.mark.parametrize("kind", list(KINDS), ids="-".join)
def test_load_runs(kernels, kind):
    count, lengths = KINDS[kind]
    found = {n: b for n, b in kernels.items() if kind[0] in n and f"ProductTileILi{kind[1]}E" in n}
    assert len(found) == count, list(found)
    for name, (body, _) in found.items():
        runs = _runs(body)
        assert len(runs) > 5, name
        assert all(r == [1024 * i for i in range(len(r))] for r in runs), name
        assert {len(r) for r in runs} == lengths, name


def test_every_kernel_with_such_loads_is_looked_at(kernels):
    of = {k for k, _ in KINDS}
    assert sum(c for c, _ in KINDS.values()) == len([n for n in kernels if any(k in n for k in of)])
    for name, (body, _) in kernels.items():
        assert not _runs(body) or any(k in name for k in of), name


def test_scratch(kernels):
    for name, (_, size) in kernels.items():
        assert size == 0 or ("ProductTileILi256ELi256E" in name and size <= 40), (name, size)


def test_no_packed_fp32(kernels):
    for name, (body, _) in kernels.items():
        assert not [ln for ln in body if re.match(r"v_pk_(add|mul|fma)_f32", ln)], name


def test_the_experts_table_is_read_behind_its_barrier(kernels):
    """Its lanes write it to LDS and what they need of one another's comes by lane: nothing is read from LDS ahead of
    the first barrier."""
    found = [(n, body) for n, (body, _) in kernels.items() if "grouped_rows_kernel" in n or "grouped_wgrad_kernel" in n]
    assert len(found) == 18
    for name, body in found:
        barrier = next(i for i, ln in enumerate(body) if ln.startswith("s_barrier"))
        assert any(ln.startswith("ds_write") for ln in body[:barrier]), name
        assert not [ln for ln in body[:barrier] if ln.startswith("ds_read")], name


def test_counted_stores(kernels):
    """Kernels whose first barrier behind a tile lets that many memory accesses be on their way (all that came before
    them, loads among them, is then there): a wave's end of a tile makes at least these, 16-byte stores one after
    another, with no branch among them and under no lane mask, and the wait has their number."""
    found = [(n, body) for n, (body, _) in kernels.items() if re.search(r"grouped_wgrad_kernel.*WgradOutE0E|plain_kernel.*EELb0EEE", n)]
    assert len(found) == 7, [n for n, _ in found]
    for name, body in found:
        bm, bn, waves, across = (int(re.search(r"ProductTileILi(\d+)ELi(\d+)ELb\dELb\dELi\dELi(\d)ELi(\d)", name).group(i)) for i in (1, 2, 3, 4))
        count = (bm * across // (16 * waves)) * (bn // (16 * across)) // 2
        stores = [i for i, ln in enumerate(body) if ln.startswith("buffer_store_dwordx4")]
        assert len(stores) == count, (name, len(stores), count)
        last_product = max(i for i, ln in enumerate(body[:stores[0]]) if ln.startswith("v_mfma"))
        assert not [ln for ln in body[last_product:stores[-1]] if re.match(r"\S+\s+exec|\S*saveexec|v_cmpx", ln)], name
        assert not [ln for ln in body[stores[0]:stores[-1]] if re.match(r"s_c?branch|s_setpc|s_barrier|\.LBB", ln)], name
        waits = [i for i, ln in enumerate(body) if re.match(rf"s_waitcnt vmcnt\({count}\) lgkmcnt\(0\)", ln)]
        behind = [next(ln for ln in body[i + 1:] if not ln.startswith(";")) for i in waits]
        assert [ln for ln in behind if ln.startswith(("s_barrier", "s_branch"))], (name, behind)
