"""What the FFN operators launch, asked of the library's own rules compiled for
the host (tests/c/forms.cpp), and the cases that the parity tests run to reach
every form. A case whose rule moves elsewhere fails the host test beside it."""
import functools
import os
import pathlib
import subprocess
import tempfile

ROOT = pathlib.Path(__file__).resolve().parent.parent
CSRC = ROOT / "paper_2606_11718_amd" / "csrc"


@functools.lru_cache(maxsize=None)
def _program() -> str:
    exe = os.path.join(tempfile.mkdtemp(prefix="ccl_forms_"), "forms")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", str(CSRC), "-I", str(CSRC / "host"),
                    str(ROOT / "tests" / "c" / "forms.cpp"), str(CSRC / "host" / "plan.cpp"), "-o", exe], check=True)
    return exe


def ask(*question, env=None) -> dict:
    """The form of one call: ("ortho", batch, rows, cols) and so on, as forms.cpp reads them."""
    line = " ".join(str(int(q)) if not isinstance(q, str) else q for q in question)
    out = subprocess.run([_program()], input=line + "\n", capture_output=True, text=True, check=True,
                         env={**os.environ, **(env or {})}).stdout.split()
    return {k: v if k == "kernel" else int(v) for k, v in (pair.split("=") for pair in out)}


# ---- ccl_orthogonalize ----

# (batch, rows, cols): sides off the grid of 128 and 256, wide and tall
ORTHO = [(1, 127, 2300), (2, 2300, 128), (8, 512, 2431), (8, 2400, 500), (12, 639, 640), (8, 1020, 1024), (12, 1150, 1270),
         (3, 4090, 1660), (8, 1024, 3840), (12, 1279, 1400), (4, 2940, 3960), (12, 1400, 1408), (8, 1408, 1400),
         (4, 3300, 3328), (8, 1536, 1530), (4, 128, 4224), (4, 4200, 100), (2, 1150, 3710), (2, 3700, 1151), (8, 4222, 128),
         (2, 1790, 4860), (6, 3710, 1536), (6, 512, 4300), (6, 4220, 510), (6, 2304, 2944)]


def ortho_forms(batch, rows, cols) -> set:
    """(product, tile, two workgroups to a CU, K ranges, ragged at the 256-row tile, tall) of its three products."""
    f = ask("ortho", batch, rows, cols)
    out = set()
    for name in ("gram", "square", "update"):
        tile, ranges, whole = f[name + "_tile"], f[name + "_ranges"], f[name + "_whole"]
        cut = "none" if ranges == 1 else "some" if whole else "all"
        ragged = tile == 256 and (f["pp"] % 256 != 0 or (name == "update" and f["qp"] % 256 != 0))
        out.add((name, tile, f[name + "_paired"], cut, ragged))
    return out


# Every form that the rules give, and is to be run; the update's also from the
# transpose (tall).
ORTHO_FORMS = {
    ("gram", 64, 0, "none", False), ("gram", 64, 0, "all", False), ("gram", 128, 0, "none", False),
    ("gram", 128, 0, "all", False), ("gram", 128, 1, "none", False), ("gram", 128, 1, "some", False),
    ("gram", 256, 0, "none", False), ("gram", 256, 0, "none", True), ("gram", 256, 0, "all", False),
    ("gram", 256, 0, "all", True), ("gram", 256, 0, "some", False), ("gram", 256, 0, "some", True),
    ("square", 64, 0, "none", False), ("square", 128, 0, "none", False), ("square", 128, 1, "none", False),
    ("square", 128, 1, "some", False), ("square", 256, 0, "none", False), ("square", 256, 0, "none", True),
    ("square", 256, 0, "some", False),
    ("update", 64, 0, "none", False), ("update", 128, 0, "none", False), ("update", 128, 1, "none", False),
    ("update", 128, 1, "some", False), ("update", 256, 0, "none", False), ("update", 256, 0, "none", True),
    ("update", 256, 0, "some", False), ("update", 256, 0, "some", True),
}
ORTHO_TALL = {("update", 64, 0, "none"), ("update", 128, 0, "none"), ("update", 128, 1, "none"), ("update", 128, 1, "some"),
              ("update", 256, 0, "none"), ("update", 256, 0, "some")}

# ---- ccl_moe_decode ----

# (tokens, hidden, ffn, experts, top_k): streaming up workgroups whose waves take
# several chunks of K, the down product on four column tiles with many lines a
# wave, in ranges and not, and column tiles past the last
MOE = [(64, 6144, 1024, 30, 8), (3, 6144, 1024, 30, 8), (48, 2048, 768, 40, 8), (64, 1040, 2064, 12, 4), (17, 4112, 1200, 20, 4),
       (2, 4112, 2064, 24, 8), (9, 528, 2064, 40, 4), (33, 16400, 512, 8, 4), (1, 8208, 1040, 9, 8), (64, 5008, 144, 512, 16)]


def moe_form(case, fp8) -> dict:
    """The form, with the chunks of K that a wave of the up product takes and the lines of a wave of the down product."""
    tokens, hidden, ffn, experts, top_k = case
    f = ask("moe", tokens, hidden, ffn, experts, top_k, fp8)
    size = 1 if fp8 else 2
    per = -(-(-(-hidden * size // 128)) // 8)
    f["chunks"] = -(-per // (2 if fp8 else 4))
    used = min(experts, tokens * top_k)
    f["lines"] = used * -(-ffn * size // 128) / (f["ranges"] * 8)
    f["clamped"] = f["down_tiles"] % f["down_nt"] != 0
    return f

# ---- ccl_gemm_fused, ccl_gemm_fused_grad ----


def _fused(M, N, K, grid_rows, rows, *, grad=False, gated=False, fp8=False, splits=1, chiplets=8, env=None, **expect):
    return dict(M=M, N=N, K=K, grid_rows=grid_rows, rows=rows, grad=grad, gated=gated, fp8=fp8, splits=splits,
                chiplets=chiplets, env=env or {}, expect=expect)


def _both(*args, **more):
    """The forward and the gradient call, plain and gated."""
    return [_fused(*args, grad=grad, gated=gated, **more) for grad in (False, True) for gated in (False, True)]


FUSED = (
    # the tiles with valid rows go round all XCDs
    _both(1024, 4224, 256, 8, 100, remap=0, kernel="gemm_kernel", tile_m=128, tile_n=128)
    + _both(2048, 6272, 256, 8, 100, remap=0, kernel="gemm_kernel", tile_m=256, tile_n=128)
    + _both(512, 8960, 256, 4, 100, remap=0, kernel="gemm_k64_kernel", tile_m=128, tile_n=128)
    + _both(1024, 12544, 256, 4, 300, remap=0, kernel="gemm_k64_kernel", tile_m=256, tile_n=128)
    + _both(512, 16896, 256, 4, 100, remap=0, kernel="gemm_k64_kernel", tile_m=128, tile_n=192, ragged=0)
    + _both(1024, 8448, 768, 8, 129, remap=0, kernel="gemm_k64_kernel", tile_m=128, tile_n=192, ragged=1)
    + _both(2048, 8960, 256, 4, 1025, remap=0, kernel="gemm_k64_kernel", tile_m=128, tile_n=320, ragged=0)
    + _both(2048, 8320, 768, 8, 1025, remap=0, kernel="gemm_k64_kernel", tile_m=128, tile_n=320, ragged=1)
    + _both(1024, 4224, 1024, 8, 100, fp8=True, remap=0, kernel="gemm_fp8s_kernel", tile_m=128, tile_n=128)
    + _both(2048, 6272, 1024, 8, 300, fp8=True, remap=0, kernel="gemm_fp8s_kernel", tile_m=256, tile_n=128)
    + [_fused(4096, 6400, 1024, 8, 2049, remap=0, kernel="gemm_a2_kernel"),
       _fused(4096, 6400, 1024, 8, 2049, grad=True, remap=0, kernel="gemm_a2_kernel")]
    + _both(4096, 6400, 1024, 8, 2049, fp8=True, remap=0, kernel="gemm_fp8p_kernel")
    # short K: 128x128 tiles, two workgroups to a CU, in place of larger ones
    + _both(2048, 4608, 256, 2, 1900, kernel="gemm_kernel", tile_m=128, tile_n=128, direct=1)
    + [_fused(4096, 4096, 128, 2, 4001, kernel="gemm_kernel", tile_m=128, tile_n=128),
       _fused(4096, 4096, 128, 2, 4001, grad=True, gated=True, kernel="gemm_kernel", tile_m=128, tile_n=128)]
    # K ranges, whole tiles without a valid row: their partials are not written
    + [c for rows in (0, 5, 100, 256) for c in
       _both(256, 512, 4096, 2, rows, chiplets=4, splits=16, direct=0, own=1, ranges=16, kernel="gemm_k64_kernel")]
    + [c for rows in (0, 5, 200) for c in
       _both(256, 512, 4096, 2, rows, chiplets=4, splits=16, fp8=True, direct=0, own=1, ranges=8, kernel="gemm_fp8s_kernel")]
    # the form for operands of 2 GiB and more, by way of one range's partials
    + [c for tile in ("128x128", "256x128", "128x256") for c in
       _both(512, 2048, 512, 1, 300, env={"CCL_GEMM_FAR": "1", "CCL_GEMM_TILE": tile}, direct=0, far=1, ranges=1)]
    # and with K ranges
    + _both(256, 512, 4096, 2, 100, chiplets=4, splits=16, env={"CCL_GEMM_FAR": "1"}, direct=0, far=1, ranges=16)
)


def fused_moved(case) -> int:
    """Bytes of C, Z and R an element of A B, for a forward call that reads a residual and keeps Z."""
    wide = 2 if case["gated"] else 1
    return 4 * wide if case["grad"] else 4 // wide + 2


def fused_form(case) -> dict:
    c = case
    return ask("fused", c["M"], c["N"], c["K"], c["chiplets"], c["grid_rows"], 4096, c["fp8"], 0, 16 if c["grad"] else c["splits"],
               c["grad"], c["gated"], c["grad"], c["rows"], fused_moved(c), env=c["env"])


def fused_name(c) -> str:
    return "-".join([f"{c['M']}x{c['N']}x{c['K']}", "grad" if c["grad"] else "fwd"] + ["gated"] * c["gated"] + ["fp8"] * c["fp8"] +
                    [f"rows{c['rows']}"] + [f"splits{c['splits']}"] * (c["splits"] > 1) + sorted(c["env"].values()))
