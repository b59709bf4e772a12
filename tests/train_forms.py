"""What the training operators launch, asked of the library's own rules compiled for
the host (tests/c/train_forms.cpp), and the cases that the parity tests run to reach
every form. A case whose rule moves elsewhere fails the host test beside it."""
import functools
import os
import pathlib
import subprocess
import tempfile

ROOT = pathlib.Path(__file__).resolve().parent.parent
CSRC = ROOT / "paper_2606_11718_amd" / "csrc"
FORWARD, GRAD, WGRAD = 0, 1, 2


@functools.lru_cache(maxsize=None)
def _program() -> str:
    exe = os.path.join(tempfile.mkdtemp(prefix="ccl_train_forms_"), "forms")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", str(CSRC), str(ROOT / "tests" / "c" / "train_forms.cpp"),
                    str(CSRC / "host" / "train.cpp"), "-o", exe], check=True)
    return exe


def ask_many(questions) -> list:
    lines = "\n".join(" ".join(str(int(q)) if not isinstance(q, str) else q for q in one) for one in questions) + "\n"
    out = subprocess.run([_program()], input=lines, capture_output=True, text=True, check=True).stdout.splitlines()
    return [{k: int(v) for k, v in (pair.split("=") for pair in line.split())} for line in out]


def ask(*question) -> dict:
    return ask_many([question])[0]


# (tile rows, K ranges or not): (direction, counts, in, out, gated). Sides off the
# grids of 64, 128 and 256, experts without rows, rows behind no whole tile.
GROUPED = {
    (64, False): [(FORWARD, [3, 0, 70, 1] * 20, 80, 96, False), (FORWARD, [5, 0, 131, 64] * 20, 464, 160, True),
                  (GRAD, [3, 0, 70, 1] * 20, 144, 80, True), (GRAD, [2] * 130, 272, 48, False)],
    (64, True): [(FORWARD, [1], 4112, 272, False), (FORWARD, [40, 0, 3], 1040, 96, True), (GRAD, [9, 0, 30], 144, 1040, True),
                 (GRAD, [5], 48, 2064, False)],
    (128, False): [(FORWARD, [300, 0, 129], 336, 288, True), (GRAD, [40, 300], 272, 272, True),
                   (WGRAD, [130, 0, 1, 127], 144, 272, False)],
    (128, True): [(FORWARD, [300, 129], 1040, 288, True), (FORWARD, [200], 528, 144, False), (GRAD, [400], 272, 1040, True),
                  (GRAD, [200, 0, 250], 144, 528, False), (WGRAD, [600, 0, 1500], 144, 272, False), (WGRAD, [3000], 16, 32, False)],
    (256, False): [(FORWARD, [700, 900], 80, 8208, False), (FORWARD, [600, 0, 1000], 144, 11040, True),
                   (FORWARD, [300] * 40, 64, 2080, True), (GRAD, [700, 900], 16368, 48, False), (GRAD, [700, 900], 16400, 144, True),
                   (WGRAD, [70, 0, 130, 1], 2000, 2032, False)],
}
# loss: (tokens, hidden, vocab)
LOGITS = {64: [(1, 2064, 1000), (64, 48, 700), (65, 80, 700), (300, 336, 2049), (64, 32, 40000)],
          128: [(300, 336, 8001), (130, 16, 16300), (300, 80, 12000)], 256: [(250, 80, 65400), (1000, 128, 16300)]}
# 256x256 tiles over whole rounds, 64x128 and 128x128 ones over the columns behind them
LOGITS_REST = {64: [(1000, 528, 16701)], 128: [(2290, 512, 8257)]}
DX_REST = [(9000, 2080, 600), (15000, 1040, 2100)]
DW_REST = [(520, 1040, 13900)]
# (tile rows, K ranges or not)
DX = {(64, True): [(3, 80, 3000), (64, 272, 2100)], (64, False): [(50, 80, 700)], (128, True): [(130, 272, 2100)],
      (128, False): [(130, 80, 700)], (256, False): [(2000, 8176, 300)], (256, True): [(400, 1040, 49999)]}
DW = {128: [(70, 272, 2100)], 256: [(70, 4080, 4001)]}
