"""GPU parity of ccl_gemm_fused and ccl_gemm_fused_grad with the fp64 oracle.

Elementwise bound, fixed by the arithmetic: the result is rounded to bf16 once
(8 significant bits: half a
spacing is at most 2^-8 relative), and what is rounded carries the fp32 errors of the K-term
accumulation (at most K 2^-23 sum |a b|, the products of bf16 or fp8 values
being exact) and of the activation (32 fp32 ulps of its argument's size),
both multiplied by what the formula multiplies them by. Rows that are not
valid are exactly zero.
"""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import ffn as OF
from oracle import gemm as OG
from oracle import layout as OL
from paper_2606_11718_amd import ccl
from tests.helpers import dev_full, from_dev, to_dev

pytestmark = pytest.mark.gpu

NAN16 = 0x7FC0


def _bytes_dev(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.uint8).reshape(-1)).to("cuda")


def _store(bits, layout, gr, gc, page):
    """Row-major bits as the call takes them."""
    return OL.pack(bits, gr, gc, page) if layout == ccl.CCL_LAYOUT_CCL else np.ascontiguousarray(bits)


def _load(t, rows, cols, layout, gr, gc, page):
    bits = from_dev(t)
    if layout == ccl.CCL_LAYOUT_CCL:
        return OL.unpack(bits, rows, cols, gr, gc, page)
    return bits.reshape(rows, cols)


def _matrix_elems(plan, cols, layout, M):
    if layout == ccl.CCL_LAYOUT_CCL:
        return ccl.ccl_plan_matrix_layout(plan, cols).total_bytes // 2
    return M * cols


def _within(got, want, err, rows, what):
    """|got - want| <= 2^-8 |want| + err elementwise on the valid rows (of the
    larger of the two: a value may round across a power of two), zeros below."""
    assert not got[rows:].any(), f"{what}: rows past the valid ones"
    g, w = got[:rows], want[:rows]
    bad = ~(np.abs(g - w) <= 2.0 ** -8 * np.maximum(np.abs(g), np.abs(w)) + err[:rows] + 1e-37)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), g[bad][:3], w[bad][:3])


# M, N, K, G, grid rows, page
SMALL = (256, 512, 256, 4, 2, 4096)
EXPERT = (512, 768, 512, 8, 4, 65536)
WIDE = (256, 2048, 256, 8, 1, 4096)
TALL = (2048, 256, 384, 8, 4, 4096)
ODD32 = (512, 512, 352, 1, 1, 4096)          # K = 11 * 32


def _forward(shape, kind, gated=False, bias=None, residual=False, keep=True, rows=None, layout=ccl.CCL_LAYOUT_CCL,
             splits=1, fp8=False, alpha=1.0, beta=1.0, in_place=False, seed=9000, spoil=False):
    M, N, K, G, Gr, P = shape
    ab = ccl.CCL_DT_FP8_E4M3 if fp8 else ccl.CCL_DT_BF16
    plan = ccl.ccl_plan_typed(M, N, K, G, Gr, P, ab, ccl.CCL_DT_BF16)
    gr, gc = ccl.ccl_plan_grid(plan)
    rows = M if rows is None else rows
    print(f"fused {M}x{N}x{K} grid {gr}x{gc} act={kind} gated={gated} rows={rows} layout={layout} splits={splits} fp8={fp8}",
          flush=True)
    draw = W.draw_array_fp8 if fp8 else W.draw_array
    A = draw(seed, M, K, "normal", 1.0)
    B = draw(seed + 1, K, N, "normal", 1.0 if fp8 else 0.06)
    Av = OG.decode_fp8_e4m3(A) if fp8 else OG.decode_bf16(A)
    Bv = OG.decode_fp8_e4m3(B) if fp8 else OG.decode_bf16(B)
    cols = N // 2 if gated else N
    R = W.draw_array(seed + 2, M, cols, "normal", 1.0) if residual else None
    if spoil and rows < M:          # what the rows past the valid ones hold must not matter
        A = A.copy()
        A[rows:] = 0x7F if fp8 else NAN16
        if residual:
            R[rows:] = NAN16
    rng = np.random.default_rng(seed + 3)
    bv = bdev = None
    if bias == "f32":
        bv = rng.standard_normal(N).astype(np.float32)
        bdev = torch.from_numpy(bv).cuda()
    elif bias == "bf16":
        bits = W.draw_array(seed + 4, 1, N, "normal", 1.0)
        bv = OG.decode_bf16(bits)[0]
        bdev = to_dev(bits).view(torch.bfloat16).reshape(-1)
    put = lambda x: _bytes_dev(_store(x, layout, gr, gc, P))  # noqa: E731
    Ad, Bd = put(A), put(B)
    Rd = put(R) if residual else None
    C = Rd.view(torch.int16) if in_place else dev_full(_matrix_elems(plan, cols, layout, M))
    Z = dev_full(_matrix_elems(plan, N, layout, M)) if keep else None
    _, need = ccl.ccl_gemm_fused_workspace(plan, splits, layout=layout)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    ccl.ccl_gemm_fused(plan, Ad, Bd, C, activation=kind, gated=gated, bias=bdev, residual=Rd, beta=beta, preact=Z,
                       alpha=alpha, rows=rows, layout=layout, splits=splits, workspace=ws, workspace_bytes=need)
    Rv = OG.decode_bf16(R) if residual else None
    with np.errstate(invalid="ignore"):
        want, Zw = OF.linear(Av, Bv, kind, gated, bv, Rv, beta, alpha, rows)
        ez = abs(alpha) * K * 2.0 ** -23 * (np.abs(Av) @ np.abs(Bv)) + 2.0 ** -22 * np.abs(Zw)
    if gated:
        g, u = OF.split_gated(Zw)
        eg, eu = OF.split_gated(ez)
        ec = 1.2 * (eg + 2.0 ** -18 * np.abs(g)) * (np.abs(u) + eu) + np.abs(g) * eu
    else:
        ec = 1.2 * (ez + 2.0 ** -18 * np.abs(Zw))
    if residual:
        ec = ec + 2.0 ** -22 * np.abs(beta * np.nan_to_num(Rv))
    _within(OG.decode_bf16(_load(C, M, cols, layout, gr, gc, P)), want, ec, rows, "C")
    if keep:
        _within(OG.decode_bf16(_load(Z, M, N, layout, gr, gc, P)), Zw, ez, rows, "Z")
    return C


ALL_ACTS = [ccl.CCL_ACT_NONE, ccl.CCL_ACT_RELU, ccl.CCL_ACT_GELU, ccl.CCL_ACT_SILU]
LAYOUTS = [ccl.CCL_LAYOUT_CCL, ccl.CCL_LAYOUT_ROWMAJOR]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kind", ALL_ACTS)
def test_activations(kind, gated, layout):
    _forward(SMALL, kind, gated, bias="f32", residual=True, layout=layout)


@pytest.mark.parametrize("shape", [EXPERT, WIDE, TALL, ODD32, (512, 1024, 1280, 8, 2, 4096)])
@pytest.mark.parametrize("gated", [False, True])
def test_shapes_and_grids(shape, gated):
    _forward(shape, ccl.CCL_ACT_SILU, gated, bias="bf16", residual=True)


@pytest.mark.parametrize("rows", [0, 1, 127, 128, 129, 300, 512])
@pytest.mark.parametrize("gated", [False, True])
def test_ragged_rows(rows, gated):
    _forward(EXPERT, ccl.CCL_ACT_GELU, gated, bias="f32", residual=True, rows=rows, spoil=True)


@pytest.mark.parametrize("splits", [2, 3, 4])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("fp8", [False, True])
def test_split_k(splits, gated, fp8):
    _forward((256, 512, 1024, 4, 2, 4096), ccl.CCL_ACT_SILU, gated, bias="f32", residual=True, splits=splits, fp8=fp8,
             rows=200, spoil=True, alpha=0.03 if fp8 else 1.0)


@pytest.mark.parametrize("tile", ["256x256", "256x128", "128x256", "128x128"])
@pytest.mark.parametrize("waves", ["8", "4"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("K", [512, 576])
def test_every_tile(monkeypatch, tile, waves, fp8, K):
    """Every kernel tile, K blocks of whole and of odd steps."""
    monkeypatch.setenv("CCL_GEMM_TILE", tile)
    monkeypatch.setenv("CCL_GEMM_WAVES", waves)
    for gated in (False, True):
        _forward((512, 512, K, 1, 1, 4096), ccl.CCL_ACT_SILU, gated, bias="f32", residual=True, fp8=fp8, rows=400,
                 alpha=0.05 if fp8 else 1.0, layout=ccl.CCL_LAYOUT_ROWMAJOR)


# 40 tile columns in each of 8 and 4 partition rows: few valid rows leave XCDs idle
@pytest.mark.parametrize("rows", [1, 128, 300, 700, 896])
@pytest.mark.parametrize("shape", [(1024, 5120, 256, 8, 8, 4096), (1024, 10240, 256, 8, 4, 4096)])
@pytest.mark.parametrize("grad", [False, True])
def test_valid_rows_of_few_partitions(shape, rows, grad):
    if grad:
        _backward(shape, ccl.CCL_ACT_SILU, True, rows=rows, spoil=True)
    else:
        _forward(shape, ccl.CCL_ACT_SILU, True, residual=True, rows=rows, spoil=True)


# past one round of the CUs on 128x192, 128x128 and 256x256 tiles, short K: 128x128
# tiles, two workgroups to a CU
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("shape,rows", [((2048, 4608, 256, 8, 2, 4096), 1900), ((1408, 6400, 96, 1, 1, 4096), None),
                                        ((4096, 4096, 128, 8, 2, 4096), 4001)])
def test_paired_workgroups(shape, rows, grad, gated):
    if grad:
        _backward(shape, ccl.CCL_ACT_GELU, gated, rows=rows, spoil=True)
    else:
        _forward(shape, ccl.CCL_ACT_GELU, gated, bias="f32", residual=True, keep=not gated, rows=rows, spoil=True)


# plans whose launch takes 128-row tiles of 192 or 320 columns, whole and odd K
# blocks (K / 8 of 64 i and of 32)
WIDE_TILES = [((256, 1920, 512, 1, 1, 4096), 192), ((256, 1920, 512, 1, 1, 4096), 320),
              ((256, 15360, 768, 8, 1, 4096), 192), ((256, 15360, 768, 8, 1, 4096), 320)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("shape,cols", WIDE_TILES)
def test_wide_tiles(monkeypatch, shape, cols, grad, gated):
    monkeypatch.setenv("CCL_GEMM_WIDE", str(cols))
    plan = ccl.ccl_plan(*shape)
    assert ccl.ccl_debug_launch(plan).tile_cols == cols
    if grad:
        _backward(shape, ccl.CCL_ACT_SILU, gated, rows=200, spoil=True)
    else:
        _forward(shape, ccl.CCL_ACT_SILU, gated, bias="f32", residual=True, rows=200, spoil=True)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("tile", ["256x256", "256x128", "128x256", "128x128"])
def test_odd_k_blocks(monkeypatch, tile, grad, gated):
    """K blocks that are odd multiples of 32: the 32-K kernels and the ragged 64-K ones."""
    monkeypatch.setenv("CCL_GEMM_TILE", tile)
    shape = (512, 2048, 768, 8, 1, 4096)          # K / 8 = 96
    if grad:
        _backward(shape, ccl.CCL_ACT_GELU, gated, rows=300)
    else:
        _forward(shape, ccl.CCL_ACT_GELU, gated, bias="bf16", residual=True, rows=300)


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("bias", [None, "f32", "bf16"])
def test_parts_of_the_epilogue(bias, residual, keep):
    _forward(EXPERT, ccl.CCL_ACT_GELU, False, bias=bias, residual=residual, keep=keep, alpha=-0.5, beta=0.25)


@pytest.mark.parametrize("alpha", [1e20, 1e30])
@pytest.mark.parametrize("kind", ALL_ACTS)
def test_pre_activations_whose_squares_overflow(kind, alpha):
    """Finite in, finite out: z or 0."""
    _forward(SMALL, kind, alpha=alpha)


def test_residual_in_place():
    _forward(EXPERT, ccl.CCL_ACT_NONE, residual=True, keep=False, in_place=True)
    _forward(EXPERT, ccl.CCL_ACT_SILU, gated=True, residual=True, keep=False, in_place=True)


def test_plain_epilogue_equals_the_gemm():
    """No activation, bias or residual: the bits of ccl_gemm."""
    M, N, K, G, Gr, P = EXPERT
    plan = ccl.ccl_plan(M, N, K, G, Gr, P)
    gr, gc = ccl.ccl_plan_grid(plan)
    A = to_dev(OL.pack(W.draw_array(1, M, K, "normal", 1.0), gr, gc, P))
    B = to_dev(OL.pack(W.draw_array(2, K, N, "normal", 0.05), gr, gc, P))
    n = ccl.ccl_plan_layout(plan, ccl.CCL_C).total_bytes // 2
    C1, C2 = dev_full(n), dev_full(n)
    ccl.ccl_gemm(plan, A, B, C1)
    _, need = ccl.ccl_gemm_fused_workspace(plan)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    ccl.ccl_gemm_fused(plan, A, B, C2, workspace=ws, workspace_bytes=need)
    assert np.array_equal(from_dev(C1), from_dev(C2))


def _backward(shape, kind, gated=False, dbias=True, rows=None, layout=ccl.CCL_LAYOUT_CCL, fp8=False, alpha=1.0,
              in_place=False, spoil=False, seed=9500):
    M, N, K, G, Gr, P = shape
    ab = ccl.CCL_DT_FP8_E4M3 if fp8 else ccl.CCL_DT_BF16
    plan = ccl.ccl_plan_typed(M, N, K, G, Gr, P, ab, ccl.CCL_DT_BF16)
    gr, gc = ccl.ccl_plan_grid(plan)
    rows = M if rows is None else rows
    cols = 2 * N if gated else N
    print(f"fused grad {M}x{N}x{K} grid {gr}x{gc} act={kind} gated={gated} rows={rows} layout={layout} fp8={fp8}", flush=True)
    draw, dec = (W.draw_array_fp8, OG.decode_fp8_e4m3) if fp8 else (W.draw_array, OG.decode_bf16)
    A = draw(seed, M, K, "normal", 1.0)
    B = draw(seed + 1, K, N, "normal", 1.0 if fp8 else 0.06)
    Zb = W.draw_array(seed + 2, M, cols, "normal", 2.0)
    Zb[0, :8] = W.round_to_bf16_bits(np.array([0.0, -0.0, 30.0, -30.0, 200.0, -200.0, 3e19, -3e19], np.float32))
    Av, Bv, Zv = dec(A), dec(B), OG.decode_bf16(Zb)
    if spoil and rows < M:
        A = A.copy()
        A[rows:] = 0x7F if fp8 else NAN16
        Zb[rows:] = NAN16
    put = lambda x: _bytes_dev(_store(x, layout, gr, gc, P))  # noqa: E731
    Ad, Bd, Zd = put(A), put(B), put(Zb)
    dZ = Zd.view(torch.int16) if in_place else dev_full(_matrix_elems(plan, cols, layout, M))
    db = torch.full((cols,), float("nan"), device="cuda") if dbias else None
    need = ccl.ccl_gemm_fused_grad_workspace(plan, gated=gated, dbias=dbias, layout=layout)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    ccl.ccl_gemm_fused_grad(plan, Ad, Bd, Zd, dZ, activation=kind, gated=gated, dbias=db, alpha=alpha, rows=rows,
                            layout=layout, workspace=ws, workspace_bytes=need)
    want, dbw = OF.linear_grad(Av, Bv, Zv, kind, gated, alpha, rows)
    ed = abs(alpha) * K * 2.0 ** -23 * (np.abs(Av) @ np.abs(Bv))
    D = np.abs(alpha * (Av @ Bv))
    if gated:
        g, u = np.abs(OF.split_gated(Zv)[0]), np.abs(OF.split_gated(Zv)[1])
        e = OF.join_gated(1.2 * u * (ed + 2.0 ** -18 * D), 1.2 * g * (ed + 2.0 ** -18 * D))
    else:
        e = 1.2 * (ed + 2.0 ** -18 * D)
    _within(OG.decode_bf16(_load(dZ, M, cols, layout, gr, gc, P)), want, e, rows, "dZ")
    if dbias:
        got = db.cpu().numpy().astype(np.float64)
        # the unrounded sums: the elements' errors and M roundings of the running sums
        tol = e[:rows].sum(0) + (M + 8) * 2.0 ** -24 * np.abs(want[:rows]).sum(0) + 1e-30
        assert (np.abs(got - dbw) <= tol).all(), np.abs(got - dbw).max()
    return dZ, db


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kind", ALL_ACTS)
def test_grad_activations(kind, gated, layout):
    _backward(SMALL, kind, gated, layout=layout)


@pytest.mark.parametrize("shape", [EXPERT, WIDE, TALL, ODD32])
@pytest.mark.parametrize("gated", [False, True])
def test_grad_shapes_and_grids(shape, gated):
    _backward(shape, ccl.CCL_ACT_SILU, gated)


@pytest.mark.parametrize("rows", [0, 1, 127, 128, 129, 300, 512])
@pytest.mark.parametrize("gated", [False, True])
def test_grad_ragged_rows(rows, gated):
    _backward(EXPERT, ccl.CCL_ACT_SILU, gated, rows=rows, spoil=True)


@pytest.mark.parametrize("tile", ["256x256", "256x128", "128x256", "128x128"])
@pytest.mark.parametrize("waves", ["8", "4"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("K", [512, 576])
def test_grad_every_tile(monkeypatch, tile, waves, fp8, K):
    monkeypatch.setenv("CCL_GEMM_TILE", tile)
    monkeypatch.setenv("CCL_GEMM_WAVES", waves)
    for gated in (False, True):
        _backward((512, 512, K, 1, 1, 4096), ccl.CCL_ACT_SILU, gated, fp8=fp8, rows=400, alpha=0.05 if fp8 else 1.0,
                  layout=ccl.CCL_LAYOUT_ROWMAJOR)


def test_grad_in_place_and_without_bias():
    _backward(EXPERT, ccl.CCL_ACT_SILU, False, dbias=False, in_place=True)
    _backward(EXPERT, ccl.CCL_ACT_SILU, True, dbias=True, in_place=True)


def test_grad_same_bits_every_time():
    a = _backward(EXPERT, ccl.CCL_ACT_SILU, True)
    b = _backward(EXPERT, ccl.CCL_ACT_SILU, True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_grad_is_the_difference_quotient_of_the_forward():
    """Forward outputs at Z +- h (through the bias) against dZ summed over rows:
    with D = 1 everywhere, sum over rows of (C(+h) - C(-h)) / 2h = dbias."""
    M, N, K = 256, 256, 256
    plan = ccl.ccl_plan(M, N, K, 1, 1, 4096)
    A = to_dev(W.draw_array(11, M, K, "normal", 1.0))
    B = to_dev(W.draw_array(12, K, N, "normal", 0.06))
    rm = ccl.CCL_LAYOUT_ROWMAJOR
    _, need = ccl.ccl_gemm_fused_workspace(plan, layout=rm)
    need = max(need, ccl.ccl_gemm_fused_grad_workspace(plan, dbias=True, layout=rm))
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    h = 0.25
    outs = []
    for s in (h, -h, 0.0):
        C, Z = dev_full(M * N), dev_full(M * N)
        bias = torch.full((N,), s, device="cuda")
        ccl.ccl_gemm_fused(plan, A, B, C, activation=ccl.CCL_ACT_SILU, bias=bias, preact=Z, layout=rm, workspace=ws,
                           workspace_bytes=ws.numel())
        outs.append(C)
    Zc = Z
    quotient = (OG.decode_bf16(from_dev(outs[0])) - OG.decode_bf16(from_dev(outs[1]))).reshape(M, N).sum(0) / (2 * h)
    one = W.round_to_bf16_bits(np.ones((M, K), np.float32))
    unit = np.zeros((K, N), np.float32)
    unit[0] = 1.0                                            # D = 1
    db, dZ = torch.empty(N, device="cuda"), dev_full(M * N)
    ccl.ccl_gemm_fused_grad(plan, to_dev(one), to_dev(W.round_to_bf16_bits(unit)), Zc, dZ, activation=ccl.CCL_ACT_SILU,
                            dbias=db, layout=rm, workspace=ws, workspace_bytes=ws.numel())
    # each quotient: h^2 / 6 of the third derivative (at most 0.4), the
    # roundings of two outputs (2^-8 of at most |z| + 1) over 2 h, and Z's own
    z = np.abs(OG.decode_bf16(from_dev(Zc))).reshape(M, N)
    tol = (h * h / 6 * 0.4 + 2 * 2.0 ** -8 * (z + 1) / (2 * h) + 2.0 ** -8 * z * 0.5).sum(0)
    assert (np.abs(quotient - db.cpu().numpy()) <= tol).all()


def test_another_stream():
    """Operands made and read on a side stream."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        _forward(EXPERT, ccl.CCL_ACT_GELU, True, residual=True)
        _backward(EXPERT, ccl.CCL_ACT_GELU, True)


def test_graph_replays():
    """A captured forward and backward call, replayed with eager work between:
    the eager bits each time."""
    M, N, K = 256, 512, 256
    plan = ccl.ccl_plan(M, N, K, 4, 2, 4096)
    rm = ccl.CCL_LAYOUT_ROWMAJOR
    A = to_dev(W.draw_array(21, M, K, "normal", 1.0))
    B = to_dev(W.draw_array(22, K, N, "normal", 0.06))
    C, Z, dZ, db = dev_full(M * N // 2), dev_full(M * N), dev_full(M * 2 * N), torch.empty(2 * N, device="cuda")
    Zin = to_dev(W.draw_array(23, M, 2 * N, "normal", 2.0))
    need = max(ccl.ccl_gemm_fused_workspace(plan, layout=rm)[1],
               ccl.ccl_gemm_fused_grad_workspace(plan, gated=True, dbias=True, layout=rm), 16)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step():
        ccl.ccl_gemm_fused(plan, A, B, C, activation=ccl.CCL_ACT_SILU, gated=True, preact=Z, rows=200, layout=rm,
                           workspace=ws, workspace_bytes=need)
        ccl.ccl_gemm_fused_grad(plan, A, B, Zin, dZ, activation=ccl.CCL_ACT_SILU, gated=True, dbias=db, rows=200,
                                layout=rm, workspace=ws, workspace_bytes=need)

    outs = (C, Z, dZ, db)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        (A.float() + 1).sum().item()
