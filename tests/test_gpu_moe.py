"""GPU parity of ccl_moe_decode with the fp64 oracle.

The choice of experts is exact. Probabilities are fp32 (exponentials and a
division: 2^-20 relative). y is rounded to bf16 once (2^-8 relative at most);
before that it carries the fp32 errors of the K-term sums (at most K 2^-23 sum
|a b|), of the activation (2^-18 of its argument) and of h, kept to 16 bits
(2^-16 relative), each multiplied by what the formula multiplies it by.
"""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import ffn as OF
from oracle import gemm as OG
from paper_2606_11718_amd import ccl

pytestmark = pytest.mark.gpu

SILU, GELU = ccl.CCL_ACT_SILU, ccl.CCL_ACT_GELU


def _weights(seed, shape, fp8, std):
    n = int(np.prod(shape))
    bits = (W.draw_array_fp8 if fp8 else W.draw_array)(seed, 1, n, "normal", 1.0 if fp8 else std).reshape(shape)
    return bits, (OG.decode_fp8_e4m3 if fp8 else OG.decode_bf16)(bits)


def _padded(bits, ld, stride):
    """(E, rows, cols) bits on the GPU as bytes, rows ld and experts stride elements apart, NaN between."""
    E, rows, cols = bits.shape
    out = np.full(E * stride, 0x7F if bits.dtype == np.uint8 else 0x7FC0, bits.dtype)
    for e in range(E):
        view = out[e * stride:e * stride + (rows - 1) * ld + cols]
        for r in range(rows):
            view[r * ld:r * ld + cols] = bits[e, r]
    return torch.from_numpy(out.view(np.uint8)).cuda()


def _run(tokens, hidden, ffn, experts, top_k, fp8=False, act=SILU, normalize=True, logits=None, pad=False, seed=1,
         want_route=True, share=None):
    print(f"moe tokens={tokens} hidden={hidden} ffn={ffn} experts={experts} top_k={top_k} fp8={fp8} act={act} "
          f"normalize={normalize} pad={pad}", flush=True)
    rng = np.random.default_rng(seed)
    xb = W.draw_array(seed + 1, tokens, hidden, "normal", 1.0)
    gub, gu = _weights(seed + 2, (experts, 2 * ffn, hidden), fp8, 1 / np.sqrt(hidden))
    db, dn = _weights(seed + 3, (experts, hidden, ffn), fp8, 1 / np.sqrt(ffn))
    if logits is None:
        logits = rng.standard_normal((tokens, experts)) * 1.5
    logits = np.ascontiguousarray(logits, np.float32)
    gs = (rng.uniform(0.5, 1.5, experts) / np.sqrt(hidden)).astype(np.float32) if fp8 else None
    ds = (rng.uniform(0.5, 1.5, experts) / np.sqrt(ffn)).astype(np.float32) if fp8 else None
    extra = dict(gate_up_ld=hidden + 16, gate_up_stride=2 * ffn * (hidden + 16) + 32, down_ld=ffn + 32,
                 down_stride=hidden * (ffn + 32) + 16) if pad else {}
    moe = ccl.ccl_moe(hidden=hidden, ffn=ffn, experts=experts, top_k=top_k, activation=act, normalize=normalize,
                      weight_type=ccl.CCL_DT_FP8_E4M3 if fp8 else ccl.CCL_DT_BF16, **extra)
    wide = 24 if pad else 0
    x = torch.full((tokens, hidden + wide), float("nan"), dtype=torch.bfloat16, device="cuda")
    x[:, :hidden] = torch.from_numpy(xb.view(np.int16)).cuda().view(torch.bfloat16)
    lg = torch.full((tokens, experts + wide), float("inf"), device="cuda")
    lg[:, :experts] = torch.from_numpy(logits).cuda()
    y = torch.full((tokens, hidden + (5 if pad else 0)), 777.0, dtype=torch.bfloat16, device="cuda")
    if pad:
        gud = _padded(gub, moe.gate_up_ld, moe.gate_up_stride)
        dd = _padded(db, moe.down_ld, moe.down_stride)
    else:
        gud, dd = (torch.from_numpy(b.view(np.uint8).reshape(-1)).cuda() for b in (gub, db))
    ids = torch.full((tokens, top_k), -7, dtype=torch.int32, device="cuda") if want_route else None
    probs = torch.full((tokens, top_k), -7.0, device="cuda") if want_route else None
    ws = torch.full((max(16, ccl.ccl_moe_workspace(moe, tokens)),), 0xFF, dtype=torch.uint8, device="cuda")
    if share is not None:
        x, lg, y, gud, dd, ids, probs, ws = share(x, lg, y, gud, dd, ids, probs, ws)
    ccl.ccl_moe_decode(moe, tokens, x, lg, gud, dd, y, ids=ids, probs=probs,
                       gate_up_scale=None if gs is None else torch.from_numpy(gs).cuda(),
                       down_scale=None if ds is None else torch.from_numpy(ds).cuda(), workspace=ws,
                       workspace_bytes=ws.numel())
    torch.cuda.synchronize()
    xv = OG.decode_bf16(xb)
    yw, iw, pw = OF.moe(xv, logits, gu, dn, top_k, act, normalize, gs, ds)
    if want_route:
        assert np.array_equal(ids.cpu().numpy(), iw)
        assert (np.abs(probs.cpu().numpy() - pw) <= 2.0 ** -20 * pw + 1e-38).all()
    # the bound on y
    tol = np.zeros_like(yw)
    for t in range(tokens):
        for e, p in zip(iw[t], pw[t]):
            if e < 0:
                continue
            sg = 1.0 if gs is None else float(gs[e])
            sd = 1.0 if ds is None else float(ds[e])
            z = sg * (gu[e] @ xv[t])
            ez = hidden * 2.0 ** -23 * sg * (np.abs(gu[e]) @ np.abs(xv[t])) + 2.0 ** -18 * np.abs(z)
            g, u, eg, eu = z[:ffn], z[ffn:], ez[:ffn], ez[ffn:]
            h = OF.act(g, act) * u
            eh = 1.2 * eg * (np.abs(u) + eu) + np.abs(g) * eu + 2.0 ** -16 * np.abs(h)
            tol[t] += p * sd * (np.abs(dn[e]) @ (eh + (ffn * 2.0 ** -23 + 2.0 ** -20) * np.abs(h)))
    got = y[:, :hidden].float().cpu().numpy().astype(np.float64)
    bad = ~(np.abs(got - yw) <= 2.0 ** -8 * np.maximum(np.abs(got), np.abs(yw)) + 1.01 * tol + 1e-37)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], yw[bad][:4])
    if pad:
        assert (y[:, hidden:] == 777.0).all()
    return y, ids


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("tokens", [1, 2, 7, 8, 9, 16, 17, 33, 64])
def test_tokens(tokens, fp8):
    _run(tokens, 256, 96, 32, 4, fp8)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hidden,ffn", [(16, 16), (48, 32), (272, 80), (1040, 16), (64, 528), (2048, 768), (4112, 144)])
def test_sizes(hidden, ffn, fp8):
    _run(5, hidden, ffn, 6, 2, fp8)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("tokens", [9, 50])
def test_narrow_layer_in_ranges(tokens, fp8):
    """Few columns of y, many steps: one column tile a workgroup, cut into ranges."""
    _run(tokens, 256, 1200, 40, 4, fp8)


@pytest.mark.parametrize("experts,top_k", [(1, 1), (2, 2), (3, 1), (16, 16), (63, 8), (64, 8), (65, 3), (128, 8), (257, 10), (512, 16)])
@pytest.mark.parametrize("tokens", [1, 3, 40])
def test_experts(experts, top_k, tokens):
    _run(tokens, 64, 32, experts, top_k)


@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("act", [ccl.CCL_ACT_NONE, ccl.CCL_ACT_RELU, GELU, SILU])
def test_activations(act, normalize):
    _run(6, 128, 64, 16, 4, act=act, normalize=normalize)


@pytest.mark.parametrize("tokens", [2, 30])
@pytest.mark.parametrize("fp8", [False, True])
def test_strides(tokens, fp8):
    _run(tokens, 128, 48, 20, 3, fp8, pad=True)


@pytest.mark.parametrize("tokens", [4, 50])
@pytest.mark.parametrize("normalize", [False, True])
def test_ties_and_masks(tokens, normalize):
    """Equal logits, -0 against 0, masked experts, rows with fewer experts than
    slots, rows with none, NaN, infinities and the type's lowest value."""
    rng = np.random.default_rng(9)
    E = 24
    lg = rng.integers(-2, 3, (tokens, E)).astype(np.float32)
    lg[rng.random((tokens, E)) < 0.2] = -0.0
    lg[rng.random((tokens, E)) < 0.3] = -np.inf
    lg[0] = -np.inf                       # nothing left
    lg[1] = -np.inf
    lg[1, 13] = -3.0                      # one expert
    lg[2, ::2] = np.nan
    lg[3] = np.finfo(np.float32).min      # masked by the lowest value: still a choice
    if tokens > 4:
        lg[4, 5] = np.inf
        lg[5, 3] = lg[5, 20] = np.inf
        lg[6] = np.nan
        lg[7] = 88.0 * rng.standard_normal(E)
    y, ids = _run(tokens, 64, 32, E, 5, normalize=normalize, logits=lg)
    assert not y[0].any() and (ids[0] == -1).all()


def test_every_token_on_the_same_experts():
    lg = np.zeros((64, 40), np.float32)
    lg[:, 7] = 3.0
    lg[:, 31] = 2.0
    _run(64, 128, 64, 40, 2, logits=lg)


def test_route_is_optional():
    _run(3, 64, 32, 16, 2, want_route=False)


def test_offsets_past_32_bits():
    """Experts that start beyond 2^31 and 2^32 bytes of the weights."""
    hidden, ffn, experts = 256, 64, 3
    moe = ccl.ccl_moe(hidden=hidden, ffn=ffn, experts=experts, top_k=3, gate_up_stride=(1 << 30) + 64,
                      down_stride=(1 << 30) + 128)
    gu = torch.zeros(2 * moe.gate_up_stride + 2 * ffn * hidden, dtype=torch.bfloat16, device="cuda")
    dn = torch.zeros(2 * moe.down_stride + hidden * ffn, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    gws, dws = [], []
    for e in range(experts):
        a = torch.randn(2 * ffn, hidden, generator=g, device="cuda").mul_(0.06).bfloat16()
        b = torch.randn(hidden, ffn, generator=g, device="cuda").mul_(0.12).bfloat16()
        gu[e * moe.gate_up_stride:][:a.numel()] = a.view(-1)
        dn[e * moe.down_stride:][:b.numel()] = b.view(-1)
        gws.append(a.float().cpu().numpy().astype(np.float64))
        dws.append(b.float().cpu().numpy().astype(np.float64))
    x = torch.randn(2, hidden, generator=g, device="cuda").bfloat16()
    lg = torch.randn(2, experts, generator=g, device="cuda")
    y = torch.empty(2, hidden, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(ccl.ccl_moe_workspace(moe, 2), dtype=torch.uint8, device="cuda")
    ccl.ccl_moe_decode(moe, 2, x, lg, gu, dn, y, workspace=ws, workspace_bytes=ws.numel())
    want, _, _ = OF.moe(x.float().cpu().numpy().astype(np.float64), lg.cpu().numpy(), np.stack(gws), np.stack(dws), 3,
                        SILU, True)
    err = OG.errors(y.float().cpu().numpy().astype(np.float64), want)
    # every value is within 2^-8 of its own, and the fp32 errors are far below
    assert err["rel_fro"] <= 2.0 ** -8


def test_side_stream_and_graph_replays():
    """Captured once, replayed on new inputs with eager work between: the bits
    of the eager call each time."""
    moe = ccl.ccl_moe(hidden=256, ffn=64, experts=16, top_k=4)
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    gu, dn = rnd(16, 128, 256).mul_(0.06).bfloat16(), rnd(16, 256, 64).mul_(0.1).bfloat16()
    x, lg = rnd(3, 256).bfloat16(), rnd(3, 16)
    y, y2 = (torch.empty(3, 256, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws, ws2 = (torch.empty(ccl.ccl_moe_workspace(moe, 3), dtype=torch.uint8, device="cuda") for _ in range(2))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ccl.ccl_moe_decode(moe, 3, x, lg, gu, dn, y, workspace=ws, workspace_bytes=ws.numel())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ccl.ccl_moe_decode(moe, 3, x, lg, gu, dn, y, workspace=ws, workspace_bytes=ws.numel())
    torch.cuda.current_stream().wait_stream(s)
    for _ in range(3):
        x.copy_(rnd(3, 256))
        lg.copy_(rnd(3, 16))
        graph.replay()
        ccl.ccl_moe_decode(moe, 3, x, lg, gu, dn, y2, workspace=ws2, workspace_bytes=ws2.numel())
        torch.cuda.synchronize()
        assert torch.equal(y, y2)
