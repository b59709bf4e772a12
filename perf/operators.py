"""The FFN operators around the GEMM, as a training or serving program calls
them through paper_2606_11718_amd.ccl. A case is one of four kinds:

  linear       C = act(alpha A B + bias) + beta R, optionally gated
               (gate and up columns interleaved in groups of 16) and with the
               pre-activation kept for the backward pass.
  linear_grad  dZ = (alpha A B) * act'(Z) of that epilogue, with the bias
               gradient (the column sums of dZ).
  moe          one whole mixture-of-experts FFN layer for a few tokens:
               routing, gate/up products, activation, down product, weighted
               sum.
  ortho        the orthogonalised update of one or a batch of weight
               gradients: five Newton-Schulz steps of an odd quintic.

Operands of the first two are row-major ("rowmajor") or stored as strips of
the chiplet-contiguous layout ("ccl"): with 4 KB pages a strip is whole pages
here, so that layout is the row-major matrix cut into a grid of blocks.

Sizes are the repository's own workloads (an expert FFN of 2048 hidden and
2 x 768 intermediate out of 128 experts, a dense FFN of 8192 hidden and 28672
intermediate) and generic ones around them.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
ACTS = ("none", "relu", "gelu", "silu")
# Standard deviations: activations N(0,1), weights N(0,0.02), gradients
# N(0,0.01). fp8 weights are stored scaled up to N(0,1) and scaled back.
ACT, WEIGHT, GRAD = 1.0, 0.02, 0.01
# The odd quintic of the Newton-Schulz steps.
QUINTIC = (3.4445, -4.7750, 2.0315)
GROUP = 16   # columns of one gate or up group of an interleaved weight


def _linear(name, M, N, K, **more):
    case = {"name": name, "kind": "linear", "M": M, "N": N, "K": K, "chiplets": 8, "grid": 2, "layout": "rowmajor",
            "ab": "bf16", "act": "gelu", "gated": False, "bias": True, "residual": False, "keep": False,
            "alpha": 1.0, "beta": 1.0, "rows": M, "splits": 1, "b_std": WEIGHT}
    case.update(more)
    return case


def _grad(name, M, N, K, **more):
    case = {"name": name, "kind": "linear_grad", "M": M, "N": N, "K": K, "chiplets": 8, "grid": 2, "layout": "rowmajor",
            "ab": "bf16", "act": "gelu", "gated": False, "bias": True, "alpha": 1.0, "rows": M, "a_std": GRAD,
            "b_std": WEIGHT}
    case.update(more)
    return case


def _moe(name, tokens, **more):
    case = {"name": name, "kind": "moe", "tokens": tokens, "hidden": 2048, "ffn": 768, "experts": 128, "top_k": 8,
            "weights": "bf16", "act": "silu", "normalize": True}
    case.update(more)
    return case


def _ortho(name, batch, rows, cols, **more):
    case = {"name": name, "kind": "ortho", "batch": batch, "rows": rows, "cols": cols, "g": "bf16", "ld_pad": 0}
    case.update(more)
    return case


def listed():
    return [
        # The smallest configuration of the repository with every part of the
        # epilogue: a launch of a few microseconds.
        _linear("small_linear", 256, 512, 256, chiplets=4, residual=True, b_std=0.06),
        # Expert FFN, fused gate and up projection, 4096 tokens, training:
        # SwiGLU in the epilogue, the pre-activations kept.
        _linear("expert_swiglu", 4096, 1536, 2048, act="silu", gated=True, bias=False, keep=True),
        # Dense FFN up projection, 8192 tokens, training, operands in CCL.
        _linear("dense_up_gelu", 8192, 28672, 8192, layout="ccl", keep=True),
        # Dense FFN down projection of five decoding tokens: bound by reading
        # the weights, split along K, added to the residual stream.
        _linear("dense_down_decode", 128, 8192, 28672, grid=1, layout="ccl", act="none", residual=True, rows=5,
                splits=4),
        # Dense SwiGLU prefill in fp8, a ragged number of tokens.
        _linear("dense_swiglu_fp8", 4096, 57344, 8192, ab="fp8", act="silu", gated=True, bias=False, alpha=0.02,
                rows=3777, b_std=1.0),
        # Expert FFN backward: the gradient of its input dY W_down^T, taken
        # through SwiGLU; interleaved gate and up gradients come out.
        _grad("expert_swiglu_grad", 4096, 768, 2048, grid=8, act="silu", gated=True, bias=False),
        # Dense FFN backward through GELU with the bias gradient, in CCL.
        _grad("dense_gelu_grad", 8192, 28672, 8192, layout="ccl"),
        # One decoding token through a layer of 128 experts, eight chosen.
        _moe("moe_one_token", 1),
        # A decoding batch of 48 tokens over the same experts in fp8: nearly
        # every expert's weights are read.
        _moe("moe_batch_fp8", 48, weights="fp8"),
        # Muon update of one expert's down projection ...
        _ortho("ortho_expert", 1, 768, 2048),
        # ... of the gate and up projections of 16 experts, fp32 gradients ...
        _ortho("ortho_expert_batch", 16, 2048, 1536, g="fp32"),
        # ... and of a dense up projection.
        _ortho("ortho_dense", 1, 8192, 28672),
    ]


def _log(rng, lo, hi):
    """A whole number of lo..hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """One more case: products of 1 to 8192 tokens and 256 to 28672 columns of
    every grid, layout, activation and type; layers of 1 to 64 tokens and 1 to
    256 experts; updates of 1 to 64 matrices of 60 to 8192 rows."""
    kind = rng.choice(["linear", "linear", "linear", "grad", "grad", "moe", "moe", "moe", "ortho", "ortho"])
    if kind in ("linear", "grad"):
        grid = rng.choice([1, 2, 4, 8])
        cols = 8 // grid
        gated = rng.random() < 0.4
        fp8 = kind == "linear" and rng.random() < 0.25
        while True:
            M = 128 * grid * _log(rng, 1, 64 // grid)
            N = 128 * cols * _log(rng, 1, 224 // cols)
            K = 256 * _log(rng, 2, 112)
            if fp8:
                K = 1024 * max(1, K // 1024)
            if 2.0 * M * N * K <= 1.5e12:
                break
        common = dict(grid=grid, layout=rng.choice(["rowmajor", "ccl"]), gated=gated,
                      act=rng.choice(["gelu", "silu"]) if gated else rng.choice(ACTS), bias=rng.random() < 0.6,
                      rows=M if rng.random() < 0.5 else rng.randint(1, M))
        if kind == "grad":
            case = _grad("", M, N, K, **common)
        else:
            case = _linear("", M, N, K, keep=rng.random() < 0.4, residual=rng.random() < 0.5,
                           beta=rng.choice([1.0, 0.5]), **common)
            if fp8:
                case.update(ab="fp8", alpha=0.02, b_std=1.0)
            if M * N <= 128 * 64 * 8 * 128:
                case["splits"] = rng.choice([1, 2, 4])
    elif kind == "moe":
        hidden, ffn = 64 * _log(rng, 4, 96), 64 * _log(rng, 2, 48)
        experts = max(1, min(_log(rng, 1, 256), 600_000_000 // (3 * hidden * ffn)))
        case = _moe("", _log(rng, 1, 64), hidden=hidden, ffn=ffn, experts=experts,
                    top_k=min(experts, _log(rng, 1, 10)), weights=rng.choice(["bf16", "fp8"]),
                    act=rng.choice(["silu", "gelu"]), normalize=rng.random() < 0.7)
    else:
        rows, cols = _log(rng, 60, 8192), _log(rng, 60, 8192)
        batch = max(1, min(_log(rng, 1, 64), int(4e11 / (5.0 * 4 * min(rows, cols) ** 2 * max(rows, cols)))))
        case = _ortho("", batch, rows, cols, g=rng.choice(["bf16", "fp32"]), ld_pad=rng.choice([0, 0, 1, 8]))
    del case["name"]
    return case


# ---------------------------------------------------------------------------
# inputs


def _normal(gen, shape, std, dtype):
    if dtype == torch.float8_e4m3fn:
        return torch.randn(shape, device=DEV, dtype=torch.bfloat16, generator=gen).mul_(std).to(dtype)
    return torch.randn(shape, device=DEV, dtype=dtype, generator=gen).mul_(std)


def _wide(case):
    """Columns of the kept or read pre-activations, and of the result."""
    N = case["N"]
    if case["kind"] == "linear":
        return N, N // 2 if case["gated"] else N
    return (2 * N, 2 * N) if case["gated"] else (N, N)


def _grid(case):
    return case["grid"], case["chiplets"] // case["grid"]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    state = {"case": case}
    if own:
        from paper_2606_11718_amd import ccl
        state["ccl"] = ccl
    kind = case["kind"]
    if kind in ("linear", "linear_grad"):
        M, N, K = case["M"], case["N"], case["K"]
        dt = torch.float8_e4m3fn if case["ab"] == "fp8" else torch.bfloat16
        gr, gc = _grid(case)
        blocks = lambda r, c: (gr, gc, r // gr, c // gc) if case["layout"] == "ccl" else (r, c)  # noqa: E731
        state["A"] = _normal(gen, blocks(M, K), case.get("a_std", ACT), dt)
        state["B"] = _normal(gen, blocks(K, N), case["b_std"], dt)
        z_cols, c_cols = _wide(case)
        state["C"] = torch.empty(blocks(M, c_cols), device=DEV, dtype=torch.bfloat16)
        if kind == "linear":
            state["bias"] = _normal(gen, (N,), 0.5, torch.float32) if case["bias"] else None
            state["R"] = _normal(gen, blocks(M, c_cols), ACT, torch.bfloat16) if case["residual"] else None
            state["Z"] = torch.empty(blocks(M, z_cols), device=DEV, dtype=torch.bfloat16) if case["keep"] else None
        else:
            state["Z"] = _normal(gen, blocks(M, z_cols), ACT, torch.bfloat16)
            state["dbias"] = torch.empty(z_cols, device=DEV, dtype=torch.float32) if case["bias"] else None
        if own:
            ab = ccl.CCL_DT_FP8_E4M3 if case["ab"] == "fp8" else ccl.CCL_DT_BF16
            state["plan"] = ccl.ccl_plan_typed(M, N, K, case["chiplets"], case["grid"], 4096, ab, ccl.CCL_DT_BF16)
            state["act"] = {"none": ccl.CCL_ACT_NONE, "relu": ccl.CCL_ACT_RELU, "gelu": ccl.CCL_ACT_GELU,
                            "silu": ccl.CCL_ACT_SILU}[case["act"]]
            state["layout"] = ccl.CCL_LAYOUT_CCL if case["layout"] == "ccl" else ccl.CCL_LAYOUT_ROWMAJOR
            if kind == "linear":
                _, need = ccl.ccl_gemm_fused_workspace(state["plan"], case["splits"], layout=state["layout"])
            else:
                need = ccl.ccl_gemm_fused_grad_workspace(state["plan"], gated=case["gated"], dbias=case["bias"],
                                                         layout=state["layout"])
            state["ws"] = torch.empty(max(need, 16), device=DEV, dtype=torch.uint8)
    elif kind == "moe":
        T, D, F, E = case["tokens"], case["hidden"], case["ffn"], case["experts"]
        fp8 = case["weights"] == "fp8"
        dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
        state["x"] = _normal(gen, (T, D), ACT, torch.bfloat16)
        state["logits"] = _normal(gen, (T, E), 1.5, torch.float32)
        # Output-major weights, as a checkpoint stores them: gate rows, then up rows.
        state["gate_up"] = _normal(gen, (E, 2 * F, D), 1.0 if fp8 else 1.0 / math.sqrt(D), dt)
        state["down"] = _normal(gen, (E, D, F), 1.0 if fp8 else 1.0 / math.sqrt(F), dt)
        scale = lambda n: torch.rand(E, device=DEV, generator=gen).add_(0.5).mul_(1.0 / math.sqrt(n))  # noqa: E731
        state["gate_up_scale"] = scale(D) if fp8 else None
        state["down_scale"] = scale(F) if fp8 else None
        state["y"] = torch.empty(T, D, device=DEV, dtype=torch.bfloat16)
        state["ids"] = torch.empty(T, case["top_k"], device=DEV, dtype=torch.int32)
        state["probs"] = torch.empty(T, case["top_k"], device=DEV, dtype=torch.float32)
        if own:
            state["moe"] = ccl.ccl_moe(
                hidden=D, ffn=F, experts=E, top_k=case["top_k"], normalize=case["normalize"],
                activation=ccl.CCL_ACT_SILU if case["act"] == "silu" else ccl.CCL_ACT_GELU,
                weight_type=ccl.CCL_DT_FP8_E4M3 if fp8 else ccl.CCL_DT_BF16)
            state["ws"] = torch.empty(ccl.ccl_moe_workspace(state["moe"], T), device=DEV, dtype=torch.uint8)
    else:
        n, r, c = case["batch"], case["rows"], case["cols"]
        dt = torch.bfloat16 if case["g"] == "bf16" else torch.float32
        # Gradients: noise and a few strong directions.
        G = _normal(gen, (n, r, c), GRAD, torch.float32)
        G += torch.matmul(_normal(gen, (n, r, 4), GRAD, torch.float32), _normal(gen, (n, 4, c), 1.0, torch.float32))
        wide = torch.zeros(n, r, c + case["ld_pad"], device=DEV, dtype=dt)
        wide[:, :, :c] = G
        state["G"] = wide[:, :, :c]
        state["O"] = torch.empty(n, r, c, device=DEV, dtype=torch.bfloat16)
        if own:
            state["ws"] = torch.empty(ccl.ccl_orthogonalize_workspace(n, r, c), device=DEV, dtype=torch.uint8)
    return state


# ---------------------------------------------------------------------------
# plain forms, in 32 bits


def _unblock(x):
    """Row-major matrix of a blocked (Gr, Gc, rows, cols) one."""
    if x is None or x.dim() == 2:
        return x
    return x.permute(0, 2, 1, 3).reshape(x.shape[0] * x.shape[2], x.shape[1] * x.shape[3])


def _block(x, case):
    if case["layout"] != "ccl":
        return x
    gr, gc = _grid(case)
    return x.reshape(gr, x.shape[0] // gr, gc, x.shape[1] // gc).permute(0, 2, 1, 3).contiguous()


def _tanh_arg(z):
    return math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(_tanh_arg(z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        t = torch.tanh(_tanh_arg(z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2.0 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _halves(z):
    """Gate and up columns of interleaved ones."""
    g = z.view(z.shape[0], -1, 2, GROUP)
    return g[:, :, 0].reshape(z.shape[0], -1), g[:, :, 1].reshape(z.shape[0], -1)


def _interleave(gate, up):
    m = gate.shape[0]
    return torch.stack([gate.view(m, -1, GROUP), up.view(m, -1, GROUP)], dim=2).reshape(m, -1)


def _plain_linear(s):
    case = s["case"]
    z = torch.matmul(_unblock(s["A"]).float(), _unblock(s["B"]).float()) * case["alpha"]
    if s["bias"] is not None:
        z = z + s["bias"]
    if case["gated"]:
        gate, up = _halves(z)
        c = _act(gate, case["act"]) * up
    else:
        c = _act(z, case["act"])
    if s["R"] is not None:
        c = c + case["beta"] * _unblock(s["R"]).float()
    live = (torch.arange(case["M"], device=DEV) < case["rows"])[:, None]
    out = {"C": _block(torch.where(live, c, torch.zeros_like(c)).to(torch.bfloat16), case)}
    if case["keep"]:
        out["Z"] = _block(torch.where(live, z, torch.zeros_like(z)).to(torch.bfloat16), case)
    return out


def _plain_grad(s):
    case = s["case"]
    d = torch.matmul(_unblock(s["A"]).float(), _unblock(s["B"]).float()) * case["alpha"]
    z = _unblock(s["Z"]).float()
    if case["gated"]:
        gate, up = _halves(z)
        dz = _interleave(d * up * _act_grad(gate, case["act"]), d * _act(gate, case["act"]))
    else:
        dz = d * _act_grad(z, case["act"])
    live = (torch.arange(case["M"], device=DEV) < case["rows"])[:, None]
    dz = torch.where(live, dz, torch.zeros_like(dz))
    out = {"C": _block(dz.to(torch.bfloat16), case)}
    if case["bias"]:
        out["dbias"] = dz.sum(0)
    return out


def _plain_moe(s):
    case = s["case"]
    T, F, E, k = case["tokens"], case["ffn"], case["experts"], case["top_k"]
    top, ids = torch.sort(s["logits"], dim=1, descending=True, stable=True)   # ties: the lowest expert
    top, ids = top[:, :k], ids[:, :k]
    e = torch.exp(top - top[:, :1])
    total = e.sum(1, keepdim=True) if case["normalize"] else torch.exp(s["logits"] - top[:, :1]).sum(1, keepdim=True)
    probs = e / total
    x = s["x"].float()
    chosen = ids.reshape(-1)
    if T * k <= E // 2:   # the chosen experts' weights only
        gate_up = torch.matmul(s["gate_up"][chosen].float(), x.repeat_interleave(k, 0)[:, :, None])[:, :, 0]
    else:                 # every expert on every token
        every = torch.matmul(x[None], s["gate_up"].float().transpose(1, 2))
        gate_up = every.transpose(0, 1).gather(1, ids[:, :, None].expand(T, k, 2 * F)).reshape(T * k, 2 * F)
    if s["gate_up_scale"] is not None:
        gate_up = gate_up * s["gate_up_scale"][chosen][:, None]
    h = _act(gate_up[:, :F], case["act"]) * gate_up[:, F:]
    if s["down_scale"] is not None:
        h = h * s["down_scale"][chosen][:, None]
    h = h * probs.reshape(-1, 1)
    if T * k <= E // 2:
        y = torch.matmul(s["down"][chosen].float(), h[:, :, None]).view(T, k, -1).sum(1)
    else:
        spread = torch.zeros(T, E, F, device=DEV).scatter_(1, ids[:, :, None].expand(T, k, F), h.view(T, k, F))
        y = torch.matmul(spread.transpose(0, 1), s["down"].float().transpose(1, 2)).sum(0)
    return {"y": y.to(torch.bfloat16), "ids": ids.to(torch.int32), "probs": probs}


def _newton_schulz(x, left):
    """Five steps x <- a x + (b S + c S S) x with S = x x^T for a wide x."""
    if left == 0:
        return x
    a, b, c = QUINTIC
    gram = torch.matmul(x, x.transpose(1, 2))
    return _newton_schulz(a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x), left - 1)


def _plain_ortho(s):
    g = s["G"].float()
    x = g / (torch.sqrt((g * g).sum((1, 2), keepdim=True)) + 1e-7)
    tall = g.shape[1] > g.shape[2]
    x = _newton_schulz(x.transpose(1, 2).contiguous() if tall else x, 5)
    return {"O": (x.transpose(1, 2) if tall else x).to(torch.bfloat16).contiguous()}


def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        return {"linear": _plain_linear, "linear_grad": _plain_grad, "moe": _plain_moe, "ortho": _plain_ortho}[kind](state)
    ccl = state["ccl"]
    if kind == "linear":
        ccl.ccl_gemm_fused(state["plan"], state["A"], state["B"], state["C"], activation=state["act"],
                           gated=case["gated"], bias=state["bias"], residual=state["R"], beta=case["beta"],
                           preact=state["Z"], alpha=case["alpha"], rows=case["rows"], layout=state["layout"],
                           splits=case["splits"], workspace=state["ws"], workspace_bytes=state["ws"].numel())
        return {"C": state["C"], "Z": state["Z"]} if case["keep"] else {"C": state["C"]}
    if kind == "linear_grad":
        ccl.ccl_gemm_fused_grad(state["plan"], state["A"], state["B"], state["Z"], state["C"], activation=state["act"],
                                gated=case["gated"], dbias=state["dbias"], alpha=case["alpha"], rows=case["rows"],
                                layout=state["layout"], workspace=state["ws"], workspace_bytes=state["ws"].numel())
        return {"C": state["C"], "dbias": state["dbias"]} if case["bias"] else {"C": state["C"]}
    if kind == "moe":
        ccl.ccl_moe_decode(state["moe"], case["tokens"], state["x"], state["logits"], state["gate_up"], state["down"],
                           state["y"], ids=state["ids"], probs=state["probs"], gate_up_scale=state["gate_up_scale"],
                           down_scale=state["down_scale"], workspace=state["ws"], workspace_bytes=state["ws"].numel())
        return {"y": state["y"], "ids": state["ids"], "probs": state["probs"]}
    G = state["G"]
    ccl.ccl_orthogonalize(case["batch"], case["rows"], case["cols"], G,
                          ccl.CCL_DT_BF16 if case["g"] == "bf16" else ccl.CCL_DT_FP32, G.stride(1), G.stride(0),
                          state["O"], workspace=state["ws"], workspace_bytes=state["ws"].numel())
    return {"O": state["O"]}


# ---------------------------------------------------------------------------
# 64-bit values, from the definitions


def _exact_act(z, act):
    """Value and derivative."""
    if act == "relu":
        on = (z > 0).double()
        return z * on, on
    if act in ("gelu", "silu"):
        # both are z * sigmoid(u(z)): u = z, or twice the tanh argument
        w = math.sqrt(8.0 / math.pi)
        u = z if act == "silu" else w * z * (1 + 0.044715 * z * z)
        du = torch.ones_like(z) if act == "silu" else w * (1 + 0.134145 * z * z)
        s = torch.sigmoid(u)
        return z * s, s + z * s * torch.sigmoid(-u) * du
    return z, torch.ones_like(z)


def _exact_product(s):
    case = s["case"]
    return case["alpha"] * (_unblock(s["A"]).double() @ _unblock(s["B"]).double())


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "linear":
        z = _exact_product(s)
        if s["bias"] is not None:
            z += s["bias"].double()
        if case["gated"]:
            cols = torch.arange(case["N"], device=DEV)
            gate = (cols // GROUP) % 2 == 0
            c = _exact_act(z[:, gate], case["act"])[0] * z[:, ~gate]
        else:
            c = _exact_act(z, case["act"])[0]
        if s["R"] is not None:
            c = c + case["beta"] * _unblock(s["R"]).double()
        c[case["rows"]:] = 0
        out = {"C": _block(c, case)}
        if case["keep"]:
            z[case["rows"]:] = 0
            out["Z"] = _block(z, case)
        return out
    if kind == "linear_grad":
        d = _exact_product(s)
        z = _unblock(s["Z"]).double()
        if case["gated"]:
            cols = torch.arange(z.shape[1], device=DEV)
            gate = (cols // GROUP) % 2 == 0
            v, dv = _exact_act(z[:, gate], case["act"])
            dz = torch.empty_like(z)
            dz[:, gate] = d * z[:, ~gate] * dv
            dz[:, ~gate] = d * v
        else:
            dz = d * _exact_act(z, case["act"])[1]
        dz[case["rows"]:] = 0
        out = {"C": _block(dz, case)}
        if case["bias"]:
            out["dbias"] = dz.sum(0)
        return out
    if kind == "moe":
        T, D, F, k = case["tokens"], case["hidden"], case["ffn"], case["top_k"]
        y = torch.zeros(T, D, device=DEV, dtype=torch.float64)
        probs = torch.zeros(T, k, device=DEV, dtype=torch.float64)
        all_logits = s["logits"].double()
        host = all_logits.cpu()
        by_expert = {}
        for t in range(T):
            row = host[t].tolist()
            order = sorted(range(len(row)), key=lambda e: (-row[e], e))[:k]
            weights = torch.softmax(host[t][order] if case["normalize"] else host[t], 0)
            for j, e in enumerate(order):
                p = float(weights[j if case["normalize"] else e])
                probs[t, j] = p
                by_expert.setdefault(e, []).append((t, p))
        for e, uses in by_expert.items():
            at = torch.tensor([t for t, _ in uses], device=DEV)
            p = torch.tensor([q for _, q in uses], device=DEV, dtype=torch.float64)
            z = s["x"][at].double() @ s["gate_up"][e].double().t().contiguous()
            if s["gate_up_scale"] is not None:
                z *= s["gate_up_scale"][e].double()
            h = _exact_act(z[:, :F], case["act"])[0] * z[:, F:]
            v = h @ s["down"][e].double().t().contiguous()
            if s["down_scale"] is not None:
                v *= s["down_scale"][e].double()
            y.index_add_(0, at, p[:, None] * v)
        return {"y": y, "ids": None, "probs": probs}
    a, b, c = QUINTIC
    out = torch.empty(case["batch"], case["rows"], case["cols"], device=DEV, dtype=torch.float64)
    for i in range(case["batch"]):
        x = s["G"][i].double()
        x = x / (x.square().sum().sqrt() + 1e-7)
        tall = x.shape[0] > x.shape[1]
        for _ in range(5):
            gram = x.t() @ x if tall else x @ x.t()
            first = x @ gram if tall else gram @ x
            x = a * x + b * first + c * (first @ gram if tall else gram @ first)
        out[i] = x
    return {"O": out}


# ---------------------------------------------------------------------------


def work(case):
    """Inputs read once, outputs written once, and the products' operations on
    the rows and experts that are used."""
    kind = case["kind"]
    if kind in ("linear", "linear_grad"):
        M, N, K = case["rows"], case["N"], case["K"]
        e = 1 if case["ab"] == "fp8" else 2
        z_cols, c_cols = _wide(case)
        b = (M * K + K * N) * e + 2 * case["M"] * c_cols
        if kind == "linear":
            b += 2 * case["M"] * z_cols * case["keep"] + 2 * M * c_cols * case["residual"] + 4 * N * case["bias"]
        else:
            b += 2 * M * z_cols + 4 * z_cols * case["bias"]
        return {"bytes": b, "flops": 2.0 * M * N * K}
    if kind == "moe":
        T, D, F, E, k = case["tokens"], case["hidden"], case["ffn"], case["experts"], case["top_k"]
        used = E * (1 - (1 - k / E) ** T)   # experts that T tokens choose, on average
        e = 1 if case["weights"] == "fp8" else 2
        return {"bytes": used * 3 * D * F * e + 4 * T * E + 4 * T * D + 8 * T * k, "flops": 6.0 * T * k * D * F}
    n, r, c = case["batch"], case["rows"], case["cols"]
    p, q = min(r, c), max(r, c)
    # Of the symmetric products x x^T and S S half are needed.
    flops = 5.0 * n * (p * (p + 1.0) * q + p * (p + 1.0) * p + 2.0 * p * p * q)
    return {"bytes": n * r * c * ((2 if case["g"] == "bf16" else 4) + 2), "flops": flops}
