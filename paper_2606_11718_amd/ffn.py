"""A gated FFN trained and served with the library: the operators as one program.

    python -m paper_2606_11718_amd.ffn [--tokens M --hidden D --ffn F --steps N]

GatedFFN holds W_up (hidden x 2 ffn, gate and up columns interleaved in groups
of 16) and W_down (ffn x hidden) and takes training steps of
    Y = X + (silu(X Wg) * (X Wu)) W_down
with the activation, gate and residual in the forward products' epilogues, the
gradient through the activation in the backward product's, weight gradients by
ccl_gemm on packed operands, and both weights moved along their orthogonalised
gradients. MoELayer serves experts of the same shape to a few tokens at a time.

torch supplies memory, the transposed weight copies, elementwise updates and the
router's logits; every other product runs in the library. Operands of the epilogue calls are row-major,
weight gradients pack theirs (one from the stored transpose).
"""
from __future__ import annotations

import argparse

import torch

from . import ccl

ROWMAJOR = ccl.CCL_LAYOUT_ROWMAJOR
GROUP = 16


def interleave(gate, up):
    """(hidden, 2 ffn) columns as a gated epilogue takes them, of (hidden, ffn) gate and up."""
    d = gate.shape[0]
    return torch.stack([gate.view(d, -1, GROUP), up.view(d, -1, GROUP)], dim=2).reshape(d, -1).contiguous()


def _plan(M, N, K, c_type=ccl.CCL_DT_BF16, chiplets=8):
    """A plan that the GEMM runs, over `chiplets` chiplets or as many fewer as that takes."""
    while True:
        try:
            plan = ccl.ccl_plan_typed(M, N, K, chiplets, 0, 4096, ccl.CCL_DT_BF16, c_type)
            ccl.ccl_debug_gemm_config(plan)
            return plan
        except ccl.CCLError as e:
            if e.status_name not in ("CCL_ERR_UNALIGNED_PARTITION", "CCL_ERR_UNSUPPORTED") or chiplets == 1:
                raise
            chiplets //= 2


class GatedFFN:
    """tokens, hidden and ffn: multiples of 128; a call may have fewer valid tokens."""

    def __init__(self, tokens: int, hidden: int, ffn: int, *, device="cuda", seed=0):
        M, D, F = tokens, hidden, ffn
        self.M, self.D, self.F, self.device = M, D, F, device
        gen = torch.Generator(device=device).manual_seed(seed)
        init = lambda r, c: torch.randn(r, c, generator=gen, device=device).div_(r ** 0.5)  # noqa: E731
        self.w_up = interleave(init(D, F), init(D, F))          # fp32 masters
        self.w_down = init(F, D).mul_(0.1)
        self.up, self.down, self.dh = _plan(M, 2 * F, D), _plan(M, D, F), _plan(M, F, D)
        self.dw_up, self.dw_down = (_plan(D, 2 * F, M, ccl.CCL_DT_FP32), _plan(F, D, M, ccl.CCL_DT_FP32))
        need = max(ccl.ccl_gemm_fused_workspace(self.up, layout=ROWMAJOR)[1],
                   ccl.ccl_gemm_fused_workspace(self.down, layout=ROWMAJOR)[1],
                   ccl.ccl_gemm_fused_grad_workspace(self.dh, gated=True, layout=ROWMAJOR),
                   ccl.ccl_orthogonalize_workspace(1, D, 2 * F), ccl.ccl_orthogonalize_workspace(1, F, D))
        self.ws = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
        self._cast()

    def _cast(self):
        self.w_up16, self.w_down16 = self.w_up.bfloat16(), self.w_down.bfloat16()
        self.w_down16_t = self.w_down16.t().contiguous()

    def _empty(self, *shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device=self.device)

    def _whole(self, name, t, cols):
        """The products read M x cols elements side by side from t's address."""
        if t.dtype != torch.bfloat16 or t.shape != (self.M, cols) or not t.is_contiguous():
            raise ValueError(f"{name} has to be a contiguous bf16 tensor of {self.M} x {cols}, not {t.dtype} of "
                             f"{tuple(t.shape)} with strides {t.stride()}")

    def forward(self, x, rows: int | None = None):
        """(y, h, z) of x (tokens x hidden, bf16), of which the first `rows` count."""
        self._whole("x", x, self.D)
        z, h, y = self._empty(self.M, 2 * self.F), self._empty(self.M, self.F), self._empty(self.M, self.D)
        common = dict(layout=ROWMAJOR, rows=rows, workspace=self.ws, workspace_bytes=self.ws.numel())
        ccl.ccl_gemm_fused(self.up, x, self.w_up16, h, activation=ccl.CCL_ACT_SILU, gated=True, preact=z, **common)
        ccl.ccl_gemm_fused(self.down, h, self.w_down16, y, residual=x, **common)
        return y, h, z

    def _weight_grad(self, plan, a, b):
        """a^T b in fp32: both packed, a from its stored transpose."""
        buf = [torch.empty(ccl.ccl_plan_layout(plan, op).total_bytes, dtype=torch.uint8, device=self.device)
               for op in (ccl.CCL_A, ccl.CCL_B, ccl.CCL_C)]
        ccl.ccl_pack(plan, ccl.CCL_A, a, a.shape[1], 1, buf[0])
        ccl.ccl_pack(plan, ccl.CCL_B, b, b.shape[1], 0, buf[1])
        ccl.ccl_gemm(plan, *buf)
        out = self._empty(a.shape[1], b.shape[1], dtype=torch.float32)
        ccl.ccl_unpack(plan, ccl.CCL_C, buf[2], out, b.shape[1])
        return out

    def _valid(self, t, rows):
        """t with zeros past its first `rows` rows, whatever it holds there (0 * NaN would reach a sum over rows)."""
        if rows is None or rows >= self.M:
            return t
        t = t.clone()
        t[rows:] = 0
        return t

    def backward(self, x, h, z, dy, rows: int | None = None):
        """Gradients of W_up and W_down from the first `rows` tokens and from forward's h and z for them."""
        for name, t, cols in (("x", x, self.D), ("h", h, self.F), ("z", z, 2 * self.F), ("dy", dy, self.D)):
            self._whole(name, t, cols)
        x, dy = self._valid(x, rows), self._valid(dy, rows)
        dz = self._empty(self.M, 2 * self.F)
        ccl.ccl_gemm_fused_grad(self.dh, dy, self.w_down16_t, z, dz, activation=ccl.CCL_ACT_SILU, gated=True, rows=rows,
                                layout=ROWMAJOR, workspace=self.ws, workspace_bytes=self.ws.numel())
        return self._weight_grad(self.dw_up, x, dz), self._weight_grad(self.dw_down, h, dy)

    def update(self, grads, lr: float):
        """Each weight along its orthogonalised gradient, scaled by its shape."""
        for w, g in zip((self.w_up, self.w_down), grads):
            r, c = w.shape
            o = self._empty(r, c)
            ccl.ccl_orthogonalize(1, r, c, g, ccl.CCL_DT_FP32, c, r * c, o, workspace=self.ws,
                                  workspace_bytes=self.ws.numel())
            w.add_(o, alpha=-lr * max(1.0, r / c) ** 0.5)
        self._cast()

    def step(self, x, target, lr: float, rows: int | None = None) -> float:
        """One training step on the mean squared error over the first `rows` tokens; the loss before it."""
        rows = self.M if rows is None else rows
        y, h, z = self.forward(x, rows)
        diff = y.float() - target.float()
        diff[rows:] = 0
        dy = (diff * (2.0 / (rows * self.D))).bfloat16()
        self.update(self.backward(x, h, z, dy, rows), lr)
        return float((diff * diff).sum() / (rows * self.D))


class MoELayer:
    """Experts as a checkpoint stores them (output-major bf16), for up to 64 tokens a call."""

    def __init__(self, hidden: int, ffn: int, experts: int, top_k: int, *, tokens: int = ccl.CCL_MOE_MAX_TOKENS,
                 device="cuda", seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=gen, device=device)  # noqa: E731
        self.router = rnd(hidden, experts).div_(hidden ** 0.5)
        self.gate_up = rnd(experts, 2 * ffn, hidden).div_(hidden ** 0.5).bfloat16()
        self.down = rnd(experts, hidden, ffn).div_(ffn ** 0.5).bfloat16()
        self.moe = ccl.ccl_moe(hidden=hidden, ffn=ffn, experts=experts, top_k=top_k)
        self.ws = torch.empty(ccl.ccl_moe_workspace(self.moe, tokens), dtype=torch.uint8, device=device)

    def decode(self, x):
        """(y, ids, probs) of x (tokens x hidden, bf16)."""
        logits = x.float() @ self.router
        t, k = x.shape[0], self.moe.top_k
        y = torch.empty_like(x)
        ids = torch.empty(t, k, dtype=torch.int32, device=x.device)
        probs = torch.empty(t, k, dtype=torch.float32, device=x.device)
        ccl.ccl_moe_decode(self.moe, t, x, logits, self.gate_up, self.down, y, ids=ids, probs=probs, workspace=self.ws,
                           workspace_bytes=self.ws.numel())
        return y, ids, probs


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--ffn", type=int, default=768)
    ap.add_argument("--experts", type=int, default=128)
    ap.add_argument("--steps", type=int, default=10)
    a = ap.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(a.tokens, a.hidden, generator=gen, device="cuda").bfloat16()
    target = x + torch.tanh(x @ torch.randn(a.hidden, a.hidden, generator=gen, device="cuda").div_(a.hidden ** 0.5).bfloat16())
    ffn = GatedFFN(a.tokens, a.hidden, a.ffn)
    for i in range(a.steps):
        print(f"step {i}: loss {ffn.step(x, target, 0.02, rows=a.tokens - 100):.5f}", flush=True)
    layer = MoELayer(a.hidden, a.ffn, a.experts, min(8, a.experts))
    for tokens in (1, 16, 64):
        y, ids, probs = layer.decode(x[:tokens])
        print(f"decode {tokens}: experts of token 0 {ids[0].tolist()}, |y| {y.float().norm().item():.3f}", flush=True)


if __name__ == "__main__":
    main()
