"""The training operators as a training step uses them: experts, loss, gradients
and AdamW one after the other, against the fp64 formulas and against differences of the
loss; captured and replayed; two steps at once on two streams; operands whose offsets
pass 32 bits; row numbers that do not ascend.

The gradients of a step pass eight roundings to bf16 (Z, Y, the experts' output, e, P',
its product, dZ, dW), each below 2^-8 / sqrt 3 = 2.3e-3 of its own value in the 2-norm,
and the logits' own error: they are of size 1 and carry those of the experts' two
products, 3.9e-3. Added up as independent ones: 2.3e-3 sqrt 8 and 3.9e-3, 7.6e-3; 2e-2
is asked for.
"""
import numpy as np
import pytest
import torch

from oracle import train as OT
from paper_2606_11718_amd import ccl

pytestmark = pytest.mark.gpu

SILU = ccl.CCL_ACT_SILU
BF = torch.bfloat16
HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.99, eps=1e-8)


class Step:
    """Rows sorted by expert -> act(gate) * up -> down -> loss, back, and AdamW of the three weights: fp32 ones with bf16
    copies that the products read; fp32 moments, 8-bit ones for the down weights."""

    def __init__(self, seed, counts=(90, 0, 1, 150, 43), behind=16, D=96, H=80, V=700):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        E, self.rows, self.gen = len(counts), sum(counts) + behind, g
        self.D, self.H, self.V, self.used = D, H, V, sum(counts)
        self.ends = torch.tensor(np.cumsum(counts), dtype=torch.int32, device="cuda")
        self.x = torch.empty(self.rows, D, dtype=BF, device="cuda")
        self.targets = torch.empty(self.rows, dtype=torch.int64, device="cuda")
        self.w = [self.rnd(E, 2 * H, D) / D ** 0.5, self.rnd(E, D, H) / H ** 0.5 * 2, self.rnd(V, D) / D ** 0.5]
        self.copy = [w.to(BF) for w in self.w]
        self.w = [c.float() for c in self.copy]
        self.g = [torch.empty_like(self.w[0]), torch.empty_like(self.copy[1]), torch.empty_like(self.copy[2])]
        bits8 = [False, True, False]
        zeros = lambda w, e: torch.zeros(w.numel(), dtype=torch.uint8 if e else torch.float32, device="cuda")  # noqa: E731
        scale = lambda w: torch.zeros(-(-w.numel() // 128), dtype=torch.uint8, device="cuda")  # noqa: E731
        self.m, self.v = ([zeros(w, e) for w, e in zip(self.w, bits8)] for _ in range(2))
        self.ms, self.vs = ([scale(w) if e else None for w, e in zip(self.w, bits8)] for _ in range(2))
        self.set = ccl.ccl_adamw(
            ccl.ccl_adamw_tensor(w, gr, m, v, exp_avg_scale=a, exp_avg_sq_scale=b, copy=c, weight_decay=0.1)
            for w, gr, m, v, a, b, c in zip(self.w, self.g, self.m, self.v, self.ms, self.vs, self.copy))
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        out = lambda n: torch.full((self.rows, n), float("nan"), dtype=BF, device="cuda")  # noqa: E731
        self.z, self.y, self.o, self.do, self.dz, self.dx = out(2 * H), out(H), out(D), out(D), out(2 * H), out(D)
        self.loss = torch.empty(self.rows, device="cuda")
        self.up = ccl.ccl_grouped(in_features=D, out_features=2 * H, experts=E, activation=SILU, gated=True)
        # the same sides without a gate: the gradient of rows that nothing was applied to
        self.up_in = ccl.ccl_grouped(in_features=D, out_features=2 * H, experts=E)
        self.down = ccl.ccl_grouped(in_features=H, out_features=D, experts=E)
        self.down_in = ccl.ccl_grouped(in_features=H, out_features=D, experts=E, activation=SILU, gated=True)
        self.head = ccl.ccl_vocab(hidden=D, vocab=V)
        need = [ccl.ccl_cross_entropy_workspace(self.head, self.rows, grad=True)]
        need += [ccl.ccl_grouped_gemm_workspace(k, self.rows, way) for k in (self.up, self.down) for way in range(3)]
        self.ws = torch.full((max(need),), 0xFF, dtype=torch.uint8, device="cuda")
        self.new_data()

    def new_data(self):
        self.x.copy_(self.rnd(self.rows, self.D))
        self.x[self.used:] = float("nan")
        self.targets.copy_(torch.randint(0, self.V, (self.rows,), generator=self.gen, device="cuda"))
        self.targets[5:9] = -100
        self.targets[self.used:] = -100
        self.step += 1

    def run(self):
        ws = dict(workspace=self.ws, workspace_bytes=self.ws.numel())
        n, (w1, w2, wo), (g1, g2, go) = self.rows, self.copy, self.g
        ccl.ccl_grouped_gemm(self.up, n, self.ends, self.x, w1, self.y, preact=self.z, **ws)
        ccl.ccl_grouped_gemm(self.down, n, self.ends, self.y, w2, self.o, **ws)
        ccl.ccl_cross_entropy_grad(self.head, n, self.o, wo, self.targets, self.loss, self.do, go, dloss_scale=1 / 256, **ws)
        ccl.ccl_grouped_gemm_grad(self.down_in, n, self.ends, self.do, w2, self.dz, preact=self.z, **ws)
        ccl.ccl_grouped_gemm_wgrad(self.down, n, self.ends, self.do, self.y, g2, **ws)
        ccl.ccl_grouped_gemm_wgrad(self.up, n, self.ends, self.dz, self.x, g1, **ws)
        ccl.ccl_grouped_gemm_grad(self.up_in, n, self.ends, self.dz, w1, self.dx, **ws)
        ccl.ccl_adamw_step(self.set, step_ptr=self.step, **HYPER)

    def state(self):
        held = [self.loss, self.dx, self.do, *self.g, *self.w, *self.copy, *self.m, *self.v, self.ms[1], self.vs[1]]
        return [t.clone() for t in held]


def _same(a, b):
    for i, (x, y) in enumerate(zip(a, b)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), i


def _f64(t):
    return t.double().cpu().numpy()


def _loss(x, ws, targets, ends):
    """(sum of losses / 256, gradients of it, dX) in 64 bits."""
    w1, w2, wo = ws
    y, z, _ = OT.grouped(x, w1, ends, SILU, True)
    o, _, _ = OT.grouped(y, w2, ends, ccl.CCL_ACT_NONE)
    loss, _, _, P = OT.cross_entropy(o, wo, targets, 1.0, np.full(len(targets), 1 / 256))
    do = P @ wo
    dz, _, _ = OT.grouped_grad(do, w2, ends, SILU, True, z)
    dx, _, _ = OT.grouped_grad(dz, w1, ends, ccl.CCL_ACT_NONE)
    return loss.sum() / 256, (OT.grouped_wgrad(dz, x, ends)[0], OT.grouped_wgrad(do, y, ends)[0], P.T @ o), dx


def test_step_against_formulas_and_differences():
    s = Step(3)
    before = [_f64(w) for w in s.w]
    s.run()
    torch.cuda.synchronize()
    u, ends = s.used, s.ends.cpu().numpy()
    x, targets = _f64(s.x[:u]), s.targets[:u].cpu().numpy()
    loss, grads, dx = _loss(x, before, targets, ends)
    assert abs(_f64(s.loss).sum() / 256 - loss) <= 2e-2 * loss
    got = [_f64(g) for g in s.g]
    for name, a, b in [*zip(("up", "down", "head"), got, grads), ("dx", _f64(s.dx[:u]), dx)]:
        assert np.linalg.norm(a - b) <= 2e-2 * np.linalg.norm(b), (name, np.linalg.norm(a - b) / np.linalg.norm(b))
    # along each weight's own gradient the loss changes by what the gradient says: h^2 and 1e-16 / h are left
    for i in range(3):
        to = got[i] / np.linalg.norm(got[i])
        at = lambda h: _loss(x, [w + h * to if k == i else w for k, w in enumerate(before)], targets, ends)[0]  # noqa: E731,B023
        slope = (at(1e-4) - at(-1e-4)) / 2e-4
        assert abs(slope - np.linalg.norm(got[i])) <= 2e-2 * abs(slope), (i, slope)
    for p0, g, p, c in zip(before, got, s.w, s.copy):
        want, _, _ = OT.adamw(p0, g, np.zeros_like(g), np.zeros_like(g), step=1, weight_decay=float(np.float32(0.1)), **HYPER)
        assert (np.abs(_f64(p) - want) <= 3 * 2.0 ** -24 * (np.abs(p0) + HYPER["lr"]) * 1.01 + 2.0 ** -20 * HYPER["lr"]).all()
        assert torch.equal(c, p.to(BF))
    assert bool((s.do[u:] == 0).all()) and bool(torch.isnan(s.dx[u:]).all())


def test_captured_steps():
    """Captured once; every replay, with eager work and other data between, leaves the bits of eager steps."""
    a, b = Step(4), Step(4)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        a.run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            a.run()
    torch.cuda.current_stream().wait_stream(stream)
    b.run()
    torch.cuda.synchronize()
    _same(a.state(), b.state())
    for i in range(4):
        a.new_data()
        b.new_data()
        if i == 2:     # other row counts too, and a batch that is not full
            for s in (a, b):
                s.ends.copy_(torch.tensor([0, 70, 70, 71, 200], dtype=torch.int32))
                s.x[200:] = float("nan")
                s.targets[200:] = -1
        graph.replay()
        b.run()
        if i % 2:
            torch.cuda.synchronize()
        _same(a.state(), b.state())


def test_two_steps_at_once():
    pairs = [(Step(k), Step(k)) for k in (5, 6)]
    streams = [torch.cuda.Stream() for _ in pairs]
    torch.cuda.synchronize()
    for _ in range(5):
        for (s, _), stream in zip(pairs, streams):
            with torch.cuda.stream(stream):
                s.run()
                s.step.add_(1)
    torch.cuda.synchronize()
    for s, alone in pairs:
        for _ in range(5):
            alone.run()
            alone.step.add_(1)
        _same(s.state(), alone.state())


def _spread(t, ld):
    """The rows of t, ld elements apart."""
    out = torch.empty((t.shape[0] - 1) * ld + t.shape[1], dtype=t.dtype, device="cuda").as_strided(t.shape, (ld, 1))
    return out.copy_(t)


FAR = 1 << 21


def test_experts_past_32_bits():
    """1100 rows 2^21 elements apart, experts 2^23: offsets past 2^31 elements and 2^32 bytes."""
    E, K, N, rows = 512, 48, 32, 1100
    gen = torch.Generator(device="cuda").manual_seed(7)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(BF)  # noqa: E731
    ends = torch.full((E,), 600, dtype=torch.int32, device="cuda")
    ends[-1] = rows
    x, dy, w = rnd(rows, K), rnd(rows, N), rnd(E, N, K)
    stride = (1 << 23) + 16
    wide = torch.empty((E - 1) * stride + N * K, dtype=BF, device="cuda").as_strided((E, N, K), (stride, K, 1)).copy_(w)
    near = ccl.ccl_grouped(in_features=K, out_features=N, experts=E)
    far = ccl.ccl_grouped(in_features=K, out_features=N, experts=E, w_stride=stride)
    y, z, dx = torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(x)
    fx, fdy = _spread(x, FAR), _spread(dy, FAR)
    ccl.ccl_grouped_gemm(near, rows, ends, x, w, y)
    out = _spread(torch.zeros_like(y), FAR)
    ccl.ccl_grouped_gemm(far, rows, ends, fx, wide, out, preact=z)
    assert torch.equal(out, y) and torch.equal(z, y)
    ccl.ccl_grouped_gemm_grad(near, rows, ends, dy, w, dx)
    out = _spread(torch.zeros_like(dx), FAR)
    ccl.ccl_grouped_gemm_grad(far, rows, ends, fdy, wide, out)
    assert torch.equal(out, dx)
    ccl.ccl_grouped_gemm_wgrad(near, rows, ends, dy, x, w)
    ccl.ccl_grouped_gemm_wgrad(far, rows, ends, fdy, fx, wide)
    assert torch.equal(wide, w)


def test_loss_past_32_bits():
    D, V, tokens = 48, 1100, 1101
    gen = torch.Generator(device="cuda").manual_seed(8)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(BF)  # noqa: E731
    x, w = rnd(tokens, D), rnd(V, D)
    t = torch.randint(0, V, (tokens,), generator=gen, device="cuda")
    near, far = ccl.ccl_vocab(hidden=D, vocab=V), ccl.ccl_vocab(hidden=D, vocab=V, w_ld=FAR)
    ws = torch.empty(ccl.ccl_cross_entropy_workspace(near, tokens, grad=True), dtype=torch.uint8, device="cuda")
    more = dict(workspace=ws, workspace_bytes=ws.numel())
    loss, lf, dx, dw = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    ccl.ccl_cross_entropy_grad(near, tokens, x, w, t, loss, dx, dw, **more)
    fdx, fdw = _spread(torch.zeros_like(x), FAR), _spread(torch.zeros_like(w), FAR)
    ccl.ccl_cross_entropy_grad(far, tokens, _spread(x, FAR), _spread(w, FAR), t, lf, fdx, fdw, **more)
    assert torch.equal(lf, loss) and torch.equal(fdx, dx) and torch.equal(fdw, dw)


def test_adamw_past_32_bits():
    """A tensor of 2^31 elements and some: those last ones as in a tensor of their own (8-bit codes, whose roundings go by
    the place, within one)."""
    tail, first = 1000, 1 << 31
    gen = torch.Generator(device="cuda").manual_seed(9)
    n = first + tail

    def make(size):
        t = dict(param=torch.zeros(size, dtype=BF, device="cuda"), grad=torch.zeros(size, dtype=BF, device="cuda"))
        for k in ("exp_avg", "exp_avg_sq"):
            t[k] = torch.zeros(size, dtype=torch.uint8, device="cuda")
            t[k + "_scale"] = torch.zeros(-(-size // 128), dtype=torch.uint8, device="cuda")
        return t
    big, small = make(n), make(tail)
    p, g = torch.randn(tail, generator=gen, device="cuda").to(BF), torch.randn(tail, generator=gen, device="cuda").to(BF)
    for t, at in ((big, first), (small, 0)):
        t["param"][at:], t["grad"][at:] = p, g
        ccl.ccl_adamw_step(ccl.ccl_adamw([ccl.ccl_adamw_tensor(**t, weight_decay=0.1)]), step=1, **HYPER)
    assert not torch.equal(small["param"], p) and torch.equal(big["param"][first:], small["param"])
    for k in ("exp_avg", "exp_avg_sq"):
        assert torch.equal(big[k + "_scale"][first // 128:], small[k + "_scale"])
        off = big[k][first:].int() - small[k].int()
        assert int(off.abs().max()) == 1
    assert not bool(big["param"][:first].any())
    m = torch.empty(n, dtype=BF, device="cuda")
    ccl.ccl_adamw_moments(n, big["exp_avg"], big["exp_avg_scale"], big["exp_avg_sq"], big["exp_avg_sq_scale"], m, None)
    want = torch.empty(tail, dtype=BF, device="cuda")
    ccl.ccl_adamw_moments(tail, big["exp_avg"][first:], big["exp_avg_scale"][first // 128:], None, None, want, None)
    assert torch.equal(m[first:], want)


@pytest.mark.parametrize("step,lr", [(0, 1e-3), (-3, 1e-3), (-(1 << 63), 1e-3), (1, float("nan")), (1, float("inf"))])
def test_steps_that_cannot_be(step, lr):
    """A step number below 1 or a rate that is not finite, read on the device: nothing is written."""
    f = lambda: torch.full((300,), 0.5, device="cuda")  # noqa: E731
    t = [f() for _ in range(4)]
    ccl.ccl_adamw_step(ccl.ccl_adamw([ccl.ccl_adamw_tensor(*t)]), lr=1.0, step_ptr=torch.tensor([step], device="cuda"),
                       lr_ptr=torch.tensor([lr], device="cuda"))
    assert all(bool((x == 0.5).all()) for x in t)


@pytest.mark.parametrize("K,N", [(80, 96), (1040, 96)])
def test_row_numbers_that_do_not_ascend(K, N):
    """They are taken as the largest so far, within the rows there are."""
    rows, g = 100, ccl.ccl_grouped(in_features=K, out_features=N, experts=5)
    gen = torch.Generator(device="cuda").manual_seed(10)
    x = torch.randn(rows, K, generator=gen, device="cuda").to(BF)
    w = torch.randn(5, N, K, generator=gen, device="cuda").to(BF)
    out = []
    for ends in ([-7, 50, 20, 90, 200], [0, 50, 50, 90, 100]):
        e = torch.tensor(ends, dtype=torch.int32, device="cuda")
        y, dx, dw = torch.zeros(rows, N, dtype=BF, device="cuda"), torch.zeros(rows, K, dtype=BF, device="cuda"), torch.zeros_like(w)
        ws = torch.empty(32 << 20, dtype=torch.uint8, device="cuda")
        more = dict(workspace=ws, workspace_bytes=ws.numel())
        ccl.ccl_grouped_gemm(g, rows, e, x, w, y, **more)
        ccl.ccl_grouped_gemm_grad(g, rows, e, y, w, dx, **more)
        ccl.ccl_grouped_gemm_wgrad(g, rows, e, y, x, dw, **more)
        out.append([y, dx, dw])
    _same(*out)


def test_a_tile_of_masked_logits():
    """256 logits of -inf beside each other (whole tiles of them, or a part): terms of 0."""
    D, V, tokens = 64, 700, 70
    gen = torch.Generator(device="cuda").manual_seed(11)
    x, w = torch.randn(tokens, D, generator=gen, device="cuda").to(BF), torch.randn(V, D, generator=gen, device="cuda").to(BF) * 0.1
    x[:, 0] = 1
    w[:256, 0] = float("-inf")
    w[300:310, 0] = float("-inf")
    live = [*range(256, 300), *range(310, V)]
    t = torch.tensor(live, device="cuda")[torch.randint(0, len(live), (tokens,), generator=gen, device="cuda")]
    head = ccl.ccl_vocab(hidden=D, vocab=V)
    ws = torch.empty(ccl.ccl_cross_entropy_workspace(head, tokens), dtype=torch.uint8, device="cuda")
    loss = torch.empty(tokens, device="cuda")
    ccl.ccl_cross_entropy(head, tokens, x, w, t, loss, workspace=ws, workspace_bytes=ws.numel())
    z = _f64(x) @ _f64(w[live]).T
    at = np.searchsorted(live, t.cpu().numpy())
    want = np.log(np.exp(z).sum(1)) - z[np.arange(tokens), at]
    dz = D * 2.0 ** -23 * (np.abs(_f64(x)) @ np.abs(_f64(w[live])).T).max()
    assert (np.abs(_f64(loss) - want) <= 2 * (dz + 2.0 ** -23 * 110)).all()
