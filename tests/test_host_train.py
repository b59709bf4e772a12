"""What the training operators and their queries refuse (every refusal comes
before the first device call)."""
import ctypes

import pytest
import torch

from paper_2606_11718_amd import ccl

P = 1 << 20
INV, UNS, MIS = "CCL_ERR_INVALID_ARG", "CCL_ERR_UNSUPPORTED", "CCL_ERR_MISALIGNED_POINTER"


def _refused(status, call, *args, **more):
    with pytest.raises(ccl.CCLError) as e:
        call(*args, **more)
    assert e.value.status_name == status, str(e.value)


# ---- experts' products ----

GROUPED = dict(in_features=64, out_features=96, experts=4)


@pytest.mark.parametrize("change,status", [
    (dict(in_features=0), INV), (dict(out_features=-16), INV), (dict(in_features=72), UNS), (dict(out_features=100), UNS),
    (dict(in_features=1 << 21), UNS), (dict(experts=0), INV), (dict(experts=513), INV), (dict(activation=4), INV),
    (dict(gated=2), INV), (dict(w_ld=56), INV), (dict(w_ld=68), MIS), (dict(w_ld=1 << 22), INV),
    (dict(w_stride=64 * 96 - 8), INV), (dict(w_stride=64 * 96 + 4), MIS), (dict(w_stride=1 << 49), INV),
])
def test_grouped_description(change, status):
    g = ccl.ccl_grouped(**{**GROUPED, **change})
    for way in (ccl.CCL_GROUPED_FORWARD, ccl.CCL_GROUPED_GRAD, ccl.CCL_GROUPED_WGRAD):
        _refused(status, ccl.ccl_grouped_gemm_workspace, g, 10, way)
    _refused(status, ccl.ccl_grouped_gemm, g, 10, P, P, P, P)
    _refused(status, ccl.ccl_grouped_gemm_grad, g, 10, P, P, P, P, preact=P)
    _refused(status, ccl.ccl_grouped_gemm_wgrad, g, 10, P, P, P, P)


def test_grouped_sizes():
    g = ccl.ccl_grouped(**GROUPED)
    _refused(INV, ccl.ccl_grouped_gemm_workspace, g, 10, 3)
    _refused(INV, ccl.ccl_grouped_gemm_workspace, g, -1, 0)
    _refused(INV, ccl.ccl_grouped_gemm_workspace, g, (1 << 30) + 1, 0)
    odd = ccl.ccl_grouped(in_features=64, out_features=48, experts=4, gated=True)
    _refused(UNS, ccl.ccl_grouped_gemm, odd, 10, P, P, P, P)              # gate and up rows of 24
    assert ccl.ccl_grouped_gemm_workspace(odd, 10, ccl.CCL_GROUPED_GRAD) >= 0
    wide = ccl.ccl_grouped(in_features=32768, out_features=32768, experts=1, gated=True)
    _refused(UNS, ccl.ccl_grouped_gemm, wide, 10, P, P, P, P)
    assert ccl.ccl_grouped_gemm_workspace(wide, 10, ccl.CCL_GROUPED_GRAD) >= 0
    many = ccl.ccl_grouped(in_features=1 << 20, out_features=1 << 20, experts=512)
    _refused(UNS, ccl.ccl_grouped_gemm_wgrad, many, 10, P, P, P, P)


@pytest.mark.parametrize("call", ["ccl_grouped_gemm", "ccl_grouped_gemm_grad", "ccl_grouped_gemm_wgrad"])
def test_grouped_pointers(call):
    f = getattr(ccl, call)
    g = ccl.ccl_grouped(**GROUPED)
    for i in range(4):
        args = [P, P, P, P]
        args[i] = None
        _refused(INV, f, g, 10, *args)
        args[i] = P + (2 if i == 0 else 8)
        _refused(MIS, f, g, 10, *args)


@pytest.mark.parametrize("call,more,status", [
    ("ccl_grouped_gemm", dict(x_ld=60), INV), ("ccl_grouped_gemm", dict(x_ld=68), MIS), ("ccl_grouped_gemm", dict(y_ld=88), INV),
    ("ccl_grouped_gemm", dict(y_ld=100), MIS), ("ccl_grouped_gemm", dict(preact=P, z_ld=88), INV),
    ("ccl_grouped_gemm", dict(preact=P + 8), MIS), ("ccl_grouped_gemm", dict(x_ld=1 << 22), INV),
    ("ccl_grouped_gemm_grad", dict(dy_ld=88), INV), ("ccl_grouped_gemm_grad", dict(dx_ld=56), INV),
    ("ccl_grouped_gemm_grad", dict(dx_ld=68), MIS), ("ccl_grouped_gemm_wgrad", dict(dy_ld=88), INV),
    ("ccl_grouped_gemm_wgrad", dict(x_ld=68), MIS), ("ccl_grouped_gemm_wgrad", dict(accumulate=2), INV),
    ("ccl_grouped_gemm_wgrad", dict(dw_type=ccl.CCL_DT_FP8_E4M3), INV),
])
def test_grouped_calls(call, more, status):
    _refused(status, getattr(ccl, call), ccl.ccl_grouped(**GROUPED), 10, P, P, P, P, **more)


def test_grouped_workspace():
    """Enough for fewer rows too, and bounded."""
    for K, N, E in ((64, 96, 4), (4096, 4096, 1), (256, 256, 4), (2048, 1536, 128), (8192, 64, 2)):
        g = ccl.ccl_grouped(in_features=K, out_features=N, experts=E)
        for way in (ccl.CCL_GROUPED_FORWARD, ccl.CCL_GROUPED_GRAD, ccl.CCL_GROUPED_WGRAD):
            need = [ccl.ccl_grouped_gemm_workspace(g, r, way) for r in (0, 1, 63, 300, 5000, 100000, 1 << 30)]
            assert need == sorted(need) and need[0] == 0 and need[-1] <= 32 << 20


def test_grouped_grad_needs_what_it_goes_through():
    for how in (dict(activation=ccl.CCL_ACT_SILU), dict(gated=True)):
        g = ccl.ccl_grouped(**GROUPED, **how)
        _refused(INV, ccl.ccl_grouped_gemm_grad, g, 10, P, P, P, P)
    gated = ccl.ccl_grouped(**GROUPED, gated=True)
    _refused(INV, ccl.ccl_grouped_gemm_grad, gated, 10, P, P, P, P, preact=P, z_ld=120)
    _refused(INV, ccl.ccl_grouped_gemm_grad, gated, 10, P, P, P, P, preact=P, dx_ld=64)


def test_grouped_grad_in_place():
    """dX is preact: its rows lie where preact's do."""
    for how, wide in ((dict(activation=ccl.CCL_ACT_SILU), 64), (dict(gated=True), 128)):
        g = ccl.ccl_grouped(**GROUPED, **how)
        with pytest.raises(ccl.CCLError, match="in place of preact"):
            ccl.ccl_grouped_gemm_grad(g, 10, 2 * P, 3 * P, 4 * P, P, preact=P, dx_ld=wide, z_ld=wide + 8)


def test_grouped_tensors():
    g = ccl.ccl_grouped(**GROUPED)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    ends, x, w, y = torch.zeros(4, dtype=torch.int32), bf(10, 64), bf(4, 96, 64), bf(10, 96)
    for bad in (dict(ends=ends.long()), dict(ends=ends[:3]), dict(x=x[:9]), dict(x=x[:, :60]), dict(x=x.float()),
                dict(x=bf(64, 10).t()), dict(w=w[:3]), dict(w=w.float()), dict(w=bf(4, 64, 96).transpose(1, 2)), dict(y=y.float()),
                dict(y=bf(10, 80))):
        a = {**dict(ends=ends, x=x, w=w, y=y), **bad}
        _refused(INV, ccl.ccl_grouped_gemm, g, 10, a["ends"], a["x"], a["w"], a["y"])
    _refused(INV, ccl.ccl_grouped_gemm_wgrad, g, 10, ends, y, x, torch.zeros(4, 96, 64, dtype=torch.float16))
    _refused(INV, ccl.ccl_grouped_gemm_wgrad, g, 10, ends, y, x, w, dw_type=ccl.CCL_DT_FP32)


# ---- vocabulary loss ----

VOCAB = dict(hidden=64, vocab=1000)


@pytest.mark.parametrize("change,status", [
    (dict(hidden=0), INV), (dict(vocab=0), INV), (dict(hidden=72), UNS), (dict(hidden=1 << 21), UNS), (dict(vocab=(1 << 20) + 1), UNS),
    (dict(block=-1), INV), (dict(block=32769), INV), (dict(scale=float("nan")), INV), (dict(scale=float("inf")), INV),
    (dict(w_ld=56), INV), (dict(w_ld=68), MIS), (dict(w_ld=1 << 22), INV),
])
def test_vocab_description(change, status):
    v = ccl.ccl_vocab(**{**VOCAB, **change})
    _refused(status, ccl.ccl_cross_entropy_workspace, v, 10)
    _refused(status, ccl.ccl_cross_entropy_workspace, v, 10, grad=True)
    _refused(status, ccl.ccl_cross_entropy, v, 10, P, P, P, P, workspace=P, workspace_bytes=1 << 40)
    _refused(status, ccl.ccl_cross_entropy_grad, v, 10, P, P, P, P, P, P, workspace=P, workspace_bytes=1 << 40)


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("change,status", [
    (dict(x=None), INV), (dict(w=None), INV), (dict(t=None), INV), (dict(x=P + 8), MIS), (dict(w=P + 8), MIS), (dict(t=P + 4), MIS),
    (dict(loss=P + 2), MIS), (dict(lse=P + 2), MIS), (dict(x_ld=60), INV), (dict(x_ld=68), MIS), (dict(workspace=None), INV),
    (dict(workspace_bytes=64), INV), (dict(workspace=P + 8), MIS), (dict(tokens=-1), INV), (dict(tokens=(1 << 30) + 1), INV),
])
def test_vocab_calls(change, status, grad):
    a = {**dict(x=P, w=P, t=P, loss=P, tokens=10), **{k: v for k, v in change.items() if k in ("x", "w", "t", "loss", "tokens")}}
    more = {**dict(workspace=P, workspace_bytes=1 << 40), **{k: v for k, v in change.items() if k not in a}}
    v = ccl.ccl_vocab(**VOCAB)
    if grad:
        _refused(status, ccl.ccl_cross_entropy_grad, v, a["tokens"], a["x"], a["w"], a["t"], a["loss"], P, P, **more)
    else:
        _refused(status, ccl.ccl_cross_entropy, v, a["tokens"], a["x"], a["w"], a["t"], a["loss"], **more)


@pytest.mark.parametrize("more,status", [
    (dict(dX=None, dW=None), INV), (dict(dX=P + 8), MIS), (dict(dW=P + 8), MIS), (dict(dw_type=ccl.CCL_DT_FP8_E4M3), INV),
    (dict(accumulate=3), INV), (dict(dx_ld=60), INV), (dict(dx_ld=68), MIS), (dict(dw_ld=60), INV), (dict(dw_ld=68), MIS),
    (dict(dloss=P + 2), MIS), (dict(dw_ld=66, dw_type=ccl.CCL_DT_FP32), MIS),
])
def test_vocab_grad_calls(more, status):
    args = {"dX": P, "dW": P, **more}
    dX, dW = args.pop("dX"), args.pop("dW")
    _refused(status, ccl.ccl_cross_entropy_grad, ccl.ccl_vocab(**VOCAB), 10, P, P, P, P, dX, dW, workspace=P,
             workspace_bytes=1 << 40, **args)


def test_vocab_no_outputs():
    _refused(INV, ccl.ccl_cross_entropy, ccl.ccl_vocab(**VOCAB), 10, P, P, P, None, workspace=P, workspace_bytes=1 << 40)


def test_vocab_tensors():
    v = ccl.ccl_vocab(**VOCAB)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    ok = dict(x=bf(10, 64), w=bf(1000, 64), t=torch.zeros(10, dtype=torch.int64), loss=torch.zeros(10))
    for bad in (dict(x=bf(9, 64)), dict(x=bf(10, 64).float()), dict(w=bf(999, 64)), dict(w=bf(1000, 80)[:, :64]), dict(w=bf(64, 1000).t()),
                dict(t=torch.zeros(10, dtype=torch.int32)), dict(t=torch.zeros(20, dtype=torch.int64)[::2]), dict(loss=torch.zeros(9)),
                dict(loss=bf(10))):
        a = {**ok, **bad}
        _refused(INV, ccl.ccl_cross_entropy, v, 10, a["x"], a["w"], a["t"], a["loss"], workspace=P, workspace_bytes=1 << 40)
    _refused(INV, ccl.ccl_cross_entropy_grad, v, 10, ok["x"], ok["w"], ok["t"], ok["loss"], bf(10, 64),
             torch.zeros(1000, 64, dtype=torch.float16), workspace=P, workspace_bytes=1 << 40)


def test_vocab_workspace():
    """Bounded by the block: what is kept does not grow with the tokens beyond it."""
    v = ccl.ccl_vocab(hidden=2048, vocab=131072)
    need = [ccl.ccl_cross_entropy_workspace(v, t, grad=True) for t in (1, 100, 8192, 15000, 16128, 16129, 100000, 1000000)]
    assert need == sorted(need) and need[-1] < (4 << 30) + (3 << 29)
    assert ccl.ccl_cross_entropy_workspace(v, 0, grad=True) == 0
    small = ccl.ccl_vocab(hidden=2048, vocab=131072, block=256)
    assert ccl.ccl_cross_entropy_workspace(small, 8192) < ccl.ccl_cross_entropy_workspace(v, 8192)


# ---- AdamW ----

def _entry(**change):
    t = ccl._AdamwTensor(P, 2 * P, 3 * P, 4 * P, 0, 0, 0, 1000, ccl.CCL_DT_FP32, ccl.CCL_DT_FP32, 32, 0.0)
    for k, v in change.items():
        setattr(t, k, v)
    return t, ()


@pytest.mark.parametrize("change,status", [
    (dict(param=None), INV), (dict(grad=None), INV), (dict(exp_avg=None), INV), (dict(exp_avg_sq=None), INV), (dict(n=-1), INV),
    (dict(n=(1 << 34) + 1), INV), (dict(param_type=1), INV), (dict(grad_type=1), INV), (dict(moment_bits=16), INV),
    (dict(moment_bits=8), INV), (dict(moment_bits=8, exp_avg_scale=P), INV), (dict(weight_decay=float("nan")), INV),
    (dict(param=P + 2), MIS), (dict(grad=P + 2), MIS), (dict(exp_avg=P + 2), MIS), (dict(exp_avg_sq=P + 2), MIS),
    (dict(copy=P + 1), MIS), (dict(param=P + 1, param_type=0), MIS), (dict(exp_avg=P), INV), (dict(copy=P + 100), INV),
])
def test_adamw_tensors(change, status):
    _refused(status, ccl.ccl_adamw_step, ccl.ccl_adamw([_entry(**change)]), lr=1e-3, step=1)


def test_adamw_the_same_tensor_twice():
    _refused(INV, ccl.ccl_adamw_step, ccl.ccl_adamw([_entry(), _entry()]), lr=1e-3, step=1)
    _refused(INV, ccl.ccl_adamw_step, ccl.ccl_adamw([_entry(), _entry(param=9 * P, exp_avg=10 * P)]), lr=1e-3, step=1)
    _refused(INV, ccl.ccl_adamw_step, ccl.ccl_adamw([_entry(), _entry(param=P - 3996, exp_avg=10 * P, exp_avg_sq=11 * P)]),
             lr=1e-3, step=1)
    eight = dict(moment_bits=8, exp_avg_scale=5 * P, exp_avg_sq_scale=6 * P)
    _refused(INV, ccl.ccl_adamw_step, ccl.ccl_adamw([_entry(**{**eight, "exp_avg_sq_scale": 5 * P})]), lr=1e-3, step=1)
    other = dict(param=9 * P, exp_avg=10 * P, exp_avg_sq=11 * P, exp_avg_scale=12 * P)
    _refused(INV, ccl.ccl_adamw_step, ccl.ccl_adamw([_entry(**eight), _entry(**{**eight, **other})]), lr=1e-3, step=1)


def test_adamw_count():
    for count in (-1, (1 << 20) + 1, 1 << 62):
        a = ccl._Adamw(1e-3, 0.9, 0.999, 1e-8, 1, None, None, None)
        assert ccl.library().ccl_adamw_step(ctypes.byref(a), ctypes.byref(_entry()[0]), count, None) == 1, count


@pytest.mark.parametrize("more", [dict(step=0), dict(step=-5), dict(step=1, lr=float("inf")), dict(step=1, beta1=1.0),
                                  dict(step=1, beta2=-0.1), dict(step=1, eps=-1e-8), dict(step=1, eps=float("nan")),
                                  dict(step=1, beta1=float("nan"))])
def test_adamw_numbers(more):
    _refused(INV, ccl.ccl_adamw_step, ccl.ccl_adamw([_entry()]), **{"lr": 1e-3, **more})


def test_adamw_binding():
    f, b8 = lambda n: torch.zeros(n), lambda n: torch.zeros(n, dtype=torch.uint8)  # noqa: E731
    make = ccl.ccl_adamw_tensor
    _refused(INV, make, f(100), f(99), f(100), f(100))
    _refused(INV, make, f(100), f(100), f(100), f(101))
    _refused(INV, make, f(100), f(100).half(), f(100), f(100))
    _refused(INV, make, f(100).double(), f(100), f(100), f(100))
    _refused(INV, make, f(100), f(100), b8(100), f(100), exp_avg_scale=b8(1), exp_avg_sq_scale=b8(1))
    _refused(INV, make, f(130), f(130), b8(130), b8(130), exp_avg_scale=b8(1), exp_avg_sq_scale=b8(2))
    _refused(INV, make, f(100), f(100), f(100), f(100), copy=f(100))
    _refused(INV, make, f(200)[::2], f(100), f(100), f(100))
    _refused(INV, ccl.ccl_adamw_moments, 130, b8(130), b8(1), b8(130), b8(2), f(130), f(130))
    _refused(INV, ccl.ccl_adamw_moments, 130, b8(130), b8(2), b8(130), b8(2), f(130), f(130).bfloat16())
    _refused(INV, ccl.ccl_adamw_moments, 130, b8(130), b8(2), b8(130), b8(2), f(130).double(), None)
    # nothing to do: no device needed
    ccl.ccl_adamw_step(ccl.ccl_adamw([]), lr=1e-3, step=1)
    ccl.ccl_adamw_step(ccl.ccl_adamw([make(f(0), f(0), f(0), f(0))]), lr=1e-3, step=1)


def test_tensors_of_another_device():
    """Tensors in host memory that would fit otherwise: refused before anything is launched."""
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    g = ccl.ccl_grouped(**GROUPED)
    ends = torch.zeros(4, dtype=torch.int32)
    _refused(INV, ccl.ccl_grouped_gemm, g, 10, ends, bf(10, 64), bf(4, 96, 64), bf(10, 96))
    _refused(INV, ccl.ccl_grouped_gemm_grad, g, 10, ends, bf(10, 96), bf(4, 96, 64), bf(10, 64))
    _refused(INV, ccl.ccl_grouped_gemm_wgrad, g, 10, ends, bf(10, 96), bf(10, 64), bf(4, 96, 64))
    v = ccl.ccl_vocab(**VOCAB)
    t, loss = torch.zeros(10, dtype=torch.int64), torch.zeros(10)
    _refused(INV, ccl.ccl_cross_entropy, v, 10, bf(10, 64), bf(1000, 64), t, loss, workspace=P, workspace_bytes=1 << 40)
    _refused(INV, ccl.ccl_cross_entropy_grad, v, 10, bf(10, 64), bf(1000, 64), t, loss, bf(10, 64), None, workspace=P,
             workspace_bytes=1 << 40)
    f = lambda n: torch.zeros(n)  # noqa: E731
    _refused(INV, ccl.ccl_adamw_step, ccl.ccl_adamw([ccl.ccl_adamw_tensor(f(9), f(9), f(9), f(9))]), lr=1e-3, step=1)
    _refused(INV, ccl.ccl_adamw_step, ccl.ccl_adamw([_entry()]), lr=1e-3, step=1, grad_scale=f(1))
    b8 = lambda n: torch.zeros(n, dtype=torch.uint8)  # noqa: E731
    _refused(INV, ccl.ccl_adamw_moments, 130, b8(130), b8(2), b8(130), b8(2), f(130), f(130))


def test_rows_of_the_output_matrix(monkeypatch):
    """W's rows lie as the description says: one row expanded to all (stride 0), rows with gaps, or rows without the gaps
    that w_ld names are refused; the calls would read behind them."""
    monkeypatch.setattr(ccl, "_here", lambda **tensors: None)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    for w_ld, bad in ((0, bf(1, 64).expand(1000, 64)), (64, bf(1, 64).expand(1000, 64)), (0, bf(1000, 72)[:, :64]),
                      (72, bf(1000, 64)), (72, bf(1, 64).expand(1000, 64))):
        v = ccl.ccl_vocab(**{**VOCAB, "w_ld": w_ld})
        for call in (lambda: ccl.ccl_cross_entropy(v, 10, P, bad, P, P, workspace=P, workspace_bytes=1 << 40),  # noqa: B023
                     lambda: ccl.ccl_cross_entropy_grad(v, 10, P, bad, P, P, P, P, workspace=P, workspace_bytes=1 << 40)):  # noqa: B023
            with pytest.raises(ccl.CCLError, match="W: rows"):
                call()


def test_workspace_tensors(monkeypatch):
    """A tensor smaller than the bytes it is given for, or with gaps, is refused, whatever it is on."""
    monkeypatch.setattr(ccl, "_here", lambda **tensors: None)
    v = ccl.ccl_vocab(**VOCAB)
    need = ccl.ccl_cross_entropy_workspace(v, 10, grad=True)
    bytes_ = lambda n: torch.zeros(n, dtype=torch.uint8)  # noqa: E731
    for ws in (bytes_(need - 1), bytes_(2 * need)[::2]):
        for call in (lambda: ccl.ccl_cross_entropy(v, 10, P, P, P, P, workspace=ws, workspace_bytes=need),  # noqa: B023
                     lambda: ccl.ccl_cross_entropy_grad(v, 10, P, P, P, P, P, P, workspace=ws, workspace_bytes=need),  # noqa: B023
                     lambda: ccl.ccl_grouped_gemm(ccl.ccl_grouped(**GROUPED), 10, P, P, P, P, workspace=ws,  # noqa: B023
                                                  workspace_bytes=need)):
            with pytest.raises(ccl.CCLError, match="contiguous bytes"):
                call()
