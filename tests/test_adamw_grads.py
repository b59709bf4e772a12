"""AdamwSet.grads: a step reads the gradients that were given last. torch drops the
old ones with zero_grad(), so that a set made once would go on with theirs."""
import pytest
import torch

from paper_2606_11718_amd import ccl

INV = 1


def _refused(call, *args):
    with pytest.raises(ccl.CCLError) as e:
        call(*args)
    assert e.value.status == INV


def _set(device, params):
    moments = [[torch.zeros(p.numel(), device=device) for _ in range(2)] for p in params]
    return ccl.ccl_adamw(ccl.ccl_adamw_tensor(p.detach(), p.grad, *mv, weight_decay=0.1) for p, mv in zip(params, moments)), moments


def test_addresses():
    params = [torch.zeros(n, requires_grad=True) for n in (100, 7)]
    for p in params:
        p.grad = torch.ones_like(p)
    s, _ = _set("cpu", params)
    new = [torch.full((100,), 2.0, dtype=torch.bfloat16), torch.full((7,), 3.0)]
    assert s.grads(g for g in new) is s
    assert [t.grad for t in s.tensors] == [g.data_ptr() for g in new]
    assert [t.grad_type for t in s.tensors] == [ccl.CCL_DT_BF16, ccl.CCL_DT_FP32]
    assert all(held[1] is g for held, g in zip(s.kept, new))
    assert [t.param for t in s.tensors] == [p.data_ptr() for p in params]


def test_refusals():
    """Nothing of a list that is refused is taken."""
    params = [torch.zeros(n, requires_grad=True) for n in (100, 7)]
    for p in params:
        p.grad = torch.ones_like(p)
    s, _ = _set("cpu", params)
    before = [t.grad for t in s.tensors]
    good = torch.zeros(100)
    for bad in ([good], [good, torch.zeros(7), torch.zeros(7)], [good, None], [good, torch.zeros(8)],
                [good, torch.zeros(7).half()], [good, torch.zeros(14)[::2]], [good, torch.zeros(7, device="meta")]):
        _refused(s.grads, bad)
        assert [t.grad for t in s.tensors] == before
    assert ccl.ccl_adamw([]).grads([]).kept == []


@pytest.mark.gpu
def test_steps_of_new_gradients():
    """Backward passes whose gradients are other tensors each time: the steps are those of moments kept by hand, with
    tolerances of four fp32 roundings a step of p's size and 2^-20 of the update (a square root, a reciprocal, products)."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    params = [torch.randn(n, device="cuda", generator=gen).requires_grad_() for n in (1000, 33)]
    want = [p.detach().double() for p in params]
    state = [[torch.zeros_like(w) for w in want] for _ in range(2)]
    held, lr, b1, b2, eps = [], 1e-2, 0.9, 0.99, 1e-8
    s = None
    for step in range(1, 4):
        for p in params:
            p.grad = None
        sum((p * p * step).sum() for p in params).backward()
        held.append([p.grad for p in params])
        if s is None:
            s, _ = _set("cuda", params)
        else:
            s.grads(p.grad for p in params)
        grads = [p.grad.double() for p in params]
        ccl.ccl_adamw_step(s, lr=lr, step=step, beta1=b1, beta2=b2, eps=eps)
        for i, g in enumerate(grads):
            m = state[0][i] = b1 * state[0][i] + (1 - b1) * g
            v = state[1][i] = b2 * state[1][i] + (1 - b2) * g * g
            decay = float(torch.tensor(0.1))
            want[i] = want[i] * (1 - lr * decay) - lr * m / (1 - b1 ** step) / ((v / (1 - b2 ** step)).sqrt() + eps)
    assert len({g.data_ptr() for g in (x[0] for x in held)}) == 3       # kept here: other storage each time
    for p, w in zip(params, want):
        off = (p.detach().double() - w).abs()
        assert bool((off <= 3 * (4 * 2.0 ** -24 * (w.abs() + 1) + 2.0 ** -20 * 3 * lr)).all()), float(off.max())
