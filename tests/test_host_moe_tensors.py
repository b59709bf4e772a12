"""Tensors that ccl_moe_decode's binding refuses: it reads their row strides, so
their types, column strides and sizes have to be those that the call reads them
by (every refusal comes before the first device call; tensors on the host stand
for those on the GPU)."""
import pytest
import torch

from paper_2606_11718_amd import ccl

T, D, F, E, K = 4, 256, 64, 16, 4
BF16, FP8 = torch.bfloat16, torch.float8_e4m3fn


def _tensors(fp8=False):
    w = FP8 if fp8 else BF16
    z = lambda *s, dtype: torch.zeros(s, dtype=dtype)  # noqa: E731
    return dict(x=z(T, D, dtype=BF16), logits=z(T, E, dtype=torch.float32), gate_up=z(E, 2 * F, D, dtype=w),
                down=z(E, D, F, dtype=w), y=z(T, D, dtype=BF16), ids=z(T, K, dtype=torch.int32),
                probs=z(T, K, dtype=torch.float32), gate_up_scale=z(E, dtype=torch.float32),
                down_scale=z(E, dtype=torch.float32))


def _status(change=None, fp8=False, layer=None, tokens=T, **more):
    args = {**_tensors(fp8), **(change or {})}
    moe = ccl.ccl_moe(**{**dict(hidden=D, ffn=F, experts=E, top_k=K,
                                weight_type=ccl.CCL_DT_FP8_E4M3 if fp8 else ccl.CCL_DT_BF16), **(layer or {})})
    # the last of the library's own checks, so that a call which passes the binding's ends there
    with pytest.raises(ccl.CCLError) as e:
        ccl.ccl_moe_decode(moe, tokens, args.pop("x"), args.pop("logits"), args.pop("gate_up"), args.pop("down"),
                           args.pop("y"), workspace=1 << 20, workspace_bytes=1, **args, **more)
    return e.value.status_name, str(e.value)


def _passes(*args, **more):
    status, text = _status(*args, **more)
    return status == "CCL_ERR_INVALID_ARG" and "workspace smaller" in text


def _refused(name, *args, **more):
    status, text = _status(*args, **more)
    return status == "CCL_ERR_INVALID_ARG" and name in text and "workspace" not in text


@pytest.mark.parametrize("fp8", [False, True])
def test_what_the_call_reads_passes(fp8):
    assert _passes(fp8=fp8)
    assert _passes(dict(ids=None, probs=None, gate_up_scale=None, down_scale=None), fp8=fp8)
    t = _tensors(fp8)
    wide = torch.zeros(T, D + 24, dtype=BF16)
    assert _passes(dict(x=wide[:, :D], y=wide[:, 8:8 + D], logits=torch.zeros(T + 3, E + 5)[:, :E]), fp8=fp8)
    assert _passes(dict(x=t["x"].view(T, 1, D), y=t["y"].view(1, T, D)), fp8=fp8)                # leading axes
    assert _passes(dict(x=t["x"].view(-1), logits=t["logits"].view(-1)), fp8=fp8)                # flat
    assert _passes(dict(x=t["x"].view(torch.int16)), fp8=fp8)                                    # raw bits
    raw = {k: t[k].view(torch.uint8).view(-1) for k in ("gate_up", "down")}
    assert _passes(raw, fp8=fp8)                                                                 # raw bytes
    gu = torch.zeros(E, 2 * F, D + 32, dtype=t["gate_up"].dtype)[:, :, :D]
    assert _passes(dict(gate_up=gu), fp8=fp8, layer=dict(gate_up_ld=D + 32))
    one = {k: t[k][:1].as_strided(t[k][:1].shape, (1, *t[k].stride()[1:])) for k in ("gate_up", "down")}
    assert _passes(one, fp8=fp8, layer=dict(experts=1, top_k=1))        # one expert: no stride between experts


@pytest.mark.parametrize("name,dtype", [
    ("logits", BF16), ("logits", torch.float64), ("logits", torch.int32), ("x", torch.float32), ("x", torch.float16),
    ("y", torch.float32), ("gate_up", torch.float32), ("gate_up", torch.float16), ("down", FP8), ("ids", torch.int64),
    ("probs", BF16), ("gate_up_scale", BF16), ("down_scale", torch.float64)])
def test_types(name, dtype):
    assert _refused(name, {name: _tensors()[name].to(dtype)})


def test_fp8_encodings():
    assert _refused("gate_up", dict(gate_up=torch.zeros(E, 2 * F, D, dtype=torch.float8_e5m2)), fp8=True)
    assert _refused("down", dict(down=torch.zeros(E, D, F, dtype=torch.float8_e4m3fnuz)), fp8=True)
    assert _refused("down", dict(down=torch.zeros(E, D, F, dtype=BF16)), fp8=True)


@pytest.mark.parametrize("name", ["x", "y", "logits", "ids", "probs"])
def test_column_strides(name):
    t = _tensors()[name]
    twice = torch.zeros(T, 2 * t.shape[1], dtype=t.dtype)
    assert _refused(name, {name: twice[:, ::2]})
    assert _refused(name, {name: torch.zeros(2 * t.shape[1], T, dtype=t.dtype).t()[:, :t.shape[1]]})


@pytest.mark.parametrize("name", ["gate_up_scale", "down_scale"])
def test_scale_strides(name):
    assert _refused(name, {name: torch.zeros(2 * E)[::2]})
    assert _refused(name, {name: torch.zeros(1).expand(E)})


@pytest.mark.parametrize("name", ["gate_up", "down"])
def test_weight_strides(name):
    t = _tensors()[name]
    e, r, c = t.shape
    assert _refused(name, {name: torch.zeros(e, c, r, dtype=BF16).transpose(1, 2)})        # input-major
    assert _refused(name, {name: torch.zeros(e, r, c + 32, dtype=BF16)[:, :, :c]})         # a gap the layer does not have
    assert _refused(name, {name: torch.zeros(1, r, c, dtype=BF16).expand(e, r, c)})


def test_sizes():
    """Tensors that end before what the call would read or write."""
    for name, t in _tensors().items():
        assert _refused(name, {name: t[:-1]}), name
    t = _tensors()
    for name in ("x", "y", "logits", "gate_up", "down"):
        assert _refused(name, {name: t[name][..., :-8]}), name
        assert _refused(name, {name: t[name].reshape(-1)[:-1]}), name
    assert _refused("x", dict(x=torch.zeros(2, T // 2, 2 * D, dtype=BF16)[:, :, :D].transpose(0, 1)))   # no one row stride


def test_an_address_or_a_stride_is_taken_as_given():
    assert _passes(dict(x=1 << 20, logits=1 << 20, y=1 << 20, gate_up=1 << 20, down=1 << 20, ids=1 << 20, probs=1 << 20))
    # columns of a wider allocation, whose row stride the caller states
    assert _passes(dict(x=torch.zeros(T * 512, dtype=BF16)), x_ld=512)
