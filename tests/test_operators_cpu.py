"""The gate, the experts' products and the layer of few tokens without a GPU: what the entry points refuse
(every check is made before anything is launched), and the reference's gradients against differences."""
import ctypes
import math

import pytest
import torch

import operators_reference as ref


@pytest.fixture(scope="module")
def ep():
    from paper_2603_13606_amd import binding, build
    if not build.is_current():
        build.build()
    binding.load()
    return binding


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def refused(ep, code, fn, *a, **kw):
    with pytest.raises(ep.EpError) as e:
        fn(*a, stream=0, **kw)
    assert e.value.code == code


@pytest.mark.parametrize("change", [
    dict(score=2), dict(score=-1), dict(renormalise=2), dict(scale=math.inf), dict(scale=math.nan), dict(num_groups=0),
    dict(num_groups=3), dict(num_groups=4, groups_kept=5), dict(num_groups=4, groups_kept=0), dict(num_groups=128, groups_kept=1),
    dict(logits=torch.zeros(4, 128, dtype=torch.int32)), dict(logits=torch.zeros(4, 1032)), dict(logits=torch.zeros(128)),
    dict(logits=torch.zeros(128, 4).t()), dict(idx=i32(4, 65), w=torch.zeros(4, 65)), dict(idx=i32(5, 8)), dict(w=torch.zeros(4, 7)),
    dict(idx=torch.zeros(4, 8)), dict(w=torch.zeros(4, 8, dtype=torch.bfloat16)), dict(bias=torch.zeros(127)),
    dict(bias=torch.zeros(128, dtype=torch.bfloat16)), dict(idx=i32(8, 4).t()),
])
def test_route_refuses(ep, change):
    a = dict(logits=torch.zeros(4, 128), idx=i32(4, 8), w=torch.zeros(4, 8), bias=None)
    kw = {k: v for k, v in change.items() if k not in a}
    a.update({k: v for k, v in change.items() if k in a})
    refused(ep, ep.EP_ERR_INVALID_ARG, ep.ep_route, a["logits"], a["idx"], a["w"], bias=a["bias"], **kw)
    if "bias" not in change and not {"num_groups", "groups_kept"} & set(kw):
        refused(ep, ep.EP_ERR_INVALID_ARG, ep.ep_route_backward, a["logits"], a["idx"], a["w"], torch.zeros_like(a["logits"]), **kw)


def test_route_backward_refuses_another_type_or_shape(ep):
    for g in (torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(4, 127), torch.zeros(3, 128)):
        refused(ep, ep.EP_ERR_INVALID_ARG, ep.ep_route_backward, torch.zeros(4, 128), i32(4, 8), torch.zeros(4, 8), g)


def odd(t):
    """The same shape, off a 16-byte boundary."""
    n = t.numel()
    return torch.zeros(n + 8, dtype=t.dtype)[1:n + 1].view(t.shape)


@pytest.mark.parametrize("change,code", [
    (dict(activation=3), 1), (dict(activation=-1), 1), (dict(gated=2), 1), (dict(first_expert=1), 1), (dict(first_expert=-1), 1),
    (dict(w=bf(3, 24, 60)), 1), (dict(w=bf(3, 20, 64)), 1), (dict(w=bf(24, 64)), 1), (dict(w=bf(3, 24, 64).float()), 1),
    (dict(w=odd(bf(3, 24, 64))), 1), (dict(x=odd(bf(10, 64))), 1), (dict(x=bf(10, 72)), 1), (dict(x=bf(10, 64).float()), 1),
    (dict(out=bf(10, 32)), 1), (dict(out=bf(10, 28)[:, :24]), 1), (dict(out=bf(24, 10).t()), 1), (dict(out=bf(1, 10, 24)), 1),
    (dict(bias=bf(3, 16)), 1), (dict(bias=bf(2, 24)), 1), (dict(bias=i32(3, 24)), 1), (dict(bias=odd(bf(3, 24))), 1),
    (dict(residual=bf(10, 32)), 1), (dict(pre=bf(10, 32)), 1), (dict(count=None), 1), (dict(count=i32(2)), 1), (dict(offset=i32(2)), 1),
    (dict(offset=None), 1), (dict(count=torch.zeros(3)), 1), (dict(gated=True), 1), (dict(w=bf(1025, 8, 64), out=bf(10, 8)), 1),
    (dict(x=bf(3, 5, 64), out=bf(3, 5, 24)), 1),                     # padded rows have no offsets
    (dict(x=bf(2, 5, 64), out=bf(2, 5, 24), offset=None), 1), (dict(x=bf(3, 5, 64), out=bf(3, 6, 24), offset=None), 1),
])
def test_expert_product_refuses(ep, change, code):
    a = dict(x=bf(10, 64), w=bf(3, 24, 64), out=bf(10, 24), bias=None, residual=None, pre=None, offset=i32(3), count=i32(3))
    kw = {k: v for k, v in change.items() if k not in a}
    a.update({k: v for k, v in change.items() if k in a})
    refused(ep, code, ep.ep_expert_product, a["x"], a["w"], a["out"], bias=a["bias"], residual=a["residual"], pre=a["pre"],
            row_offset=a["offset"], row_count=a["count"], **kw)


def test_outputs_whose_rows_share_memory_are_refused(ep):
    """Expanded outputs, or windows that reach into each other; interleaved ones are fine (empty here: nothing is launched)."""
    x, cnt = bf(3, 5, 64), i32(3)
    for out in (bf(1, 5, 24).expand(3, 5, 24), bf(216).as_strided((3, 5, 24), (48, 24, 1))):
        refused(ep, ep.EP_ERR_INVALID_ARG, ep.ep_expert_product, x, bf(3, 24, 64), out, row_count=cnt)
        refused(ep, ep.EP_ERR_INVALID_ARG, ep.ep_expert_product, x, bf(3, 24, 64), bf(3, 5, 24), pre=out, row_count=cnt)
        refused(ep, ep.EP_ERR_INVALID_ARG, ep.ep_expert_product_backward, x, bf(3, 64, 24), grad_x=out, row_count=cnt)
    for gw in (bf(1, 24, 64).expand(3, 24, 64), bf(24, 64).as_strided((3, 16, 64), (64, 64, 1))):
        refused(ep, ep.EP_ERR_INVALID_ARG, ep.ep_expert_product_backward, bf(3, 5, gw.shape[1]), x=x, grad_weights=gw, row_count=cnt)
    none = bf(3, 0, 64)
    ep.ep_expert_product(none, bf(3, 24, 64), bf(0, 3, 24).transpose(0, 1), row_count=cnt, stream=0)


def test_expert_product_refuses_far_rows(ep):
    """Rows 2^22 elements apart, and a gated expert whose weights span 2^31 bytes."""
    d = ep.tensor_desc(bf(10, 64), ep.EP_TAG_TOKENS)
    d.stride[0] = 1 << 22
    w = ep.tensor_desc(bf(1, 64, 64), ep.EP_TAG_EXPERT_WEIGHTS)
    out, cnt, off = ep.tensor_desc(bf(10, 64), ep.EP_TAG_TOKENS), ep.tensor_desc(i32(1), ep.EP_TAG_ROW_COUNT), ep.tensor_desc(i32(1), ep.EP_TAG_ROW_OFFSET)
    cfg = ep._product_config(ep.EP_ACT_NONE, False)

    def call(x, w, out):
        ins = (ep.ep_tensor_t * 4)(x, w, cnt, off)
        return ep.load().ep_expert_product(None, ctypes.byref(cfg), ins, 4, (ep.ep_tensor_t * 1)(out), 1, None)
    assert call(d, w, out) == ep.EP_ERR_INVALID_ARG
    cfg = ep._product_config(ep.EP_ACT_SILU, True)
    w.stride[1] = 1 << 24
    assert call(ep.tensor_desc(bf(10, 64), ep.EP_TAG_TOKENS), w, ep.tensor_desc(bf(10, 32), ep.EP_TAG_TOKENS)) == ep.EP_ERR_INVALID_ARG
    w.stride[1], w.shape[1] = (1 << 22) - 8, 512
    assert call(ep.tensor_desc(bf(10, 64), ep.EP_TAG_TOKENS), w, ep.tensor_desc(bf(10, 256), ep.EP_TAG_TOKENS)) == ep.EP_ERR_UNSUPPORTED
    cfg.size = 4
    assert call(ep.tensor_desc(bf(10, 64), ep.EP_TAG_TOKENS), w, out) == ep.EP_ERR_INVALID_ARG


@pytest.mark.parametrize("change", [
    dict(w=None, gw=None), dict(w=None), dict(x=None), dict(gb=bf(3, 24).float()), dict(gw=None), dict(gw=bf(3, 24, 72)),
    dict(gw=i32(3, 24, 64)), dict(pre=bf(10, 24)), dict(gp=bf(10, 24)), dict(activation=1), dict(gated=True),
    dict(gx=bf(10, 72)), dict(go=bf(10, 32)), dict(accumulate=2),
])
def test_expert_product_backward_refuses(ep, change):
    a = dict(go=bf(10, 24), w=bf(3, 24, 64), x=bf(10, 64), pre=None, gp=None, gx=bf(10, 64), gw=bf(3, 24, 64), gb=bf(3, 24))
    kw = {k: v for k, v in change.items() if k not in a}
    a.update({k: v for k, v in change.items() if k in a})
    refused(ep, ep.EP_ERR_INVALID_ARG, ep.ep_expert_product_backward, a["go"], a["w"], x=a["x"], pre=a["pre"], grad_pre=a["gp"],
            grad_x=a["gx"], grad_weights=a["gw"], grad_bias=a["gb"], row_offset=i32(3), row_count=i32(3), **kw)


@pytest.mark.parametrize("change,code", [
    (dict(x=bf(129, 64), idx=i32(129, 2), wt=None, out=bf(129, 64)), 4), (dict(idx=i32(3, 2)), 1), (dict(idx=i32(4, 65), wt=None), 1),
    (dict(wt=torch.zeros(4, 3)), 1), (dict(up=bf(5, 32, 72)), 1), (dict(up=bf(4, 32, 64)), 1), (dict(down=bf(5, 64, 24)), 1),
    (dict(down=bf(5, 72, 16)), 1), (dict(out=bf(4, 72)), 1), (dict(out=odd(bf(4, 64))), 1), (dict(ws=None), 1),
    (dict(ws=torch.zeros(64, dtype=torch.uint8)), 1), (dict(ws=torch.zeros(1 << 16)), 1), (dict(bu=bf(5, 16)), 1), (dict(bd=bf(5, 72)), 1),
    (dict(res=bf(3, 64)), 1), (dict(activation=9), 1), (dict(first_expert=-1), 1), (dict(gated=False), 1),
])
def test_expert_layer_refuses(ep, change, code):
    a = dict(x=bf(4, 64), idx=i32(4, 2), wt=torch.zeros(4, 2), up=bf(5, 32, 64), down=bf(5, 64, 16), out=bf(4, 64),
             ws=torch.zeros(1 << 16, dtype=torch.uint8), bu=None, bd=None, res=None)
    kw = dict(dict(activation=1, gated=True), **{k: v for k, v in change.items() if k not in a})
    a.update({k: v for k, v in change.items() if k in a})
    refused(ep, code, ep.ep_expert_layer, a["x"], a["idx"], a["wt"], a["up"], a["down"], a["out"], a["ws"], bias_up=a["bu"],
            bias_down=a["bd"], residual=a["res"], **kw)


def test_empty_calls_launch_nothing(ep):
    """No tokens, or windows without a row in any tensor: success, without a GPU."""
    ep.ep_route(torch.zeros(0, 16), i32(0, 2), torch.zeros(0, 2), stream=0)
    ep.ep_route_backward(torch.zeros(0, 16), i32(0, 2), torch.zeros(0, 2), torch.zeros(0, 16), stream=0)
    ep.ep_expert_layer(bf(0, 64), i32(0, 2), None, bf(5, 16, 64), bf(5, 64, 16), bf(0, 64), torch.zeros(0, dtype=torch.uint8), stream=0)


def test_layer_plan(ep):
    p = ep.ep_expert_layer_plan(128, 8, 256, 7168, 2048)
    # the rows between the products, one per entry; the entries by expert: a count, ids, starts and one more, the entries
    assert p.slots == 256 and p.workspace_bytes >= 128 * 8 * 2048 * 2 + (1 + 256 + 256 + 1 + 128 * 8) * 2
    assert ep.ep_expert_layer_plan(3, 2, 256, 64, 16).slots == 6
    for bad in ((129, 8, 8, 64, 16), (-1, 8, 8, 64, 16), (1, 0, 8, 64, 16), (1, 65, 8, 64, 16), (1, 1, 0, 64, 16), (1, 1, 1025, 64, 16),
                (1, 1, 8, 60, 16), (1, 1, 8, 64, 12), (1, 1, 8, 64, 1 << 18), (128, 64, 8, 64, 1 << 17)):
        with pytest.raises(ep.EpError):
            ep.ep_expert_layer_plan(*bad)


# ------------------------------------------------------------------ the reference's gradients against differences


def differences(f, v, h=1e-5):
    """Central differences of a scalar function."""
    g = torch.zeros_like(v)
    for i in range(v.numel()):
        old = float(v.view(-1)[i])
        v.view(-1)[i] = old + h
        up = float(f())
        v.view(-1)[i] = old - h
        g.view(-1)[i] = (up - float(f())) / (2 * h)
        v.view(-1)[i] = old
    return g


@pytest.mark.parametrize("activation,gated", [("none", False), ("silu", False), ("gelu", False), ("silu", True), ("gelu", True)])
def test_reference_product_gradients_are_differences(activation, gated):
    gen = torch.Generator().manual_seed(3)
    x, w, b = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((3, 8), (8, 8), (8,)))
    g = torch.randn(3, 4 if gated else 8, generator=gen, dtype=torch.float64)
    f = lambda: (ref.product(x, w, b, None, activation, gated)[0] * g).sum()  # noqa: E731
    pre = x @ w.t() + b
    got = ref.product_grad(g, w, x, pre if activation != "none" or gated else None, activation, gated)
    for name, v in (("grad_x", x), ("grad_w", w), ("grad_b", b)):
        assert torch.allclose(got[name][0], differences(f, v), rtol=1e-6, atol=1e-8), name


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_reference_route_gradients_are_differences(score, renormalise):
    gen = torch.Generator().manual_seed(5)
    l = torch.randn(4, 10, generator=gen, dtype=torch.float64)
    l[1, 3] = -math.inf
    g = torch.randn(4, 3, generator=gen, dtype=torch.float64)
    idx, w, _ = ref.route(l, 3, None, score, renormalise, scale=2.5)
    got, _ = ref.route_grad(l, idx, g, score, renormalise, 2.5)

    def f():
        again, v, _ = ref.route(l, 3, None, score, renormalise, scale=2.5)
        assert torch.equal(again, idx)
        return (v * g).sum()
    want = differences(f, l)
    there = l > -math.inf
    assert torch.allclose(got[there], want[there], rtol=1e-6, atol=1e-8) and (got[~there] == 0).all()
