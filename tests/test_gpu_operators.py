"""The gate, the experts' products and the layer of few tokens on the GPU against 64-bit definitions
(operators_reference.py, which also says how the bounds are counted)."""
import math

import pytest
import torch

import operators_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
POISON = float("nan")   # what rows outside the windows and fresh outputs hold


@pytest.fixture(scope="module")
def ep():
    import ep_harness
    ep_harness.ensure_built()
    assert torch.cuda.is_available()
    from paper_2603_13606_amd import binding
    return binding


def gen_of(seed):
    g = torch.Generator(DEV)
    g.manual_seed(seed)
    return g


def normal(gen, *shape, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=gen, device=DEV) * std).to(dtype)


def strided(t, pad=8):
    """The same values in rows that are `pad` elements longer (the gaps are NaN)."""
    big = torch.full((*t.shape[:-1], t.shape[-1] + pad), POISON, dtype=t.dtype, device=t.device)
    big[..., :t.shape[-1]] = t
    return big[..., :t.shape[-1]]


def within(got, want, bound, what):
    got, want, bound = got.double().cpu(), want.cpu(), bound.cpu()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {(((got - want).abs() / bound).nan_to_num(1e9)).max():.3g} bounds"


# ---------------------------------------------------------------------- the gate

ROUTES = [
    # T, E, K, dtype, rule
    (1, 8, 1, "f32", dict()),
    (5, 8, 8, "bf16", dict(renormalise=False)),
    (67, 60, 4, "f32", dict(score="sigmoid")),
    (64, 64, 6, "bf16", dict(score="sigmoid", renormalise=False, scale=2.5)),
    (33, 65, 7, "f32", dict(renormalise=False)),
    (31, 128, 2, "f32", dict(bias=True)),
    (40, 256, 8, "bf16", dict(score="sigmoid", bias=True, groups=8, kept=4, scale=2.5)),
    (40, 256, 8, "f32", dict(groups=8, kept=3, renormalise=False)),
    (17, 1000, 7, "f32", dict(masked=0.3, renormalise=False)),
    (9, 1024, 64, "bf16", dict(score="sigmoid")),
    (9, 1024, 64, "f32", dict(bias=True, groups=64, kept=5)),
    (12, 24, 8, "f32", dict(groups=24, kept=5)),               # groups of one
    (12, 24, 16, "f32", dict(groups=3, kept=1)),               # more entries than the kept groups have experts
    (50, 40, 8, "f32", dict(masked=0.95)),                     # fewer routable experts than entries, often none
    (50, 40, 8, "bf16", dict(masked=0.95, bias=True, groups=5, kept=2, score="sigmoid")),
    (2050, 16, 2, "bf16", dict()),
]


def route_case(T, E, dtype, rule, seed=0):
    gen = gen_of(T * E + seed)
    l = torch.randn((T, E), generator=gen, device=DEV) * 2
    if rule.get("masked"):
        l[torch.rand((T, E), generator=gen, device=DEV) < rule["masked"]] = -math.inf
    l = l.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    b = torch.randn(E, generator=gen, device=DEV) * 0.2 if rule.get("bias") else None
    return gen, l, b, {k: v for k, v in rule.items() if k not in ("masked", "bias")}


def call_route(ep, l, K, b, rule):
    T = l.shape[0]
    idx = torch.full((T, K), -7, dtype=torch.int32, device=DEV)
    w = torch.full((T, K), POISON, device=DEV)
    ep.ep_route(l, idx, w, bias=b, score=ep.EP_SCORE_SIGMOID if rule.get("score") == "sigmoid" else ep.EP_SCORE_SOFTMAX,
                renormalise=rule.get("renormalise", True), num_groups=rule.get("groups", 1), groups_kept=rule.get("kept", 1),
                scale=rule.get("scale", 1.0))
    return idx, w


def check_route(ep, l, K, b, rule):
    idx, w = call_route(ep, l, K, b, rule)
    want_idx, want_w, rel = ref.route(l, K, b, **rule)
    assert torch.equal(idx.cpu(), want_idx)
    within(w, want_w, rel * want_w.abs() + ref.TINY, "weights")
    return idx, w


@pytest.mark.parametrize("T,E,K,dtype,rule", ROUTES)
def test_route(ep, T, E, K, dtype, rule):
    _, l, b, rule = route_case(T, E, dtype, rule)
    check_route(ep, l, K, b, rule)
    check_route(ep, strided(l, 3), K, b, rule)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias,groups", [(False, 1), (True, 1), (False, 4)])
def test_route_special_logits(ep, dtype, score, bias, groups):
    """Ties go to the lowest id (both zeros are equal); the lowest finite value is routable, -inf and NaN are not;
    +inf counts as the largest finite number; a token without routable experts gets nothing."""
    E, low = 72, torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min
    l = torch.zeros((9, E), device=DEV)
    l[1] = torch.where(torch.arange(E, device=DEV) % 2 == 0, -0.0, 0.0)
    l[2] = torch.arange(E, device=DEV) % 3
    l[3] = -math.inf
    l[4] = math.nan
    l[5] = low
    l[6, 5], l[6, 70] = math.inf, math.inf
    l[7, ::2], l[7, 1] = math.nan, -math.inf
    l[8] = -math.inf
    l[8, 71] = low
    l = l.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    b = torch.zeros(E, device=DEV) if bias else None
    for renormalise in (True, False):
        idx, w = check_route(ep, l, 5, b, dict(score=score, renormalise=renormalise, groups=groups, kept=2 if groups > 1 else 1))
        assert idx[3].tolist() == idx[4].tolist() == [-1] * 5 and (w[3:5] == 0).all()
        assert idx[8].tolist() == [71, -1, -1, -1, -1] and idx[0].tolist() == [0, 1, 2, 3, 4]
        assert torch.isfinite(w).all()


def test_route_bias_can_take_experts_out(ep):
    l = torch.zeros((3, 8), device=DEV)
    b = torch.tensor([0.0, math.nan, -math.inf, 1.0, 0.0, 0.0, 0.0, 2.0], device=DEV)
    idx, w = call_route(ep, l, 8, b, {})
    assert idx[0].tolist() == [7, 3, 0, 4, 5, 6, -1, -1]
    assert w[0].tolist() == pytest.approx([1 / 6] * 6 + [0, 0], rel=1e-6)


@pytest.mark.parametrize("T,E,K,dtype,rule", ROUTES)
def test_route_backward(ep, T, E, K, dtype, rule):
    gen, l, b, rule = route_case(T, E, dtype, rule, 1)
    idx, _ = call_route(ep, l, K, b, rule)
    if K > 1 and T > 3:
        idx[1, 1] = idx[1, 0]      # the same expert twice
        idx[2, 0] = E              # no expert at all
        idx[3, 0] = -5
    g = torch.randn((T, K), generator=gen, device=DEV)
    rule = {k: v for k, v in rule.items() if k not in ("groups", "kept")}
    want, bound = ref.route_grad(l, idx, g, **rule)
    score = ep.EP_SCORE_SIGMOID if rule.get("score") == "sigmoid" else ep.EP_SCORE_SOFTMAX
    for ll in (l, strided(l, 5)):
        out = torch.full((T, E + 3), POISON, dtype=l.dtype, device=DEV)
        ep.ep_route_backward(ll, idx, g, out[:, :E], score=score, renormalise=rule.get("renormalise", True), scale=rule.get("scale", 1.0))
        within(out[:, :E], want, bound, "grad_logits")
        assert out[:, E:].isnan().all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_one_renormalised_weight_has_no_gradient(ep, score):
    """It is the scale whatever the logits are."""
    l = torch.randn((70, 96), generator=gen_of(3), device=DEV)
    rule = dict(score=getattr(ep, "EP_SCORE_" + score.upper()), scale=2.5)
    idx, w, grad = torch.empty((70, 1), dtype=torch.int32, device=DEV), torch.empty((70, 1), device=DEV), torch.full((70, 96), POISON, device=DEV)
    ep.ep_route(l, idx, w, **rule)
    assert (w == 2.5).all()
    ep.ep_route_backward(l, idx, torch.randn((70, 1), generator=gen_of(4), device=DEV), grad, **rule)
    assert (grad == 0).all()


# ---------------------------------------------------------------------- experts' products

# rows per expert, Kd, output columns
SHAPES = [
    ([1], 8, 8), ([0, 5, 0], 64, 24), ([17, 1, 0, 64], 72, 136), ([128, 127, 129, 3], 200, 128), ([300], 1000, 264),
    ([0, 0], 64, 64), ([5] * 70, 128, 40), ([700, 2, 513], 328, 520),
]
ACTS = [("none", False), ("silu", False), ("gelu", False), ("silu", True), ("gelu", True), ("none", True)]


class Case:
    """Inputs of the products: windows with rows in front, between and behind that belong to nobody (NaN)."""

    def __init__(self, counts, Kd, No, gated, padded, seed=0):
        gen = gen_of(seed + Kd)
        self.counts, self.Kd, self.No, self.N, self.L = counts, Kd, No, (2 if gated else 1) * No, len(counts)
        self.padded = padded
        if padded:
            self.C = max(counts) + 3
            self.first = [e * self.C for e in range(self.L)]
            self.rows = self.L * self.C
        else:
            self.first, at = [], 2
            for n in counts:
                self.first.append(at)
                at += n + 1
            self.rows = at + 4
        self.live = torch.zeros(self.rows, dtype=torch.bool, device=DEV)
        for f, n in zip(self.first, counts):
            self.live[f:f + n] = True
        self.w = normal(gen, self.L, self.N, Kd, std=Kd ** -0.5)
        self.gen = gen
        self.count = torch.tensor(counts, dtype=torch.int32, device=DEV)
        self.offset = None if padded else torch.tensor(self.first, dtype=torch.int32, device=DEV)

    def shape(self, cols):
        return (self.L, self.C, cols) if self.padded else (self.rows, cols)

    def tokens(self, cols):
        t = normal(self.gen, self.rows, cols)
        t[~self.live] = POISON
        return t.view(self.shape(cols))

    def fresh(self, cols):
        return torch.full(self.shape(cols), POISON, dtype=torch.bfloat16, device=DEV)

    def check(self, got, expect, what):
        """expect(e, slice) -> value and bound; rows of nobody are as they were."""
        flat = got.reshape(self.rows, -1)
        assert flat[~self.live].isnan().all(), what + ": rows outside the windows were written"
        for e, (f, n) in enumerate(zip(self.first, self.counts)):
            if n:
                within(flat[f:f + n], *expect(e, slice(f, f + n)), f"{what} of expert {e}")


@pytest.mark.parametrize("counts,Kd,No", SHAPES)
@pytest.mark.parametrize("activation,gated", ACTS)
@pytest.mark.parametrize("padded", [False, True])
def test_expert_product(ep, counts, Kd, No, activation, gated, padded):
    c = Case(counts, Kd, No, gated, padded)
    x, act = c.tokens(Kd), getattr(ep, "EP_ACT_" + activation.upper())
    for variant in range(3):
        bias = normal(c.gen, c.L, c.N, dtype=[torch.float32, torch.bfloat16][variant - 1]) if variant else None
        res = c.tokens(No) if variant == 1 else None
        pre = c.fresh(c.N) if variant == 2 else None
        out = c.fresh(No)
        xx, w = (strided(x), strided(c.w, 16)) if variant == 1 else (x, c.w)
        ep.ep_expert_product(xx, w, out, bias=bias, residual=res, pre=pre, row_offset=c.offset, row_count=c.count, activation=act, gated=gated)
        flat, fres = x.reshape(c.rows, Kd), res.reshape(c.rows, No) if res is not None else None

        def expect(e, s):
            return ref.product(flat[s], c.w[e], bias[e] if bias is not None else None, fres[s] if res is not None else None, activation, gated)
        c.check(out, lambda e, s: expect(e, s)[:2], "out")
        if pre is not None:
            c.check(pre, lambda e, s: expect(e, s)[2:], "pre")
    if not padded:                  # in place on the residual, into a view with longer rows
        res = strided(c.tokens(No))
        want = res.clone()
        ep.ep_expert_product(x, c.w, res, residual=res, row_offset=c.offset, row_count=c.count, activation=act, gated=gated)
        c.check(res, lambda e, s: ref.product(x[s], c.w[e], None, want[s], activation, gated)[:2], "out on the residual")


@pytest.mark.parametrize("counts,Kd,No", SHAPES)
@pytest.mark.parametrize("activation,gated", ACTS)
@pytest.mark.parametrize("padded", [False, True])
def test_expert_product_backward(ep, counts, Kd, No, activation, gated, padded):
    c = Case(counts, Kd, No, gated, padded, seed=1)
    act = getattr(ep, "EP_ACT_" + activation.upper())
    x, g = c.tokens(Kd), c.tokens(No)
    elementwise = activation != "none" or gated
    pre = c.tokens(c.N) if elementwise else None
    flat = lambda t: t.reshape(c.rows, -1)  # noqa: E731
    want = [ref.product_grad(flat(g)[f:f + n], c.w[e], flat(x)[f:f + n], flat(pre)[f:f + n] if elementwise else None, activation, gated)
            for e, (f, n) in enumerate(zip(c.first, c.counts))]
    for wide, accumulate in ((True, False), (True, True), (False, True), (False, False)):
        t = torch.float32 if wide else torch.bfloat16
        start_w, start_b = (normal(c.gen, c.L, c.N, Kd, dtype=t), normal(c.gen, c.L, c.N, dtype=t)) if accumulate else (
            torch.full((c.L, c.N, Kd), POISON, dtype=t, device=DEV), torch.full((c.L, c.N), POISON, dtype=t, device=DEV))
        gw, gb = start_w.clone(), start_b.clone()
        gp, gx = c.fresh(c.N) if elementwise else None, c.fresh(Kd)
        keep = pre.clone() if elementwise else None
        if wide and accumulate and elementwise:
            gp = keep               # on the spot of the pre-activation
        ep.ep_expert_product_backward(strided(g) if wide else g, strided(c.w) if wide else c.w, x=x, pre=keep, grad_pre=gp, grad_x=gx,
                                      grad_weights=gw, grad_bias=gb, row_offset=c.offset, row_count=c.count, activation=act, gated=gated,
                                      accumulate=accumulate)
        if elementwise:
            c.check(gp, lambda e, s: want[e]["grad_pre"], "grad_pre")
        c.check(gx, lambda e, s: want[e]["grad_x"], "grad_x")
        for got, start, name in ((gw, start_w, "grad_w"), (gb, start_b, "grad_b")):
            for e in range(c.L):
                v, b = want[e][name]
                if accumulate:
                    v = v + start[e].double()
                    b = b + ref.U32 * v.abs()
                within(got[e], v, b + (0 if wide else ref.BF16 * (v.abs() + b)), f"{name} of expert {e}")
    # parts of it alone give the same bits
    gx2 = c.fresh(Kd)
    gp2 = c.fresh(c.N) if elementwise else None
    ep.ep_expert_product_backward(g, c.w, pre=pre, grad_pre=gp2, grad_x=gx2, row_offset=c.offset, row_count=c.count, activation=act, gated=gated)
    assert torch.equal(gx2.view(torch.int16), gx.view(torch.int16))
    gw2 = torch.empty((c.L, c.N, Kd), dtype=torch.bfloat16, device=DEV)
    ep.ep_expert_product_backward(g, None, x=x, pre=pre, grad_pre=gp2, grad_weights=gw2, row_offset=c.offset, row_count=c.count,
                                  activation=act, gated=gated)
    assert torch.equal(gw2, gw)


def cycle(counts, n):
    return [counts[i % len(counts)] for i in range(n)]


# Enough tiles for every compute unit: tall windows, short ones, both, last rounds that are part full; 1 to 25 contraction steps.
MANY = [
    (cycle([140, 129, 250, 256, 257, 130, 200], 70), 264, 264), (cycle([1, 128, 0, 17, 64, 65, 100], 140), 72, 136),
    (cycle([1, 128, 0, 17, 64, 65, 100], 140), 72, 120), (cycle([10, 200, 128, 129, 0, 300, 64], 140), 320, 200),
    (cycle([150, 131], 140), 40, 16), (cycle([160, 3], 90), 128, 264), (cycle([130, 20, 280], 40), 1600, 1000),
    (cycle([600, 90, 0], 12), 200, 2056), (cycle([3, 8], 1024), 64, 48),
    (cycle([65, 1, 0, 190], 40), 2056, 264), (cycle([70, 30], 40), 264, 2056),   # two rounds of the smallest tiles, forward and backward
]


@pytest.mark.parametrize("counts,Kd,No", MANY)
@pytest.mark.parametrize("activation,gated,options", [("none", False, "bias residual"), ("silu", True, "bias pre"), ("gelu", False, "residual pre"),
                                                      ("gelu", True, "bias residual pre")])
def test_expert_product_with_many_tiles(ep, counts, Kd, No, activation, gated, options):
    c = Case(counts, Kd, No, gated, padded=activation == "silu", seed=2)
    x = c.tokens(Kd)
    bias = normal(c.gen, c.L, c.N, dtype=torch.bfloat16 if gated else torch.float32) if "bias" in options else None
    res = c.tokens(No) if "residual" in options else None
    pre = c.fresh(c.N) if "pre" in options else None
    out = c.fresh(No)
    ep.ep_expert_product(x, c.w, out, bias=bias, residual=res, pre=pre, row_offset=c.offset, row_count=c.count,
                         activation=getattr(ep, "EP_ACT_" + activation.upper()), gated=gated)
    flat, fres = x.reshape(c.rows, Kd), res.reshape(c.rows, No) if res is not None else None
    want = [ref.product(flat[f:f + n], c.w[e], bias[e] if bias is not None else None, fres[f:f + n] if res is not None else None, activation, gated)
            for e, (f, n) in enumerate(zip(c.first, c.counts))]
    c.check(out, lambda e, s: want[e][:2], "out")
    if pre is not None:
        c.check(pre, lambda e, s: want[e][2:], "pre")


@pytest.mark.parametrize("counts,Kd,No", MANY)
@pytest.mark.parametrize("activation,gated,wide,accumulate", [("none", False, True, True), ("silu", True, False, False), ("gelu", False, True, False),
                                                              ("gelu", True, False, True)])
def test_expert_product_backward_with_many_tiles(ep, counts, Kd, No, activation, gated, wide, accumulate):
    c = Case(counts, Kd, No, gated, padded=activation == "silu", seed=3)
    x, g = c.tokens(Kd), c.tokens(No)
    pre = c.tokens(c.N) if activation != "none" or gated else None
    gp, gx = c.fresh(c.N) if pre is not None else None, c.fresh(Kd)
    t = torch.float32 if wide else torch.bfloat16
    start_w, start_b = normal(c.gen, c.L, c.N, Kd, dtype=t), normal(c.gen, c.L, c.N, dtype=t)
    gw, gb = start_w.clone(), start_b.clone()
    ep.ep_expert_product_backward(g, c.w, x=x, pre=pre, grad_pre=gp, grad_x=gx, grad_weights=gw, grad_bias=gb, row_offset=c.offset,
                                  row_count=c.count, activation=getattr(ep, "EP_ACT_" + activation.upper()), gated=gated, accumulate=accumulate)
    flat = lambda t: t.reshape(c.rows, -1)  # noqa: E731
    want = [ref.product_grad(flat(g)[f:f + n], c.w[e], flat(x)[f:f + n], flat(pre)[f:f + n] if pre is not None else None, activation, gated)
            for e, (f, n) in enumerate(zip(c.first, c.counts))]
    if pre is not None:
        c.check(gp, lambda e, s: want[e]["grad_pre"], "grad_pre")
    c.check(gx, lambda e, s: want[e]["grad_x"], "grad_x")
    for got, start, name in ((gw, start_w, "grad_w"), (gb, start_b, "grad_b")):
        for e in range(c.L):
            v, b = want[e][name]
            if accumulate:
                v = v + start[e].double()
                b = b + ref.U32 * v.abs()
            within(got[e], v, b + (0 if wide else ref.BF16 * (v.abs() + b)), f"{name} of expert {e}")


def test_expert_product_windows_beyond_the_tensors_are_cut(ep):
    """Offsets and counts that do not fit: negative, beyond the end, across it."""
    gen = gen_of(9)
    x, w = normal(gen, 40, 64), normal(gen, 6, 24, 64, std=0.1)
    offset = torch.tensor([0, 30, 40, -3, 1 << 30, 5], dtype=torch.int32, device=DEV)
    count = torch.tensor([5, 100, 7, 4, 1 << 30, -2], dtype=torch.int32, device=DEV)
    big = torch.full((64, 24), POISON, dtype=torch.bfloat16, device=DEV)
    ep.ep_expert_product(x, w, big[8:48], row_offset=offset, row_count=count)
    assert big[:8].isnan().all() and big[48:].isnan().all() and big[13:38].isnan().all()
    for e, s in ((0, slice(0, 5)), (1, slice(30, 40))):
        within(big[8:48][s], *ref.product(x[s], w[e])[:2], f"expert {e}")
    gw = torch.full((6, 24, 64), POISON, device=DEV)
    ep.ep_expert_product_backward(big[8:48], x=x, grad_weights=gw, row_offset=offset, row_count=count)
    assert (gw[2:] == 0).all() and torch.isfinite(gw).all()


def test_expert_product_interleaved_windows(ep):
    """Padded windows that lie between each other: [C, L, .] seen as [L, C, .]."""
    gen = gen_of(17)
    counts, C, Kd, No = [5, 0, 9, 70], 70, 136, 72
    L, cnt = len(counts), torch.tensor([5, 0, 9, 70], dtype=torch.int32, device=DEV)
    x, w = normal(gen, C, L, Kd).transpose(0, 1), normal(gen, L, No, Kd, std=0.1)
    out = torch.full((C, L, No), POISON, dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    ep.ep_expert_product(x, w, out, row_count=cnt)
    gx = torch.full((C, L, Kd), POISON, dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    gw = torch.empty((No, L, Kd), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    g = normal(gen, L, C, No)
    ep.ep_expert_product_backward(g, w, x=x, grad_x=gx, grad_weights=gw, row_count=cnt)
    for e, n in enumerate(counts):
        assert out[e, n:].isnan().all() and gx[e, n:].isnan().all()
        want = ref.product_grad(g[e, :n], w[e], x[e, :n])
        within(gw[e], want["grad_w"][0], want["grad_w"][1] + ref.BF16 * (want["grad_w"][0].abs() + want["grad_w"][1]), "grad_w")
        if n:
            within(out[e, :n], *ref.product(x[e, :n], w[e])[:2], "out")
            within(gx[e, :n], *want["grad_x"], "grad_x")


def test_no_rows_at_all(ep):
    """Windows without rows: nothing is written but the zeros of the weights' gradients."""
    w, cnt = torch.randn((3, 24, 64), device=DEV).bfloat16(), torch.zeros(3, dtype=torch.int32, device=DEV)
    out = torch.full((3, 5, 24), POISON, dtype=torch.bfloat16, device=DEV)
    x, gw, gb = torch.full((3, 5, 64), POISON, dtype=torch.bfloat16, device=DEV), torch.full((3, 24, 64), POISON, device=DEV), torch.full((3, 24), POISON, device=DEV)
    ep.ep_expert_product(x, w, out, row_count=cnt)
    gx = x.clone()
    ep.ep_expert_product_backward(out, w, x=x, grad_x=gx, grad_weights=gw, grad_bias=gb, row_count=cnt)
    assert out.isnan().all() and gx.isnan().all() and (gw == 0).all() and (gb == 0).all()
    gw.fill_(POISON)
    ep.ep_expert_product_backward(out[:, :0], x=x[:, :0], grad_weights=gw, row_count=cnt)
    assert (gw == 0).all()


def test_expert_product_special_values(ep):
    """A row's NaN or infinity stays in its row; an expert's in its expert."""
    gen = gen_of(11)
    counts, off = torch.tensor([20, 20], dtype=torch.int32, device=DEV), torch.tensor([0, 20], dtype=torch.int32, device=DEV)
    x, w = normal(gen, 40, 136), normal(gen, 2, 40, 136, std=0.1)
    x[3, 7], x[25, 0] = math.nan, math.inf
    out = torch.empty((40, 40), dtype=torch.bfloat16, device=DEV)
    ep.ep_expert_product(x, w, out, row_offset=off, row_count=counts, activation=ep.EP_ACT_GELU)
    ok = torch.ones(40, dtype=torch.bool, device=DEV)
    ok[3] = ok[25] = False
    assert out[3].isnan().all() and not torch.isfinite(out[25]).all() and torch.isfinite(out[ok]).all()
    w[1, 3] = math.nan
    x = normal(gen, 40, 136)
    ep.ep_expert_product(x, w, out, row_offset=off, row_count=counts)
    assert torch.isfinite(out[:20]).all() and out[20:, 3].isnan().all() and torch.isfinite(out[20:, :3]).all()


def test_expert_product_far_rows(ep):
    """Row and expert offsets beyond 2^31 elements: an expert's weights and rows at the far end of large storage."""
    gen = gen_of(13)
    stride = 1 << 21
    store = torch.zeros(1200 * stride, dtype=torch.bfloat16, device=DEV)     # 5 GB
    rows = store.as_strided((1200, 64), (stride, 1))
    rows[1150:1190] = normal(gen, 40, 64)
    w = store.as_strided((2, 24, 64), (1100 * stride, 64, 1), 4096)
    w[1] = normal(gen, 24, 64, std=0.1)
    out = torch.full((1200, 24), POISON, dtype=torch.bfloat16, device=DEV)
    off, cnt = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([0, 1150], [0, 40]))
    ep.ep_expert_product(rows, w, out, row_offset=off, row_count=cnt)
    within(out[1150:1190], *ref.product(rows[1150:1190], w[1])[:2], "far rows")
    assert out[:1150].isnan().all() and out[1190:].isnan().all()
    g = normal(gen, 1200, 24)
    gx, gw = store.as_strided((1200, 64), (stride, 1), 128), torch.empty((2, 24, 64), device=DEV)
    ep.ep_expert_product_backward(g, w, x=rows, grad_x=gx, grad_weights=gw, row_offset=off, row_count=cnt)
    want = ref.product_grad(g[1150:1190], w[1], rows[1150:1190])
    within(gx[1150:1190], *want["grad_x"], "grad_x")
    within(gw[1], *want["grad_w"], "grad_w")
    assert (gw[0] == 0).all()


# ---------------------------------------------------------------------- the layer of few tokens

LAYERS = [
    # T, K, L, H, inner, activation, gated, options
    (1, 1, 1, 8, 8, "none", False, {}),
    (1, 8, 16, 200, 72, "silu", True, {}),
    (2, 2, 8, 64, 16, "gelu", False, dict(bias=torch.float32, residual=True)),
    (13, 6, 10, 264, 136, "gelu", True, dict(bias=torch.bfloat16, residual=True, masked=0.5)),
    (16, 4, 4, 128, 64, "silu", True, dict(first=3)),
    (17, 2, 2, 72, 200, "silu", False, dict(weights=False)),
    (40, 3, 1, 96, 40, "silu", True, dict(first=2, masked=0.2)),      # one expert names more than two groups of 16
    (128, 8, 64, 136, 72, "silu", True, dict(bias=torch.float32)),
    (128, 2, 2, 64, 24, "gelu", False, dict(residual=True)),          # more than 64 tokens per expert
    (100, 5, 1024, 32, 16, "silu", True, {}),
    (5, 64, 70, 40, 24, "silu", True, {}),
    (7, 3, 5, 64, 32, "silu", True, dict(masked=1.0, residual=True)),  # nobody is routed here
    (7, 3, 5, 64, 32, "silu", True, dict(masked=1.0)),
    # enough runs of rows for every wavefront; more output columns than compute units can take by eights; whole lines or not
    (64, 8, 64, 128, 1040, "silu", True, dict(bias=torch.bfloat16)),
    (128, 8, 64, 72, 1088, "gelu", False, dict(residual=True)),
    (128, 4, 8, 128, 8256, "silu", True, {}),
    (9, 2, 4, 2368, 64, "silu", True, dict(residual=True)),
    (9, 2, 4, 2312, 72, "gelu", False, dict(bias=torch.float32)),
    (70, 1, 1, 2304, 128, "silu", True, {}),
    (128, 2, 1, 2120, 200, "silu", False, dict(first=1)),
    (128, 64, 1024, 48, 16, "silu", True, dict(masked=0.1)),          # as many entries as there can be
    (50, 2, 4, 4168, 136, "silu", True, {}),
]


def layer_case(T, K, L, H, inner, gated, opt, seed=0):
    gen = gen_of(T + 7 * H + seed)
    N, first = (2 if gated else 1) * inner, opt.get("first", 0)
    c = dict(x=normal(gen, T, H), w_up=normal(gen, L, N, H, std=H ** -0.5), w_down=normal(gen, L, H, inner, std=inner ** -0.5))
    ids = torch.randint(0, L + 2 * first, (T, K), generator=gen, device=DEV, dtype=torch.int32)   # duplicates within a token are legal
    ids[torch.rand((T, K), generator=gen, device=DEV) < opt.get("masked", 0.0)] = -1
    c["idx"] = ids
    c["wts"] = torch.randn((T, K), generator=gen, device=DEV) if opt.get("weights", True) else None
    b = opt.get("bias")
    c["b_up"], c["b_down"] = (normal(gen, L, N, dtype=b), normal(gen, L, H, dtype=b)) if b else (None, None)
    c["res"] = normal(gen, T, H) if opt.get("residual") else None
    return c


def call_layer(ep, c, out, activation, gated, first=0, garbage=0xff):
    T, H = c["x"].shape
    n = ep.ep_expert_layer_plan(T, c["idx"].shape[1], c["w_up"].shape[0], H, c["w_down"].shape[2]).workspace_bytes
    store = torch.full((n + 256,), garbage, dtype=torch.uint8, device=DEV)
    ep.ep_expert_layer(c["x"], c["idx"], c["wts"], c["w_up"], c["w_down"], out, store[:n], bias_up=c["b_up"], bias_down=c["b_down"],
                       residual=c["res"], activation=getattr(ep, "EP_ACT_" + activation.upper()), gated=gated, first_expert=first)
    assert (store[n:] == garbage).all(), "written behind the workspace"
    return out


@pytest.mark.parametrize("T,K,L,H,inner,activation,gated,opt", LAYERS)
def test_expert_layer(ep, T, K, L, H, inner, activation, gated, opt):
    c = layer_case(T, K, L, H, inner, gated, opt)
    first = opt.get("first", 0)
    want, bound = ref.layer(c["x"], c["idx"], c["wts"], c["w_up"], c["w_down"], c["b_up"], c["b_down"], c["res"], activation, gated, first)
    out = torch.full((T, H + 8), POISON, dtype=torch.bfloat16, device=DEV)
    call_layer(ep, c, out[:, :H], activation, gated, first)
    within(out[:, :H], want, bound, "out")
    assert out[:, H:].isnan().all()
    again = torch.empty((T, H), dtype=torch.bfloat16, device=DEV)
    call_layer(ep, dict(c, x=strided(c["x"]), w_up=strided(c["w_up"]), w_down=strided(c["w_down"], 24)), again, activation, gated, first, garbage=0)
    assert torch.equal(again, out[:, :H]), "strides, or what the workspace held, changed the result"
    if c["res"] is not None:
        call_layer(ep, c, c["res"], activation, gated, first)
        assert torch.equal(c["res"], again)
    else:
        call_layer(ep, c, c["x"], activation, gated, first)
        assert torch.equal(c["x"], again)


def test_expert_layer_keeps_experts_apart(ep):
    """NaN and infinities in the weights of experts reach the tokens that name them and no others."""
    c = layer_case(40, 2, 12, 72, 40, True, {}, seed=3)
    c["idx"] = torch.randint(0, 12, (40, 2), generator=gen_of(1), device=DEV, dtype=torch.int32)
    clean = call_layer(ep, c, torch.empty((40, 72), dtype=torch.bfloat16, device=DEV), "silu", True)
    c["w_up"][3], c["w_down"][7], c["w_down"][8, 5] = math.nan, math.inf, math.nan
    c["x"][0, 0] = math.nan
    out = call_layer(ep, c, torch.empty((40, 72), dtype=torch.bfloat16, device=DEV), "silu", True)
    touched = ((c["idx"] == 3) | (c["idx"] == 7) | (c["idx"] == 8)).any(dim=1)
    touched[0] = True
    assert torch.equal(out[~touched], clean[~touched]) and torch.isfinite(out[~touched]).all() and (~touched).sum() > 10
    assert out[(c["idx"] == 3).any(dim=1)].isnan().all()


# ---------------------------------------------------------------------- together, streams, graphs


def test_results_do_not_depend_on_timing(ep):
    c = layer_case(64, 6, 24, 1000, 264, True, dict(bias=torch.float32), seed=5)
    a = call_layer(ep, c, torch.empty((64, 1000), dtype=torch.bfloat16, device=DEV), "silu", True)
    p = Case([700, 2, 513, 0, 90], 328, 520, False, False)
    x, g = p.tokens(328), p.tokens(520)
    outs = []
    for _ in range(3):
        out, gx, gw, gb = p.fresh(520), p.fresh(328), torch.empty_like(p.w, dtype=torch.float32), torch.empty((5, 520), device=DEV)
        ep.ep_expert_product(x, p.w, out, row_offset=p.offset, row_count=p.count)
        ep.ep_expert_product_backward(g, p.w, x=x, grad_x=gx, grad_weights=gw, grad_bias=gb, row_offset=p.offset, row_count=p.count)
        b = call_layer(ep, c, torch.empty((64, 1000), dtype=torch.bfloat16, device=DEV), "silu", True)
        assert torch.equal(a, b)
        outs.append([t.view(torch.int16).clone() for t in (out, gx)] + [gw, gb])
    for other in outs[1:]:
        assert all(torch.equal(s, t) for s, t in zip(outs[0], other))


def moe_inputs(T, E, H, inner, gated, seed):
    gen = gen_of(seed)
    N = (2 if gated else 1) * inner
    return dict(logits=torch.randn((T, E), generator=gen, device=DEV), x=normal(gen, T, H), w1=normal(gen, E, N, H, std=H ** -0.5),
                b1=normal(gen, E, N, std=0.3, dtype=torch.float32), w2=normal(gen, E, H, inner, std=inner ** -0.5), g=normal(gen, T, H))


def moe_reference(v, K, gated, score="softmax"):
    """The layer in float64 autograd, dense over the experts."""
    leaf = {k: v[k].double().cpu().requires_grad_(True) for k in ("logits", "x", "w1", "b1", "w2")}
    idx, _, _ = ref.route(v["logits"], K, None, score)
    s = torch.softmax(leaf["logits"], 1) if score == "softmax" else torch.sigmoid(leaf["logits"])
    w = s.gather(1, idx.long())
    w = w / w.sum(1, keepdim=True)
    out = torch.zeros_like(leaf["x"])
    for e in range(v["w1"].shape[0]):
        t, k = torch.nonzero(idx == e, as_tuple=True)
        pre = leaf["x"][t] @ leaf["w1"][e].t() + leaf["b1"][e]
        n = pre.shape[1] // 2
        h = torch.nn.functional.silu(pre[:, :n]) * pre[:, n:] if gated else torch.nn.functional.silu(pre)
        out = out.index_add(0, t, w[t, k][:, None] * (h @ leaf["w2"][e].t()))
    (out * v["g"].double().cpu()).sum().backward()
    return idx, out.detach(), {k: t.grad for k, t in leaf.items()}


@pytest.mark.parametrize("mode,T,E,H,inner,K,gated", [("ht", 100, 16, 128, 72, 4, True), ("ll", 60, 8, 72, 40, 2, False), ("ht", 1, 8, 64, 24, 2, True)])
def test_a_whole_layer_forward_and_backward(ep, mode, T, E, H, inner, K, gated):
    """Gate, dispatch, two products, combine through the buffer and its autograd functions, against float64.
    Rounding to bf16 happens once per stage (h, y, out; their gradients), each of half a step, 2^-8: in the 2-norm
    a result behind at most 8 of them is off by no more than 8 * 2^-8 of its size."""
    from paper_2603_13606_amd import buffer as B
    v = moe_inputs(T, E, H, inner, gated, T)
    want_idx, want, grads = moe_reference(v, K, gated)
    buf = B.EPBuffer(2, E, H, K, max_tokens_per_rank=T, mode=mode)
    try:
        leaf = {k: v[k].clone().requires_grad_(True) for k in ("logits", "x", "w1", "b1", "w2")}
        idx, w = B.EPRouteFn.apply(leaf["logits"], K)
        assert torch.equal(idx.cpu(), want_idx)
        _, _, _, h, _ = buf.dispatch(leaf["x"].detach(), idx, w.detach())
        rows = B.EPDispatchFn.apply(leaf["x"], buf, h)
        mid = B.EPExpertProductFn.apply(rows, leaf["w1"], leaf["b1"], None, buf, h, "silu", gated)
        y = B.EPExpertProductFn.apply(mid, leaf["w2"], None, None, buf, h)
        out = B.EPCombineFn.apply(y, w, buf, h)
        few = buf.expert_layer(v["x"], idx, w.detach(), v["w1"], v["w2"], bias_up=v["b1"], activation="silu", gated=gated)

        def near(a, b, what):
            a, b = a.detach().double().cpu(), b.double()
            assert float((a - b).norm()) <= 8 * ref.BF16 * float(b.norm()), what
        near(out, want, "out")
        near(few, want, "the layer of few tokens")
        (out.float() * v["g"].float()).sum().backward()
        for k in leaf:
            assert torch.isfinite(leaf[k].grad).all(), k
            near(leaf[k].grad, grads[k], "gradient of " + k)
        buf.destroy_handle(h)
    finally:
        buf.close()


def test_products_of_some_experts_with_a_handle(ep):
    """A program that owns experts [first, first + L) passes their weights only: the other windows are untouched;
    rows beyond the output are skipped and flagged."""
    E, K, T, H = 12, 3, 50, 64
    gen = gen_of(31)
    idx, w = torch.empty((T, K), dtype=torch.int32, device=DEV), torch.empty((T, K), device=DEV)
    ep.ep_route(torch.randn((T, E), generator=gen, device=DEV), idx, w)
    x, weights = normal(gen, T, H), normal(gen, 5, 40, H, std=0.1)
    for mode in (ep.EP_MODE_HT, ep.EP_MODE_LL):
        g = ep.ep_group_create(ep.make_config(4, E, H, K, T, mode=mode))
        h = ep.ep_layout(g, idx)
        ll = mode == ep.EP_MODE_LL
        recv = torch.full((E, T, H) if ll else (T * K, H), POISON, dtype=torch.bfloat16, device=DEV)
        ep.ep_dispatch(h, x, recv)
        out = torch.full((*recv.shape[:-1], 40), POISON, dtype=torch.bfloat16, device=DEV)
        ep.ep_expert_product(recv, weights, out, handle=h, first_expert=4)
        info = ep.ep_handle_query(h)
        off, kept = ep.read_device_i32(info.expert_offset, E + 1).tolist(), ep.read_device_i32(info.expert_kept, E).tolist()
        fr, fo = recv.reshape(-1, H), out.reshape(-1, 40)
        live = torch.zeros(fo.shape[0], dtype=torch.bool, device=DEV)
        for e in range(4, 9):
            s = slice(off[e], off[e] + kept[e])
            live[s] = True
            within(fo[s], *ref.product(fr[s], weights[e - 4])[:2], f"expert {e}")
        assert fo[~live].isnan().all() and live.any()
        for bad in (dict(first_expert=8), dict(first_expert=4, row_count=idx[0])):
            with pytest.raises(ep.EpError) as err:
                ep.ep_expert_product(recv, weights, out, handle=h, **bad)
            assert err.value.code == ep.EP_ERR_INVALID_ARG
        if not ll:
            short = out[:off[9] - 1]
            ep.ep_expert_product(recv, weights, short, handle=h, first_expert=4)
            assert ep.ep_handle_query(h, ok=(ep.EP_ERR_OVERFLOW,)).status & ep.STATUS_OUTPUT_OVERFLOW
        ep.ep_handle_destroy(h)
        ep.ep_group_destroy(g)


def test_calls_in_a_graph(ep):
    """Gate, layer, products and their backward pass captured once and replayed on changing inputs, with eager work
    between the replays; two graphs with a workspace each."""
    T, E, K, H, inner = 24, 16, 4, 136, 72
    v = moe_inputs(T, E, H, inner, True, 77)
    off = torch.arange(0, 4 * E, 4, dtype=torch.int32, device=DEV)
    cnt = torch.full((E,), 4, dtype=torch.int32, device=DEV)
    n = ep.ep_expert_layer_plan(T, K, E, H, inner).workspace_bytes

    def buffers():
        e = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device=DEV)  # noqa: E731
        return dict(idx=e(T, K, dtype=torch.int32), w=e(T, K, dtype=torch.float32), out=e(T, H), ws=e(n, dtype=torch.uint8), mid=e(4 * E, inner),
                    pre=e(4 * E, 2 * inner), gp=e(4 * E, 2 * inner), gx=e(4 * E, H), gw=e(E, 2 * inner, H), gl=e(T, E, dtype=torch.float32))

    x, logits, rows, gmid = v["x"].clone(), v["logits"].clone(), normal(gen_of(5), 4 * E, H), normal(gen_of(6), 4 * E, inner)

    def step(b):
        ep.ep_route(logits, b["idx"], b["w"])
        ep.ep_expert_layer(x, b["idx"], b["w"], v["w1"], v["w2"], b["out"], b["ws"], bias_up=v["b1"], activation=ep.EP_ACT_SILU, gated=True)
        ep.ep_expert_product(rows, v["w1"], b["mid"], bias=v["b1"], pre=b["pre"], row_offset=off, row_count=cnt, activation=ep.EP_ACT_SILU, gated=True)
        ep.ep_expert_product_backward(gmid, v["w1"], x=rows, pre=b["pre"], grad_pre=b["gp"], grad_x=b["gx"], grad_weights=b["gw"],
                                      row_offset=off, row_count=cnt, activation=ep.EP_ACT_SILU, gated=True)
        ep.ep_route_backward(logits, b["idx"], b["w"], b["gl"])

    graphs = []
    side = torch.cuda.Stream()
    for _ in range(2):
        b = buffers()
        with torch.cuda.stream(side):
            step(b)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(b)
        graphs.append((graph, b))
    eager = buffers()
    for i in range(4):
        x.copy_(normal(gen_of(100 + i), T, H))
        logits.copy_(torch.randn((T, E), generator=gen_of(200 + i), device=DEV))
        rows.copy_(normal(gen_of(300 + i), 4 * E, H))
        cnt.copy_(torch.randint(0, 5, (E,), generator=gen_of(400 + i), device=DEV, dtype=torch.int32))
        for t in (eager, graphs[0][1], graphs[1][1]):
            for k in t:
                t[k].zero_()
        step(eager)
        torch.cuda.synchronize()
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, b in graphs:
            for k in b:
                if k != "ws":
                    assert torch.equal(b[k], eager[k]), (i, k)


def test_calls_on_another_stream(ep):
    c = layer_case(20, 4, 10, 520, 264, True, {}, seed=9)
    want = call_layer(ep, c, torch.empty((20, 520), dtype=torch.bfloat16, device=DEV), "silu", True)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    n = ep.ep_expert_layer_plan(20, 4, 10, 520, 264).workspace_bytes
    outs = [torch.empty((20, 520), dtype=torch.bfloat16, device=DEV) for _ in range(8)]
    ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):          # two at once, a workspace each
        ep.ep_expert_layer(c["x"], c["idx"], c["wts"], c["w_up"], c["w_down"], out, ws[i % 2], activation=ep.EP_ACT_SILU, gated=True,
                           stream=(s1, s2)[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    with pytest.raises(ValueError):
        ep._one_device([c["x"], type("T", (), {"is_cuda": True, "device": torch.device("cuda", 1)})()])
