"""The gate and the experts' operators at the limits of their ranges, on the GPU against 64-bit definitions."""
import math

import pytest
import torch

import operators_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def ep():
    import ep_harness
    ep_harness.ensure_built()
    assert torch.cuda.is_available()
    from paper_2603_13606_amd import binding
    return binding


def within(got, want, bound, what):
    got, want, bound = got.double().cpu(), want.cpu(), bound.cpu()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, first at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]}"


# ---------------------------------------------------------------------- gate: renormalised sigmoid scores near 0


def faint_logits(E=24):
    """Tokens whose selected scores are near the smallest float32 or below it; every entry names another expert."""
    rows = [[-80.0, -80.0, -80.0, -80.0], [-88.5, -88.5, -88.25, -88.0], [-87.0, -88.7, -88.8, -95.0], [-6.0, -7.5, -6.5, -30.0],
            [-9.0, -9.5, -60.0, -92.0], [-100.0, -100.0, -101.5, -100.25], [-300.0, -299.0, -300.0, -320.0], [-700.0, -701.0, -700.5, -707.0],
            [3.0, -2.0, -90.0, 40.0], [-20.0, -20.0, -20.5, -21.0]]
    l = torch.full((len(rows), E), -math.inf, device=DEV)
    for t, r in enumerate(rows):
        for k, v in enumerate(r):
            l[t, (5 * k + 3 * t) % E] = v
    return l


def quotients(l, idx):
    """Weights of the selected and 1 - score, in 64 bits."""
    lk = torch.gather(l.double().cpu(), 1, idx.cpu().long())
    return torch.softmax(torch.nn.functional.logsigmoid(lk), dim=1), torch.sigmoid(-lk)


# Roundings: differences of logits of up to 100 (a step each of the exponent's argument), exponential, 1 + e, divisions, a sum of 4.
STEPS = (100 + 24) * ref.U32
# A score below the smallest normal float32 may be lost beside one of 2^-16 or more.
LOST = 2.0 ** -110


def gradient_of(p, rest, g, idx, shape):
    """Gradient of the logits from p = w / scale and g = scale * gradient of w, and the sum of what it is made of."""
    out, mag = (torch.zeros(shape, dtype=torch.float64) for _ in range(2))
    at = idx.cpu().long()
    out.scatter_add_(1, at, p * rest * (g - (g * p).sum(1, keepdim=True)))
    mag.scatter_add_(1, at, p * rest * (g.abs() + (g * p).abs().sum(1, keepdim=True)))
    return out, mag


def check_gradient(ep, l, idx, size):
    g = size * torch.tensor([1.0, -1.0, 2.0, -0.5], device=DEV).repeat(l.shape[0], 1)
    grad = torch.full_like(l, math.nan)
    ep.ep_route_backward(l, idx, g, grad, score=ep.EP_SCORE_SIGMOID, scale=2.5)
    p, rest = quotients(l, idx)
    want, mag = gradient_of(p, rest, 2.5 * g.double().cpu(), idx, l.shape)
    within(grad, want, 2 * STEPS * mag + size * 16 * LOST, "grad_logits")


@pytest.mark.parametrize("size", [1.0, 65536.0])
def test_gradients_of_faint_scores_are_finite(ep, size):
    """(g - mean) * score / sum, not (g - mean) / sum * score: with a loss scale in g the first quotient alone overflows."""
    l = faint_logits()
    l = l[(l.masked_fill(l == -math.inf, 0.0) >= -88.6).all(dim=1)].contiguous()
    assert l.shape[0] == 4
    check_gradient(ep, l, torch.stack([torch.nonzero(r > -math.inf).flatten() for r in l]).to(torch.int32), size)


@pytest.mark.parametrize("bias,dtype", [(False, torch.float32), (True, torch.float32), (False, torch.bfloat16)])
def test_faint_scores_keep_their_weights(ep, bias, dtype):
    """Renormalised weights add up to the scale however small the scores are, and have gradients."""
    l = faint_logits().to(dtype)
    b = torch.zeros(l.shape[1], device=DEV) if bias else None
    idx = torch.empty((l.shape[0], 4), dtype=torch.int32, device=DEV)
    w = torch.empty((l.shape[0], 4), device=DEV)
    ep.ep_route(l, idx, w, bias=b, score=ep.EP_SCORE_SIGMOID, scale=2.5)
    assert all(sorted(i) == torch.nonzero(r > -math.inf).flatten().tolist() for i, r in zip(idx.tolist(), l))
    if dtype == torch.float32:
        p, _ = quotients(l, idx)
        within(w, 2.5 * p, 2.5 * (STEPS * p + LOST), "weights")
        for size in (1.0, 65536.0):
            check_gradient(ep, l, idx, size)
    assert torch.allclose(w.sum(1), torch.full_like(w[:, 0], 2.5), rtol=4 * ref.U32, atol=0)


def test_scores_below_64_bits_are_zero(ep):
    l = torch.tensor([[-708.3, -709.0, -800.0], [-709.0, -710.0, -3e38]], device=DEV)
    idx, w = torch.empty((2, 2), dtype=torch.int32, device=DEV), torch.empty((2, 2), device=DEV)
    ep.ep_route(l, idx, w, score=ep.EP_SCORE_SIGMOID)
    assert idx.tolist() == [[0, 1], [0, 1]] and w.tolist() == [[1.0, 0.0], [0.0, 0.0]]
    grad = torch.full_like(l, math.nan)
    ep.ep_route_backward(l, idx, torch.tensor([[1.0, 2.0], [3.0, 4.0]], device=DEV), grad, score=ep.EP_SCORE_SIGMOID)
    assert (grad == 0).all()


# ---------------------------------------------------------------------- gate: more tokens than wavefronts of a launch


def many_tokens(dtype, E=16, T=70001):
    gen = torch.Generator(DEV)
    gen.manual_seed(11)
    l = torch.randn((T, E), generator=gen, device=DEV) * 2
    l[torch.rand((T, E), generator=gen, device=DEV) < 0.2] = -math.inf
    return gen, l.to(dtype)


@pytest.mark.parametrize("groups,kept", [(1, 1), (4, 2)])
def test_route_many_tokens(ep, groups, kept):
    """Wavefronts take several tokens each: everything of the first one, group keys included, gives way to the next."""
    _, l = many_tokens(torch.float32)
    (T, E), K = l.shape, 3
    idx, w = torch.full((T, K), -7, dtype=torch.int32, device=DEV), torch.full((T, K), math.nan, device=DEV)
    ep.ep_route(l, idx, w, renormalise=False, num_groups=groups, groups_kept=kept, scale=1.5)
    s, _, there = ref.route_scores(l.double().cpu(), "softmax")
    key = torch.where(there, s, -math.inf)
    if groups > 1:
        two = key.view(T, groups, -1).topk(2, dim=2).values
        worth = two[:, :, 0] + two[:, :, 1].clamp(min=0.0)
        best = worth.sort(dim=1, descending=True, stable=True).indices[:, :kept]
        key = key.masked_fill(~torch.zeros(T, groups, dtype=torch.bool).scatter(1, best, True).repeat_interleave(E // groups, 1), -math.inf)
    top, order = key.sort(dim=1, descending=True, stable=True)
    some = top[:, :K] > -math.inf
    assert torch.equal(idx.cpu(), torch.where(some, order[:, :K], -1).to(torch.int32))
    want = torch.where(some, 1.5 * s.gather(1, order[:, :K]), 0.0)
    within(w, want, (20 + E + 16) * ref.U32 * want + ref.TINY, "weights")


@pytest.mark.parametrize("dtype,score,renormalise", [(torch.float32, "softmax", False), (torch.bfloat16, "sigmoid", True)])
def test_route_backward_many_tokens(ep, dtype, score, renormalise):
    gen, l = many_tokens(dtype)
    (T, E), K = l.shape, 3
    idx = torch.randint(-1, E, (T, K), generator=gen, device=DEV, dtype=torch.int32)
    g = torch.randn((T, K), generator=gen, device=DEV)
    grad = torch.full_like(l, math.nan)
    ep.ep_route_backward(l, idx, g, grad, score=getattr(ep, "EP_SCORE_" + score.upper()), renormalise=renormalise)
    within(grad, *ref.route_grad(l, idx, g, score, renormalise), "grad_logits")


def test_a_bias_takes_experts_out_of_the_choice_only(ep):
    """The scores are those of the logits: plain softmax weights count the experts that the bias keeps from being chosen, as the
    backward pass does, which knows no bias."""
    l = torch.tensor([[0.5, 2.0, 1.0, -1.0, 0.0, -math.inf, 0.25, 1.5]], device=DEV)
    b = torch.tensor([0.0, math.nan, -math.inf, 1.0, 0.0, 0.0, 0.0, 2.0], device=DEV)
    idx, w = torch.empty((1, 8), dtype=torch.int32, device=DEV), torch.empty((1, 8), device=DEV)
    ep.ep_route(l, idx, w, bias=b, renormalise=False)
    assert idx.tolist() == [[7, 3, 0, 6, 4, -1, -1, -1]]
    leaf = l.double().cpu().requires_grad_(True)
    s = torch.softmax(leaf, dim=1)
    want = torch.cat([s[:, [7, 3, 0, 6, 4]], torch.zeros(1, 3)], dim=1)
    within(w, want.detach(), 40 * ref.U32 * want.detach(), "weights")
    g = torch.tensor([[1.0, -2.0, 0.5, 3.0, -1.0, 7.0, 7.0, 7.0]], device=DEV)
    (want * g.double().cpu()).sum().backward()
    grad = torch.full_like(l, math.nan)
    ep.ep_route_backward(l, idx, g, grad, renormalise=False)
    assert grad[0, 5] == 0
    there = [0, 1, 2, 3, 4, 6, 7]
    within(grad[:, there], leaf.grad[:, there], torch.full((1, 7), 8 * 60 * ref.U32, dtype=torch.float64), "grad_logits")


# ---------------------------------------------------------------------- the buffer's products and the life of a handle


def test_a_handle_outlives_a_product_that_is_held_back(ep):
    """Weight gradients queued behind other work on a side stream; meanwhile the handle is combined with, destroyed, and its place
    taken by the next routing, all on the communication stream: the product still sees its own windows."""
    from paper_2603_13606_amd import buffer as B
    T, E, H, K, N = 64, 8, 128, 2, 40
    gen = torch.Generator(DEV)
    gen.manual_seed(3)
    normal = lambda *s: torch.randn(s, generator=gen, device=DEV).bfloat16()  # noqa: E731
    x, y, g = normal(T, H), normal(T * K, H), normal(T * K, N)
    one = torch.stack([torch.arange(T) % 3, 3 + torch.arange(T) % 5], 1).to(torch.int32).to(DEV)
    two = torch.full((T, K), 7, dtype=torch.int32, device=DEV)
    two[:, 0] = 6
    buf = B.EPBuffer(2, E, H, K, max_tokens_per_rank=T, max_handles=1)
    try:
        recv, _, _, h, _ = buf.dispatch(x, one)
        want, got = (torch.full((E, N, H), math.nan, device=DEV) for _ in range(2))
        buf.expert_product_backward(g, h, x=recv, grad_weights=want)
        torch.cuda.synchronize()
        ev = buf.capture()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
            buf.expert_product_backward(g, h, x=recv, grad_weights=got)
        buf.combine(y, h, previous_event=ev)
        buf.destroy_handle(h)
        _, _, _, other, _ = buf.dispatch(x, two, previous_event=ev)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.isfinite(want).all()
        buf.destroy_handle(other)
    finally:
        buf.close()


def test_products_on_a_stream_of_somebody_else(ep):
    """The same results on a stream that torch did not make, behind what is queued there and before what follows."""
    from paper_2603_13606_amd import buffer as B
    T, E, H, K, N = 50, 8, 64, 2, 24
    gen = torch.Generator(DEV)
    gen.manual_seed(5)
    normal = lambda *s: torch.randn(s, generator=gen, device=DEV).bfloat16()  # noqa: E731
    idx = torch.randint(0, E, (T, K), generator=gen, device=DEV, dtype=torch.int32)
    x, w, g = normal(T, H), normal(E, N, H), normal(T * K, N)
    owner = torch.cuda.Stream()
    theirs = torch.cuda.ExternalStream(owner.cuda_stream)
    buf = B.EPBuffer(2, E, H, K, max_tokens_per_rank=T)
    try:
        recv, _, _, h, _ = buf.dispatch(x, idx)
        rows = buf.get_num_recv_tokens(h)
        want, _ = buf.expert_product(recv, w, h)
        want_gx, _ = buf.expert_product_backward(g, h, w)
        torch.cuda.synchronize()
        late = torch.zeros_like(recv)
        with torch.cuda.stream(theirs):
            torch.cuda._sleep(2_000_000)
            late.copy_(recv)
            out, _ = buf.expert_product(late, w, h)
            out = out.clone()
            gx, _ = buf.expert_product_backward(g, h, w)
            gx = gx.clone()
        torch.cuda.synchronize()
        assert torch.equal(out[:rows], want[:rows]) and torch.equal(gx, want_gx)
        buf.destroy_handle(h)
    finally:
        buf.close()


# ---------------------------------------------------------------------- gelu far below 0


def gelu_inputs():
    """Every bf16 number from -13 to -1/64, and some above."""
    v = torch.arange(0x3c80, 0x4151, device=DEV).to(torch.int16).view(torch.bfloat16)
    return torch.cat([-v, torch.linspace(0, 12, 96, device=DEV).bfloat16()])[:-((v.numel() + 96) % 8) or None].reshape(-1, 8).contiguous()


# Of the value: half a step of bf16, and 2^-15 for what float32 and the part's exponential do to arguments of up to 85.
GELU = ref.BF16 + 2.0 ** -15


@pytest.mark.parametrize("gated", [False, True])
def test_gelu_is_as_exact_far_below_zero(ep, gated):
    v = gelu_inputs()
    n = v.shape[0]
    eye = torch.eye(8, device=DEV, dtype=torch.bfloat16)[None]
    off, cnt = torch.zeros(1, dtype=torch.int32, device=DEV), torch.full((1,), n, dtype=torch.int32, device=DEV)
    out = torch.full_like(v, math.nan)
    if gated:   # the up projection is 1: its weights are 0, its bias 1
        w, b = torch.cat([eye, torch.zeros_like(eye)], 1), torch.tensor([[0.0] * 8 + [1.0] * 8], device=DEV)
    else:
        w, b = eye, None
    ep.ep_expert_product(v, w, out, bias=b, row_offset=off, row_count=cnt, activation=ep.EP_ACT_GELU, gated=gated)
    want = ref.act("gelu", v.double())
    within(out, want, GELU * want.abs() + ref.TINY, "gelu")
    pre = torch.cat([v, torch.ones_like(v)], 1) if gated else v
    grad = torch.full_like(pre, math.nan)
    ep.ep_expert_product_backward(torch.ones_like(v), w, pre=pre, grad_pre=grad, grad_x=torch.empty_like(v), row_offset=off, row_count=cnt,
                                  activation=ep.EP_ACT_GELU, gated=gated)
    d, cdf = ref.act_grad("gelu", v.double()), ref.act("gelu", v.double()) / v.double().where(v != 0, 1.0)
    within(grad[:, :8], d, ref.BF16 * d.abs() + 2.0 ** -15 * (cdf.abs() + (d - cdf).abs()) + ref.TINY, "its derivative")
    if gated:
        within(grad[:, 8:], want, GELU * want.abs() + ref.TINY, "gelu in the backward pass")
