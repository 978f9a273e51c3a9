"""The gate, the experts' products and the layer of a few tokens: what they are measured on.

Three operators around layout, dispatch and combine, in five forms (`op`):

  route       gate logits [T, E] -> the K experts of each token and their gate weights (ep_route)
  route_grad  its backward pass: gradient of the gate weights -> gradient of the logits
  product     the experts' product on the windows that a dispatch fills: x W^T with bias, activation and
              residual, rows grouped by expert, the row counts on the device (ep_expert_product)
  product_grad  its backward pass: gradients of the pre-activation, the rows, the weights and the bias
  layer       the whole layer for a few tokens, without windows (ep_expert_layer)

`run` computes them in plain torch operations in 32 bits (64 where the order of gate scores is decided), or,
with `own` set, by the framework's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"

_ROUTE = dict(T=128, E=256, K=8, dtype="f32", score="softmax", renormalise=True, bias=False, groups=1, kept=1, scale=1.0,
              masked=0.0)      # share of the logits that are -inf; a twentieth as many tokens have nothing else
_PRODUCT = dict(rows=1024, L=8, Kd=7168, No=2048, gated=True, act="silu", bias=False, residual=False, C=0,  # C: padded windows [L, C, Kd]
                empty=0,       # experts without rows
                spread=0.4,    # of the rows over the experts: counts go by exp(spread * N(0, 1))
                wgrad="bf16")  # type of the gradients of weights and bias
_LAYER = dict(T=1, L=64, K=8, H=7168, inner=2048, gated=True, act="silu", bias=False, residual=False,
              masked=0.0)      # share of the ids that are -1 (experts of other ranks)


def _case(name, op, **kw):
    d = _ROUTE if op.startswith("route") else _PRODUCT if op.startswith("product") else _LAYER
    return dict(d, **kw, op=op, name=name)


def listed():
    return [
        # the gate of a decode step: 128 tokens, latency is all
        _case("route_decode", "route"),
        # the gate of a prefill batch with a selection bias and group-limited choice
        _case("route_prefill", "route", T=4096, dtype="bf16", score="sigmoid", bias=True, groups=8, kept=4, scale=2.5),
        # odd sizes: 1000 experts, top-7, experts masked out (some tokens left with none), plain softmax weights
        _case("route_masked", "route", T=611, E=1000, K=7, renormalise=False, masked=0.3),
        # the gate's backward pass in a training step on 128 experts; without renormalisation every logit has a gradient
        _case("route_train", "route_grad", T=8192, E=128, K=8, renormalise=False),
        # up and gate projection of a decode step: a rank with 8 of 256 experts receives 32 x 128 tokens' top-8 into padded windows
        _case("product_decode", "product", rows=1024, C=512),
        # the same in prefill: 32 ranks' 4096 tokens, concatenated windows
        _case("product_prefill", "product", rows=32768),
        # down projection with bias and residual, odd sizes, ragged rows, experts without any
        _case("product_ragged", "product", rows=3001, L=48, Kd=1000, No=2888, gated=False, act="gelu", bias=True, residual=True, empty=7, spread=1.0),
        # training: backward of the up projection, all gradients
        _case("product_train_up", "product_grad", rows=16384, L=8, Kd=4096, No=1408, bias=True),
        # training: backward of a small down projection without activation, float32 gradients, odd sizes
        _case("product_train_down", "product_grad", rows=2003, L=16, Kd=1000, No=520, gated=False, act="none", bias=True, empty=2, wgrad="f32"),
        # one token of a decode step
        _case("layer_one", "layer"),
        # a ragged handful of tokens on a rank that owns half of the experts
        _case("layer_ragged", "layer", T=13, L=40, K=6, H=2888, inner=1000, gated=False, act="gelu", bias=True, residual=True, masked=0.5),
        # the decode batch, every expert named
        _case("layer_batch", "layer", T=128, L=128, H=4096, inner=1408),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "route_grad", "product", "product", "product_grad", "layer", "layer"])
    if op.startswith("route"):
        c = dict(_ROUTE, op=op, T=_log_int(rng, 1, 16384), E=rng.choice([8, 16, 60, 64, 96, 128, 160, 256, 384, 1000, 1024]),
                 dtype=rng.choice(["f32", "bf16"]), score=rng.choice(["softmax", "sigmoid"]), renormalise=rng.random() < 0.6,
                 scale=rng.choice([1.0, 2.5]), masked=rng.choice([0.0, 0.0, 0.3]))
        c["K"] = min(c["E"], rng.choice([1, 2, 4, 6, 7, 8, 8, 16]))
        c["bias"] = rng.random() < 0.4
        if op == "route" and rng.random() < 0.3 and c["E"] % 4 == 0:
            c["groups"], c["kept"] = 4, rng.choice([1, 2, 3])
        return c
    if op.startswith("product"):
        c = dict(_PRODUCT, op=op, L=_log_int(rng, 1, 64), gated=rng.random() < 0.5, act=rng.choice(["none", "silu", "gelu"]),
                 bias=rng.random() < 0.5, residual=op == "product" and rng.random() < 0.3, spread=rng.choice([0.0, 0.4, 1.0]),
                 Kd=8 * _log_int(rng, 16, 896), No=8 * _log_int(rng, 16, 512))
        if c["act"] == "none":
            c["gated"] = False
        one = c["Kd"] * c["No"] * (2 if c["gated"] else 1)
        c["L"] = max(1, min(c["L"], 1200000000 // one))
        # a plain form works on expert windows of the longest one's length: that bounds the rows of a case
        most = 1.2e12 / (6 if op == "product_grad" else 2) / one
        c["rows"] = _log_int(rng, 1, max(1, min(8192, int(most))))
        c["empty"] = rng.choice([0, 0, c["L"] // 4])
        if op == "product" and rng.random() < 0.4:
            c["C"] = max(8, 4 * c["rows"] // c["L"])
        if op == "product_grad" and c["act"] == "none":
            c["wgrad"] = rng.choice(["bf16", "f32"])
        return c
    c = dict(_LAYER, op=op, T=_log_int(rng, 1, 128), L=rng.choice([1, 8, 24, 40, 64, 96]), K=rng.choice([1, 2, 4, 6, 8]), H=8 * _log_int(rng, 32, 640),
             inner=8 * _log_int(rng, 16, 176), gated=rng.random() < 0.6, act=rng.choice(["silu", "gelu"]), bias=rng.random() < 0.4,
             residual=rng.random() < 0.4, masked=rng.choice([0.0, 0.0, 0.5]))
    c["K"] = min(c["K"], c["L"])
    return c


# ---------------------------------------------------------------------- inputs


def _normal(gen, *shape, std=1.0, dtype=torch.bfloat16):
    t = torch.randn(shape, generator=gen, device=DEV, dtype=dtype)
    return t.mul_(std) if std != 1.0 else t


def _row_counts(c, seed):
    """Rows per expert: `rows` in all, some experts with none; within C for padded windows."""
    rng = random.Random(seed)
    p = [math.exp(c["spread"] * rng.gauss(0.0, 1.0)) for _ in range(c["L"])]
    for e in rng.sample(range(c["L"]), min(c["empty"], c["L"] - 1)):
        p[e] = 0.0
    total = sum(p)
    n = [int(c["rows"] * v / total) for v in p]
    left = c["rows"] - sum(n)
    for e in sorted(range(c["L"]), key=lambda e: -p[e])[:left]:
        n[e] += 1
    return [min(v, c["C"]) for v in n] if c["C"] else n


def _prepare_route(c, s, gen):
    T, E, K = c["T"], c["E"], c["K"]
    logits = _normal(gen, T, E, dtype=torch.float32)
    if c["masked"]:
        gone = torch.rand((T, E), generator=gen, device=DEV) < c["masked"]
        gone |= torch.rand((T, 1), generator=gen, device=DEV) < c["masked"] / 20
        logits.masked_fill_(gone, -math.inf)
    s["logits"] = logits.to(torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)
    s["bias"] = _normal(gen, E, std=0.1, dtype=torch.float32) if c["bias"] else None
    s["topk_idx"] = torch.zeros((T, K), dtype=torch.int32, device=DEV)
    s["topk_w"] = torch.zeros((T, K), device=DEV)
    if c["op"] == "route_grad":
        order = s["logits"].float() + torch.rand((T, E), generator=gen, device=DEV)  # any K different experts will do
        top, idx = torch.topk(order, K, dim=1)
        s["topk_idx"] = torch.where(top > -math.inf, idx, -1).to(torch.int32)
        s["grad_w"] = _normal(gen, T, K, dtype=torch.float32)
        s["grad_logits"] = torch.zeros_like(s["logits"])


def _prepare_product(c, s, gen, seed):
    L, Kd, No, C = c["L"], c["Kd"], c["No"], c["C"]
    N = 2 * No if c["gated"] else No
    n = _row_counts(c, seed)
    s["most"] = max(n)
    s["count"] = torch.tensor(n, dtype=torch.int32, device=DEV)
    first = [e * C for e in range(L)] if C else [sum(n[:e]) for e in range(L)]
    s["offset"] = torch.tensor(first, dtype=torch.int32, device=DEV)
    lead = (L, C) if C else (c["rows"],)
    s["x"] = _normal(gen, *lead, Kd)
    s["w"] = _normal(gen, L, N, Kd, std=Kd ** -0.5)
    s["bias"] = _normal(gen, L, N, std=0.1) if c["bias"] else None
    if c["op"] == "product":
        s["residual"] = _normal(gen, *lead, No) if c["residual"] else None
        s["out"] = torch.zeros((*lead, No), dtype=torch.bfloat16, device=DEV)
        return
    s["grad_out"] = _normal(gen, *lead, No)
    s["pre"] = _normal(gen, *lead, N) if c["act"] != "none" else None  # as the forward pass kept it
    wt = torch.float32 if c["wgrad"] == "f32" else torch.bfloat16
    s["grad_pre"] = torch.zeros((*lead, N), dtype=torch.bfloat16, device=DEV) if c["act"] != "none" else None
    s["grad_x"] = torch.zeros((*lead, Kd), dtype=torch.bfloat16, device=DEV)
    s["grad_w"] = torch.zeros((L, N, Kd), dtype=wt, device=DEV)
    s["grad_bias"] = torch.zeros((L, N), dtype=wt, device=DEV) if c["bias"] else None


def _prepare_layer(c, s, gen):
    T, L, K, H, inner = c["T"], c["L"], c["K"], c["H"], c["inner"]
    N = 2 * inner if c["gated"] else inner
    s["x"] = _normal(gen, T, H)
    top, idx = torch.topk(torch.randn((T, L), generator=gen, device=DEV), K, dim=1)
    gone = torch.rand((T, K), generator=gen, device=DEV) < c["masked"]
    s["topk_idx"] = torch.where(gone, -1, idx).to(torch.int32).contiguous()
    s["topk_w"] = torch.softmax(top, dim=1).contiguous()
    s["w_up"] = _normal(gen, L, N, H, std=H ** -0.5)
    s["w_down"] = _normal(gen, L, H, inner, std=inner ** -0.5)
    s["b_up"] = _normal(gen, L, N, std=0.1) if c["bias"] else None
    s["b_down"] = _normal(gen, L, H, std=0.1) if c["bias"] else None
    s["residual"] = _normal(gen, T, H) if c["residual"] else None
    s["out"] = torch.zeros((T, H), dtype=torch.bfloat16, device=DEV)


def prepare(case, seed):
    c = case
    gen = torch.Generator(DEV)
    gen.manual_seed(seed)
    s = {"c": c}
    if c["op"].startswith("route"):
        _prepare_route(c, s, gen)
    elif c["op"].startswith("product"):
        _prepare_product(c, s, gen, seed)
    else:
        _prepare_layer(c, s, gen)
    return s


# ---------------------------------------------------------------------- plain forms


def _act(name, v):
    if name == "silu":
        return v / (1.0 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    return v


def _act_grad(name, v):
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-v))
        return s * (1.0 + v * (1.0 - s))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(v)


def _scores(c, l):
    """Gate scores in the type of l; 0 for an expert that is masked out."""
    if c["score"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-l))
    top = l.max(dim=1, keepdim=True).values
    p = torch.exp(l - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    return p / p.sum(dim=1, keepdim=True).clamp(min=1e-300 if l.dtype == torch.float64 else 1e-30)


def _plain_route(s):
    c, K = s["c"], s["c"]["K"]
    l = s["logits"].float()
    there = l > -math.inf
    if s["bias"] is None and c["groups"] == 1:
        key = l
    else:  # scores next to each other: their order is decided in 64 bits
        key = _scores(c, l.double())
        if s["bias"] is not None:
            key = key + s["bias"].double()
        key = torch.where(there, key, -math.inf)
        if c["groups"] > 1:
            two = torch.sort(key.reshape(l.shape[0], c["groups"], -1), dim=2, descending=True).values[:, :, :2]
            none = two[:, :, 0] == -math.inf
            worth = torch.where(none, -math.inf, torch.where(two == -math.inf, 0.0, two).sum(dim=2))
            order = torch.sort(worth, dim=1, descending=True, stable=True).indices
            keep = torch.zeros_like(worth, dtype=torch.bool).scatter(1, order[:, :c["kept"]], True)
            key = torch.where(keep.repeat_interleave(l.shape[1] // c["groups"], dim=1), key, -math.inf)
    best, idx = torch.sort(key, dim=1, descending=True, stable=True)
    best, idx = best[:, :K], idx[:, :K]
    w = torch.where(best > -math.inf, torch.gather(_scores(c, l), 1, idx), 0.0)
    if c["renormalise"]:
        w = w / w.sum(dim=1, keepdim=True).clamp(min=1e-30)
    return {"topk_idx": torch.where(best > -math.inf, idx, -1).to(torch.int32), "topk_w": w * c["scale"]}


def _plain_route_grad(s):
    c = s["c"]
    l, g = s["logits"].float(), s["grad_w"]
    there = s["topk_idx"] >= 0
    idx = s["topk_idx"].long().clamp(min=0)
    p = _scores(c, l)
    pk = torch.where(there, torch.gather(p, 1, idx), 0.0)
    total = pk.sum(dim=1, keepdim=True).clamp(min=1e-30) if c["renormalise"] else torch.ones_like(pk[:, :1])
    dp = torch.where(there, g, 0.0) * (c["scale"] / total)
    if c["renormalise"]:
        dp = torch.where(there, dp - (dp * pk).sum(dim=1, keepdim=True) / total, 0.0)
    if c["score"] == "sigmoid":
        dl = torch.zeros_like(l).scatter_add(1, idx, dp * pk * (1.0 - pk))
    else:
        dl = p * (torch.zeros_like(l).scatter_add(1, idx, dp) - (dp * pk).sum(dim=1, keepdim=True))
    return {"grad_logits": dl.to(s["logits"].dtype)}


def _windows(s):
    """Row numbers [L, most] of every expert's rows and which of them there are."""
    at = torch.arange(max(s["most"], 1), device=DEV)
    there = at[None] < s["count"][:, None]
    return torch.where(there, s["offset"][:, None].long() + at[None], 0), there


def _gather(t, rows, there):
    return torch.where(there[..., None], t.reshape(-1, t.shape[-1])[rows], 0).float()


def _scatter(like, rows, there, v):
    """v in the rows of its experts, zeros elsewhere (the last row takes what has no place)."""
    n = like.numel() // like.shape[-1]
    out = torch.zeros((n + 1, like.shape[-1]), dtype=like.dtype, device=DEV)
    out[torch.where(there, rows, n)] = v.to(like.dtype)
    return out[:n].reshape(like.shape)


def _plain_product(s):
    c = s["c"]
    rows, there = _windows(s)
    pre = torch.bmm(_gather(s["x"], rows, there), s["w"].float().transpose(1, 2))
    if s["bias"] is not None:
        pre = pre + s["bias"].float()[:, None]
    if c["gated"]:
        y = _act(c["act"], pre[..., :c["No"]]) * pre[..., c["No"]:]
    else:
        y = _act(c["act"], pre)
    if s["residual"] is not None:
        y = y + _gather(s["residual"], rows, there)
    return {"out": _scatter(s["out"], rows, there, y)}


def _plain_product_grad(s):
    c, No = s["c"], s["c"]["No"]
    rows, there = _windows(s)
    d = _gather(s["grad_out"], rows, there)
    out = {}
    if c["act"] != "none":
        pre = _gather(s["pre"], rows, there)
        if c["gated"]:
            d = torch.cat([d * pre[..., No:] * _act_grad(c["act"], pre[..., :No]), d * _act(c["act"], pre[..., :No])], dim=-1)
        else:
            d = d * _act_grad(c["act"], pre)
        out["grad_pre"] = _scatter(s["grad_pre"], rows, there, d)
    out["grad_x"] = _scatter(s["grad_x"], rows, there, torch.bmm(d, s["w"].float()))
    out["grad_w"] = torch.bmm(d.transpose(1, 2).contiguous(), _gather(s["x"], rows, there)).to(s["grad_w"].dtype)
    if s["grad_bias"] is not None:
        out["grad_bias"] = d.sum(dim=1).to(s["grad_bias"].dtype)
    return out


def _plain_layer(s):
    """Every expert that is named works on every token; the gate weights pick."""
    c, L = s["c"], s["c"]["L"]
    ids = s["topk_idx"].long()
    gate = torch.zeros((c["T"], L + 1), device=DEV).scatter_add(1, torch.where(ids >= 0, ids, L), s["topk_w"])[:, :L]
    named = torch.unique(ids[ids >= 0])
    x = s["x"].float()[None].expand(named.shape[0], -1, -1)
    pre = torch.bmm(x, s["w_up"][named].float().transpose(1, 2))
    if s["b_up"] is not None:
        pre = pre + s["b_up"][named].float()[:, None]
    h = _act(c["act"], pre[..., :c["inner"]]) * pre[..., c["inner"]:] if c["gated"] else _act(c["act"], pre)
    y = torch.bmm(h, s["w_down"][named].float().transpose(1, 2))
    if s["b_down"] is not None:
        y = y + s["b_down"][named].float()[:, None]
    out = (gate[:, named].t()[..., None] * y).sum(dim=0)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return {"out": out.to(torch.bfloat16)}


# ---------------------------------------------------------------------- the framework's calls


def _own_call(s):
    """The call of a pass with its descriptors built once, as a program that makes it every step keeps it."""
    from paper_2603_13606_amd import binding as ep
    c, op = s["c"], s["c"]["op"]
    act = {"none": ep.EP_ACT_NONE, "silu": ep.EP_ACT_SILU, "gelu": ep.EP_ACT_GELU}.get(c.get("act", "none"))
    if op.startswith("route"):
        rule = dict(score=ep.EP_SCORE_SIGMOID if c["score"] == "sigmoid" else ep.EP_SCORE_SOFTMAX, renormalise=c["renormalise"],
                    scale=c["scale"])
        if op == "route":
            call = ep.prepare_route(s["logits"], s["topk_idx"], s["topk_w"], bias=s["bias"], num_groups=c["groups"],
                                    groups_kept=c["kept"], **rule)
            return call, {"topk_idx": s["topk_idx"], "topk_w": s["topk_w"]}
        call = ep.prepare_route_backward(s["logits"], s["topk_idx"], s["grad_w"], s["grad_logits"], **rule)
        return call, {"grad_logits": s["grad_logits"]}
    if op == "layer":
        n = ep.ep_expert_layer_plan(c["T"], c["K"], c["L"], c["H"], c["inner"]).workspace_bytes
        s["workspace"] = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)
        call = ep.prepare_expert_layer(s["x"], s["topk_idx"], s["topk_w"], s["w_up"], s["w_down"], s["out"], s["workspace"],
                                       bias_up=s["b_up"], bias_down=s["b_down"], residual=s["residual"], activation=act,
                                       gated=c["gated"])
        return call, {"out": s["out"]}
    windows = dict(row_count=s["count"], row_offset=None if c["C"] else s["offset"], activation=act, gated=c["gated"])
    if op == "product":
        call = ep.prepare_expert_product(s["x"], s["w"], s["out"], bias=s["bias"], residual=s["residual"], **windows)
        return call, {"out": s["out"]}
    call = ep.prepare_expert_product_backward(s["grad_out"], s["w"], x=s["x"], pre=s["pre"], grad_pre=s["grad_pre"], grad_x=s["grad_x"],
                                              grad_weights=s["grad_w"], grad_bias=s["grad_bias"], **windows)
    return call, {k: s[k] for k in ("grad_pre", "grad_x", "grad_w", "grad_bias") if s[k] is not None}


def run(state):
    s = state
    if own:
        if "call" not in s:
            s["call"], s["outputs"] = _own_call(s)
        s["call"](stream_ptr=torch.cuda.current_stream().cuda_stream)
        return s["outputs"]
    return {"route": _plain_route, "route_grad": _plain_route_grad, "product": _plain_product, "product_grad": _plain_product_grad,
            "layer": _plain_layer}[s["c"]["op"]](s)


def work(case):
    c = case
    if c["op"].startswith("route"):
        n = c["T"] * c["E"]
        size = 2 if c["dtype"] == "bf16" else 4
        if c["op"] == "route":
            return {"bytes": n * size + 8 * c["T"] * c["K"] + (4 * c["E"] if c["bias"] else 0), "flops": 4 * n}
        return {"bytes": 2 * n * size + 8 * c["T"] * c["K"], "flops": 6 * n}
    if c["op"].startswith("product"):
        N = 2 * c["No"] if c["gated"] else c["No"]
        rows, L = c["rows"], min(c["L"], c["rows"]) - min(c["empty"], c["L"] - 1)
        w = 2 * max(L, 1) * N * c["Kd"]
        if c["op"] == "product":
            io = 2 * rows * (c["Kd"] + c["No"] * (2 if c["residual"] else 1))
            return {"bytes": w + io, "flops": 2 * rows * N * c["Kd"]}
        io = 2 * rows * (2 * c["Kd"] + c["No"] + (2 * N if c["act"] != "none" else 0))
        grads = (4 if c["wgrad"] == "f32" else 2) * c["L"] * N * c["Kd"]
        return {"bytes": w + io + grads, "flops": 4 * rows * N * c["Kd"]}
    entries = c["T"] * c["K"] * (1.0 - c["masked"])
    named = max(1.0, c["L"] * (1.0 - (1.0 - c["K"] * (1.0 - c["masked"]) / c["L"]) ** c["T"]))
    one = (3 if c["gated"] else 2) * c["H"] * c["inner"]
    return {"bytes": 2 * named * one + 2 * c["T"] * c["H"] * (3 if c["residual"] else 2) + 8 * c["T"] * c["K"], "flops": 2 * entries * one}


# ---------------------------------------------------------------------- the definitions in 64 bits


def _exact_score(c, l):
    if c["score"] == "sigmoid":
        return torch.sigmoid(l)
    return torch.softmax(l, dim=1).nan_to_num(0.0)  # a token without experts


def _exact_route(s):
    c, T, K = s["c"], s["c"]["T"], s["c"]["K"]
    l = s["logits"].double()
    score = _exact_score(c, l)
    key = score if s["bias"] is None else score + s["bias"].double()
    key = key.masked_fill(l == -math.inf, -math.inf)
    if s["bias"] is None and c["groups"] == 1:
        key = l  # the same order, without the ties of scores that round alike
    if c["groups"] > 1:
        size = c["E"] // c["groups"]
        worth = torch.full((T, c["groups"]), -math.inf, dtype=torch.float64, device=DEV)
        for g in range(c["groups"]):
            part = key[:, g * size:(g + 1) * size].topk(min(2, size), dim=1).values
            worth[:, g] = part[:, 0] + (part[:, 1:].clamp(min=-1e300).sum(dim=1).masked_fill((part[:, 1:] == -math.inf).any(dim=1), 0.0) if size > 1 else 0.0)
        chosen = (-worth).argsort(dim=1, stable=True)[:, :c["kept"]]
        member = torch.arange(c["E"], device=DEV) // size
        key = key.masked_fill(~(member[None, :, None] == chosen[:, None, :]).any(dim=2), -math.inf)
    order = (-key).argsort(dim=1, stable=True)[:, :K]
    ok = key.gather(1, order) > -math.inf
    w = score.gather(1, order) * ok
    if c["renormalise"]:
        w = torch.where(ok, w / w.sum(dim=1, keepdim=True), 0.0)
    return {"topk_idx": torch.where(ok, order, -1).to(torch.int32), "topk_w": w * c["scale"]}


def _exact_route_grad(s):
    """The derivative, by autograd of the weights' definition in 64 bits."""
    c = s["c"]
    l = s["logits"].double()
    leaf = l.masked_fill(l == -math.inf, 0.0).requires_grad_(True)
    score = _exact_score(c, leaf.masked_fill(l == -math.inf, -math.inf) if c["score"] == "softmax" else leaf)
    ok = s["topk_idx"] >= 0
    w = score.gather(1, s["topk_idx"].long().clamp(min=0)) * ok
    if c["renormalise"]:
        total = w.sum(dim=1, keepdim=True)
        w = w / torch.where(total > 0, total, 1.0)
    (w * s["grad_w"].double() * c["scale"]).sum().backward()
    return {"grad_logits": leaf.grad.nan_to_num(0.0).masked_fill(l == -math.inf, 0.0)}


def _exact_act(name, v):
    return torch.nn.functional.silu(v) if name == "silu" else torch.nn.functional.gelu(v) if name == "gelu" else v


def _exact_mid(c, pre, No):
    return _exact_act(c["act"], pre[:, :No]) * pre[:, No:] if c["gated"] else _exact_act(c["act"], pre)


def _exact_product(s):
    c = s["c"]
    out = torch.zeros((s["out"].numel() // c["No"], c["No"]), dtype=torch.float64, device=DEV)
    x = s["x"].reshape(-1, c["Kd"])
    for e, (at, n) in enumerate(zip(s["offset"].tolist(), s["count"].tolist())):
        pre = x[at:at + n].double() @ s["w"][e].double().t()
        if s["bias"] is not None:
            pre += s["bias"][e].double()
        out[at:at + n] = _exact_mid(c, pre, c["No"])
        if s["residual"] is not None:
            out[at:at + n] += s["residual"].reshape(-1, c["No"])[at:at + n].double()
    return {"out": out.reshape(s["out"].shape)}


def _exact_product_grad(s):
    c, No, Kd = s["c"], s["c"]["No"], s["c"]["Kd"]
    names = [k for k in ("grad_pre", "grad_x", "grad_w", "grad_bias") if s[k] is not None]
    out = {k: torch.zeros(s[k].shape, dtype=torch.float64, device=DEV) for k in names}
    for e, (at, n) in enumerate(zip(s["offset"].tolist(), s["count"].tolist())):
        d = s["grad_out"][at:at + n].double()
        if s["pre"] is not None:
            pre = s["pre"][at:at + n].double().requires_grad_(True)
            (_exact_mid(c, pre, No) * d).sum().backward()
            d = pre.grad
            out["grad_pre"][at:at + n] = d
        out["grad_x"][at:at + n] = d @ s["w"][e].double()
        out["grad_w"][e] = d.t() @ s["x"][at:at + n].double()
        if s["grad_bias"] is not None:
            out["grad_bias"][e] = d.sum(dim=0)
    return out


def _exact_layer(s):
    c = s["c"]
    out = s["residual"].double() if s["residual"] is not None else torch.zeros((c["T"], c["H"]), dtype=torch.float64, device=DEV)
    ids = s["topk_idx"].cpu()
    for e in sorted(set(ids[ids >= 0].tolist())):
        t, k = torch.nonzero(ids == e, as_tuple=True)
        t, k = t.to(DEV), k.to(DEV)
        pre = s["x"][t].double() @ s["w_up"][e].double().t()
        if s["b_up"] is not None:
            pre += s["b_up"][e].double()
        y = _exact_mid(c, pre, c["inner"]) @ s["w_down"][e].double().t()
        if s["b_down"] is not None:
            y += s["b_down"][e].double()
        out.index_add_(0, t, y * s["topk_w"][t, k].double()[:, None])
    return {"out": out}


def exact(case, seed):
    s = prepare(case, seed)
    return {"route": _exact_route, "route_grad": _exact_route_grad, "product": _exact_product, "product_grad": _exact_product_grad,
            "layer": _exact_layer}[case["op"]](s)
