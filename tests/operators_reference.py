"""The gate, the experts' products and the layer of few tokens in 64 bits, with bounds of what rounding may
change (test glue; nothing here calls the library).

Bounds count roundings.  A sum of n products in float32 is off by at most (n + 2) * 2^-23 * sum |terms| (one
step, twice half a step, per addition), a result rounded to bf16 by 2^-8 of its value, the float32
activations by 2^-18 of |v| (exponent, reciprocal, product; |v| <= 30 scales the exponent's error)."""
from __future__ import annotations

import math

import torch

U32 = 2.0 ** -23
BF16 = 2.0 ** -8
ACT = 2.0 ** -18
TINY = 2.0 ** -120


def act(name, v):
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu":
        return v * 0.5 * torch.erfc(-v / math.sqrt(2.0))
    return v


def act_grad(name, v):
    if name == "silu":
        s = torch.sigmoid(v)
        return s + v * s * torch.sigmoid(-v)
    if name == "gelu":
        return 0.5 * torch.erfc(-v / math.sqrt(2.0)) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(v)


# ------------------------------------------------------------------ the gate


def route_scores(l, score):
    there = l > -math.inf          # false for NaN too
    l = torch.where(there, l.clamp(max=torch.finfo(torch.float32).max), -math.inf)
    if score == "sigmoid":
        return torch.where(there, torch.sigmoid(l), 0.0), l, there
    top = l.max(dim=1, keepdim=True).values
    p = torch.where(there, torch.exp(l - torch.where(top > -math.inf, top, 0.0)), 0.0)
    total = p.sum(dim=1, keepdim=True)
    return torch.where(total > 0, p / total, 0.0), l, there


def route(logits, K, bias=None, score="softmax", renormalise=True, groups=1, kept=1, scale=1.0):
    """idx, w and a relative bound of w, token by token as the definition reads."""
    T, E = logits.shape
    l = logits.double().cpu()
    s, l, there = route_scores(l, score)
    key = l.clone() if bias is None and groups == 1 else s + (bias.double().cpu() if bias is not None else 0.0)
    key = torch.where(there & (key > -math.inf), key, -math.inf)
    idx = torch.full((T, K), -1, dtype=torch.int32)
    w = torch.zeros((T, K), dtype=torch.float64)
    for t in range(T):
        k = key[t].tolist()
        if groups > 1:
            size = E // groups
            worth = []
            for g in range(groups):
                two = sorted(k[g * size:(g + 1) * size], reverse=True)[:2]
                worth.append(-math.inf if two[0] == -math.inf else sum(v for v in two if v > -math.inf))
            best = sorted(range(groups), key=lambda g: (-worth[g], g))[:kept]
            k = [v if e // size in best else -math.inf for e, v in enumerate(k)]
        order = [e for e in sorted(range(E), key=lambda e: (-k[e], e)) if k[e] > -math.inf][:K]
        if order:
            idx[t, :len(order)] = torch.tensor(order, dtype=torch.int32)
            v = s[t][order]
            total = v.sum()
            w[t, :len(order)] = v / (total if total > 0 else 1.0) if renormalise else v
    if renormalise and score == "softmax":  # a sum that is 0 in 64 bits: relative to the selected's largest
        for t in range(T):
            n = int((idx[t] >= 0).sum())
            if n:
                v = torch.softmax(l[t][idx[t, :n].long()], dim=0)
                w[t, :n] = v
    # exponent's argument: a rounding of |l - top|; then exponential, E additions, two divisions
    reach = torch.where(there, (l - torch.where(there, l, -math.inf).max(dim=1, keepdim=True).values).abs(), 0.0).max(dim=1, keepdim=True).values
    reach = torch.maximum(reach, torch.where(there, l.abs(), 0.0).max(dim=1, keepdim=True).values if score == "sigmoid" else reach)
    return idx, w * scale, (reach.clamp(max=200.0) + E + 16) * U32


def route_grad(logits, idx, g, score="softmax", renormalise=True, scale=1.0):
    """Gradient of the logits and a bound."""
    T, E = logits.shape
    s, l, there = route_scores(logits.double().cpu(), score)
    idx = idx.cpu().long()
    ok = (idx >= 0) & (idx < E)
    at = idx.clamp(0, E - 1)
    ok &= torch.gather(there, 1, at)
    g = torch.where(ok, g.double().cpu() * scale, 0.0)
    if renormalise and score == "softmax":
        lk = torch.where(ok, torch.gather(l, 1, at), -math.inf)
        sk = torch.where(ok, torch.softmax(lk, dim=1).nan_to_num(0.0), 0.0)
        d, mag = sk * (g - (g * sk).sum(1, keepdim=True)), sk * (g.abs() + (g * sk).abs().sum(1, keepdim=True))
        out, size = torch.zeros_like(l).scatter_add(1, at, d), torch.zeros_like(l).scatter_add(1, at, mag)
    elif score == "softmax":
        sk = torch.where(ok, torch.gather(s, 1, at), 0.0)
        dot, mag = (g * sk).sum(1, keepdim=True), (g * sk).abs().sum(1, keepdim=True)
        out = s * (torch.zeros_like(l).scatter_add(1, at, g) - dot)
        size = s * (torch.zeros_like(l).scatter_add(1, at, g.abs()) + mag)
    else:
        sk = torch.where(ok, torch.gather(s, 1, at), 0.0)
        rest = torch.where(ok, torch.sigmoid(-torch.gather(l, 1, at)), 0.0)
        d, mag = g, g.abs()
        if renormalise:
            total = sk.sum(1, keepdim=True)
            total = torch.where(total > 0, total, 1.0)
            d = (g - (g * sk).sum(1, keepdim=True) / total) / total
            mag = (g.abs() + (g * sk).abs().sum(1, keepdim=True) / total) / total
        out, size = torch.zeros_like(l).scatter_add(1, at, d * sk * rest), torch.zeros_like(l).scatter_add(1, at, mag * sk * rest)
    reach = torch.where(there, l.abs(), 0.0).max(dim=1, keepdim=True).values.clamp(max=200.0)
    bound = size * (2 * reach + E + 2 * idx.shape[1] + 32) * U32 * 2 + TINY
    if logits.dtype == torch.bfloat16:
        bound = bound + BF16 * out.abs()
    return out, bound


# ------------------------------------------------------------------ products


def product(x, w, bias=None, residual=None, activation="none", gated=False):
    """One expert: x [n, Kd], w [N, Kd].  out, its bound, pre, its bound."""
    x, w = x.double(), w.double()
    pre = x @ w.t()
    size = x.abs() @ w.abs().t()
    if bias is not None:
        pre = pre + bias.double()
        size = size + bias.double().abs()
    d = size * (x.shape[1] + 2) * U32
    if gated:
        n = w.shape[0] // 2
        a, u = act(activation, pre[:, :n]), pre[:, n:]
        da = 1.2 * d[:, :n] + ACT * pre[:, :n].abs()
        out, err = a * u, da * u.abs() + a.abs() * d[:, n:] + da * d[:, n:]
    else:
        out, err = act(activation, pre), 1.2 * d + (ACT * pre.abs() if activation != "none" else 0.0)
    if residual is not None:
        out = out + residual.double()
        err = err + U32 * (out.abs() + residual.double().abs())
    return out, err * (1 + BF16) + BF16 * out.abs() + TINY, pre, d * (1 + BF16) + BF16 * pre.abs() + TINY


def product_grad(g, w, x, pre=None, activation="none", gated=False):
    """One expert: gradients {grad_pre, grad_x, grad_w, grad_b} with bounds, as float32 results of what the
    bf16 grad_pre carries on (a result kept in bf16 is off by BF16 of its value more)."""
    g, w, x = g.double(), w.double(), x.double()
    if pre is None:
        gp, e = g, torch.zeros_like(g)
    else:
        pre = pre.double()
        if gated:
            n = w.shape[0] // 2
            a, u = pre[:, :n], pre[:, n:]
            gp = torch.cat([g * u * act_grad(activation, a), g * act(activation, a)], dim=1)
            mag = torch.cat([(g * u).abs() * (1 + a.abs()), g.abs() * a.abs()], dim=1)
        else:
            gp, mag = g * act_grad(activation, pre), g.abs() * (1 + pre.abs())
        e = BF16 * gp.abs() + 2 * ACT * mag + TINY
    gx, ex = gp @ w, e @ w.abs() + (w.shape[0] + 2) * U32 * (gp.abs() @ w.abs())
    gw, ew = gp.t() @ x, e.t() @ x.abs() + (x.shape[0] + 2) * U32 * (gp.abs().t() @ x.abs())
    gb, eb = gp.sum(0), e.sum(0) + (x.shape[0] + 2) * U32 * gp.abs().sum(0)
    return {"grad_pre": (gp, e), "grad_x": (gx, ex + BF16 * (gx.abs() + ex) + TINY), "grad_w": (gw, ew + TINY), "grad_b": (gb, eb + TINY)}


def layer(x, idx, wts, w_up, w_down, b_up=None, b_down=None, residual=None, activation="silu", gated=True, first=0):
    """out [T, H] and its bound."""
    T, H = x.shape
    out = residual.double() if residual is not None else torch.zeros((T, H), dtype=torch.float64, device=x.device)
    size, err = out.abs().clone(), torch.zeros_like(out)
    for t in range(T):
        for k in range(idx.shape[1]):
            e = int(idx[t, k]) - first
            if not 0 <= e < w_up.shape[0]:
                continue
            s = float(wts[t, k]) if wts is not None else 1.0
            h, eh, _, _ = product(x[t:t + 1], w_up[e], b_up[e] if b_up is not None else None, None, activation, gated)
            wd = w_down[e].double()
            y, ey, mag = h @ wd.t(), eh @ wd.abs().t(), h.abs() @ wd.abs().t()
            if b_down is not None:
                y, mag = y + b_down[e].double(), mag + b_down[e].double().abs()
            out[t] += s * y[0]
            err[t] += abs(s) * ey[0] * (1 + 2 * BF16)
            size[t] += abs(s) * mag[0]
    err = err + size * (w_down.shape[2] * max(1, idx.shape[1]) + 16) * U32
    return out, err * (1 + BF16) + BF16 * out.abs() + TINY
