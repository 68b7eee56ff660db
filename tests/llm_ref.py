"""64-bit references of the 4-bit layer, the routing and the experts' products, with bounds of what FP32 sums and the stated roundings
may differ by.  Written from the definitions in include/bolt.h, with torch in float64 on whatever device the inputs are."""
import math

import torch

U16, U32 = 2.0 ** -11, 2.0 ** -23  # half an ulp of binary16, an ulp of binary32 (products and sums may each be half of one off)
TINY = 2.0 ** -24                  # the smallest binary16


def act(v, name):
    if name == "none":
        return v
    if name == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if name == "gelu":
        return v * torch.special.ndtr(v)
    if name == "hardswish":
        return v * torch.clamp(v + 3, 0, 6) / 6
    if name == "softplus":
        return torch.logaddexp(v, torch.zeros_like(v))
    if name == "silu":
        return v * torch.sigmoid(v)
    raise ValueError(name)


STEEP = 1.2  # no activation here is steeper
CLOSE = 2e-5  # relative error of the activations in FP32 (their own comments say 4e-6 to 1e-5)


def w4_matrix(q, scales, zeros, group):
    """[N][K] of one matrix from bytes [N][K / 2]."""
    N, K = q.shape[0], q.shape[1] * 2
    v = torch.empty((N, K), dtype=torch.float64, device=q.device)
    v[:, 0::2], v[:, 1::2] = (q & 15).double(), (q >> 4).double()
    g = torch.arange(K, device=q.device) // group
    z = 8.0 if zeros is None else zeros.double()[:, g]
    return scales.double()[:, g] * (v - z)


def product(x, W, bias, alpha=1.0, beta=1.0, shift=0.0):
    """x . W^T in 64 bits, and how far an FP32 sum in any order may be off (`shift`: relative rounding of W)."""
    v = alpha * (x @ W.t().contiguous())
    size = abs(alpha) * (x.abs() @ W.abs().t().contiguous())
    if bias is not None:
        v = v + beta * bias
        size = size + abs(beta) * bias.abs()
    return v, size * ((x.shape[1] + 16) * U32 + shift)


def linear(x, W, bias, name, alpha=1.0, beta=1.0, shift=0.0):
    """The layer and the bound of its rounded result."""
    v, off = product(x, W, bias, alpha, beta, shift)
    y = act(v, name)
    return y, off * STEEP + y.abs() * (CLOSE + U16) + TINY


def expert(x, up, b_up, down, b_down, name, gated):
    """One expert on rows x, and the bound of its FP32 rows: the hidden values are rounded to binary16."""
    u, off = product(x, up, b_up)
    if gated:
        F = u.shape[1] // 2
        g = act(u[:, :F], name)
        h = g * u[:, F:]
        dh = (off[:, :F] * STEEP + g.abs() * CLOSE) * (u[:, F:].abs() + off[:, F:]) + g.abs() * off[:, F:]
    else:
        h = act(u, name)
        dh = off * STEEP + h.abs() * CLOSE
    dh = dh + (h.abs() + dh) * U16 + TINY
    r, off = product(h, down, b_down)
    return r, off * (1 + 1e-3) + dh @ down.abs().t().contiguous()


def experts(x, ups, b_up, downs, b_down, ids, weights, name, gated):
    """y and its bound; ups(e), downs(e) give the matrices in 64 bits."""
    y = torch.zeros(x.shape[0], downs(0).shape[0], dtype=torch.float64, device=x.device)
    off, size = torch.zeros_like(y), torch.zeros_like(y)
    for e in torch.unique(ids).tolist():
        if e < 0:
            continue
        t, j = (ids == e).nonzero(as_tuple=True)
        r, d = expert(x[t].double(), ups(e), None if b_up is None else b_up[e].double(), downs(e),
                      None if b_down is None else b_down[e].double(), name, gated)
        w = weights[t, j].double()[:, None]
        y.index_add_(0, t, w * r)
        off.index_add_(0, t, w.abs() * d)
        size.index_add_(0, t, (w * r).abs())
    return y, off + size * (ids.shape[1] + 2) * U32 + y.abs() * U16 + TINY


def lists(ids, E):
    """offsets and order of routed ids, from a stable sort."""
    flat = ids.reshape(-1).cpu()
    on = (flat >= 0).nonzero().reshape(-1)
    by = on[torch.sort(flat[on], stable=True).indices]
    order = torch.full((flat.numel(),), -1, dtype=torch.int32)
    order[:by.numel()] = by.int()
    offsets = torch.zeros(E + 1, dtype=torch.int32)
    offsets[1:] = torch.bincount(flat[on].long(), minlength=E).cumsum(0).int()
    return offsets, order


def route(logits, bias, mask, k, score, groups, top_groups, renormalize, scale):
    """ids, weights (64 bits) and the smallest distance between keys that compete for a place of each token."""
    x = logits.double()
    x = torch.where(torch.isnan(x), torch.full_like(x, -torch.finfo(torch.float32).max), x)
    x = x.clamp(-torch.finfo(torch.float32).max, torch.finfo(torch.float32).max)
    T, E = x.shape
    s = torch.softmax(x, 1) if score == "softmax" else torch.sigmoid(x)
    key = x if bias is None else s + bias.double()
    gap = torch.full((T,), math.inf, dtype=torch.float64)
    if top_groups < groups:
        of = (s if score == "sigmoid" and bias is None else key).reshape(T, groups, E // groups)
        value = of.amax(2) if score == "softmax" else of.topk(min(2, E // groups), 2).values.sum(2)
        sorted_, idx = value.sort(dim=1, descending=True, stable=True)
        gap = torch.minimum(gap, sorted_[:, top_groups - 1] - sorted_[:, top_groups])
        keep = torch.zeros(T, groups, dtype=torch.bool).scatter_(1, idx[:, :top_groups], True)
        key = key.masked_fill(~keep.repeat_interleave(E // groups, 1), -math.inf)
    sorted_, idx = key.sort(dim=1, descending=True, stable=True)
    n = min(k + 1, sorted_.shape[1])
    if n > 1:
        gap = torch.minimum(gap, (sorted_[:, :n - 1] - sorted_[:, 1:n]).amin(1))
    ids = idx[:, :k]
    w = torch.gather(s, 1, ids)
    if renormalize:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, torch.zeros_like(w))
    w = w * scale
    if mask is not None:
        off = (mask == 0)[:, None]
        ids, w = ids.masked_fill(off, -1), w.masked_fill(off, 0.0)
    return ids.int(), w, gap
