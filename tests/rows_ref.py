"""64-bit references of the norm, the rows in 8 bits, the layers that read them and the projections with adapters, with bounds of what FP32
arithmetic and the stated roundings may differ by.  Written from the definitions in include/bolt.h."""
import torch

import llm_ref as ref

U8 = 2.0 ** -4         # half a step of E4M3, relative
TINY8 = 2.0 ** -10     # half its smallest step
MOST8 = 448.0
H16, H32 = 2.0 ** -11, 2.0 ** -24  # half a step of binary16 and of binary32, relative
TINY16 = 2.0 ** -25    # half the smallest step of binary16
# The sum of a row's squares: a lane adds 32 at most one after the other (each a rounded square), 6 levels of lanes and 16 waves follow; the
# mean, eps, root and quotient are four more roundings, and the root halves what came before it.  v itself is rounded once, twice in its square.
NORM = ((32 + 6 + 16 + 2 + 2) / 2 + 4) * H32


def norm(x, residual, weight, eps, offset):
    """v, n and the relative bound of n in FP32."""
    v = x.double() if residual is None else x.double() + residual.double()
    n = v / torch.sqrt((v * v).mean(1, keepdim=True) + eps) * (offset + weight.double())
    return v, n, NORM + 5 * H32  # (v, offset + weight, two products)


def within(got, want, bound, what=""):
    got = got.double()
    assert torch.isfinite(got).all(), what
    err = (got - want).abs()
    worst = (err - bound).max().item() if err.numel() else 0.0
    assert worst <= 0.0, (what, worst, (err / bound.clamp(min=1e-300)).max().item())


def check_half(got, want, rel, what=""):
    within(got, want, want.abs() * (H16 * (1 + rel) + rel) + TINY16, what)


def check_q(q, scales, n, rel, what=""):
    """q and scales of rows n."""
    s = n.abs().amax(1) / MOST8
    within(scales, s, s * (rel + 2 * H32), what + " scales")
    t = n / s.clamp(min=1e-300)[:, None]
    within(q, t, t.abs() * (U8 * (1 + 4 * rel + 8 * H32) + 4 * rel + 8 * H32) + TINY8, what + " q")


def lora(x, W, bias, ids, down, up, scales, act, alpha=1.0, beta=1.0, shift=0.0, apart=True):
    """The projection with adapters and the bound of its rounded result.  apart: the adapters' share is rounded to binary16 before it is added."""
    v, size = x @ W.t().contiguous(), x.abs() @ W.abs().t().contiguous()
    off = size * ((x.shape[1] + 16) * ref.U32 + shift)
    for a in range(down.shape[0]):
        rows = (ids == a).nonzero().view(-1)
        if not len(rows):
            continue
        s = 1.0 if scales is None else scales[a].double()
        d, u = down[a].double(), up[a].double()
        low = s * (x[rows] @ d.t().contiguous())
        dlow = abs(s) * (x[rows].abs() @ d.abs().t().contiguous()) * (x.shape[1] + 24) * ref.U32
        dlow = dlow + (low.abs() + dlow) * H16 + TINY16
        share = low @ u.t().contiguous()
        dshare = dlow @ u.abs().t().contiguous() + (low.abs() + dlow) @ u.abs().t().contiguous() * (d.shape[0] + 8) * ref.U32
        if apart:
            dshare = dshare + (share.abs() + dshare) * H16 + TINY16
        v[rows] += share
        off[rows] += dshare
        size[rows] += share.abs()
    v, off = alpha * v, abs(alpha) * off
    if bias is not None:
        v, size = v + beta * bias, size + abs(beta) * bias.abs()
    off = off + (abs(alpha) * size + v.abs()) * 4 * ref.U32
    y = ref.act(v, act)
    return y, off * ref.STEEP + y.abs() * (ref.CLOSE + ref.U16) + ref.TINY
