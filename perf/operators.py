"""The sparse-MLP and 4-bit operators as cases that can be timed and compared: what a program that serves a language
model on this library calls next to its FP16 GEMMs.

Kinds of cases and what they stand for:
  w4       a linear layer whose weights are held in 4 bits with a scale (and a zero point) for every group of a row
  route    the choice of experts for every token, from the router's logits, with the lists that the experts' products need
  experts  the experts' products for routed tokens: up projection, activation (gated or not), down projection, weighted sum

With `own` false, `run` computes a case with elementary torch operations in 32 bits; with `own` true it calls the library.
"""
import math

import torch

own = False

ACTS = ("none", "relu", "gelu", "hardswish", "softplus", "silu")


def listed():
    return [
        # One token through a square projection: the smallest call, bound by 8 MB of weights and the launch.
        dict(name="w4_one_token", kind="w4", M=1, N=4096, K=4096, group=128, zeros=False, bias=False, act="none"),
        # A few sequences decoding together through an MLP's first half; widths that are no multiples of a tile or group.
        dict(name="w4_few_rows", kind="w4", M=13, N=6152, K=5000, group=64, zeros=True, bias=True, act="gelu"),
        # A large batch of sequences, between weight bound and compute bound.
        dict(name="w4_batch", kind="w4", M=100, N=8192, K=2048, group=128, zeros=True, bias=False, act="none"),
        # A prompt: thousands of rows, bound by the matrix cores.
        dict(name="w4_prompt", kind="w4", M=4096, N=8192, K=4096, group=32, zeros=False, bias=True, act="relu"),
        # One decoded token chooses its experts: latency.
        dict(name="route_one_token", kind="route", T=1, E=64, k=8, score="softmax", groups=1, top_groups=1, bias=False,
             renorm=True, logits="f16", masked=0.0),
        # A prompt (with padding tokens) under a router with a bias for balance and a choice of groups first.
        dict(name="route_groups", kind="route", T=4099, E=256, k=8, score="sigmoid", groups=8, top_groups=4, bias=True,
             renorm=True, logits="f32", masked=0.05),
        # A large prefill batch: every token's logits once through the chip.
        dict(name="route_many", kind="route", T=65536, E=128, k=4, score="softmax", groups=1, top_groups=1, bias=False,
             renorm=False, logits="f16", masked=0.0),
        # One decoded token through its 8 experts: 100 MB of FP16 weights.
        dict(name="experts_one_token", kind="experts", T=1, E=64, k=8, width=2048, hidden=1024, gated=True, act="silu",
             weights="f16", group=0, bias=False, masked=0.0),
        # A decode batch over many small experts held in 4 bits: few tokens for each, nearly every expert is read.
        dict(name="experts_decode_w4", kind="experts", T=29, E=128, k=8, width=2048, hidden=768, gated=True, act="silu",
             weights="w4", group=64, bias=False, masked=0.0),
        # A short prompt over few experts, no gate, with biases, odd widths.
        dict(name="experts_odd", kind="experts", T=700, E=8, k=2, width=1000, hidden=2504, gated=False, act="gelu",
             weights="f16", group=0, bias=True, masked=0.1),
        # A prefill batch over many experts: the largest, bound by the matrix cores.
        dict(name="experts_prefill", kind="experts", T=8192, E=64, k=6, width=2048, hidden=1024, gated=True, act="silu",
             weights="f16", group=0, bias=False, masked=0.0),
        # A prefill batch whose experts are held in 4 bits.
        dict(name="experts_prefill_w4", kind="experts", T=3001, E=32, k=4, width=1536, hidden=1280, gated=True, act="silu",
             weights="w4", group=128, bias=False, masked=0.02),
    ]


# ----------------------------------------------------------------------------------------------------------------
# draws from the same ranges
# ----------------------------------------------------------------------------------------------------------------
def _log(rng, lo, hi, step=1):
    """An integer in [lo, hi], its logarithm uniform, rounded to a multiple of `step`."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(("w4", "w4", "route", "experts", "experts"))
    while True:
        if kind == "w4":
            case = dict(kind=kind, M=_log(rng, 1, 4096), N=_log(rng, 256, 12288, 8), K=_log(rng, 256, 12288, 8),
                        group=rng.choice((32, 64, 128)), zeros=rng.random() < 0.5, bias=rng.random() < 0.5,
                        act=rng.choice(ACTS))
            if case["M"] * case["N"] * case["K"] > 4096 * 8192 * 4096 or case["N"] * case["K"] > 64 << 20 or 3072 in case.values():
                continue
            return case
        if kind == "route":
            groups = rng.choice((1, 1, 2, 4, 8))
            E = groups * _log(rng, max(2, 8 // groups), 512 // groups)
            top_groups = rng.randint(1, groups)
            score = rng.choice(("softmax", "sigmoid"))
            case = dict(kind=kind, T=_log(rng, 1, 65536), E=E, k=rng.randint(1, min(10, E // groups * top_groups)), score=score,
                        groups=groups, top_groups=top_groups, bias=score == "sigmoid" and rng.random() < 0.7,
                        renorm=rng.random() < 0.7, logits=rng.choice(("f16", "f32")), masked=rng.choice((0.0, 0.1)))
            if case["T"] * E > 65536 * 128 or 3072 in case.values():
                continue
            return case
        w4 = rng.random() < 0.4
        E = _log(rng, 4, 128)
        case = dict(kind=kind, T=_log(rng, 1, 8192), E=E, k=rng.randint(1, min(8, E)), width=_log(rng, 256, 4096, 8),
                    hidden=_log(rng, 256, 4096, 8), gated=rng.random() < 0.7, act=rng.choice(ACTS[1:]),
                    weights="w4" if w4 else "f16", group=rng.choice((32, 64, 128)) if w4 else 0, bias=rng.random() < 0.3,
                    masked=rng.choice((0.0, 0.1)))
        size = case["width"] * case["hidden"] * (3 if case["gated"] else 2)
        if size * E > 64 * 3 * 2048 * 1024 or size * case["T"] * case["k"] > 8192 * 6 * 3 * 2048 * 1024 or 3072 in case.values():
            continue
        return case


# ----------------------------------------------------------------------------------------------------------------
# what a program has in hand before the call
# ----------------------------------------------------------------------------------------------------------------
class _State:
    def __init__(self, **kw):
        self.__dict__.update(kw)


def _w4_weights(count, N, K, group, zeros, gen):
    """4-bit weights as a quantiser leaves them: two to a byte (even k in the low half), a scale and a zero point per group."""
    groups = -(-K // group)
    q = torch.randint(0, 256, (count, N, K // 2), dtype=torch.uint8, device="cuda", generator=gen)
    scales = ((torch.rand((count, N, groups), device="cuda", generator=gen) + 0.5) * (0.2 / math.sqrt(K))).half()
    z = torch.randint(4, 12, (count, N, groups), dtype=torch.uint8, device="cuda", generator=gen) if zeros else None
    return q, scales, z


def _pack(w, N, K, group):
    import paper_2110_15238_amd as bolt
    q, scales, z = w
    packed = torch.empty(bolt.bolt_w4_packed_bytes(N, K, group, q.shape[0]), dtype=torch.uint8, device="cuda")
    return bolt.bolt_w4_pack(N, K, group, q, scales, z, packed)


def _half(gen, *shape, std=1.0):
    t = torch.empty(shape, dtype=torch.float16, device="cuda")
    return t.normal_(0.0, std, generator=gen)


def _prepare_w4(case, gen):
    M, N, K, G = case["M"], case["N"], case["K"], case["group"]
    s = _State(A=_half(gen, M, K), w=_w4_weights(1, N, K, G, case["zeros"], gen), bias=_half(gen, N) if case["bias"] else None)
    if own:
        import paper_2110_15238_amd as bolt
        s.desc = bolt.gemm_w4_desc(M, N, K, G, act=case["act"])
        s.packed = _pack(s.w, N, K, G)
        s.D = torch.empty((M, N), dtype=torch.float16, device="cuda")
        s.workspace = torch.empty(bolt.bolt_gemm_w4_workspace_bytes(s.desc), dtype=torch.uint8, device="cuda")
    return s


def _decisions_hang_on_rounding(case, logits, bias):
    """Tokens for which two keys that compete for a place (or two groups at the cut) are closer than 32-bit rounding can
    tell apart: either choice is right there, so the inputs hold none of them."""
    s = torch.sigmoid(logits.double())
    key = s if bias is None else s + bias.double()
    T, E, g, n = case["T"], case["E"], case["groups"], case["top_groups"]
    grouped = key.view(T, g, E // g)
    value = grouped.topk(min(2, E // g), dim=2).values.sum(2).sort(dim=1, descending=True)
    close = torch.zeros(T, dtype=torch.bool, device=key.device)
    if n < g:
        close |= value.values[:, n - 1] - value.values[:, n] < 1e-5
    keep = torch.zeros((T, g), dtype=torch.bool, device=key.device).scatter_(1, value.indices[:, :n], True)
    left = torch.where(keep[:, :, None], grouped, -1.0).view(T, E).topk(min(case["k"] + 1, n * (E // g)), dim=1).values
    if left.shape[1] > 1:
        close |= (left[:, :-1] - left[:, 1:]).amin(1) < 1e-5
    return close


def _prepare_route(case, gen):
    T, E = case["T"], case["E"]
    dtype = torch.float16 if case["logits"] == "f16" else torch.float32
    drift = torch.randn(E, device="cuda", generator=gen) * 0.5  # some experts are asked for more often
    bias = torch.randn(E, device="cuda", generator=gen) * 0.05 if case["bias"] else None
    logits = (torch.randn((T, E), device="cuda", generator=gen) + drift).to(dtype)
    if case["score"] == "sigmoid":
        for _ in range(20):
            close = _decisions_hang_on_rounding(case, logits, bias)
            logits = torch.where(close[:, None], (torch.randn((T, E), device="cuda", generator=gen) + drift).to(dtype), logits)
    mask = (torch.rand(T, device="cuda", generator=gen) >= case["masked"]).to(torch.uint8) if case["masked"] else None
    s = _State(logits=logits, bias=bias, mask=mask)
    if own:
        import paper_2110_15238_amd as bolt
        s.desc = bolt.moe_route_desc(T, E, case["k"], score=case["score"], groups=case["groups"], top_groups=case["top_groups"],
                                     renormalize=case["renorm"], logits=case["logits"])
        new = lambda *shape, dtype=torch.int32: torch.empty(shape, dtype=dtype, device="cuda")
        s.ids, s.weights = new(T, case["k"]), new(T, case["k"], dtype=torch.float32)
        s.offsets, s.order = new(E + 1), new(T * case["k"])
        s.workspace = new(bolt.bolt_moe_route_workspace_bytes(s.desc), dtype=torch.uint8)
    return s


def _prepare_experts(case, gen):
    T, E, k, D, F = case["T"], case["E"], case["k"], case["width"], case["hidden"]
    U = 2 * F if case["gated"] else F
    # the routing as bolt_moe_route leaves it: choices of unequal popularity, lists by expert
    logits = torch.randn((T, E), device="cuda", generator=gen) + 0.5 * torch.randn(E, device="cuda", generator=gen)
    top = logits.softmax(1).topk(k, dim=1)
    weights, ids = top.values / top.values.sum(1, keepdim=True), top.indices.int()
    if case["masked"]:
        off = torch.rand(T, device="cuda", generator=gen) < case["masked"]
        weights, ids = weights.masked_fill(off[:, None], 0.0), ids.masked_fill(off[:, None], -1)
    by = torch.where(ids < 0, E, ids).view(-1).sort(stable=True)
    order = torch.where(by.values < E, by.indices.int(), -1).contiguous()
    offsets = torch.searchsorted(by.values.int(), torch.arange(E + 1, dtype=torch.int32, device="cuda")).int()
    s = _State(x=_half(gen, T, D), ids=ids.contiguous(), weights=weights.float().contiguous(), offsets=offsets, order=order,
               b_up=_half(gen, E, U, std=0.1) if case["bias"] else None, b_down=_half(gen, E, D, std=0.1) if case["bias"] else None)
    if case["weights"] == "w4":
        s.w_up, s.w_down = _w4_weights(E, U, D, case["group"], False, gen), _w4_weights(E, D, F, case["group"], False, gen)
    else:
        s.w_up, s.w_down = _half(gen, E, U, D, std=1 / math.sqrt(D)), _half(gen, E, D, F, std=1 / math.sqrt(F))
    if own:
        import paper_2110_15238_amd as bolt
        s.desc = bolt.moe_desc(T, E, k, D, F, act=case["act"], gated=case["gated"], weights=case["weights"], group=case["group"])
        s.up, s.down = s.w_up, s.w_down
        if case["weights"] == "w4":
            s.up, s.down = _pack(s.w_up, U, D, case["group"]), _pack(s.w_down, D, F, case["group"])
        s.y = torch.empty((T, D), dtype=torch.float16, device="cuda")
        s.workspace = torch.empty(bolt.bolt_moe_workspace_bytes(s.desc), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"w4": _prepare_w4, "route": _prepare_route, "experts": _prepare_experts}[case["kind"]](case, gen)
    s.case = case
    return s


# ----------------------------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------------------------
def _act(v, act):
    if act == "relu":
        return torch.clamp(v, min=0.0)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "hardswish":
        return v * torch.clamp(v + 3.0, 0.0, 6.0) / 6.0
    if act == "softplus":
        return torch.clamp(v, min=0.0) + torch.log1p(torch.exp(-torch.abs(v)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _plain_weights(w, K, group, e=0):
    q, scales, zeros = w
    v = torch.stack((q[e] & 15, q[e] >> 4), dim=2).view(q.shape[1], K).float()
    z = 8.0 if zeros is None else zeros[e].float().repeat_interleave(group, dim=1)[:, :K]
    return (v - z) * scales[e].float().repeat_interleave(group, dim=1)[:, :K]


def _plain_w4(s):
    c = s.case
    v = s.A.float() @ _plain_weights(s.w, c["K"], c["group"]).t()
    if s.bias is not None:
        v = v + s.bias.float()
    return _act(v, c["act"]).half()


def _plain_route(s):
    c = s.case
    T, E, k, g = c["T"], c["E"], c["k"], c["groups"]
    x = s.logits.float()
    if c["score"] == "softmax":
        score = torch.exp(x - x.amax(1, keepdim=True))
        score = score / score.sum(1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-x))
    key = x if s.bias is None else score + s.bias
    if c["top_groups"] < g:
        by_group = (key if c["score"] == "softmax" else score if s.bias is None else key).view(T, g, E // g)
        value = by_group.sort(dim=2, descending=True).values[:, :, :1 if c["score"] == "softmax" else 2].sum(2)
        best = value.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        keep = torch.zeros((T, g), dtype=torch.bool, device=x.device).scatter_(1, best, True)
        key = torch.where(keep[:, :, None], key.view(T, g, E // g), -math.inf).view(T, E)
    ids = key.sort(dim=1, descending=True, stable=True).indices[:, :k]
    w = torch.gather(score, 1, ids)
    if c["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    if s.mask is not None:
        off = (s.mask == 0)[:, None]
        w, ids = w.masked_fill(off, 0.0), ids.masked_fill(off, -1)
    by = torch.where(ids < 0, E, ids).view(-1).sort(stable=True)
    order = torch.where(by.values < E, by.indices, -1)
    counts = (by.values[None, :] == torch.arange(E, device=x.device)[:, None]).sum(1) if T * k * E <= 1 << 28 else \
        torch.zeros(E + 1, dtype=torch.int64, device=x.device).index_add_(0, by.values, torch.ones_like(by.values))[:E]
    offsets = torch.cat((torch.zeros(1, dtype=torch.int64, device=x.device), counts.cumsum(0)))
    return {"ids": ids.int(), "weights": w, "offsets": offsets.int(), "order": order.int()}


def _plain_experts(s):
    c = s.case
    T, E, k, D, F = c["T"], c["E"], c["k"], c["width"], c["hidden"]
    at = s.offsets.tolist()  # the sizes of the products below
    x = s.x.float()
    rows = torch.zeros((T * k, D), dtype=torch.float32, device=x.device)
    w = s.weights.view(-1, 1)
    for e in range(E):
        if at[e] == at[e + 1]:
            continue
        slots = s.order[at[e]:at[e + 1]].long()
        if c["weights"] == "w4":
            up, down = _plain_weights(s.w_up, D, c["group"], e), _plain_weights(s.w_down, F, c["group"], e)
        else:
            up, down = s.w_up[e].float(), s.w_down[e].float()
        u = x[slots // k] @ up.t()
        if s.b_up is not None:
            u = u + s.b_up[e].float()
        h = _act(u[:, :F], c["act"]) * u[:, F:] if c["gated"] else _act(u, c["act"])
        r = h @ down.t()
        if s.b_down is not None:
            r = r + s.b_down[e].float()
        rows[slots] = r * w[slots]
    return rows.view(T, k, D).sum(1).half()


def run(s):
    kind = s.case["kind"]
    if not own:
        return {"w4": _plain_w4, "route": _plain_route, "experts": _plain_experts}[kind](s)
    import paper_2110_15238_amd as bolt
    if kind == "w4":
        return bolt.bolt_gemm_w4(s.desc, s.A, s.packed, s.bias, s.D, s.workspace)
    if kind == "route":
        bolt.bolt_moe_route(s.desc, s.logits, s.bias, s.mask, s.ids, s.weights, s.offsets, s.order, s.workspace)
        return {"ids": s.ids, "weights": s.weights, "offsets": s.offsets, "order": s.order}
    return bolt.bolt_moe_experts(s.desc, s.x, s.up, s.b_up, s.down, s.b_down, s.ids, s.weights, s.offsets, s.order, s.y, s.workspace)


def work(case):
    if case["kind"] == "w4":
        M, N, K = case["M"], case["N"], case["K"]
        groups = -(-K // case["group"])
        weights = N * K // 2 + N * groups * (3 if case["zeros"] else 2)
        return {"bytes": weights + 2 * M * K + 2 * M * N + (2 * N if case["bias"] else 0), "flops": 2 * M * N * K}
    T, E, k = case["T"], case["E"], case["k"]
    if case["kind"] == "route":
        inputs = T * E * (2 if case["logits"] == "f16" else 4) + (4 * E if case["bias"] else 0) + (T if case["masked"] else 0)
        return {"bytes": inputs + 12 * T * k + 4 * (E + 1), "flops": 8 * T * E}
    D, F, up = case["width"], case["hidden"], 2 if case["gated"] else 1
    on = T * (1.0 - case["masked"])
    asked = E * (1.0 - (1.0 - k / E) ** on)  # experts with a token, if all are asked for equally often
    params = (up + 1) * D * F
    if case["weights"] == "w4":
        one = params // 2 + 2 * (up * F * -(-D // case["group"]) + D * -(-F // case["group"]))
    else:
        one = 2 * params
    if case["bias"]:
        one += 2 * (up * F + D)
    return {"bytes": int(asked * one + 4 * T * D + 12 * T * k + 4 * (E + 1)), "flops": int(2 * on * k * params)}


# ----------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ----------------------------------------------------------------------------------------------------------------
def _exact_act(v, act):
    return {"none": lambda: v, "relu": lambda: torch.relu(v), "gelu": lambda: v * torch.special.ndtr(v),
            "hardswish": lambda: v * torch.relu(v + 3).minimum(torch.full_like(v, 6)) / 6,
            "softplus": lambda: torch.logaddexp(v, torch.zeros_like(v)), "silu": lambda: v * torch.sigmoid(v)}[act]()


def _exact_matrix(w, K, group, e=0):
    q, scales, zeros = w
    N = q.shape[1]
    v = torch.empty((N, K), dtype=torch.float64, device=q.device)
    v[:, 0::2], v[:, 1::2] = (q[e] % 16).double(), (q[e] // 16).double()
    of = torch.arange(K, device=q.device) // group
    return scales[e].double()[:, of] * (v - (8 if zeros is None else zeros[e].double()[:, of]))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "w4":
        v = torch.mm(s.A.double(), _exact_matrix(s.w, case["K"], case["group"]).transpose(0, 1).contiguous())
        return _exact_act(v + (0 if s.bias is None else s.bias.double()), case["act"])
    if case["kind"] == "route":
        T, E, k, g = case["T"], case["E"], case["k"], case["groups"]
        x = s.logits.double()
        score = torch.softmax(x, 1) if case["score"] == "softmax" else torch.sigmoid(x)
        # places by pairwise precedence: a higher key, or the same key at a lower index, goes first
        key = x if s.bias is None else score + s.bias.double()
        if case["top_groups"] < g:
            v = (key if case["score"] == "softmax" else score if s.bias is None else key).reshape(T, g, -1)
            v = v.amax(2) if case["score"] == "softmax" else v.topk(min(2, E // g), dim=2).values.sum(2)
            i = torch.arange(g, device=x.device)
            ahead = ((v[:, None, :] > v[:, :, None]) | ((v[:, None, :] == v[:, :, None]) & (i[None, None, :] < i[None, :, None]))).sum(2)
            key = key.masked_fill((ahead >= case["top_groups"]).repeat_interleave(E // g, dim=1), -math.inf)
        chosen = torch.argsort(-key, dim=1, stable=True)[:, :k]
        w = torch.take_along_dim(score, chosen, 1)
        if case["renorm"]:
            w = w / w.sum(1, keepdim=True)
        if s.mask is not None:
            w = w * (s.mask != 0)[:, None]
        return {"ids": None, "weights": w, "offsets": None, "order": None}
    T, k, D, F = case["T"], case["k"], case["width"], case["hidden"]
    y = torch.zeros((T, D), dtype=torch.float64, device=s.x.device)
    for e in range(case["E"]):
        t, j = (s.ids == e).nonzero(as_tuple=True)
        if not len(t):
            continue
        if case["weights"] == "w4":
            up, down = _exact_matrix(s.w_up, D, case["group"], e), _exact_matrix(s.w_down, F, case["group"], e)
        else:
            up, down = s.w_up[e].double(), s.w_down[e].double()
        u = torch.mm(s.x[t].double(), up.transpose(0, 1).contiguous())
        if s.b_up is not None:
            u += s.b_up[e].double()
        h = _exact_act(u[:, :F], case["act"]) * u[:, F:] if case["gated"] else _exact_act(u, case["act"])
        r = torch.mm(h, down.transpose(0, 1).contiguous())
        if s.b_down is not None:
            r += s.b_down[e].double()
        y.index_add_(0, t, r * s.weights[t, j].double()[:, None])  # (a token's experts differ, so no index comes twice)
    return y
