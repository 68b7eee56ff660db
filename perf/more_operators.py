"""What stands around the shared products of a served language model, as cases that can be timed and compared: the norm in front of a
product, with the residual stream's addition and rows in 8 bits; the linear layer that reads such rows; and a projection shared by requests
that each bring a low-rank adapter.

Kinds of cases and what they stand for:
  norm  root-mean-square norm of x + residual: the new residual stream, the normed rows in FP16, in 8 bits (E4M3) with a scale per row, or both
  q8    a linear layer whose activations and weights are held in 8 bits, with a scale for every row of either
  lora  a linear layer, FP16 or 4-bit weights, plus scale * (x . down^T) . up^T of the adapter that each row's request names, if any

With `own` false, `run` computes a case with elementary torch operations in 32 bits; with `own` true it calls the library.
"""
import math

import torch

own = False

ACTS = ("none", "relu", "gelu", "hardswish", "softplus")
MOST_Q8 = 448.0  # the largest E4M3


def listed():
    return [
        # One decoded token between two layers: latency.
        dict(name="norm_one_token", kind="norm", rows=1, width=4096, residual=True, y=True, q=False, offset=0.0),
        # A decode batch in front of an 8-bit projection that has adapters too: both forms of the rows; a width that is no power of two.
        dict(name="norm_batch_both", kind="norm", rows=133, width=12296, residual=True, y=True, q=True, offset=1.0),
        # A prompt in front of an 8-bit projection.
        dict(name="norm_prompt_q8", kind="norm", rows=4099, width=5120, residual=True, y=False, q=True, offset=0.0),
        # A large prefill batch, the residual stream read and written once: bound by memory.
        dict(name="norm_many", kind="norm", rows=32768, width=4096, residual=True, y=True, q=False, offset=0.0),
        # One token through a square projection: 17 MB of weights and the launch.
        dict(name="q8_one_token", kind="q8", M=1, N=4096, K=4096, bias=False, act="none"),
        # A decode batch through an MLP's first half; sizes that are no multiples of a tile.
        dict(name="q8_batch", kind="q8", M=45, N=6152, K=5008, bias=True, act="gelu"),
        # A short prompt through an MLP's second half: a long reduction, few tiles.
        dict(name="q8_short_prompt", kind="q8", M=333, N=4096, K=11008, bias=False, act="none"),
        # A prompt: bound by the matrix cores.
        dict(name="q8_prompt", kind="q8", M=4096, N=8192, K=4096, bias=True, act="relu"),
        # One token of one request.
        dict(name="lora_one_token", kind="lora", M=1, N=4096, K=4096, weights="f16", group=0, adapters=8, rank=16, runs=False, without=0.0,
             bias=False, act="none"),
        # A decode batch, every row another request, some without an adapter; 4-bit weights, odd sizes.
        dict(name="lora_decode_w4", kind="lora", M=29, N=6152, K=5000, weights="w4", group=64, adapters=32, rank=32, runs=False, without=0.1,
             bias=True, act="gelu"),
        # Prompts of several requests in one batch, rows of a request one behind the other.
        dict(name="lora_mixed", kind="lora", M=700, N=4104, K=4096, weights="f16", group=0, adapters=6, rank=24, runs=True, without=0.2,
             bias=True, act="none"),
        # A large prefill batch of a few requests: the largest, bound by the matrix cores.
        dict(name="lora_prompt", kind="lora", M=4096, N=8192, K=4096, weights="f16", group=0, adapters=4, rank=64, runs=True, without=0.0,
             bias=False, act="none"),
    ]


# ----------------------------------------------------------------------------------------------------------------
# draws from the same ranges
# ----------------------------------------------------------------------------------------------------------------
def _log(rng, lo, hi, step=1):
    """An integer in [lo, hi], its logarithm uniform, rounded to a multiple of `step`."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(("norm", "q8", "lora"))
    while True:
        if kind == "norm":
            y, q = rng.choice(((True, False), (False, True), (True, True)))
            case = dict(kind=kind, rows=_log(rng, 1, 32768), width=_log(rng, 64, 16384, 8), residual=rng.random() < 0.7, y=y, q=q,
                        offset=rng.choice((0.0, 1.0)))
            if case["rows"] * case["width"] <= 24000 * 4096:
                return case
            continue
        M, N = _log(rng, 1, 4096), _log(rng, 256, 12288, 8)
        bias, act = rng.random() < 0.5, rng.choice(ACTS)
        if kind == "q8":
            case = dict(kind=kind, M=M, N=N, K=_log(rng, 256, 12288, 16), bias=bias, act=act)
        else:
            w4 = rng.random() < 0.4
            case = dict(kind=kind, M=M, N=N, K=_log(rng, 256, 12288, 8), weights="w4" if w4 else "f16",
                        group=rng.choice((32, 64, 128)) if w4 else 0, adapters=_log(rng, 1, 64), rank=_log(rng, 8, 128, 8),
                        runs=M > 64 or rng.random() < 0.2, without=rng.choice((0.0, 0.0, 0.2)), bias=bias, act=act)
            if case["adapters"] * case["rank"] * M > 256 * 4096:
                continue
        if M * N * case["K"] <= 4000 * 8192 * 4096 and N * case["K"] <= 64 << 20:
            return case


# ----------------------------------------------------------------------------------------------------------------
# what a program has in hand before the call
# ----------------------------------------------------------------------------------------------------------------
class _State:
    def __init__(self, **kw):
        self.__dict__.update(kw)


def _half(gen, *shape, std=1.0):
    t = torch.empty(shape, dtype=torch.float16, device="cuda")
    return t.normal_(0.0, std, generator=gen)


def _empty(*shape, dtype=torch.float16):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _prepare_norm(case, gen):
    rows, width = case["rows"], case["width"]
    # a residual stream: some channels are much larger than the others
    loud = torch.where(torch.rand(width, device="cuda", generator=gen) < 0.01, 12.0, 1.0).half()
    x, residual = _half(gen, rows, width, std=0.5), _half(gen, rows, width, std=2.0).mul_(loud) if case["residual"] else None
    s = _State(x=x, residual=residual, weight=_half(gen, width, std=0.2).add_(1.0 - case["offset"]), eps=1e-5)
    if own:
        import paper_2110_15238_amd as bolt
        s.desc = bolt.rms_norm_desc(rows, width, eps=s.eps, weight_offset=case["offset"])
        s.sum = _empty(rows, width) if case["residual"] else None
        s.y = _empty(rows, width) if case["y"] else None
        s.q = _empty(rows, width, dtype=torch.float8_e4m3fn) if case["q"] else None
        s.scales = _empty(rows, dtype=torch.float32) if case["q"] else None
    return s


def _rows_in_8_bits(gen, rows, width, std):
    """Rows as a quantiser leaves them: the largest value of a row is the type's largest."""
    v = torch.empty((rows, width), dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen)
    scale = v.abs().amax(1) / MOST_Q8
    return (v / scale[:, None]).clamp(-MOST_Q8, MOST_Q8).to(torch.float8_e4m3fn), scale


def _prepare_q8(case, gen):
    M, N, K = case["M"], case["N"], case["K"]
    A, a_scales = _rows_in_8_bits(gen, M, K, 1.0)
    W, w_scales = _rows_in_8_bits(gen, N, K, 1 / math.sqrt(K))
    s = _State(A=A, a_scales=a_scales, W=W, w_scales=w_scales, bias=_half(gen, N) if case["bias"] else None)
    if own:
        import paper_2110_15238_amd as bolt
        s.desc = bolt.gemm_q8_desc(M, N, K, act=case["act"])
        s.D = _empty(M, N)
        s.workspace = _empty(bolt.bolt_gemm_q8_workspace_bytes(s.desc), dtype=torch.uint8)
    return s


def _w4_weights(N, K, group, gen):
    """4-bit weights as a quantiser leaves them: two to a byte (even k in the low half), a scale per group, zero point 8."""
    q = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda", generator=gen)
    return q, ((torch.rand((N, -(-K // group)), device="cuda", generator=gen) + 0.5) * (0.2 / math.sqrt(K))).half()


def _prepare_lora(case, gen):
    M, N, K, n, rank = case["M"], case["N"], case["K"], case["adapters"], case["rank"]
    ids = torch.randint(0, n, (M,), dtype=torch.int32, device="cuda", generator=gen)
    if case["runs"]:
        # requests of unequal length, one behind the other
        ends = torch.rand(n, device="cuda", generator=gen).cumsum(0)
        ids = torch.searchsorted(ends / ends[-1] * M, torch.arange(M, device="cuda") + 0.5).clamp(max=n - 1).int()
        off = torch.rand(n, device="cuda", generator=gen)[ids.long()] < case["without"]
    else:
        off = torch.rand(M, device="cuda", generator=gen) < case["without"]
    s = _State(A=_half(gen, M, K), ids=ids.masked_fill(off, -1), down=_half(gen, n, rank, K, std=1 / math.sqrt(K)),
               up=_half(gen, n, N, rank, std=0.2 / math.sqrt(rank)), scales=torch.rand(n, device="cuda", generator=gen) + 0.5,
               bias=_half(gen, N) if case["bias"] else None)
    s.W = _w4_weights(N, K, case["group"], gen) if case["weights"] == "w4" else _half(gen, N, K, std=1 / math.sqrt(K))
    if own:
        import paper_2110_15238_amd as bolt
        s.desc = bolt.gemm_lora_desc(M, N, K, n, rank, weights=case["weights"], group=case["group"], act=case["act"])
        s.weights = s.W
        if case["weights"] == "w4":
            s.weights = _empty(bolt.bolt_w4_packed_bytes(N, K, case["group"], 1), dtype=torch.uint8)
            bolt.bolt_w4_pack(N, K, case["group"], *s.W, None, s.weights)
        s.D = _empty(M, N)
        s.workspace = _empty(bolt.bolt_gemm_lora_workspace_bytes(s.desc), dtype=torch.uint8)
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"norm": _prepare_norm, "q8": _prepare_q8, "lora": _prepare_lora}[case["kind"]](case, gen)
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
    return v


def _norm_outputs(case, sum_, y, q, scales):
    """What a case asks for: the new residual stream where there is one, FP16 rows, 8-bit rows with their scales."""
    out = {}
    if case["residual"]:
        out["sum"] = sum_
    if case["y"]:
        out["y"] = y
    if case["q"]:
        out["q"], out["scales"] = q, scales
    return out


def _plain_norm(s):
    c = s.case
    v = s.x.float()
    if s.residual is not None:
        v = v + s.residual.float()
    n = v * torch.rsqrt((v * v).mean(1, keepdim=True) + s.eps) * (s.weight.float() + c["offset"])
    q = scales = None
    if c["q"]:
        scales = n.abs().amax(1) / MOST_Q8
        q = torch.where(scales[:, None] > 0, n / scales[:, None], 0.0).clamp(-MOST_Q8, MOST_Q8).to(torch.float8_e4m3fn)
    return _norm_outputs(c, v.half() if c["residual"] else None, n.half() if c["y"] else None, q, scales)


def _plain_q8(s):
    v = (s.A.float() @ s.W.float().t()) * s.a_scales[:, None] * s.w_scales[None, :]
    if s.bias is not None:
        v = v + s.bias.float()
    return _act(v, s.case["act"]).half()


def _plain_lora(s):
    c = s.case
    M, N, K, n, rank = c["M"], c["N"], c["K"], c["adapters"], c["rank"]
    x = s.A.float()
    if c["weights"] == "w4":
        q, scales = s.W
        w = torch.stack((q & 15, q >> 4), dim=2).view(N, K).float() - 8.0
        w = w * scales.float().repeat_interleave(c["group"], dim=1)[:, :K]
    else:
        w = s.W.float()
    # every row through every adapter, all but its own times zero
    mine = torch.where(s.ids[:, None] == torch.arange(n, device=x.device)[None, :], s.scales[None, :], 0.0)
    h = (x @ s.down.float().view(n * rank, K).t()).view(M, n, rank) * mine[:, :, None]
    v = x @ w.t() + h.view(M, n * rank) @ s.up.float().transpose(1, 2).reshape(n * rank, N)
    if s.bias is not None:
        v = v + s.bias.float()
    return _act(v, c["act"]).half()


def run(s):
    kind = s.case["kind"]
    if not own:
        return {"norm": _plain_norm, "q8": _plain_q8, "lora": _plain_lora}[kind](s)
    import paper_2110_15238_amd as bolt
    if kind == "norm":
        bolt.bolt_rms_norm(s.desc, s.x, s.residual, s.weight, s.sum, s.y, s.q, s.scales)
        return _norm_outputs(s.case, s.sum, s.y, s.q, s.scales)
    if kind == "q8":
        return bolt.bolt_gemm_q8(s.desc, s.A, s.a_scales, s.W, s.w_scales, s.bias, s.D, s.workspace)
    return bolt.bolt_gemm_lora(s.desc, s.A, s.weights, s.bias, s.ids, s.down, s.up, s.scales, s.D, s.workspace)


def work(case):
    if case["kind"] == "norm":
        rows, width = case["rows"], case["width"]
        each = 2 + (4 if case["residual"] else 0) + (2 if case["y"] else 0) + (1 if case["q"] else 0)
        return {"bytes": rows * width * each + 2 * width + (4 * rows if case["q"] else 0), "flops": rows * width * 6}
    M, N, K = case["M"], case["N"], case["K"]
    bias = 2 * N if case["bias"] else 0
    if case["kind"] == "q8":
        return {"bytes": N * K + M * K + 2 * M * N + 4 * (M + N) + bias, "flops": 2 * M * N * K}
    weights = N * K // 2 + 2 * N * -(-K // case["group"]) if case["weights"] == "w4" else 2 * N * K
    n, on = case["adapters"], M * (1.0 - case["without"])
    asked = n * (1.0 - case["without"]) if case["runs"] else n * (1.0 - (1.0 - 1.0 / n) ** on)  # adapters with a row
    return {"bytes": int(weights + 2 * M * K + 2 * M * N + 4 * (M + n) + bias + asked * 2 * case["rank"] * (K + N)),
            "flops": int(2 * M * N * K + 2 * on * case["rank"] * (K + N))}


# ----------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ----------------------------------------------------------------------------------------------------------------
def _exact_act(v, act):
    return {"none": lambda: v, "relu": lambda: torch.relu(v), "gelu": lambda: v * torch.special.ndtr(v),
            "hardswish": lambda: v * torch.relu(v + 3).minimum(torch.full_like(v, 6)) / 6,
            "softplus": lambda: torch.logaddexp(v, torch.zeros_like(v))}[act]()


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        v = s.x.double() if s.residual is None else torch.add(s.x.double(), s.residual.double())
        length = torch.linalg.vector_norm(v, dim=1, keepdim=True)
        n = v / torch.sqrt(length ** 2 / case["width"] + s.eps) * (case["offset"] + s.weight.double())
        largest = torch.linalg.vector_norm(n, ord=math.inf, dim=1)
        return _norm_outputs(case, v, n, n * (MOST_Q8 / largest)[:, None], largest / MOST_Q8)
    bias = 0 if s.bias is None else s.bias.double()
    if case["kind"] == "q8":
        A, W = s.A.double() * s.a_scales.double()[:, None], s.W.double() * s.w_scales.double()[:, None]
        return _exact_act(torch.mm(A, W.transpose(0, 1).contiguous()) + bias, case["act"])
    x = s.A.double()
    if case["weights"] == "w4":
        q, scales = s.W
        of = torch.arange(case["K"], device=q.device) // case["group"]
        w = torch.empty((case["N"], case["K"]), dtype=torch.float64, device=q.device)
        w[:, 0::2], w[:, 1::2] = (q % 16).double(), (q // 16).double()
        w = scales.double()[:, of] * (w - 8)
    else:
        w = s.W.double()
    v = torch.mm(x, w.transpose(0, 1).contiguous())
    for a in range(case["adapters"]):
        rows = (s.ids == a).nonzero().view(-1)
        if len(rows):
            h = torch.mm(x[rows], s.down[a].double().transpose(0, 1).contiguous())
            v.index_add_(0, rows, torch.mm(h, s.up[a].double().transpose(0, 1).contiguous()) * s.scales[a].double())
    return _exact_act(v + bias, case["act"])
