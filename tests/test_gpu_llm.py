"""GPU: the 4-bit layer, the routing and the experts' products against 64-bit references.  Bounds follow from the lengths of the FP32 sums
and the stated roundings (tests/llm_ref.py); with small integers every sum is exact and results have to be equal."""
import math

import pytest

import llm_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def bolt():
    import paper_2110_15238_amd as b
    return b


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _half(g, *shape, std=1.0):
    return torch.empty(shape, dtype=torch.float16, device="cuda").normal_(0.0, std, generator=g)


def _w4(bolt, g, count, N, K, group, zeros=False, ones=False):
    """q, scales, zeros as the caller has them, and the packed form."""
    groups = -(-K // group)
    q = torch.randint(0, 256, (count, N, K // 2), dtype=torch.uint8, device="cuda", generator=g)
    s = torch.ones(count, N, groups, dtype=torch.float16, device="cuda") if ones else \
        ((torch.rand((count, N, groups), device="cuda", generator=g) + 0.1) * (0.4 / math.sqrt(K))).half()
    z = torch.randint(0, 16, (count, N, groups), dtype=torch.uint8, device="cuda", generator=g) if zeros else None
    packed = torch.full((bolt.bolt_w4_packed_bytes(N, K, group, count),), 0xff, dtype=torch.uint8, device="cuda")
    bolt.bolt_w4_pack(N, K, group, q, s, z, packed)
    return (q, s, z), packed


def _matrix(raw, group, e=0):
    q, s, z = raw
    return ref.w4_matrix(q[e], s[e], None if z is None else z[e], group)


def _within(got, want, bound, what=""):
    err = (got.double() - want).abs()
    assert torch.isfinite(got.double()).all(), what
    worst = (err - bound).max().item() if err.numel() else 0.0
    assert worst <= 0.0, (what, worst, (err / bound).max().item())


# ---- 4-bit layer ----------------------------------------------------------------------------------------------------------
# M on both sides of every kernel's rows; K: one chunk, a short step, whole steps, a short group, more steps than are held in registers
W4 = [(1, 8, 8, 32), (1, 24, 128, 128), (2, 40, 136, 64), (5, 72, 120, 32), (16, 264, 1000, 128), (16, 136, 1032, 64), (13, 200, 4104, 32),
      (7, 16, 4104, 128), (17, 8, 8, 64), (17, 264, 520, 32), (33, 136, 1032, 128), (64, 4104, 264, 64), (100, 1000, 2056, 128), (129, 520, 392, 32),
      (300, 2056, 136, 64), (513, 1032, 1000, 128), (700, 72, 4104, 32)]


@pytest.mark.parametrize("M,N,K,group", W4)
@pytest.mark.parametrize("zeros,act", [(False, "none"), (True, "silu")])
def test_gemm_w4(bolt, M, N, K, group, zeros, act):
    g = _gen(M * 7 + N)
    raw, packed = _w4(bolt, g, 1, N, K, group, zeros)
    A, bias = _half(g, M, K), _half(g, N) if zeros else None
    d = bolt.gemm_w4_desc(M, N, K, group, act=act, alpha=0.75 if zeros else 1.0, beta=-1.5)
    ws = torch.empty(bolt.bolt_gemm_w4_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    D = bolt.bolt_gemm_w4(d, A, packed, bias, torch.full((M, N), float("nan"), dtype=torch.float16, device="cuda"), ws)
    want, bound = ref.linear(A.double(), _matrix(raw, group), None if bias is None else bias.double(), act, d.alpha, d.beta)
    _within(D, want, bound)


@pytest.mark.parametrize("act", ["relu", "gelu", "hardswish", "softplus"])
@pytest.mark.parametrize("M", [3, 40])
def test_gemm_w4_activations(bolt, M, act):
    g = _gen(M)
    raw, packed = _w4(bolt, g, 1, 136, 264, 64)
    A, bias = _half(g, M, 264, std=3.0), _half(g, 136)
    d = bolt.gemm_w4_desc(M, 136, 264, 64, act=act)
    D = bolt.bolt_gemm_w4(d, A, packed, bias, torch.empty((M, 136), dtype=torch.float16, device="cuda"))
    _within(D, *ref.linear(A.double(), _matrix(raw, 64), bias.double(), act))


@pytest.mark.parametrize("act", ["none", "silu"])
def test_gemm_w4_unpacked(bolt, act):
    """So many rows that the weights are unpacked: each is rounded to binary16, half an ulp relative."""
    M, N, K = 4096, 8192, 1032
    d = bolt.gemm_w4_desc(M, N, K, 32, act=act, alpha=0.5)
    need = bolt.bolt_gemm_w4_workspace_bytes(d)
    assert need == N * K * 2
    g = _gen(5)
    raw, packed = _w4(bolt, g, 1, N, K, 32, True)
    A, bias = _half(g, M, K), _half(g, N)
    D = bolt.bolt_gemm_w4(d, A, packed, bias, torch.empty((M, N), dtype=torch.float16, device="cuda"),
                          torch.empty(need, dtype=torch.uint8, device="cuda"))
    _within(D, *ref.linear(A.double(), _matrix(raw, 32), bias.double(), act, 0.5, shift=ref.U16))


def test_gemm_w4_unpacked_takes_alpha_zero(bolt):
    M, N, K = 4096, 8192, 520
    d = bolt.gemm_w4_desc(M, N, K, 32, act="silu", alpha=0.0, beta=2.0)
    g = _gen(6)
    raw, packed = _w4(bolt, g, 1, N, K, 32)
    bias = _half(g, N)
    D = bolt.bolt_gemm_w4(d, _half(g, M, K), packed, bias, torch.empty((M, N), dtype=torch.float16, device="cuda"),
                          torch.empty(bolt.bolt_gemm_w4_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    want = ref.act(2.0 * bias.double(), "silu")
    _within(D, want.expand(M, N), (want.abs() * (ref.CLOSE + ref.U16) + ref.TINY).expand(M, N))


@pytest.mark.parametrize("M,N,K,group", [(1, 24, 40, 32), (16, 136, 264, 64), (17, 72, 136, 128), (65, 264, 72, 32), (200, 40, 264, 64)])
def test_gemm_w4_is_exact_on_integers(bolt, M, N, K, group):
    """Small integers: every product and sum is exact, so a value in a wrong place or a lost column shows."""
    g = _gen(M + K)
    raw, packed = _w4(bolt, g, 1, N, K, group, True, ones=True)
    A = torch.randint(-1, 2, (M, K), device="cuda", generator=g).half()
    D = bolt.bolt_gemm_w4(bolt.gemm_w4_desc(M, N, K, group), A, packed, None, torch.empty((M, N), dtype=torch.float16, device="cuda"))
    want = A.double() @ _matrix(raw, group).t().contiguous()
    assert want.abs().max() <= 2048 and torch.equal(D.double(), want)


@pytest.mark.parametrize("M", [4, 33, 300])
def test_gemm_w4_strides_and_untouched_padding(bolt, M):
    N, K, lda, ldd = 72, 200, 264, 136
    g = _gen(M)
    raw, packed = _w4(bolt, g, 1, N, K, 64)
    A = torch.full((M, lda), float("nan"), dtype=torch.float16, device="cuda")
    A[:, :K] = _half(g, M, K)
    D = torch.full((M, ldd), 7.0, dtype=torch.float16, device="cuda")
    bolt.bolt_gemm_w4(bolt.gemm_w4_desc(M, N, K, 64, lda=lda, ldd=ldd), A, packed, None, D)
    _within(D[:, :N], *ref.linear(A[:, :K].double(), _matrix(raw, 64), None, "none"))
    assert (D[:, N:] == 7.0).all()


@pytest.mark.parametrize("M", [9, 40, 200])
def test_gemm_w4_rows_do_not_meet(bolt, M):
    """A row of infinities and NaN spoils its own results only."""
    N, K = 136, 264
    g = _gen(M)
    raw, packed = _w4(bolt, g, 1, N, K, 128)
    A = _half(g, M, K)
    clean = A.clone()
    A[3, 5], A[3, 100], A[M - 1, 0] = float("inf"), float("nan"), float("-inf")
    run = lambda a: bolt.bolt_gemm_w4(bolt.gemm_w4_desc(M, N, K, 128), a, packed, None, torch.empty((M, N), dtype=torch.float16, device="cuda"))
    got, want = run(A), run(clean)
    others = [i for i in range(M) if i not in (3, M - 1)]
    assert torch.equal(got[others], want[others]) and not torch.isfinite(got[3]).any()


def test_gemm_w4_without_rows(bolt):
    _, packed = _w4(bolt, _gen(0), 1, 16, 128, 128)
    D = torch.full((1, 16), 3.0, dtype=torch.float16, device="cuda")
    bolt.bolt_gemm_w4(bolt.gemm_w4_desc(0, 16, 128, 128), D, packed, None, D)
    assert (D == 3.0).all()


# ---- routing ------------------------------------------------------------------------------------------------------------------
def _route(bolt, logits, k, bias=None, mask=None, score="softmax", groups=1, top_groups=1, renormalize=True, scale=1.0, ld=None):
    T, E = logits.shape
    ld = E if ld is None else ld
    held = torch.full((max(T, 1), ld), float("nan"), dtype=logits.dtype, device="cuda")
    held[:T, :E] = logits.cuda()
    d = bolt.moe_route_desc(T, E, k, score=score, groups=groups, top_groups=top_groups, renormalize=renormalize, scale=scale,
                            logits="f16" if logits.dtype is torch.float16 else "f32", ld=ld)
    new = lambda *s, dtype=torch.int32: torch.full(s, -7, dtype=dtype, device="cuda")
    out = new(T, k), new(T, k, dtype=torch.float32), new(E + 1), new(T * k)
    bolt.bolt_moe_route(d, held, None if bias is None else bias.cuda(), None if mask is None else mask.cuda(), *out,
                        torch.empty(bolt.bolt_moe_route_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    ids, w, offsets, order = (t.cpu() for t in out)
    want_ids, want_w, gap = ref.route(logits, bias, mask, k, score, groups, top_groups, renormalize, scale)
    return ids, w, offsets, order, want_ids, want_w, gap


def _check_route(got, E, exact_keys):
    """exact_keys: keys are logits, so ties are ties; else tokens whose places hang on 1e-5 are left out of the comparison of ids."""
    ids, w, offsets, order, want_ids, want_w, gap = got
    sure = torch.ones_like(gap, dtype=torch.bool) if exact_keys else gap > 1e-5
    assert sure.float().mean() > 0.5 or not len(sure)
    assert torch.equal(ids[sure], want_ids[sure])
    # a score is an exponential (4 units in the last place), a sum over E and two quotients
    err = (w[sure].double() - want_w[sure]).abs()
    assert (err <= want_w[sure].abs() * (E + 16) * ref.U32 + 1e-37).all()
    o, r = ref.lists(ids, E)
    assert torch.equal(offsets, o) and torch.equal(order, r)


@pytest.mark.parametrize("T", [0, 1, 2, 63, 256, 257, 1030, 9000])
@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (63, 5), (64, 8), (65, 1), (128, 4), (200, 16), (512, 10)])
def test_route_softmax(bolt, T, E, k):
    """FP16 logits: many equal ones, which go by the lower index."""
    if T == 9000 and E not in (64, 200):
        pytest.skip("one width on either side is enough")
    g = torch.Generator().manual_seed(T + E)
    logits = (torch.randn(T, E, generator=g) * 2).half()
    logits[:, ::3] = (logits[:, ::3] * 2).round() / 2
    mask = (torch.rand(T, generator=g) > 0.2).to(torch.uint8) if T % 2 else None
    _check_route(_route(bolt, logits, k, mask=mask, renormalize=E % 2 == 0, scale=2.5, ld=E + (3 if E % 2 else 0)), E, True)


@pytest.mark.parametrize("T", [1, 37, 300, 8200])
@pytest.mark.parametrize("E,k,groups,top_groups", [(64, 6, 1, 1), (256, 8, 8, 4), (160, 6, 16, 3), (48, 2, 4, 1), (16, 3, 16, 5), (510, 9, 2, 1)])
@pytest.mark.parametrize("biased", [True, False])
def test_route_sigmoid(bolt, T, E, k, groups, top_groups, biased):
    g = torch.Generator().manual_seed(T * E)
    logits = torch.randn(T, E, generator=g) * 1.5
    bias = torch.randn(E, generator=g) * 0.1 if biased else None
    got = _route(bolt, logits, k, bias=bias, score="sigmoid", groups=groups, top_groups=top_groups, renormalize=T != 37, scale=0.5)
    _check_route(got, E, False)


@pytest.mark.parametrize("T", [16, 17, 48, 49, 64, 65])
@pytest.mark.parametrize("E,k,groups,top_groups", [(28, 4, 1, 1), (256, 16, 16, 9), (256, 16, 1, 1), (352, 5, 1, 1), (512, 10, 8, 4)])
@pytest.mark.parametrize("half", [True, False])
def test_route_around_the_kernels_limits(bolt, T, E, k, groups, top_groups, half):
    """The numbers of tokens at which lanes per token and launches change; 64 tokens of 16 slots fill what a workgroup keeps."""
    g = torch.Generator().manual_seed(T * E + groups)
    logits = torch.randn(T, E, generator=g) * 1.5
    mask = (torch.rand(T, generator=g) > 0.2).to(torch.uint8) if T % 2 else None
    if half:
        return _check_route(_route(bolt, logits.half(), k, mask=mask, groups=groups, top_groups=top_groups), E, True)
    bias = torch.randn(E, generator=g) * 0.1
    _check_route(_route(bolt, logits, k, bias=bias, mask=mask, score="sigmoid", groups=groups, top_groups=top_groups), E, False)


@pytest.mark.parametrize("T", [5, 700])
@pytest.mark.parametrize("biased", [True, False])
def test_route_softmax_groups(bolt, T, biased):
    g = torch.Generator().manual_seed(T)
    logits = torch.randn(T, 96, generator=g)
    bias = torch.rand(96, generator=g) * 0.05 if biased else None
    _check_route(_route(bolt, logits, 4, bias=bias, groups=6, top_groups=2, renormalize=False), 96, False)


@pytest.mark.parametrize("T", [6, 300])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_rows_of_nothing(bolt, T, score):
    """Rows of minus infinity, of the type's lowest value, of NaN, with one live expert, with plus infinity: a choice and finite weights."""
    E, inf = 40, float("inf")
    logits = torch.randn(T, E, generator=torch.Generator().manual_seed(1))
    logits[0], logits[1], logits[2] = -inf, torch.finfo(torch.float32).min, float("nan")
    logits[3] = -inf
    logits[3, 17] = 0.25
    logits[4, 9], logits[4, 30] = inf, inf
    logits[5, ::2] = float("nan")
    ids, w, offsets, order, want_ids, want_w, _ = _route(bolt, logits, 3, score=score)
    assert torch.equal(ids, want_ids) and torch.isfinite(w).all()
    assert (w.double() - want_w).abs().max() <= 1e-5
    assert ids[0].tolist() == [0, 1, 2] and ids[2].tolist() == [0, 1, 2] and ids[3].tolist() == [17, 0, 1] and ids[4, :2].tolist() == [9, 30]
    o, r = ref.lists(ids, E)
    assert torch.equal(offsets, o) and torch.equal(order, r)


@pytest.mark.parametrize("T", [3, 400])
def test_route_without_any_token(bolt, T):
    got = _route(bolt, torch.randn(T, 32), 4, mask=torch.zeros(T, dtype=torch.uint8))
    assert (got[0] == -1).all() and (got[1] == 0).all() and (got[2] == 0).all() and (got[3] == -1).all()


def test_route_everything_to_one_expert(bolt):
    logits = torch.zeros(3000, 128)
    logits[:, 77] = 5.0
    _check_route(_route(bolt, logits, 1), 128, True)


# ---- experts ------------------------------------------------------------------------------------------------------------------
def _routed(g, T, E, k, off=0.0, skew=0.0, only=None):
    """ids, weights, offsets, order on the GPU; skew: how unequal the experts are asked for; only: all first places go to this expert."""
    logits = torch.randn((T, E), device="cuda", generator=g) + skew * torch.randn(E, device="cuda", generator=g)
    if only is not None:
        logits[:, only] = 100.0
    top = logits.topk(k, dim=1)
    weights, ids = torch.softmax(top.values / 4, 1), top.indices.int()
    if off:
        gone = torch.rand(T, device="cuda", generator=g) < off
        ids, weights = ids.masked_fill(gone[:, None], -1), weights.masked_fill(gone[:, None], 0.0)
    offsets, order = ref.lists(ids, E)
    return ids.contiguous(), weights.contiguous(), offsets.cuda(), order.cuda()


def _run_experts(bolt, T, E, k, D, F, act, gated, kind, group=64, bias=False, off=0.0, skew=0.0, only=None, seed=0, ldx=None, ldy=None):
    g = _gen(seed + T * 31 + E)
    U = 2 * F if gated else F
    plan = _routed(g, T, E, k, off, skew, only)
    ldx, ldy = ldx or D, ldy or D
    x = torch.full((T, ldx), float("nan"), dtype=torch.float16, device="cuda")
    x[:, :D] = _half(g, T, D)
    bu, bd = (_half(g, E, U, std=0.5), _half(g, E, D, std=0.5)) if bias else (None, None)
    if kind == "w4":
        raw_u, up = _w4(bolt, g, E, U, D, group, True)
        raw_d, down = _w4(bolt, g, E, D, F, group, False)
        ups, downs = (lambda e: _matrix(raw_u, group, e)), (lambda e: _matrix(raw_d, group, e))
    else:
        up, down = _half(g, E, U, D, std=1 / math.sqrt(D)), _half(g, E, D, F, std=1 / math.sqrt(F))
        ups, downs = (lambda e: up[e].double()), (lambda e: down[e].double())
    d = bolt.moe_desc(T, E, k, D, F, act=act, gated=gated, weights=kind, group=group, ldx=ldx, ldy=ldy)
    y = torch.full((T, ldy), 7.0, dtype=torch.float16, device="cuda")
    # the workspace starts as NaN: nothing may come from where no row was written
    ws = torch.full((bolt.bolt_moe_workspace_bytes(d) // 2,), float("nan"), dtype=torch.float16, device="cuda")
    bolt.bolt_moe_experts(d, x, up, bu, down, bd, *plan, y, ws)
    want, bound = ref.experts(x[:, :D], ups, bu, downs, bd, plan[0], plan[1], act, gated)
    _within(y[:, :D], want, bound, (T, E, k, D, F, act, gated, kind))
    assert (y[:, D:] == 7.0).all()
    return plan, y


# few rows; some ten with few and many workgroups; 64-, 128- and 256-row tiles; short last blocks; reductions of one chunk, of odd lengths
EXPERTS = [(1, 1, 1, 8, 8), (1, 8, 2, 264, 136), (3, 4, 4, 1032, 72), (20, 16, 4, 520, 264), (7, 70, 5, 136, 2056), (40, 4, 2, 264, 520), (33, 2, 2, 1000, 136),
           (150, 4, 2, 520, 136), (200, 64, 8, 264, 72), (400, 8, 2, 392, 1000), (600, 3, 2, 264, 264), (1500, 4, 2, 136, 72)]


@pytest.mark.parametrize("T,E,k,D,F", EXPERTS)
@pytest.mark.parametrize("gated,act,bias,off", [(True, "silu", False, 0.0), (False, "gelu", True, 0.3)])
@pytest.mark.parametrize("kind,group", [("f16", 0), ("w4", 32), ("w4", 64), ("w4", 128)])
def test_experts(bolt, T, E, k, D, F, gated, act, bias, off, kind, group):
    _run_experts(bolt, T, E, k, D, F, act, gated, kind, group, bias, off, skew=1.0)


@pytest.mark.parametrize("T,E,k,D,F", [(900, 4, 2, 2056, 1032), (1300, 6, 3, 1032, 2056), (2100, 4, 1, 4104, 520)])
@pytest.mark.parametrize("gated,bias", [(True, True), (False, False)])
@pytest.mark.parametrize("kind", ["f16", "w4"])
def test_experts_many_rows(bolt, T, E, k, D, F, gated, bias, kind):
    """Enough rows and columns for the 256 x 256 (FP16) and 128 x 256 (4 bits) tiles, in several rounds."""
    _run_experts(bolt, T, E, k, D, F, "relu", gated, kind, 128, bias, 0.1, skew=0.5)


@pytest.mark.parametrize("T", [30, 500])
@pytest.mark.parametrize("kind", ["f16", "w4"])
def test_experts_all_to_one(bolt, T, kind):
    _run_experts(bolt, T, 16, 1, 264, 136, "hardswish", True, kind, 64, True, only=11)


@pytest.mark.parametrize("T", [3, 90, 700])
@pytest.mark.parametrize("kind", ["f16", "w4"])
def test_experts_strides(bolt, T, kind):
    _run_experts(bolt, T, 4, 2, 136, 264, "softplus", False, kind, 32, ldx=200, ldy=264)


@pytest.mark.parametrize("T", [5, 80, 600])
@pytest.mark.parametrize("kind", ["f16", "w4"])
def test_experts_without_any_token(bolt, T, kind):
    _, y = _run_experts(bolt, T, 4, 2, 72, 136, "silu", True, kind, 64, True, off=2.0)
    assert (y == 0).all()


@pytest.mark.parametrize("T,E", [(2, 6), (40, 3), (300, 5), (1200, 3)])
def test_experts_are_exact_on_integers(bolt, T, E):
    """Integers and powers of two: no rounding anywhere, so a row in a wrong place or added twice shows."""
    g = _gen(T)
    D, F, k = 264, 136, 2
    ids, weights, offsets, order = _routed(g, T, E, k, 0.1, 1.0)
    weights = torch.where(ids < 0, 0.0, torch.tensor([1.0, 2.0], device="cuda").expand(T, 2)).contiguous()
    x = (torch.randint(0, 24, (T, D), device="cuda", generator=g) == 0).half()
    up = (torch.randint(0, 12, (E, F, D), device="cuda", generator=g) == 0).half()
    down = torch.randint(-1, 2, (E, D, F), device="cuda", generator=g).half()
    d = bolt.moe_desc(T, E, k, D, F, act="relu", gated=False)
    y = bolt.bolt_moe_experts(d, x, up, None, down, None, ids, weights, offsets, order, torch.empty((T, D), dtype=torch.float16, device="cuda"),
                              torch.empty(bolt.bolt_moe_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    want, _ = ref.experts(x, lambda e: up[e].double(), None, lambda e: down[e].double(), None, ids, weights, "relu", False)
    assert want.abs().max() <= 2048 and torch.equal(y.double(), want)


@pytest.mark.parametrize("T", [4, 60, 700])
@pytest.mark.parametrize("kind", ["f16", "w4"])
def test_experts_rows_do_not_meet(bolt, T, kind):
    """A token of infinities spoils its own row only, though it shares tiles with others."""
    E, k, D, F = 4, 2, 136, 72
    g = _gen(T)
    plan = _routed(g, T, E, k)
    x = _half(g, T, D)
    if kind == "w4":
        up, down = _w4(bolt, g, E, 2 * F, D, 32)[1], _w4(bolt, g, E, D, F, 32)[1]
    else:
        up, down = _half(g, E, 2 * F, D, std=0.1), _half(g, E, D, F, std=0.1)
    d = bolt.moe_desc(T, E, k, D, F, weights=kind, group=32)
    ws = torch.empty(bolt.bolt_moe_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    run = lambda v: bolt.bolt_moe_experts(d, v, up, None, down, None, *plan, torch.empty((T, D), dtype=torch.float16, device="cuda"), ws)
    want = run(x)
    spoiled = x.clone()
    spoiled[1] = float("inf")
    got = run(spoiled)
    keep = [i for i in range(T) if i != 1]
    assert torch.equal(got[keep], want[keep]) and not torch.isfinite(got[1]).any()


@pytest.mark.parametrize("T", [2, 300, 3000])
def test_experts_weights_past_32_bits(bolt, T):
    """5.4 GB of weights, the only expert in use is the last."""
    E, D, F = 40, 4096, 8192
    g = _gen(T)
    up = torch.zeros((E, 2 * F, D), dtype=torch.float16, device="cuda")
    down = torch.zeros((E, D, F), dtype=torch.float16, device="cuda")
    up[-1], down[-1] = _half(g, 2 * F, D, std=1 / 64), _half(g, D, F, std=1 / 90)
    x, ids = _half(g, T, D), torch.full((T, 1), E - 1, dtype=torch.int32, device="cuda")
    w = torch.ones((T, 1), device="cuda")
    offsets, order = (t.cuda() for t in ref.lists(ids, E))
    d = bolt.moe_desc(T, E, 1, D, F)
    y = bolt.bolt_moe_experts(d, x, up, None, down, None, ids, w, offsets, order, torch.empty((T, D), dtype=torch.float16, device="cuda"),
                              torch.empty(bolt.bolt_moe_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    some = torch.randperm(T, device="cuda", generator=g)[:64]
    want, bound = ref.experts(x[some], lambda e: up[e].double(), None, lambda e: down[e].double(), None, ids[some], w[some], "silu", True)
    _within(y[some], want, bound)


def test_experts_without_tokens(bolt):
    t = torch.zeros(64, dtype=torch.float16, device="cuda")
    i = torch.zeros(9, dtype=torch.int32, device="cuda")
    d = bolt.moe_desc(0, 1, 1, 8, 8, gated=False)
    bolt.bolt_moe_experts(d, t, t, None, t, None, i, torch.zeros(1, device="cuda"), i, i, t, None)


# ---- together, on other streams, in graphs ---------------------------------------------------------------------------------------
class _Layer:
    """Router GEMM, routing, experts and a 4-bit layer over buffers of its own."""

    def __init__(self, bolt, T, kind, seed=0):
        self.bolt, g = bolt, _gen(seed)
        E, k, D, F = 32, 4, 264, 136
        self.x, self.router = _half(g, T, D), _half(g, E, D, std=0.3)
        new = lambda *s, dtype: torch.zeros(s, dtype=dtype, device="cuda")
        self.logits = new(T, E, dtype=torch.float16)
        self.gd = bolt.gemm_desc(T, E, D, act="none", b_layout=bolt.LAYOUT_NK)
        self.rd = bolt.moe_route_desc(T, E, k)
        self.plan = new(T, k, dtype=torch.int32), new(T, k, dtype=torch.float32), new(E + 1, dtype=torch.int32), new(T * k, dtype=torch.int32)
        self.rws = new(bolt.bolt_moe_route_workspace_bytes(self.rd), dtype=torch.uint8)
        if kind == "w4":
            self.up, self.down = _w4(bolt, g, E, 2 * F, D, 64)[1], _w4(bolt, g, E, D, F, 64)[1]
        else:
            self.up, self.down = _half(g, E, 2 * F, D, std=0.06), _half(g, E, D, F, std=0.08)
        self.md = bolt.moe_desc(T, E, k, D, F, weights=kind, group=64)
        self.mws = new(bolt.bolt_moe_workspace_bytes(self.md), dtype=torch.uint8)
        self.y, self.out = new(T, D, dtype=torch.float16), new(T, 72, dtype=torch.float16)
        self.ld, self.head = bolt.gemm_w4_desc(T, 72, D, 32, act="gelu"), _w4(bolt, g, 1, 72, D, 32)[1]
        self.lws = new(bolt.bolt_gemm_w4_workspace_bytes(self.ld), dtype=torch.uint8)

    def run(self):
        b = self.bolt
        b.bolt_gemm_epilogue(self.gd, self.x, self.router, None, self.logits)
        b.bolt_moe_route(self.rd, self.logits, None, None, *self.plan, self.rws)
        b.bolt_moe_experts(self.md, self.x, self.up, None, self.down, None, *self.plan, self.y, self.mws)
        b.bolt_gemm_w4(self.ld, self.y, self.head, None, self.out, self.lws)
        return [t.clone() for t in (*self.plan, self.y, self.out)]


@pytest.mark.parametrize("T", [1, 40, 600])
@pytest.mark.parametrize("kind", ["f16", "w4"])
def test_same_results_every_time_on_any_stream(bolt, T, kind):
    layer = _Layer(bolt, T, kind)
    want = layer.run()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = [layer.run() for _ in range(3)]
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda.synchronize()
    for run in got:
        assert all(torch.equal(a, b) for a, b in zip(run, want))


@pytest.mark.parametrize("T", [1, 40, 600])
@pytest.mark.parametrize("kind", ["f16", "w4"])
def test_graph_replays(bolt, T, kind):
    """Captured once, replayed on new inputs, with eager work and synchronisation between the replays."""
    layer = _Layer(bolt, T, kind, seed=T)
    layer.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = layer.run()
    for i in range(4):
        layer.x.copy_(_half(_gen(100 + i), *layer.x.shape))
        graph.replay()
        torch.cuda.synchronize()
        held = [t.clone() for t in outs]
        want = layer.run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), i


def test_general_path_takes_the_same_arguments(bolt, monkeypatch):
    """Through ctypes, as without the call extension."""
    layer = _Layer(bolt, 20, "w4")
    want = layer.run()
    monkeypatch.setattr(bolt.binding, "_fast", bolt.binding._NoFast())
    assert all(torch.equal(a, b) for a, b in zip(layer.run(), want))


def test_buffers_that_are_too_small_are_refused(bolt):
    layer = _Layer(bolt, 600, "w4")
    b = bolt
    with pytest.raises(AssertionError, match="A: "):
        b.bolt_gemm_w4(layer.ld, layer.y[:10].contiguous(), layer.head, None, layer.out)
    with pytest.raises(AssertionError, match="packed: "):
        b.bolt_gemm_w4(layer.ld, layer.y, layer.head[:100], None, layer.out)
    with pytest.raises(AssertionError, match="w_up: "):
        b.bolt_moe_experts(layer.md, layer.x, layer.down, None, layer.down, None, *layer.plan, layer.y, layer.mws)
    with pytest.raises(b.BoltError) as e:
        b.bolt_moe_experts(layer.md, layer.x, layer.up, None, layer.down, None, *layer.plan, layer.y, layer.mws[:16])
    assert e.value.status == 4
