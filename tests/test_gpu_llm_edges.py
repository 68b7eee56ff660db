"""GPU: where the 4-bit layer, the routing and the experts' products could go wrong: values, masks and sizes that tests/test_gpu_llm.py does
not reach.  Bounds as there (tests/llm_ref.py)."""
import math

import pytest

import llm_ref as ref
from test_gpu_llm import _check_route, _gen, _half, _matrix, _route, _run_experts, _w4, _within, bolt  # noqa: F401  (the fixture among them)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _gemm(bolt, d, A, packed, bias=None):
    ws = torch.empty(bolt.bolt_gemm_w4_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    return bolt.bolt_gemm_w4(d, A, packed, bias, torch.full((d.M, d.N), float("nan"), dtype=torch.float16, device="cuda"), ws)


# ---- 4-bit layer ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("M,N,K,group,act", [(2048, 256, 8192, 128, "none"), (2048, 256, 8192, 32, "silu"), (512, 1024, 12288, 128, "none"),
                                             (1024, 1024, 4096, 64, "silu"), (1536, 512, 1032, 32, "silu")])
def test_gemm_w4_narrow_layers_run_on_the_weights_as_they_are(bolt, M, N, K, group, act):
    """Few output tiles: unpacking first is slower there, and rounds the weights.  Two columns of A differ from zero in a row, so the FP32 sum
    adds next to nothing to the bound, and rounded weights would leave it."""
    g = _gen(K)
    raw, packed = _w4(bolt, g, 1, N, K, group, True)
    A = torch.zeros((M, K), dtype=torch.float16, device="cuda")
    rows = torch.arange(M, device="cuda")
    A[rows, rows * 5 % K], A[rows, (rows * 7 + 64) % K] = 1.0, 1.0
    d = bolt.gemm_w4_desc(M, N, K, group, act=act)
    y = ref.act(A.double() @ _matrix(raw, group).t().contiguous(), act)
    size = A.double() @ _matrix(raw, group).abs().t().contiguous()
    _within(_gemm(bolt, d, A, packed), y, size * 3 * ref.U32 * ref.STEEP + y.abs() * ((ref.CLOSE if act == "silu" else 0) + ref.U16) + ref.TINY)


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("K,group", [(1032, 32), (2056, 64), (4104, 128)])
def test_gemm_w4_unpacked_takes_weights_beyond_a_half(bolt, act, K, group):
    """scale * (q - z) past 65504: finite at every number of rows, in the columns that hold such weights and in the others."""
    M, N = 4096, 8200
    g = _gen(group)
    groups = -(-K // group)
    q = torch.randint(0, 256, (1, N, K // 2), dtype=torch.uint8, device="cuda", generator=g)
    s = ((torch.rand((1, N, groups), device="cuda", generator=g) + 0.1) * (0.4 / math.sqrt(K))).half()
    z = torch.randint(0, 16, (1, N, groups), dtype=torch.uint8, device="cuda", generator=g)
    for n, k, v in ((5, 3, 6e4), (5, 4, -5e3), (300, 0, 4368.0), (8199, groups - 1, 65504.0), (4000, 1, 4364.0)):
        s[0, n, k] = v
    packed = torch.empty(bolt.bolt_w4_packed_bytes(N, K, group), dtype=torch.uint8, device="cuda")
    bolt.bolt_w4_pack(N, K, group, q, s, z, packed)
    A, bias = _half(g, M, K, std=1e-3), _half(g, N)
    W = _matrix((q, s, z), group)
    assert W.abs().max() > 65520  # (infinite as a half)
    want, bound = ref.linear(A.double(), W, bias.double(), act, 0.5, shift=ref.U16)
    inside = want.abs() < 6e4
    d = bolt.gemm_w4_desc(M, N, K, group, act=act, alpha=0.5)
    got = _gemm(bolt, d, A, packed, bias)
    _within(got[inside], want[inside], bound[inside])
    assert inside.double().mean() > 0.99
    few = _gemm(bolt, bolt.gemm_w4_desc(8, N, K, group, act=act, alpha=0.5), A[:8].contiguous(), packed, bias)
    assert (torch.isfinite(few) == torch.isfinite(got[:8])).all()


def test_gemm_w4_unpacked_keeps_scales_that_are_not_finite_to_their_columns(bolt):
    M, N, K, group = 4096, 8192, 520, 32
    g = _gen(9)
    raw, _ = _w4(bolt, g, 1, N, K, group)
    raw[1][0, 77, 2], raw[1][0, 4100, 0] = float("inf"), float("nan")
    packed = torch.empty(bolt.bolt_w4_packed_bytes(N, K, group), dtype=torch.uint8, device="cuda")
    bolt.bolt_w4_pack(N, K, group, *raw, packed)
    A = _half(g, M, K)
    got = _gemm(bolt, bolt.gemm_w4_desc(M, N, K, group), A, packed)
    others = torch.ones(N, dtype=torch.bool, device="cuda")
    others[[77, 4100]] = False
    assert not torch.isfinite(got[:, ~others]).any()
    W = _matrix(raw, group)[others]
    _within(got[:, others], *ref.linear(A.double(), W, None, "none", shift=ref.U16))


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("alpha", [1e-36, 1e-39])
@pytest.mark.parametrize("with_bias", [True, False])
def test_gemm_w4_unpacked_takes_an_alpha_next_to_zero(bolt, act, alpha, with_bias):
    """beta / alpha times the bias, where the sums of many rows start, is past 32 bits."""
    M, N, K = 4096, 8192, 520
    g = _gen(11)
    raw, packed = _w4(bolt, g, 1, N, K, 32)
    A, bias = _half(g, M, K), _half(g, N, std=1000.0) if with_bias else None
    d = bolt.gemm_w4_desc(M, N, K, 32, act=act, alpha=alpha, beta=0.5)
    _within(_gemm(bolt, d, A, packed, bias), *ref.linear(A.double(), _matrix(raw, 32), None if bias is None else bias.double(), act, d.alpha, d.beta))


# few rows: walks with waves that have no step, a short last step; some ten, with sets of waves that end apart; tiles
@pytest.mark.parametrize("M", [1, 13, 20, 64, 200, 700])
@pytest.mark.parametrize("K,group", [(8, 32), (136, 32), (264, 64), (392, 128), (4232, 128)])
def test_gemm_w4_infinite_scales(bolt, M, K, group):
    """All values above zero, so an infinite scale anywhere in a row gives infinity: zeros that stand for missing steps must not meet it."""
    N = 72
    g = _gen(M + K)
    groups = -(-K // group)
    q = torch.randint(1, 16, (1, N, K // 2, 2), dtype=torch.uint8, device="cuda", generator=g)
    q = q[..., 0] | q[..., 1] << 4
    s = torch.full((1, N, groups), 2.0 ** -8, dtype=torch.float16, device="cuda")
    z = torch.zeros((1, N, groups), dtype=torch.uint8, device="cuda")
    s[0, 3, 0], s[0, 40, groups - 1], s[0, 71, groups // 2] = float("inf"), float("inf"), float("inf")
    packed = torch.empty(bolt.bolt_w4_packed_bytes(N, K, group), dtype=torch.uint8, device="cuda")
    bolt.bolt_w4_pack(N, K, group, q, s, z, packed)
    A = torch.rand((M, K), device="cuda", generator=g).half() * 0.1 + 0.01
    got = _gemm(bolt, bolt.gemm_w4_desc(M, N, K, group), A, packed)
    spoiled = torch.zeros(N, dtype=torch.bool, device="cuda")
    spoiled[[3, 40, 71]] = True
    assert (got[:, spoiled] == float("inf")).all() and torch.isfinite(got[:, ~spoiled]).all()


# tiles of 64 x 128 and of 128 x 256, which fewer than 512 rows take from some thousand outputs on; ragged rows, columns and last steps
LARGE_TILES = [(100, 12296, 72), (333, 8200, 520), (400, 8200, 1032), (333, 12296, 520), (500, 8200, 1096), (411, 12296, 72)]


@pytest.mark.parametrize("M,N,K", LARGE_TILES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros,act", [(True, "none"), (False, "silu")])
def test_gemm_w4_large_tiles(bolt, M, N, K, group, zeros, act):
    g = _gen(M + K)
    raw, packed = _w4(bolt, g, 1, N, K, group, zeros)
    A, bias = _half(g, M, K), _half(g, N) if zeros else None
    d = bolt.gemm_w4_desc(M, N, K, group, act=act, alpha=0.5, beta=-2.0)
    assert bolt.bolt_gemm_w4_workspace_bytes(d) == 0  # (not unpacked)
    _within(_gemm(bolt, d, A, packed, bias), *ref.linear(A.double(), _matrix(raw, group), None if bias is None else bias.double(), act, 0.5, -2.0))


@pytest.mark.parametrize("M,N,K", [*LARGE_TILES, (13, 72, 4104), (100, 72, 4104), (700, 72, 4104), (40, 4104, 4232)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_gemm_w4_is_exact_on_integers_in_large_tiles_and_deep_layers(bolt, M, N, K, group):
    """Every product and sum is exact on the weights as they are, so a value in a wrong place or a lost column shows."""
    g = _gen(M + K)
    raw, packed = _w4(bolt, g, 1, N, K, group, True, ones=True)
    A = torch.randint(-1, 2, (M, K), device="cuda", generator=g).half() * (torch.randint(0, 4, (M, K), device="cuda", generator=g) == 0)
    d = bolt.gemm_w4_desc(M, N, K, group)
    assert bolt.bolt_gemm_w4_workspace_bytes(d) == 0
    want = A.double() @ _matrix(raw, group).t().contiguous()
    assert want.abs().max() <= 2048 and torch.equal(_gemm(bolt, d, A, packed).double(), want)


# ---- experts ------------------------------------------------------------------------------------------------------------------
# few rows (walks; deep reductions, D = 2120), some ten rows with two sets of waves (5 and 3 steps), tiles of 64 rows
@pytest.mark.parametrize("T", [2, 40, 500])
@pytest.mark.parametrize("D,F", [(8, 8), (72, 136), (264, 136), (2120, 2120)])
@pytest.mark.parametrize("where", ["up", "down"])
def test_experts_infinite_weights(bolt, T, D, F, where):
    """All values above zero, so an infinite weight of the first columns, or of the last, gives infinity in its outputs."""
    E, k = 4, 2
    g = _gen(T + D)
    above = lambda *s, top: (torch.rand(s, device="cuda", generator=g) * top).half() + 2.0 ** -12
    x, up, down = above(T, D, top=0.1), above(E, F, D, top=0.05), above(E, D, F, top=0.05)
    ids = torch.stack((torch.randint(0, 3, (T,), device="cuda", generator=g), torch.full((T,), 3, device="cuda")), 1).int()
    weights = torch.full((T, k), 0.5, device="cuda")
    offsets, order = (t.cuda() for t in ref.lists(ids, E))
    held = up if where == "up" else down
    held[0, 5, 0], held[1, 2, held.shape[2] - 1], held[2, 0, min(33, held.shape[2] - 2)] = float("inf"), float("inf"), float("inf")
    d = bolt.moe_desc(T, E, k, D, F, act="relu", gated=False)
    y = bolt.bolt_moe_experts(d, x, up, None, down, None, ids, weights, offsets, order, torch.empty((T, D), dtype=torch.float16, device="cuda"),
                              torch.empty(bolt.bolt_moe_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    want, _ = ref.experts(x, lambda e: up[e].double(), None, lambda e: down[e].double(), None, ids, weights, "relu", False)
    assert not torch.isnan(want).any() and torch.isinf(want).any()
    assert torch.equal(torch.isposinf(y), torch.isposinf(want)) and not torch.isnan(y).any()


@pytest.mark.parametrize("T,E,k,D,F", [(900, 4, 2, 2056, 1032), (1300, 6, 3, 1032, 2056), (2100, 4, 1, 4104, 520)])
@pytest.mark.parametrize("gated,act,bias", [(True, "silu", False), (False, "relu", True)])
@pytest.mark.parametrize("group", [32, 64])
def test_experts_many_rows_of_4_bits(bolt, T, E, k, D, F, gated, act, bias, group):
    """Tiles of 64 x 128 and 128 x 256 with several groups in a step."""
    _run_experts(bolt, T, E, k, D, F, act, gated, "w4", group, bias, 0.1, skew=0.5)


@pytest.mark.parametrize("T,k", [(600, 2), (512, 1)])
@pytest.mark.parametrize("kind", ["f16", "w4"])
@pytest.mark.parametrize("gated", [True, False])
def test_experts_rows_past_2_gib(bolt, T, k, kind, gated):
    """x from 2 GiB on (a wide stride) runs on the kernel of few rows, many blocks of them per expert."""
    assert T * (1 << 21) * 2 >= 1 << 31
    _run_experts(bolt, T, 4, k, 72, 136, "silu", gated, kind, 64, True, 0.1, skew=1.0, ldx=1 << 21)


@pytest.mark.parametrize("T", [3, 50])
@pytest.mark.parametrize("kind", ["f16", "w4"])
def test_experts_matrices_past_2_gib(bolt, T, kind):
    """One expert's gate and value rows take 2 GiB as halves.  Small integers in the first and last hidden units and zeros between: exact."""
    E, D, F, edge, group = 2, 1024, 1 << 19, 100, 128
    g = _gen(T)
    units = torch.cat((torch.arange(edge), torch.arange(F - edge, F))).cuda()
    x = (torch.randint(0, 24, (T, D), device="cuda", generator=g) == 0).half()
    small = (torch.randint(0, 12, (E, 4 * edge, D), device="cuda", generator=g) == 0).half()  # gate rows, then value rows
    back = torch.randint(-1, 2, (E, D, 2 * edge), device="cuda", generator=g).half()
    up, down = torch.zeros((E, 2 * F, D), dtype=torch.float16, device="cuda"), torch.zeros((E, D, F), dtype=torch.float16, device="cuda")
    up[:, torch.cat((units, F + units))], down[:, :, units] = small, back

    def pack(w):
        q = torch.empty((*w.shape[:2], w.shape[2] // 2), dtype=torch.uint8, device="cuda")
        for e in range(E):
            v = (w[e] + 8).to(torch.uint8)
            q[e] = v[:, 0::2] | v[:, 1::2] << 4
        packed = torch.empty(bolt.bolt_w4_packed_bytes(w.shape[1], w.shape[2], group, E), dtype=torch.uint8, device="cuda")
        ones = torch.ones((E, w.shape[1], w.shape[2] // group), dtype=torch.float16, device="cuda")
        return bolt.bolt_w4_pack(w.shape[1], w.shape[2], group, q, ones, None, packed)

    if kind == "w4":
        up, down = pack(up), pack(down)
    ids = torch.randint(0, E, (T, 1), device="cuda", generator=g).int()
    ids[-1] = E - 1
    offsets, order = (t.cuda() for t in ref.lists(ids, E))
    d = bolt.moe_desc(T, E, 1, D, F, act="relu", gated=True, weights=kind, group=group)
    y = bolt.bolt_moe_experts(d, x, up, None, down, None, ids, torch.ones((T, 1), device="cuda"), offsets, order,
                              torch.empty((T, D), dtype=torch.float16, device="cuda"),
                              torch.empty(bolt.bolt_moe_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    want, _ = ref.experts(x, lambda e: small[e].double(), None, lambda e: back[e].double(), None, ids, torch.ones((T, 1), device="cuda"), "relu", True)
    assert 0 < want.abs().max() <= 2048 and torch.equal(y.double(), want)


# ---- routing ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T", [3, 40, 300])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_route_sigmoid_scores_next_to_the_smallest(bolt, T, dtype):
    """1 / (1 + exp(-x)) is a number in 32 bits down to x = -88.72 (denormal from -87.3 on): equal ones share the weight, and none is
    left below."""
    logits = torch.full((T, 24), -88.5, dtype=dtype)  # (exact in a half)
    logits[1] = -89.0
    ids, w, _, _, _, _, _ = _route(bolt, logits, 4, score="sigmoid")
    assert (ids == torch.arange(4)).all()
    keep = [i for i in range(T) if i != 1]
    assert (w[keep] - 0.25).abs().max() <= 1e-6 and (w[1] == 0).all()


ROUTES = [(64, 6, 1, 1), (200, 8, 8, 3), (256, 10, 1, 1), (48, 2, 4, 1), (500, 4, 10, 5), (16, 3, 16, 5)]


@pytest.mark.parametrize("T", [1, 17, 64, 300, 8200])
@pytest.mark.parametrize("E,k,groups,top_groups", ROUTES)
@pytest.mark.parametrize("score,biased", [("sigmoid", False), ("sigmoid", True), ("softmax", True)])
def test_route_half_logits(bolt, T, E, k, groups, top_groups, score, biased):
    """FP16 logits where the tests beside it have FP32 ones: packed keys under sigmoid, and keys of score and bias."""
    g = torch.Generator().manual_seed(T * E)
    logits = (torch.randn(T, E, generator=g) * 1.5).half()
    bias = torch.randn(E, generator=g) * (0.1 if score == "sigmoid" else 0.02) if biased else None
    mask = (torch.rand(T, generator=g) > 0.2).to(torch.uint8) if T % 2 else None
    got = _route(bolt, logits, k, bias=bias, mask=mask, score=score, groups=groups, top_groups=top_groups, renormalize=T != 300, scale=1.5)
    _check_route(got, E, not biased and groups == 1)


@pytest.mark.parametrize("T", [16385, 40000])
@pytest.mark.parametrize("E,k,groups,top_groups,score,half,biased", [
    (64, 8, 1, 1, "softmax", True, False), (128, 4, 1, 1, "softmax", True, False), (256, 8, 8, 4, "sigmoid", False, True),
    (200, 6, 1, 1, "softmax", False, False), (100, 3, 1, 1, "sigmoid", True, False), (256, 8, 1, 1, "softmax", False, False)])
def test_route_several_rounds(bolt, T, E, k, groups, top_groups, score, half, biased):
    """More tokens than workgroups route at once: the next token's logits are requested ahead, whole pieces or one by one."""
    g = torch.Generator().manual_seed(T + E)
    logits = torch.randn(T, E, generator=g) * 1.5
    bias = torch.randn(E, generator=g) * 0.1 if biased else None
    mask = (torch.rand(T, generator=g) > 0.1).to(torch.uint8) if T % 2 else None
    got = _route(bolt, logits.half() if half else logits, k, bias=bias, mask=mask, score=score, groups=groups, top_groups=top_groups)
    _check_route(got, E, not biased and groups == 1)


@pytest.mark.parametrize("T", [6, 40, 300])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [True, False])
@pytest.mark.parametrize("groups,top_groups", [(1, 1), (5, 2)])
def test_route_rows_of_nothing_in_either_type(bolt, T, half, score, biased, groups, top_groups):
    """Minus infinity, the type's lowest value, NaN, one live expert, plus infinity: a choice and finite weights, with a bias and groups too."""
    E, inf, dtype = 40, float("inf"), torch.float16 if half else torch.float32
    g = torch.Generator().manual_seed(2)
    logits = torch.randn(T, E, generator=g).to(dtype)
    logits[0], logits[1], logits[2] = -inf, torch.finfo(dtype).min, float("nan")
    logits[3] = -inf
    logits[3, 17] = 0.25
    logits[4, 9], logits[4, 10] = inf, inf
    logits[5, ::2] = float("nan")
    bias = torch.linspace(0.3, 0.0, E) if biased else None
    ids, w, offsets, order, want_ids, want_w, gap = _route(bolt, logits, 3, bias=bias, score=score, groups=groups, top_groups=top_groups)
    held = torch.tensor([0, 1, 2, 3])  # (places that hang on rounding are none of these rows')
    assert torch.equal(ids[held], want_ids[held]) and torch.isfinite(w).all()
    sure = gap > 1e-5
    assert torch.equal(ids[sure], want_ids[sure]) and (w[sure].double() - want_w[sure]).abs().max() <= 1e-5
    assert ids[0].tolist() == [0, 1, 2] and ids[2].tolist() == [0, 1, 2] and ids[4, 0] == 9
    o, r = ref.lists(ids, E)
    assert torch.equal(offsets, o) and torch.equal(order, r)
