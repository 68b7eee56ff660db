"""GPU: where the 4-bit layer, the routing and the experts' products could go wrong: values, masks and sizes that tests/test_gpu_llm.py does
not reach.  Bounds as there (tests/llm_ref.py)."""
import math

import pytest

import llm_ref as ref
from test_gpu_llm import _gen, _half, _matrix, _w4, _within, bolt  # noqa: F401  (the fixture among them)

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


# ---- routing ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T", [3, 40, 300])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_route_sigmoid_scores_next_to_the_smallest(bolt, T, dtype):
    """1 / (1 + exp(-x)) is a number in 32 bits down to x = -88.72 (denormal from -87.3 on): equal ones share the weight, and none is
    left below."""
    from test_gpu_llm import _route
    logits = torch.full((T, 24), -88.5, dtype=dtype)  # (exact in a half)
    logits[1] = -89.0
    ids, w, _, _, _, _, _ = _route(bolt, logits, 4, score="sigmoid")
    assert (ids == torch.arange(4)).all()
    keep = [i for i in range(T) if i != 1]
    assert (w[keep] - 0.25).abs().max() <= 1e-6 and (w[1] == 0).all()
