"""GPU: 8-bit layers and projections with adapters where a kernel, a size or a range is easily left out (tests/rows_cases.py), against the 64-bit references
of tests/rows_ref.py."""
import math

import pytest

import llm_ref as ref
import rows_cases as cases
import rows_ref as rows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from test_gpu_rows import F8, _gen, _half, _lora, _nan, _q8, _w4, _w4_gen, bolt  # noqa: E402, F401


# ---- the adapters' share through memory ---------------------------------------------------------------------------------
@pytest.mark.parametrize("size", [c[0] for c in cases.SHARE])
def test_the_share_has_the_range_of_fp32_whatever_the_table(bolt, size):  # noqa: F811
    """A share far beyond 65504 and an alpha that brings the result back: finite, and right without the rounding of a share, by a table of the two adapters that
    the rows ask for as by one that holds many more."""
    M, N, K, n, rank, weights, group = size
    g = _gen(M + N + K)
    A = _half(g, M, K)
    if weights == "w4":
        W, W64 = _w4(bolt, g, N, K, group)
    else:
        W = _half(g, N, K, std=1 / math.sqrt(K))
        W64 = W.double()
    down, up = _half(g, n, rank, K, std=20 / math.sqrt(K)), _half(g, n, N, rank, std=2000.0)
    scales, bias = torch.rand(n, device="cuda", generator=g) + 0.5, _half(g, N, std=100.0)
    ids = torch.randint(-1, 2, (M,), dtype=torch.int32, device="cuda", generator=g)
    unpacks = weights == "w4" and M >= 512  # (weights of many rows may be rounded to FP16 once)
    want, bound = rows.lora(A.double(), W64, bias.double(), ids, down[:2], up[:2], scales[:2], "none", 2.0 ** -7, -1.5, shift=ref.U16 if unpacks else 0.0, apart=False)
    assert (want - bias.double() * -1.5).abs().max() * 2 ** 7 > 2 * 65504 and want.abs().max() < 60000
    for held in (2, n):
        d = bolt.gemm_lora_desc(M, N, K, held, rank, weights=weights, group=group, alpha=2.0 ** -7, beta=-1.5)
        ws = _nan(bolt.bolt_gemm_lora_workspace_bytes(d), dtype=torch.uint8)
        rows.within(bolt.bolt_gemm_lora(d, A, W, bias, ids, down, up, scales, _nan(M, N), ws), want, bound, "%d adapters" % held)


@pytest.mark.parametrize("size", [c[0] for c in cases.IN_TILES])
@pytest.mark.parametrize("how", ["runs", "mixed"])
def test_the_share_in_the_tiles(bolt, size, how):  # noqa: F811
    M, N, K, n, rank, weights, group = size
    D, _, c = _lora(bolt, M, N, K, n, rank, weights, group, how)
    W64 = c["W"].double() if weights == "f16" else _w4(bolt, _w4_gen(c, M, N, K), N, K, group)[1]
    rows.within(D, *rows.lora(c["A"].double(), W64, c["bias"].double(), c["ids"], c["down"], c["up"], c["scales"], "none", 0.75, -1.5, apart=False))


@pytest.mark.parametrize("size", [c[0] for c in cases.SHARE + cases.IN_TILES])
def test_the_share_is_not_rounded(bolt, size):  # noqa: F811
    """Whole numbers, all rows of A alike, and a bias that takes the share away but for what binary16 would lose of it: sums are exact in FP32, so that the
    one rounding left is the result's."""
    M, N, K, n, rank, weights, group = size
    g = _gen(M + N)
    whole = lambda most, *s: torch.randint(-most, most + 1, s, device="cuda", generator=g).half()
    A, down = whole(1, 1, K).expand(M, K).contiguous(), whole(1, n, rank, K)
    up = whole(max(1, min(2000, int(8000 * 1.7 / math.sqrt(K * 0.44 * rank)))), n, N, rank)
    if weights == "w4":
        q = torch.randint(0, 256, (1, N, K // 2), dtype=torch.uint8, device="cuda", generator=g)
        scale = torch.ones((1, N, -(-K // group)), dtype=torch.float16, device="cuda")
        W = bolt.bolt_w4_pack(N, K, group, q, scale, None, _nan(bolt.bolt_w4_packed_bytes(N, K, group), dtype=torch.uint8))
        W64 = ref.w4_matrix(q[0], scale[0], None, group)
    else:
        W = whole(8, N, K)
        W64 = W.double()
    low = down[0].double() @ A[0].double()
    share = up[0].double() @ low
    bias = -share.half()
    assert low.abs().max() <= 2048 and share.abs().max() < 65504 and (share.half().double() != share).any()
    ids = torch.randint(-1, 1, (M,), dtype=torch.int32, device="cuda", generator=g)
    d = bolt.gemm_lora_desc(M, N, K, n, rank, weights=weights, group=group)
    D = bolt.bolt_gemm_lora(d, A, W, bias, ids, down, up, None, _nan(M, N), _nan(bolt.bolt_gemm_lora_workspace_bytes(d), dtype=torch.uint8))
    base = W64 @ A[0].double() + bias.double()
    assert (base + share).abs().max() <= 2048
    for id_, want in ((-1, base), (0, base + share)):
        assert torch.equal(D[ids == id_], want.half().expand(int((ids == id_).sum()), N)), id_


# ---- 8-bit layers --------------------------------------------------------------------------------------------------------
def _layer(A, sa, W, sw, bias, act="none", alpha=1.0, beta=1.0):
    """The layer in 64 bits and the bound of its rounded result.  Its sums are FP32 over groups of eight neighbouring k; in a group the matrix cores align the
    products to the one of the largest exponent, 2^E for two operands whose exponents add up to E, and cut each towards zero below 2^(E - 13).  E4M3 has four
    significant bits, so that a product of exponent E ends at 2^(E - 6) and loses nothing; each of the other seven loses less than 2^(E - 13).  (Exponents
    of zeros and of subnormal values are the smallest normal one, -6.)"""
    sa, sw = (torch.ones(1, device="cuda") if s is None else s for s in (sa, sw))
    want, bound = ref.linear(A.double() * sa.double()[:, None], W.double() * sw.double()[:, None], bias, act, alpha, beta)
    power = lambda v: torch.exp2(torch.floor(torch.log2(v.float().abs().clamp(min=2.0 ** -6))))
    a, w, cut = power(A), power(W), torch.zeros_like(want)
    for k in range(0, A.shape[1], 8):
        top = torch.zeros(want.shape, device="cuda")
        for i in range(k, k + 8):
            torch.maximum(top, a[:, i, None] * w[None, :, i], out=top)
        cut += top
    return want, bound + ref.STEEP * abs(alpha) * 7 * 2.0 ** -13 * cut * sa.double()[:, None] * sw.double()[None, :]


@pytest.mark.parametrize("M,N,K", [(1, 264, 16), (16, 1032, 48), (40, 1032, 16), (70, 2056, 32), (200, 12288, 16), (400, 4104, 32), (2050, 8200, 16)])
def test_q8_of_short_reductions(bolt, M, N, K):  # noqa: F811
    """Where a sum has few groups what the matrix cores cut off shows next to FP16's rounding: every value is within its bound, and values that differ little
    in size, of which nothing is cut, are rounded once."""
    g = _gen(M + K)
    (A, sa), (W, sw) = _q8(g, M, K), _q8(g, N, K, std=1 / math.sqrt(K))
    rows.within(bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K), A, sa, W, sw, None, _nan(M, N)), *_layer(A, sa, W, sw, None))
    near = lambda R: torch.randint(0x38, 0x40, (R, K), device="cuda", generator=g).to(torch.uint8).view(F8)  # (1 to 1.875: products end at 2^-6, below 2^2)
    A, W = near(M), near(N)
    D = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K), A, None, W, None, None, _nan(M, N))
    assert torch.equal(D, (A.double() @ W.double().t().contiguous()).half())


# ---- 8-bit layers on 256 x 256 tiles ------------------------------------------------------------------------------------
def _rows_of(M):
    """The rows that are compared: all of few, of many those of the first row block, of some in the middle and of the last."""
    return torch.arange(M, device="cuda") if M < 1000 else torch.cat([torch.arange(a, b, device="cuda") for a, b in ((0, 300), (M // 2, M // 2 + 200), (M - 300, M))])


@pytest.mark.parametrize("M,N,K", cases.Q8_LARGE)
@pytest.mark.parametrize("act,full", [("none", False), ("silu", True), ("gelu", True), ("softplus", True)])
def test_large_q8(bolt, M, N, K, act, full):  # noqa: F811
    g = _gen(M + N + K)
    (A, sa), (W, sw) = _q8(g, M, K), _q8(g, N, K, std=1 / math.sqrt(K))
    bias = _half(g, N) if full else None
    d = bolt.gemm_q8_desc(M, N, K, act=act, alpha=0.75 if full else 1.0, beta=-1.5)
    D, at = bolt.bolt_gemm_q8(d, A, sa, W, sw, bias, _nan(M, N)), _rows_of(M)
    rows.within(D[at], *_layer(A[at], sa[at], W, sw, None if bias is None else bias.double(), act, d.alpha, d.beta))


@pytest.mark.parametrize("M,N,K", cases.Q8_LARGE)
def test_large_q8_is_exact_on_integers(bolt, M, N, K):  # noqa: F811
    """Small integers and scales that are powers of two, all rows and columns: a value in a wrong place, a lost column or a scale of another row shows."""
    g = _gen(M + K)
    integers = lambda R: torch.randint(-2, 3, (R, K), device="cuda", generator=g).float().to(F8)
    powers = lambda R: 2.0 ** torch.randint(-2, 1, (R,), device="cuda", generator=g).float()
    A, W, sa, sw, bias = integers(M), integers(N), powers(M), powers(N), torch.randint(-4, 5, (N,), device="cuda", generator=g).half()
    sums = A.float() @ W.float().t()  # (whole numbers far below 2^24: exact)
    assert sums.abs().max() <= 1024
    D = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K), A, sa, W, sw, None, _nan(M, N))
    assert torch.equal(D, (sums * sa[:, None] * sw[None, :]).half())
    D = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K, act="relu"), A, None, W, None, bias, _nan(M, N))
    assert torch.equal(D, (sums + bias.float()).clamp(min=0).half())


@pytest.mark.parametrize("M,N,K", [(262, 22344, 1296), (19742, 1032, 1040)])
def test_large_q8_strides_and_untouched_padding(bolt, M, N, K):  # noqa: F811
    lda, ldd = K + 48, N + 56
    g = _gen(M)
    (a, sa), (W, sw) = _q8(g, M, K), _q8(g, N, K)
    A = _nan(M, lda, dtype=F8)
    A.view(torch.uint8)[:, :K] = a.view(torch.uint8)
    D, at = torch.full((M, ldd), 7.0, dtype=torch.float16, device="cuda"), _rows_of(M)
    bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K, lda=lda, ldd=ldd), A, sa, W, sw, None, D)
    rows.within(D[at][:, :N], *_layer(a[at], sa[at], W, sw, None))
    assert (D[:, N:] == 7.0).all()


@pytest.mark.parametrize("M,N,K", [(262, 22344, 1296), (19742, 1032, 1040), (4365, 16688, 144)])
def test_large_q8_rows_and_columns_do_not_meet(bolt, M, N, K):  # noqa: F811
    """A NaN in a row or an infinity in its scale spoils that row only, a NaN in a weight row that column only."""
    g = _gen(M)
    (A, sa), (W, sw) = _q8(g, M, K), _q8(g, N, K, std=0.1)
    clean = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K), A, sa, W, sw, None, _nan(M, N))
    A.view(torch.uint8)[M - 2, 5], W.view(torch.uint8)[N - 2, K - 1] = 0x7f, 0x7f
    sa[7] = float("inf")
    D = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K), A, sa, W, sw, None, _nan(M, N))
    keep_r, keep_c = torch.ones(M, dtype=torch.bool, device="cuda"), torch.ones(N, dtype=torch.bool, device="cuda")
    keep_r[M - 2] = keep_r[7] = keep_c[N - 2] = False
    assert torch.isnan(D[M - 2]).all() and torch.isnan(D[:, N - 2]).all() and not torch.isfinite(D[7]).any()
    assert torch.equal(D[keep_r][:, keep_c], clean[keep_r][:, keep_c])


@pytest.mark.parametrize("M,N,K", cases.Q8_LARGE)
def test_large_q8_of_bias_alone(bolt, M, N, K):  # noqa: F811
    """alpha 0: -1.5 times the bias is a number of FP32, rounded once."""
    g = _gen(M)
    (A, sa), (W, sw), bias = _q8(g, M, K), _q8(g, N, K), _half(g, N)
    D = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K, alpha=0.0, beta=-1.5), A, sa, W, sw, bias, _nan(M, N))
    assert torch.equal(D, (bias.float() * -1.5).half().expand(M, N))


# ---- weights on both sides of 2 GiB -------------------------------------------------------------------------------------
@pytest.mark.parametrize("N,K", cases.Q8_WEIGHTS)
def test_q8_of_weights_about_2_gib(bolt, N, K):  # noqa: F811
    """On 256 x 256 tiles up to the last byte that 31 bits reach, on others beyond."""
    M, g = 520, _gen(8)
    W = torch.randint(0, 256, (N, K), dtype=torch.uint8, device="cuda", generator=g).bitwise_and_(0xb7).view(F8)  # (below 1, of both signs)
    A, sa = _q8(g, M, K)
    D = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K), A, sa, W, None, None, _nan(M, N))
    for at in (slice(0, 300), slice(N // 2, N // 2 + 300), slice(N - 300, N)):
        rows.within(D[:, at], *_layer(A, sa, W[at], None, None))


@pytest.mark.parametrize("N,K", cases.F16_WEIGHTS)
@pytest.mark.parametrize("n", [2, 600])
def test_projections_of_weights_about_2_gib(bolt, N, K, n):  # noqa: F811
    M, rank, g = 520, 8, _gen(9)
    A, W, down, up = _half(g, M, K), _half(g, N, K, std=0.01), _half(g, n, rank, K, std=0.01), _half(g, n, N, rank, std=0.1)
    ids = torch.randint(-1, 2, (M,), dtype=torch.int32, device="cuda", generator=g)
    d = bolt.gemm_lora_desc(M, N, K, n, rank)
    D = bolt.bolt_gemm_lora(d, A, W, None, ids, down, up, None, _nan(M, N), _nan(bolt.bolt_gemm_lora_workspace_bytes(d), dtype=torch.uint8))
    for at in (slice(0, 300), slice(N // 2, N // 2 + 300), slice(N - 300, N)):
        rows.within(D[:, at], *rows.lora(A.double(), W[at].double(), None, ids, down[:2], up[:2, at], None, "none", apart=False))
