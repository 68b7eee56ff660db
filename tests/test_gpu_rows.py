"""GPU: the norm with its residual, rows in 8 bits, the layers that read them, projections with low-rank adapters, against 64-bit references
(tests/rows_ref.py); with small integers every sum is exact and results have to be equal."""
import math

import pytest

import llm_ref as ref
import rows_ref as rows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F8 = torch.float8_e4m3fn


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


def _nan(*shape, dtype=torch.float16):
    return torch.full((*shape[:-1], shape[-1] * dtype.itemsize), 0xff, dtype=torch.uint8, device="cuda").view(dtype)  # (a NaN in each of the types)


def _q8(g, R, K, std=1.0):
    """Rows in 8 bits with scales, as a quantiser leaves them."""
    v = torch.empty((R, K), dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g)
    s = (v.abs().amax(1) / 448).clamp(min=1e-12)
    return (v / s[:, None]).clamp(-448, 448).to(F8), s


# ---- norm ---------------------------------------------------------------------------------------------------------------
# widths on both sides of every kernel's
WIDTHS = [8, 64, 512, 520, 1024, 1032, 2048, 2056, 4096, 4104, 8192, 8200, 16384, 16392, 32768]


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("R,residual,y,q,offset", [(1, True, True, True, 0.0), (3, False, True, False, 1.0), (5, True, False, True, 1.0), (131, True, True, True, 0.0)])
def test_rms_norm(bolt, width, R, residual, y, q, offset):
    g = _gen(width + R)
    x, w = _half(g, R, width), _half(g, width, std=0.3)
    w += 1.0 - offset
    r = _half(g, R, width, std=3.0) if residual else None
    s = _nan(R, width) if residual else None
    Y, Q, S = _nan(R, width) if y else None, _nan(R, width, dtype=F8) if q else None, _nan(R, dtype=torch.float32) if q else None
    bolt.bolt_rms_norm(bolt.rms_norm_desc(R, width, eps=1e-5, weight_offset=offset), x, r, w, s, Y, Q, S)
    v, n, rel = rows.norm(x, r, w, 1e-5, offset)
    if residual:
        rows.check_half(s, v, rows.H32, "sum")
    if y:
        rows.check_half(Y, n, rel, "y")
    if q:
        rows.check_q(Q, S, n, rel)


@pytest.mark.parametrize("width", [72, 1200, 5000, 12000])
def test_rms_norm_strides_and_untouched_padding(bolt, width):
    R, ld = 37, width + 24
    g = _gen(width)
    big = lambda std=1.0: torch.full((R, ld), float("nan"), dtype=torch.float16, device="cuda").index_copy_(1, torch.arange(width, device="cuda"), _half(g, R, width, std=std))
    x, r, w = big(), big(2.0), _half(g, width)
    s, Y = torch.full((R, ld), 7.0, dtype=torch.float16, device="cuda"), torch.full((R, ld), 7.0, dtype=torch.float16, device="cuda")
    Q, S = torch.full((R, ld), 7.0, device="cuda").to(F8), _nan(R, dtype=torch.float32)
    bolt.bolt_rms_norm(bolt.rms_norm_desc(R, width, ld, ld, ld, ld, ld), x, r, w, s, Y, Q, S)
    v, n, rel = rows.norm(x[:, :width], r[:, :width], w, 1e-5, 0.0)
    rows.check_half(s[:, :width], v, rows.H32)
    rows.check_half(Y[:, :width], n, rel)
    rows.check_q(Q[:, :width], S, n, rel)
    for t in (s, Y, Q):
        assert (t[:, width:].float() == 7.0).all()


@pytest.mark.parametrize("width", [512, 4096, 9000])
@pytest.mark.parametrize("where", ["x", "residual"])
def test_rms_norm_in_place(bolt, width, where):
    """The new residual stream over either input, and the normed rows over the other."""
    g = _gen(width)
    x, r, w = _half(g, 40, width), _half(g, 40, width), _half(g, width)
    v, n, rel = rows.norm(x, r, w, 1e-5, 0.0)
    s, Y = (x, r) if where == "x" else (r, x)
    bolt.bolt_rms_norm(bolt.rms_norm_desc(40, width), x, r, w, s, Y)
    rows.check_half(s, v, rows.H32)
    rows.check_half(Y, n, rel)


@pytest.mark.parametrize("width", [256, 1536, 6144, 20000])
def test_rms_norm_special_rows(bolt, width):
    """A NaN or an infinity spoils its own row and nothing else; a row of zeros is zeros; sums beyond FP16 are infinite in `sum` alone."""
    g = _gen(width)
    x, r, w = _half(g, 12, width), _half(g, 12, width), _half(g, width)
    x[2, width // 2], x[5, width - 1], r[7, 0] = float("nan"), float("inf"), -float("inf")
    x[9], r[9] = 0.0, 0.0
    x[10], r[10] = 60000.0, 60000.0
    s, Y, Q, S = _nan(12, width), _nan(12, width), _nan(12, width, dtype=F8), _nan(12, dtype=torch.float32)
    bolt.bolt_rms_norm(bolt.rms_norm_desc(12, width), x, r, w, s, Y, Q, S)
    v, n, rel = rows.norm(x, r, w, 1e-5, 0.0)
    fine = torch.tensor([i for i in range(12) if i not in (2, 5, 7, 9)], device="cuda")
    rows.check_half(Y[fine], n[fine], rel)
    rows.check_q(Q[fine], S[fine], n[fine], rel)
    assert torch.isinf(s[10]).all() and (Y[9] == 0).all() and (Q[9].float() == 0).all() and S[9] == 0
    for i in (2, 5, 7):
        assert torch.isnan(S[i]) and torch.isnan(Q[i].float()).all()
        assert torch.equal(torch.isnan(Y[i]).double(), torch.isnan(n[i]).double())


def test_rms_norm_without_eps_and_of_tiny_rows(bolt):
    """Rows of the smallest halves: their squares are far below FP16 and above FP32's smallest."""
    g = _gen(3)
    x = torch.randint(-3, 4, (9, 1024), device="cuda", generator=g).half() * 2.0 ** -24
    x[:, 0] = 2.0 ** -24
    w, Y, Q, S = _half(g, 1024), _nan(9, 1024), _nan(9, 1024, dtype=F8), _nan(9, dtype=torch.float32)
    bolt.bolt_rms_norm(bolt.rms_norm_desc(9, 1024, eps=0.0), x, None, w, None, Y, Q, S)
    _, n, rel = rows.norm(x, None, w, 0.0, 0.0)
    rows.check_half(Y, n, rel)
    rows.check_q(Q, S, n, rel)


def test_rms_norm_of_more_rows_than_workgroups(bolt):
    """Over 2^20 rows: workgroups take several, one behind the other."""
    R, width = (1 << 20) + 77, 1032
    g = _gen(4)
    x, w, Y = _half(g, R, width), _half(g, width), _nan(R, width)
    bolt.bolt_rms_norm(bolt.rms_norm_desc(R, width), x, None, w, None, Y)
    for at in (slice(0, 300), slice(R - 400, R)):
        _, n, rel = rows.norm(x[at], None, w, 1e-5, 0.0)
        rows.check_half(Y[at], n, rel)


@pytest.mark.parametrize("R,width", [(1, 8), (300, 136), (17, 4096), (64, 11008), (3, 32768)])
def test_quantize_rows(bolt, R, width):
    g = _gen(R)
    x = _half(g, R, width, std=2.0)
    Q, S = bolt.bolt_quantize_rows(x, _nan(R, width, dtype=F8), _nan(R, dtype=torch.float32))
    rows.check_q(Q, S, x.double(), 0.0)


def test_quantize_rows_is_exact_on_values_of_the_type(bolt):
    """Every finite E4M3 times a power of two per row, the largest among them: scales and values come back bit for bit."""
    every = torch.arange(256, dtype=torch.int32, device="cuda").to(torch.uint8).view(F8).float()
    every = every[torch.isfinite(every)].repeat(4)[:1000]
    powers = 2.0 ** torch.arange(-8, 7, device="cuda").float()
    x = (every[None, :] * powers[:, None]).half()
    assert torch.equal(x.float(), every[None, :] * powers[:, None])
    Q, S = bolt.bolt_quantize_rows(x, _nan(15, 1000, dtype=F8), _nan(15, dtype=torch.float32))
    assert torch.equal(S, powers) and torch.equal(Q.float(), every.expand(15, 1000))


def test_quantize_rows_special_rows_and_strides(bolt):
    x = torch.full((6, 80), float("nan"), dtype=torch.float16, device="cuda")[:, 8:72]
    x.copy_(torch.randn(6, 64, device="cuda"))
    x[1], x[2, 3], x[3, 5] = 0.0, float("inf"), float("nan")
    Q = torch.full((6, 96), 1.0, device="cuda").to(F8)
    S = _nan(6, dtype=torch.float32)
    bolt.bolt_quantize_rows(x, Q[:, 16:80], S)
    fine = torch.tensor([0, 4, 5], device="cuda")
    rows.check_q(Q[fine][:, 16:80], S[fine], x[fine].double(), 0.0)
    assert (Q[1, 16:80].float() == 0).all() and S[1] == 0 and torch.isinf(S[2]) and torch.isnan(S[3]) and torch.isnan(Q[3, 16:80].float()).all()
    assert (Q[:, :16].float() == 1.0).all() and (Q[:, 80:].float() == 1.0).all()


# ---- layers of 8-bit operands -------------------------------------------------------------------------------------------
# every tile by its own sizes, whole and ragged reductions, outputs that end inside a tile
Q8 = [(1, 8, 16), (1, 264, 4096), (3, 1032, 528), (16, 4104, 1040), (13, 200, 11008), (17, 8, 16), (31, 4096, 2064), (45, 6152, 1008), (64, 1000, 4112),
      (100, 8192, 272), (129, 2056, 1040), (257, 4104, 784), (300, 520, 5008), (333, 12288, 144), (513, 1032, 2000), (1000, 3000, 912), (2048, 4096, 528),
      (2100, 8200, 400), (2050, 8200, 2000)]


@pytest.mark.parametrize("M,N,K", Q8)
@pytest.mark.parametrize("full,act", [(False, "none"), (True, "silu")])
def test_gemm_q8(bolt, M, N, K, full, act):
    g = _gen(M + N + K)
    (A, sa), (W, sw) = _q8(g, M, K), _q8(g, N, K, std=1 / math.sqrt(K))
    bias = _half(g, N) if full else None
    d = bolt.gemm_q8_desc(M, N, K, act=act, alpha=0.75 if full else 1.0, beta=-1.5)
    assert bolt.bolt_gemm_q8_workspace_bytes(d) == 0
    D = bolt.bolt_gemm_q8(d, A, sa, W, sw, bias, _nan(M, N))
    want, bound = ref.linear(A.double() * sa.double()[:, None], W.double() * sw.double()[:, None], None if bias is None else bias.double(), act, d.alpha, d.beta)
    rows.within(D, want, bound)


@pytest.mark.parametrize("act", ["relu", "gelu", "hardswish", "softplus"])
@pytest.mark.parametrize("M", [5, 70, 2060])
def test_gemm_q8_activations(bolt, M, act):
    N, K = (136, 272) if M < 1000 else (8200, 1040)
    g = _gen(M)
    (A, sa), (W, sw), bias = _q8(g, M, K, std=3.0), _q8(g, N, K, std=0.1), _half(g, N)
    D = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K, act=act), A, sa, W, sw, bias, _nan(M, N))
    rows.within(D, *ref.linear(A.double() * sa.double()[:, None], W.double() * sw.double()[:, None], bias.double(), act))


@pytest.mark.parametrize("M,N,K", [(1, 24, 48), (16, 136, 272), (17, 72, 144), (40, 1032, 1040), (65, 264, 80), (130, 2056, 400), (200, 12288, 272), (400, 4104, 272),
                                   (700, 4104, 144), (2050, 8200, 272), (2050, 8200, 1040)])
def test_gemm_q8_is_exact_on_integers(bolt, M, N, K):
    """Small integers and scales that are powers of two: a value in a wrong place, a lost column or a scale of another row shows."""
    g = _gen(M + K)
    integers = lambda R: torch.randint(-2, 3, (R, K), device="cuda", generator=g).float().to(F8)
    powers = lambda R: 2.0 ** torch.randint(-2, 1, (R,), device="cuda", generator=g).float()
    A, W, sa, sw = integers(M), integers(N), powers(M), powers(N)
    D = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K), A, sa, W, sw, None, _nan(M, N))
    sums = A.double() @ W.double().t().contiguous()
    assert sums.abs().max() <= 2048
    assert torch.equal(D.double(), sums * sa.double()[:, None] * sw.double()[None, :])
    D = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K), A, None, W, None, None, _nan(M, N))
    assert torch.equal(D.double(), sums)


@pytest.mark.parametrize("M", [4, 33, 300, 2060])
def test_gemm_q8_strides_and_untouched_padding(bolt, M):
    N, K, lda, ldd = (72, 208, 272, 136) if M < 1000 else (8200, 1040, 1104, 8264)
    g = _gen(M)
    (a, sa), (W, sw) = _q8(g, M, K), _q8(g, N, K)
    A = _nan(M, lda, dtype=F8)
    A.view(torch.uint8)[:, :K] = a.view(torch.uint8)
    D = torch.full((M, ldd), 7.0, dtype=torch.float16, device="cuda")
    bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K, lda=lda, ldd=ldd), A, sa, W, sw, None, D)
    rows.within(D[:, :N], *ref.linear(a.double() * sa.double()[:, None], W.double() * sw.double()[:, None], None, "none"))
    assert (D[:, N:] == 7.0).all()


@pytest.mark.parametrize("M", [9, 40, 200, 2060])
def test_gemm_q8_rows_and_columns_do_not_meet(bolt, M):
    """A NaN in a row or in its scale spoils that row only, one in a weight row that column only."""
    N, K = (136, 272) if M < 1000 else (8200, 1040)
    g = _gen(M)
    (A, sa), (W, sw) = _q8(g, M, K), _q8(g, N, K, std=0.1)
    clean = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K), A, sa, W, sw, None, _nan(M, N))
    A.view(torch.uint8)[3, 5], W.view(torch.uint8)[N - 2, K - 1] = 0x7f, 0x7f
    sa[7] = float("inf")
    D = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K), A, sa, W, sw, None, _nan(M, N))
    keep_r, keep_c = torch.ones(M, dtype=torch.bool, device="cuda"), torch.ones(N, dtype=torch.bool, device="cuda")
    keep_r[3] = keep_r[7] = keep_c[N - 2] = False
    assert torch.isnan(D[3]).all() and torch.isnan(D[:, N - 2]).all() and not torch.isfinite(D[7]).any()
    assert torch.equal(D[keep_r][:, keep_c], clean[keep_r][:, keep_c])


@pytest.mark.parametrize("M", [9, 40, 200, 2060])
def test_gemm_q8_of_bias_alone(bolt, M):
    """alpha 0: -1.5 times the bias is a number of FP32, rounded once."""
    N, K = 4104, 272
    g = _gen(M)
    (A, sa), (W, sw), bias = _q8(g, M, K), _q8(g, N, K), _half(g, N)
    D = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K, alpha=0.0, beta=-1.5), A, sa, W, sw, bias, _nan(M, N))
    assert torch.equal(D, (bias.float() * -1.5).half().expand(M, N))


def test_gemm_q8_of_weights_past_2_gib(bolt):
    """Offsets into W pass 31 bits; the 256 x 256 tiles, which the sizes would have, give way."""
    M, N, K = 260, 200008, 12288
    g = _gen(8)
    W = torch.randint(0, 256, (N, K), dtype=torch.uint8, device="cuda", generator=g).bitwise_and_(0x37).view(F8)
    A, sa = _q8(g, M, K)
    D = bolt.bolt_gemm_q8(bolt.gemm_q8_desc(M, N, K, alpha=1e-3), A, sa, W, None, None, _nan(M, N))
    for at in (slice(0, 40), slice(N - 40, N)):
        rows.within(D[:, at], *ref.linear(A.double() * sa.double()[:, None], W[at].double(), None, "none", 1e-3))


# ---- projections with adapters ------------------------------------------------------------------------------------------
def _w4(bolt, g, N, K, group):
    q = torch.randint(0, 256, (1, N, K // 2), dtype=torch.uint8, device="cuda", generator=g)
    s = ((torch.rand((1, N, -(-K // group)), device="cuda", generator=g) + 0.1) * (0.4 / math.sqrt(K))).half()
    packed = bolt.bolt_w4_pack(N, K, group, q, s, None, _nan(bolt.bolt_w4_packed_bytes(N, K, group), dtype=torch.uint8))
    return packed, ref.w4_matrix(q[0], s[0], None, group)


def _ids(g, M, n, how):
    """runs: rows of an adapter together; else each row its own.  Some have none: below zero, or past the last."""
    if how == "runs":
        ids = (torch.arange(M, device="cuda") * (n + 1) // M).int() - 1
    else:
        ids = torch.randint(-1, n + 1, (M,), dtype=torch.int32, device="cuda", generator=g)
        ids[ids == n] = 1 << 30
        ids[ids == -1] = -(1 << 31)
    return ids


def _lora(bolt, M, N, K, n, rank, weights, group, how, full=True, act="none", lda=None, ldd=None, seed=0):
    g = _gen(M + N + K + rank + seed)
    A = torch.full((M, lda or K), float("nan"), dtype=torch.float16, device="cuda")
    A[:, :K] = _half(g, M, K)
    if weights == "w4":
        W, W64 = _w4(bolt, g, N, K, group)
    else:
        W = _half(g, N, K, std=1 / math.sqrt(K))
        W64 = W.double()
    down, up = _half(g, n, rank, K, std=1 / math.sqrt(K)), _half(g, n, N, rank, std=0.5 / math.sqrt(rank))
    scales = torch.rand(n, device="cuda", generator=g) + 0.5 if full else None
    bias = _half(g, N) if full else None
    ids = _ids(g, M, n, how)
    d = bolt.gemm_lora_desc(M, N, K, n, rank, weights=weights, group=group, lda=lda, ldd=ldd, alpha=0.75 if full else 1.0, beta=-1.5, act=act)
    ws = _nan(bolt.bolt_gemm_lora_workspace_bytes(d), dtype=torch.uint8)
    D = torch.full((M, ldd or N), 7.0, dtype=torch.float16, device="cuda")
    bolt.bolt_gemm_lora(d, A, W, bias, ids, down, up, scales, D, ws)
    # (4-bit weights of many rows may be rounded to FP16 once)
    want = lambda: rows.lora(A[:, :K].double(), W64, None if bias is None else bias.double(), ids, down, up, scales, act, d.alpha, d.beta,
                             shift=ref.U16 if weights == "w4" and M >= 512 else 0.0)
    return D, want, dict(A=A, W=W, bias=bias, ids=ids, down=down, up=up, scales=scales, d=d, ws=ws)


LORA = [(1, 8, 8, 1, 8), (1, 4104, 4096, 5, 16), (2, 264, 72, 3, 24), (16, 520, 1000, 40, 8), (13, 5000, 264, 4, 128), (16, 8200, 136, 20, 40), (17, 72, 200, 2, 16),
        (33, 264, 1032, 40, 72), (64, 1000, 4104, 70, 32), (65, 520, 264, 3, 64), (130, 4104, 72, 6, 24), (300, 136, 2056, 9, 128), (513, 1032, 1000, 4, 16),
        (1100, 264, 520, 30, 8)]


@pytest.mark.parametrize("M,N,K,n,rank", LORA)
@pytest.mark.parametrize("weights,group", [("f16", 0), ("w4", 32), ("w4", 64), ("w4", 128)])
@pytest.mark.parametrize("how", ["runs", "mixed"])
def test_gemm_lora(bolt, M, N, K, n, rank, weights, group, how):
    D, want, _ = _lora(bolt, M, N, K, n, rank, weights, group, how, full=how == "mixed")
    rows.within(D, *want())


@pytest.mark.parametrize("M,N,K,n,rank", [(3300, 4200, 136, 3, 64), (3329, 4104, 72, 40, 72), (2100, 6152, 72, 500, 128), (3300, 4200, 64, 1, 8), (3300, 4200, 2056, 3, 64),
                                           (3329, 4104, 2056, 5, 72), (3329, 4104, 2056, 40, 128), (700, 4104, 1032, 6, 128), (300, 4104, 1032, 3, 72),
                                           (1500, 4104, 1032, 9, 24)])
@pytest.mark.parametrize("how", ["runs", "mixed"])
def test_gemm_lora_on_large_tiles(bolt, M, N, K, n, rank, how):
    """Every tile for many rows, with the adapters in it and, where there can be many, their share from memory: one adapter, several in a tile."""
    D, want, _ = _lora(bolt, M, N, K, n, rank, "f16", 0, how, act="relu")
    rows.within(D, *want())


@pytest.mark.parametrize("M,N,K,n,rank", [(33, 4104, 1032, 4, 24), (64, 4104, 1032, 2, 128), (90, 2056, 520, 8, 40), (100, 8200, 264, 5, 16), (300, 4104, 1032, 2, 72),
                                           (300, 4104, 520, 8, 8), (450, 4104, 1032, 1, 64)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("how", ["runs", "mixed"])
def test_gemm_lora_of_few_adapters_on_packed_tiles(bolt, M, N, K, n, rank, group, how):
    D, want, c = _lora(bolt, M, N, K, n, rank, "w4", group, how)
    rows.within(D, *want())
    # one adapter's infinity stays with its rows (infinities of both signs: no activation behind them, a ReLU makes zeros of NaN)
    c["up"][0] = float("inf")
    again = bolt.bolt_gemm_lora(c["d"], c["A"], c["W"], c["bias"], c["ids"], c["down"], c["up"], c["scales"], _nan(M, N), c["ws"].fill_(0xff))
    others = c["ids"] != 0
    assert torch.equal(again[others], D[others]) and not torch.isfinite(again[~others]).all()


@pytest.mark.parametrize("M,N,K,n,rank", [(8, 8200, 264, 5, 24), (9, 8200, 264, 5, 24), (12, 12296, 136, 16, 8), (13, 12296, 136, 40, 72), (16, 8208, 1032, 3, 16), (16, 8192, 264, 3, 16)])
@pytest.mark.parametrize("weights,group", [("f16", 0), ("w4", 32), ("w4", 128)])
@pytest.mark.parametrize("how", ["runs", "mixed"])
def test_gemm_lora_of_wide_projections(bolt, M, N, K, n, rank, weights, group, how):
    """Few rows, on the kernel for them and on tiles; a share that goes through memory, and alpha 0."""
    D, want, c = _lora(bolt, M, N, K, n, rank, weights, group, how)
    rows.within(D, *want())
    c["d"].alpha = 0.0
    D = bolt.bolt_gemm_lora(c["d"], c["A"], c["W"], c["bias"], c["ids"], c["down"], c["up"], c["scales"], _nan(M, N), c["ws"])
    assert torch.equal(D, (c["bias"].float() * -1.5).half().expand(M, N))


@pytest.mark.parametrize("how", ["runs", "mixed"])
def test_gemm_lora_over_unpacked_weights(bolt, how):
    M, N, K = 4096, 8192, 1032
    D, want, c = _lora(bolt, M, N, K, 5, 24, "w4", 32, how)
    rows.within(D, *want())
    d = c["d"]
    assert bolt.bolt_gemm_lora_workspace_bytes(d) >= N * K * 2 + M * N * 2


def test_gemm_lora_over_unpacked_weights_beyond_a_half(bolt):
    """A scale that takes weights out of FP16's range: the layer computes those outputs from the packed weights, with the adapters' share."""
    M, N, K, group, n, rank = 4096, 8192, 1032, 32, 3, 16
    g = _gen(77)
    q = torch.randint(0, 256, (1, N, K // 2), dtype=torch.uint8, device="cuda", generator=g)
    s = ((torch.rand((1, N, -(-K // group)), device="cuda", generator=g) + 0.1) * (0.4 / math.sqrt(K))).half()
    s[0, 100, 3] = 20000.0
    packed = bolt.bolt_w4_pack(N, K, group, q, s, None, _nan(bolt.bolt_w4_packed_bytes(N, K, group), dtype=torch.uint8))
    A, down, up = _half(g, M, K, std=0.01), _half(g, n, rank, K), _half(g, n, N, rank)
    ids = _ids(g, M, n, "mixed")
    d = bolt.gemm_lora_desc(M, N, K, n, rank, weights="w4", group=group)
    D = bolt.bolt_gemm_lora(d, A, packed, None, ids, down, up, None, _nan(M, N), _nan(bolt.bolt_gemm_lora_workspace_bytes(d), dtype=torch.uint8))
    want, bound = rows.lora(A.double(), ref.w4_matrix(q[0], s[0], None, group), None, ids, down, up, None, "none", shift=ref.U16)
    here = want.abs() < 60000
    assert here.float().mean() > 0.99
    rows.within(torch.where(here, D.double(), torch.zeros_like(want)), torch.where(here, want, torch.zeros_like(want)), bound)


@pytest.mark.parametrize("act", ["relu", "gelu", "hardswish", "softplus"])
@pytest.mark.parametrize("M,weights,group", [(3, "f16", 0), (40, "f16", 0), (7, "w4", 64), (70, "w4", 128)])
def test_gemm_lora_activations(bolt, M, weights, group, act):
    D, want, _ = _lora(bolt, M, 136, 264, 4, 16, weights, group, "mixed", act=act)
    rows.within(D, *want())


@pytest.mark.parametrize("M,N,K", [(1, 24, 40), (16, 136, 264), (17, 72, 136), (65, 264, 72), (300, 136, 264), (700, 1032, 264), (3300, 4200, 72), (3300, 4200, 1032)])
@pytest.mark.parametrize("how", ["runs", "mixed"])
def test_gemm_lora_is_exact_on_integers(bolt, M, N, K, how):
    g = _gen(M + K)
    n, rank = 5, 24
    ints = lambda *s: torch.randint(-1, 2, s, device="cuda", generator=g).half()
    A, W, down, up = ints(M, K), ints(N, K), ints(n, rank, K), ints(n, N, rank)
    down[:, :, 16:] = 0  # (so that every sum stays a whole number below 2048)
    scales = torch.tensor([1.0, 2.0, 0.0, -1.0, 0.5], device="cuda") * 2
    ids = _ids(g, M, n, how)
    d = bolt.gemm_lora_desc(M, N, K, n, rank)
    D = bolt.bolt_gemm_lora(d, A, W, None, ids, down, up, scales, _nan(M, N), _nan(bolt.bolt_gemm_lora_workspace_bytes(d), dtype=torch.uint8))
    want = A.double() @ W.double().t().contiguous()
    for a in range(n):
        at = (ids == a).nonzero().view(-1)
        if len(at):
            want[at] += scales[a].double() * (A[at].double() @ down[a].double().t().contiguous()) @ up[a].double().t().contiguous()
    assert want.abs().max() <= 2048 and torch.equal(D.double(), want)


@pytest.mark.parametrize("M", [4, 16, 33, 300])
@pytest.mark.parametrize("weights,group", [("f16", 0), ("w4", 64)])
def test_gemm_lora_strides_and_untouched_padding(bolt, M, weights, group):
    D, want, _ = _lora(bolt, M, 72, 200, 3, 16, weights, group, "mixed", lda=264, ldd=136)
    rows.within(D[:, :72], *want())
    assert (D[:, 72:] == 7.0).all()


@pytest.mark.parametrize("K", [72, 2056])
def test_gemm_lora_large_tiles_strides(bolt, K):
    D, want, _ = _lora(bolt, 3300, 4200, K, 3, 16, "f16", 0, "mixed", lda=K + 64, ldd=4264)
    rows.within(D[:, :4200], *want())
    assert (D[:, 4200:] == 7.0).all()


@pytest.mark.parametrize("M,N,K", [(1, 264, 520), (16, 264, 520), (40, 264, 520), (300, 264, 520), (3300, 4200, 72), (3300, 4200, 2056)])
@pytest.mark.parametrize("weights,group", [("f16", 0), ("w4", 64)])
def test_gemm_lora_without_adapters_is_the_projection(bolt, M, N, K, weights, group):
    """No row has an adapter, and all of them hold NaN: the outputs are those of the projection alone."""
    _, _, c = _lora(bolt, M, N, K, 3, 16, weights, group, "mixed")
    ids = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    nan = lambda t: torch.full_like(t, float("nan"))
    D = bolt.bolt_gemm_lora(c["d"], c["A"], c["W"], c["bias"], ids, nan(c["down"]), nan(c["up"]), nan(c["scales"]), _nan(M, N), c["ws"].fill_(0xff))
    plain = rows.lora(c["A"].double(), c["W"].double() if weights == "f16" else _w4(bolt, _w4_gen(c, M, N, K), N, K, group)[1], c["bias"].double(), ids, c["down"],
                      c["up"], c["scales"], "none", 0.75, -1.5, shift=ref.U16 if weights == "w4" and M >= 512 else 0.0)
    rows.within(D, *plain)


def _w4_gen(c, M, N, K):
    """The generator of _lora's weights, at the place where it makes them."""
    g = _gen(M + N + K + c["d"].rank)
    _half(g, M, K)
    return g


@pytest.mark.parametrize("M,N,K", [(16, 264, 520), (40, 264, 520), (300, 264, 520), (3300, 4200, 72), (3300, 4200, 2056)])
@pytest.mark.parametrize("weights,group", [("f16", 0), ("w4", 64)])
@pytest.mark.parametrize("where", ["down", "up", "scale", "row"])
def test_gemm_lora_adapters_do_not_meet(bolt, M, N, K, weights, group, where):
    """An infinity or NaN of one adapter, or of one row, reaches its own rows only."""
    D, _, c = _lora(bolt, M, N, K, 4, 40, weights, group, "mixed")
    bad = torch.zeros(M, dtype=torch.bool, device="cuda")
    if where == "row":
        c["A"][M // 2, 7] = float("inf")
        bad[M // 2] = True
    else:
        bad = c["ids"] == 2
        if where == "down":
            c["down"][2, 3, 5] = float("nan")
        elif where == "up":
            c["up"][2] = float("inf")
        else:
            c["scales"][2] = float("inf")
    again = bolt.bolt_gemm_lora(c["d"], c["A"], c["W"], c["bias"], c["ids"], c["down"], c["up"], c["scales"], _nan(M, N), c["ws"].fill_(0xff))
    assert bad.any() and torch.equal(again[~bad], D[~bad])
    assert not torch.isfinite(again[bad]).all(dim=1).any()


@pytest.mark.parametrize("M,N", [(1, 4104), (29, 264), (300, 1032), (700, 4104), (3300, 4200)])
def test_gemm_lora_gives_the_same_bits_again(bolt, M, N):
    D, _, c = _lora(bolt, M, N, 2056 if M > 3000 else 264, 7, 24, "f16", 0, "mixed")
    for _ in range(3):
        again = bolt.bolt_gemm_lora(c["d"], c["A"], c["W"], c["bias"], c["ids"], c["down"], c["up"], c["scales"], _nan(M, N), c["ws"].fill_(0xff))
        assert torch.equal(D, again)


@pytest.mark.parametrize("M,N,K", [(4, 264, 520), (29, 264, 520), (300, 1032, 264), (600, 1032, 264), (3300, 4200, 72), (3300, 4200, 2056)])
@pytest.mark.parametrize("weights,group", [("f16", 0), ("w4", 64)])
def test_gemm_lora_of_bias_alone(bolt, M, N, K, weights, group):
    """alpha 0, with which no sum can start at beta / alpha times the bias: -1.5 times the bias is a number of FP32, rounded once."""
    _, _, c = _lora(bolt, M, N, K, 5, 24, weights, group, "mixed")
    d = bolt.gemm_lora_desc(M, N, K, 5, 24, weights=weights, group=group, alpha=0.0, beta=-1.5)
    D = bolt.bolt_gemm_lora(d, c["A"], c["W"], c["bias"], c["ids"], c["down"], c["up"], c["scales"], _nan(M, N),
                            _nan(bolt.bolt_gemm_lora_workspace_bytes(d), dtype=torch.uint8))
    assert torch.equal(D, (c["bias"].float() * -1.5).half().expand(M, N))


@pytest.mark.parametrize("M,N,K", [(4, 264, 520), (29, 1032, 520), (300, 1032, 264), (3300, 4200, 72)])
@pytest.mark.parametrize("weights,group", [("f16", 0), ("w4", 64)])
def test_gemm_lora_in_a_graph_of_other_requests(bolt, M, N, K, weights, group):
    """What a graph has captured goes by the ids that a replay finds: one adapter for all rows, one each, none at all."""
    _, _, c = _lora(bolt, M, N, K, 40, 24, weights, group, "runs")
    call = lambda D: bolt.bolt_gemm_lora(c["d"], c["A"], c["W"], c["bias"], c["ids"], c["down"], c["up"], c["scales"], D, c["ws"])
    D = _nan(M, N)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(D)
    rows_of = torch.arange(M, device="cuda", dtype=torch.int32)
    for ids in (rows_of % 40, rows_of * 0 + 39, rows_of * 0 - 1, rows_of * 40 // M):
        c["ids"].copy_(ids)
        want = call(_nan(M, N)).clone()
        c["ws"].fill_(0xff)
        D.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(D, want)


def test_gemm_lora_of_adapters_past_2_gib(bolt):
    """Offsets into the adapters pass 32 bits."""
    M, N, K, n, rank = 6, 8200, 8192, 2100, 128
    g = _gen(9)
    down, up = torch.zeros((n, rank, K), dtype=torch.float16, device="cuda"), torch.zeros((n, N, rank), dtype=torch.float16, device="cuda")
    ids = torch.tensor([n - 1, 0, 1025, -1, n - 2, n], dtype=torch.int32, device="cuda")
    for a in (0, 1025, n - 2, n - 1):
        down[a], up[a] = _half(g, rank, K, std=0.01), _half(g, N, rank, std=0.1)
    for rows_ in (M, 40):
        i = ids.repeat(8)[:rows_].contiguous()
        A, W = _half(g, rows_, K), _half(g, N, K, std=0.01)
        d = bolt.gemm_lora_desc(rows_, N, K, n, rank)
        D = bolt.bolt_gemm_lora(d, A, W, None, i, down, up, None, _nan(rows_, N), _nan(bolt.bolt_gemm_lora_workspace_bytes(d), dtype=torch.uint8))
        used = torch.tensor([0, 1025, n - 2, n - 1], device="cuda")
        short = torch.full_like(i, -1)
        for j, a in enumerate(used.tolist()):
            short[i == a] = j
        rows.within(D, *rows.lora(A.double(), W.double(), None, short, down[used], up[used], None, "none"))


# ---- together -----------------------------------------------------------------------------------------------------------
class _Block:
    """What runs between two attention layers: norm of the new residual stream in both forms, an 8-bit projection of one, a projection with the
    requests' adapters of the other, its output quantised again for an 8-bit projection back to the stream's width."""

    def __init__(self, bolt, M, width, hidden, seed=1):
        g = _gen(seed)
        self.bolt, self.M = bolt, M
        self.x, self.stream, self.weight = _half(g, M, width), _half(g, M, width, std=2.0), _half(g, width, std=0.2) + 1
        (self.W, self.sw), (self.V, self.sv) = _q8(g, hidden, width, std=1 / math.sqrt(width)), _q8(g, width, hidden, std=1 / math.sqrt(hidden))
        self.P, self.down, self.up = _half(g, hidden, width, std=1 / math.sqrt(width)), _half(g, 4, 16, width, std=0.02), _half(g, 4, hidden, 16, std=0.1)
        self.scales, self.ids = torch.rand(4, device="cuda", generator=g), _ids(g, M, 4, "mixed")
        self.sum, self.y, self.q, self.s = _nan(M, width), _nan(M, width), _nan(M, width, dtype=F8), _nan(M, dtype=torch.float32)
        self.a, self.b, self.bq, self.bs, self.out = _nan(M, hidden), _nan(M, hidden), _nan(M, hidden, dtype=F8), _nan(M, dtype=torch.float32), _nan(M, width)
        self.norm, self.up_desc, self.down_desc = bolt.rms_norm_desc(M, width), bolt.gemm_q8_desc(M, hidden, width, act="silu"), bolt.gemm_q8_desc(M, width, hidden)
        self.lora = bolt.gemm_lora_desc(M, hidden, width, 4, 16)
        self.ws = _nan(bolt.bolt_gemm_lora_workspace_bytes(self.lora), dtype=torch.uint8)

    def __call__(self):
        b = self.bolt
        b.bolt_rms_norm(self.norm, self.x, self.stream, self.weight, self.sum, self.y, self.q, self.s)
        b.bolt_gemm_q8(self.up_desc, self.q, self.s, self.W, self.sw, None, self.a)
        b.bolt_gemm_lora(self.lora, self.y, self.P, None, self.ids, self.down, self.up, self.scales, self.b, self.ws)
        b.bolt_quantize_rows(self.b, self.bq, self.bs)
        b.bolt_gemm_q8(self.down_desc, self.bq, self.bs, self.V, self.sv, None, self.out)

    def check(self):
        """Each step from what the step before it wrote."""
        v, n, rel = rows.norm(self.x, self.stream, self.weight, 1e-5, 0.0)
        rows.check_half(self.sum, v, rows.H32)
        rows.check_half(self.y, n, rel)
        rows.check_q(self.q, self.s, n, rel)
        rows.within(self.a, *ref.linear(self.q.double() * self.s.double()[:, None], self.W.double() * self.sw.double()[:, None], None, "silu"))
        rows.within(self.b, *rows.lora(self.y.double(), self.P.double(), None, self.ids, self.down, self.up, self.scales, "none"))
        rows.check_q(self.bq, self.bs, self.b.double(), 0.0)
        rows.within(self.out, *ref.linear(self.bq.double() * self.bs.double()[:, None], self.V.double() * self.sv.double()[:, None], None, "none"))


@pytest.mark.parametrize("M", [1, 20, 400])
def test_block(bolt, M):
    b = _Block(bolt, M, 1024, 2056 // 16 * 16)
    b()
    b.check()


@pytest.mark.parametrize("M", [1, 48, 600])
def test_block_in_a_graph(bolt, M):
    """Captured and replayed, with new inputs and eager work between the replays; every replay equals the eager result."""
    b = _Block(bolt, M, 1024, 1536)
    b()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b()
    for i in range(4):
        b.x.normal_(generator=_gen(100 + i))
        b.stream.normal_(generator=_gen(200 + i))
        b.ids.copy_(_ids(_gen(300 + i), M, 4, "mixed"))
        b()
        eager = [t.clone() for t in (b.sum, b.y, b.s, b.a, b.b, b.bs, b.out)]
        q = b.q.view(torch.uint8).clone()
        for t in (b.sum, b.y, b.a, b.b, b.out):
            t.fill_(float("nan"))
        b.ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        for want, got in zip(eager, (b.sum, b.y, b.s, b.a, b.b, b.bs, b.out)):
            assert torch.equal(want, got)
        assert torch.equal(q, b.q.view(torch.uint8))
    b.check()


def test_blocks_on_two_streams(bolt):
    """Two at once, each on a stream and with buffers of its own."""
    blocks = [_Block(bolt, M, 1024, 1536, seed=M) for M in (40, 300)]
    streams = [torch.cuda.Stream() for _ in blocks]
    torch.cuda.synchronize()
    for _ in range(5):
        for b, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                b()
    torch.cuda.synchronize()
    for b in blocks:
        b.check()


def test_python_refuses_other_tensors(bolt):
    x, w, y = torch.zeros(4, 64, dtype=torch.float16, device="cuda"), torch.ones(64, dtype=torch.float16, device="cuda"), torch.zeros(4, 64, dtype=torch.float16, device="cuda")
    d = bolt.rms_norm_desc(4, 64)
    for bad in (dict(x=x.float()), dict(x=x[:3]), dict(x=x.t()), dict(x=x.cpu()), dict(y=y[:, :32]), dict(weight=w[:32]), dict(residual=x[:1])):
        a = dict(x=x, residual=None, weight=w, y=y)
        a.update(bad)
        with pytest.raises(AssertionError):
            bolt.bolt_rms_norm(d, **a)
    with pytest.raises(AssertionError):
        bolt.bolt_rms_norm(d, x, None, w, None, None, torch.zeros(4, 64, dtype=torch.uint8, device="cuda"), torch.zeros(4, device="cuda"))
    with pytest.raises(bolt.BoltError):
        bolt.bolt_rms_norm(d, x, None, w, None, None, torch.zeros(4, 64, device="cuda").to(F8), None)
    q, W, D = torch.zeros(4, 64, device="cuda").to(F8), torch.zeros(16, 64, device="cuda").to(F8), torch.zeros(4, 16, dtype=torch.float16, device="cuda")
    for bad in (dict(A=q[:3]), dict(A=x), dict(W=W[:8]), dict(D=D[:2]), dict(a_scales=torch.ones(3, device="cuda")), dict(w_scales=torch.ones(16, device="cuda").half())):
        a = dict(A=q, a_scales=None, W=W, w_scales=None, bias=None, D=D)
        a.update(bad)
        with pytest.raises(AssertionError):
            bolt.bolt_gemm_q8(bolt.gemm_q8_desc(4, 16, 64), **a)
    l = bolt.gemm_lora_desc(4, 16, 64, 2, 8)
    good = dict(A=x, W=torch.zeros(16, 64, dtype=torch.float16, device="cuda"), bias=None, ids=torch.zeros(4, dtype=torch.int32, device="cuda"),
                down=torch.zeros(2, 8, 64, dtype=torch.float16, device="cuda"), up=torch.zeros(2, 16, 8, dtype=torch.float16, device="cuda"), scales=None, D=D,
                workspace=torch.zeros(bolt.bolt_gemm_lora_workspace_bytes(l), dtype=torch.uint8, device="cuda"))
    for bad in (dict(ids=good["ids"].long()), dict(ids=good["ids"][:3]), dict(down=good["down"][:1]), dict(up=good["up"][:1]), dict(W=q), dict(scales=torch.ones(1, device="cuda"))):
        with pytest.raises(AssertionError):
            bolt.bolt_gemm_lora(l, **{**good, **bad})
    with pytest.raises(bolt.BoltError):
        bolt.bolt_gemm_lora(l, **{**good, "workspace": None})


@pytest.mark.parametrize("weights", ["f16", "w4"])
def test_example_runs(weights):
    """The example checks its own rows against float64 and raises if they are off."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, os.path.join(root, "examples", "served_layer.py"), "--tokens", "1", "24", "300", "--width", "1024", "--hidden",
                          "1536", "--weights", weights], capture_output=True, text=True, timeout=110)
    assert out.returncode == 0 and out.stdout.count("us per pass") == 3, out.stdout + out.stderr
