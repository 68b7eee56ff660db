"""GPU: 8-bit layers and projections with adapters where a kernel, a size or a range is easily left out (tests/rows_cases.py), against the 64-bit references
of tests/rows_ref.py."""
import math

import pytest

import llm_ref as ref
import rows_cases as cases
import rows_ref as rows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from test_gpu_rows import F8, _gen, _half, _nan, _q8, _w4, bolt  # noqa: E402, F401


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
