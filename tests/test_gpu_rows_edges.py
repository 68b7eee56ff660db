"""GPU: 8-bit layers and projections with adapters where a kernel, a size or a range is easily left out (tests/rows_cases.py), against the 64-bit references
of tests/rows_ref.py."""
import math

import pytest

import llm_ref as ref
import rows_cases as cases
import rows_ref as rows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from test_gpu_rows import _gen, _half, _nan, _w4, bolt  # noqa: E402, F401


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
