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
