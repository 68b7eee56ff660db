"""CPU-only: what the 4-bit layer, the routing and the experts' products refuse, and with which status; sizes of their buffers."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2110_15238_amd", "libbolt.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libbolt.so not built (run __graft_entry__.build())")

OK, INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE, LAUNCH, ILLEGAL = range(7)
A16 = 0x1000  # an address that is never read: every call here is refused before a launch


@pytest.fixture(scope="module")
def bolt():
    import paper_2110_15238_amd as b
    return b


def test_struct_layouts(bolt):
    assert C.sizeof(bolt.GemmW4Desc) == 36 and C.sizeof(bolt.MoeRouteDesc) == 40 and C.sizeof(bolt.MoeDesc) == 44


def test_packed_bytes(bolt):
    # 16 rows x 128 columns are 1024 bytes; 2 bytes of scale and 1 of zero point per row and group of the padded matrix
    assert bolt.bolt_w4_packed_bytes(16, 128, 128) == 1024 + 16 * 3
    assert bolt.bolt_w4_packed_bytes(8, 8, 32) == 1024 + 16 * 4 * 3
    assert bolt.bolt_w4_packed_bytes(24, 136, 64, 3) == 3 * (2 * 2 * 1024 + 2 * 2 * 2 * 16 * 3)
    for bad in ((0, 128, 128, 1), (16, 0, 128, 1), (16, 128, 96, 1), (12, 128, 128, 1), (16, 100, 32, 1), (16, 128, 128, 0)):
        assert bolt.bolt_w4_packed_bytes(*bad) == 0
    assert bolt.bolt_w4_packed_bytes(1 << 20, 1 << 14, 128) > 1 << 33  # counted in 64 bits


def _gemm(bolt, d, A=A16, packed=A16, bias=None, D=A16, ws=None, ws_bytes=0):
    return bolt.binding.raw().bolt_gemm_w4(C.byref(d), A, packed, bias, D, ws, ws_bytes, None)


def test_gemm_w4_refusals(bolt):
    D = bolt.gemm_w4_desc
    raw = bolt.binding.raw()
    assert raw.bolt_gemm_w4(None, A16, A16, None, A16, None, 0, None) == INVALID
    assert _gemm(bolt, D(0, 64, 128, 64)) == OK  # nothing to do
    for bad in (D(-1, 64, 128, 64), D(1, 0, 128, 64), D(1, 64, 0, 64), D(1, 64, 128, 48), D(1, 64, 128, 64, lda=64), D(1, 64, 128, 64, ldd=32)):
        assert _gemm(bolt, bad) == INVALID
    bad = D(1, 64, 128, 64)
    bad.act = 6
    assert _gemm(bolt, bad) == INVALID
    for bad in (D(1, 60, 128, 64), D(1, 64, 124, 64), D(1, 64, 128, 64, lda=132), D(1, 64, 128, 64, ldd=68)):
        assert _gemm(bolt, bad) == ALIGNMENT
    assert _gemm(bolt, D(1, 64, 128, 64, lda=(1 << 21) + 8)) == UNSUPPORTED
    good = D(1, 64, 128, 64)
    assert _gemm(bolt, good, A=None) == INVALID and _gemm(bolt, good, packed=None) == INVALID and _gemm(bolt, good, D=None) == INVALID
    assert _gemm(bolt, good, A=A16 + 2) == ALIGNMENT and _gemm(bolt, good, bias=A16 + 8) == ALIGNMENT
    big = D(4096, 8192, 4096, 128)
    need = bolt.bolt_gemm_w4_workspace_bytes(big)
    assert need == 8192 * 4096 * 2 and bolt.bolt_gemm_w4_workspace_bytes(good) == 0
    assert _gemm(bolt, big) == WORKSPACE and _gemm(bolt, big, ws=A16, ws_bytes=need - 1) == WORKSPACE
    assert _gemm(bolt, big, ws=A16 + 4, ws_bytes=need) == ALIGNMENT


def test_silu_is_refused_where_it_is_not_offered(bolt):
    assert bolt.bolt_check(bolt.OP_GEMM, bolt.gemm_desc(64, 64, 64, act="silu")) == INVALID
    assert bolt.bolt_check(bolt.OP_CONV2D, bolt.conv_desc(1, 8, 8, 64, 64, 1, 1, act="silu")) == INVALID


def test_pack_refusals(bolt):
    f = bolt.binding.raw().bolt_w4_pack
    n = bolt.bolt_w4_packed_bytes(64, 128, 64)
    assert f(64, 128, 63, 1, A16, A16, None, A16, n, None) == INVALID
    assert f(60, 128, 64, 1, A16, A16, None, A16, n, None) == ALIGNMENT
    assert f(64, 128, 64, 0, A16, A16, None, A16, n, None) == INVALID
    assert f(64, 128, 64, 1, None, A16, None, A16, n, None) == INVALID
    assert f(64, 128, 64, 1, A16 + 4, A16, None, A16, n, None) == ALIGNMENT
    assert f(64, 128, 64, 1, A16, A16, None, A16, n - 1, None) == WORKSPACE


def _route(bolt, d, logits=A16, bias=None, mask=None, ids=A16, weights=A16, offsets=A16, order=A16, ws=None, ws_bytes=0):
    return bolt.binding.raw().bolt_moe_route(C.byref(d), logits, bias, mask, ids, weights, offsets, order, ws, ws_bytes, None)


def test_route_refusals(bolt):
    D = bolt.moe_route_desc
    for bad in (D(-1, 8, 2), D(4, 0, 1), D(4, 8, 0), D(4, 8, 9), D(4, 8, 2, groups=3), D(4, 8, 2, groups=0), D(4, 8, 2, groups=2, top_groups=3),
                D(4, 8, 5, groups=2, top_groups=1), D(4, 8, 2, ld=7)):
        assert _route(bolt, bad) == INVALID
    for field, value in (("score", 2), ("logits_type", 2)):
        bad = D(4, 8, 2)
        setattr(bad, field, value)
        assert _route(bolt, bad) == INVALID
    for bad in (D(4, 513, 2), D(4, 64, 17), D(4, 34, 2, groups=17), D(1 << 30, 8, 4)):
        assert _route(bolt, bad) == UNSUPPORTED
    good = D(4, 8, 2)
    for name in ("logits", "ids", "weights", "offsets", "order"):
        assert _route(bolt, good, **{name: None}) == INVALID
        assert _route(bolt, good, **{name: A16 + 4}) == ALIGNMENT
    many = D(1000, 128, 4)
    need = bolt.bolt_moe_route_workspace_bytes(many)
    assert need > 0 and bolt.bolt_moe_route_workspace_bytes(good) == 0
    assert _route(bolt, many) == WORKSPACE and _route(bolt, many, ws=A16, ws_bytes=need - 1) == WORKSPACE


def _experts(bolt, d, ws=A16, ws_bytes=1 << 40, **kw):
    names = ("x", "w_up", "b_up", "w_down", "b_down", "ids", "weights", "offsets", "order", "y")
    at = {n: A16 for n in names}
    at.update(b_up=None, b_down=None)
    at.update(kw)
    return bolt.binding.raw().bolt_moe_experts(C.byref(d), *[at[n] for n in names], ws, ws_bytes, None)


def test_experts_refusals(bolt):
    D = bolt.moe_desc
    for bad in (D(-1, 8, 2, 64, 64), D(4, 0, 1, 64, 64), D(4, 8, 0, 64, 64), D(4, 8, 9, 64, 64), D(4, 8, 2, 0, 64), D(4, 8, 2, 64, 0),
                D(4, 8, 2, 64, 64, ldx=56), D(4, 8, 2, 64, 64, ldy=56), D(4, 8, 2, 64, 64, weights="w4", group=16)):
        assert _experts(bolt, bad) == INVALID
    for field, value in (("act", 6), ("gated", 2), ("weights", 2)):
        bad = D(4, 8, 2, 64, 64)
        setattr(bad, field, value)
        assert _experts(bolt, bad) == INVALID
    for bad in (D(4, 8, 2, 60, 64), D(4, 8, 2, 64, 60), D(4, 8, 2, 64, 64, ldx=68), D(4, 8, 2, 64, 64, ldy=68)):
        assert _experts(bolt, bad) == ALIGNMENT
    for bad in (D(4, 513, 2, 64, 64), D(4, 64, 17, 64, 64), D(1 << 30, 8, 4, 64, 64), D(4, 8, 2, 64, (1 << 20) + 8)):
        assert _experts(bolt, bad) == UNSUPPORTED
    # x past 2 GiB runs on the kernel of few rows, which has no grid for this many
    assert _experts(bolt, D(300000, 8, 8, 4096, 4096)) == UNSUPPORTED
    good = D(4, 8, 2, 64, 64)
    for name in ("x", "w_up", "w_down", "ids", "weights", "offsets", "order", "y"):
        assert _experts(bolt, good, **{name: None}) == INVALID
        assert _experts(bolt, good, **{name: A16 + 8}) == ALIGNMENT
    need = bolt.bolt_moe_workspace_bytes(good)
    assert need >= 4 * 2 * (64 * 2 + 64 * 4)
    assert _experts(bolt, good, ws=None) == WORKSPACE and _experts(bolt, good, ws_bytes=need - 1) == WORKSPACE
    assert _experts(bolt, D(0, 8, 2, 64, 64), ws=None, ws_bytes=0) == OK


def test_python_calls_check_their_tensors(bolt):
    """Tensors on the CPU, of another type or too small are refused before anything reaches the library."""
    import torch
    h = torch.zeros(64, 64, dtype=torch.float16)
    with pytest.raises(AssertionError, match="CUDA float16"):
        bolt.bolt_gemm_w4(bolt.gemm_w4_desc(4, 64, 64, 64), h, torch.zeros(1, dtype=torch.uint8), None, h)
    with pytest.raises(AssertionError, match="logits: expects a contiguous CUDA float32"):
        bolt.bolt_moe_route(bolt.moe_route_desc(4, 8, 2, logits="f32"), h, None, None, h, h, h, h)
    with pytest.raises(AssertionError, match="x: expects|w_up: expects"):
        bolt.bolt_moe_experts(bolt.moe_desc(4, 8, 2, 64, 64), h, h, None, h, None, h, h, h, h, h, None)
