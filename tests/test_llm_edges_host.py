"""CPU-only: sizes at the edge of what the operators of language models accept.  Every call is one that is refused or has nothing to do, so
no address is read."""
import ctypes as C
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2110_15238_amd", "libbolt.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libbolt.so not built (run __graft_entry__.build())")

OK, INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE, LAUNCH, ILLEGAL = range(7)
A16, MUCH = 0x1000, 1 << 50
MOST = (1 << 31) - (1 << 16)  # rows, or slots


@pytest.fixture(scope="module")
def bolt():
    import paper_2110_15238_amd as b
    return b


def _route(bolt, d):
    return bolt.binding.raw().bolt_moe_route(C.byref(d), A16, None, None, A16, A16, A16, A16, A16, MUCH, None)


def _experts(bolt, d):
    return bolt.binding.raw().bolt_moe_experts(C.byref(d), A16, A16, None, A16, None, A16, A16, A16, A16, A16, A16, MUCH, None)


def _gemm(bolt, d):
    return bolt.binding.raw().bolt_gemm_w4(C.byref(d), A16, A16, None, A16, A16, MUCH, None)


def test_slots_that_32_bits_cannot_count_past_are_refused(bolt):
    """2^31 - 16 slots: the last wave's share of the lists would end at 2^31.  The most that is accepted leaves room for it."""
    for tokens, k in ((134217727, 16), ((1 << 31) - 1, 1), (MOST + 1, 1)):
        assert _route(bolt, bolt.moe_route_desc(tokens, 16, k)) == UNSUPPORTED
        assert bolt.bolt_moe_route_workspace_bytes(bolt.moe_route_desc(tokens, 16, k)) == 0
        assert _experts(bolt, bolt.moe_desc(tokens, 16, k, 8, 8)) == UNSUPPORTED
        assert bolt.bolt_moe_workspace_bytes(bolt.moe_desc(tokens, 16, k, 8, 8)) == 0
    for tokens, k in ((MOST // 16, 16), (MOST, 1)):
        assert 256 * 16 * 4 >= bolt.bolt_moe_route_workspace_bytes(bolt.moe_route_desc(tokens, 16, k)) > 0
        assert bolt.bolt_moe_workspace_bytes(bolt.moe_desc(tokens, 16, k, 8, 8)) >= tokens * k * (8 * 2 + 8 * 4)


def test_rows_that_32_bits_cannot_count_past_are_refused(bolt):
    for rows in ((1 << 31) - 1, MOST + 1):
        assert _gemm(bolt, bolt.gemm_w4_desc(rows, 8, 8, 32)) == UNSUPPORTED


def test_launches_of_two_to_the_32_threads_are_refused(bolt):
    """2^30 rows of 8 outputs (17 GB on either side) are 2^24 tiles of 64 x 128, 512 threads each; 2^30 slots of 8 x 8 experts (a GB of x)
    2^23 of 128 x 256."""
    assert _gemm(bolt, bolt.gemm_w4_desc(1 << 30, 8, 8, 32)) == UNSUPPORTED
    assert _gemm(bolt, bolt.gemm_w4_desc(1 << 30, 8, 8, 32, alpha=0.0)) == UNSUPPORTED  # (alpha 0: weights as they are packed)
    assert _experts(bolt, bolt.moe_desc(1 << 26, 16, 16, 8, 8, weights="w4", group=32)) == UNSUPPORTED


@pytest.mark.parametrize("weights,group,width", [("f16", 0, 4096), ("w4", 128, 8192), ("w4", 32, 4096)])
def test_many_rows_past_2_gib_are_refused_where_the_deep_kernel_would_take_2_to_the_32_threads(bolt, weights, group, width):
    """The deep kernel of few rows has a workgroup for every 16 rows and 32 weight rows.  (Gated groups of 32 take it from 17 steps of 128 on.)"""
    assert _experts(bolt, bolt.moe_desc(300000, 8, 8, width, 4096, weights=weights, group=group)) == UNSUPPORTED


def test_addresses_of_device_variables_are_looked_up_for_each_device(tmp_path):
    """The zeros that stand for a missing bias lie elsewhere on every GPU of a process.  The lookup on the host alone, with made-up devices; and
    nothing in the library asks for such an address but through it."""
    csrc = os.path.join(ROOT, "paper_2110_15238_amd", "csrc")
    (tmp_path / "t.cpp").write_text("""
#include "per_device.hpp"
int main() {
  static bolt::PerDevice known;
  int asked = 0, zeros[3];
  auto get = [&](int device) { return known.get(device, [&]() -> void* { ++asked; return device == 2 ? nullptr : &zeros[device]; }); };
  for (int i = 0; i < 3; ++i)
    if (get(0) != &zeros[0] || get(1) != &zeros[1] || get(2)) return 1;
  return asked != 3 || get(-1) || get(bolt::PerDevice::kMaxDevices);
}
""")
    subprocess.run(["g++", "-std=c++17", "-I" + csrc, "-o", str(tmp_path / "t"), str(tmp_path / "t.cpp"), "-pthread"], check=True)
    subprocess.run([str(tmp_path / "t")], check=True)
    calls = [f for f in sorted(os.listdir(csrc)) if f.endswith((".hip", ".hpp")) for _ in re.findall("hipGetSymbolAddress[(]", open(os.path.join(csrc, f)).read())]
    assert calls == ["bolt_device.hpp"]


def test_without_rows_no_address_is_asked_for(bolt):
    """A tensor without elements has a null address."""
    raw = bolt.binding.raw()
    assert raw.bolt_gemm_w4(C.byref(bolt.gemm_w4_desc(0, 64, 128, 64)), None, None, None, None, None, 0, None) == OK
    assert raw.bolt_moe_experts(C.byref(bolt.moe_desc(0, 8, 2, 64, 64)), *[None] * 11, 0, None) == OK


@pytest.mark.parametrize("experts", [8, 128, 256, 257, 512])
def test_workspace_of_the_routing_does_not_fall_as_tokens_grow(bolt, experts):
    near = {n + d for n in (16, 48, 64, 512, 8192, 16384, 24576, 65536, 1 << 20, 1 << 26) for d in range(-65, 66, 13)} | {1, 48, 49, 64, 65, 8192, 8193, 16384, 16385}
    tokens = sorted(n for n in near if n > 0)
    held = [bolt.bolt_moe_route_workspace_bytes(bolt.moe_route_desc(n, experts, 4)) for n in tokens]
    assert held == sorted(held) and held[0] == 0 and held[-1] == 256 * experts * 4


def test_workspace_of_the_experts_does_not_fall_as_tokens_grow(bolt):
    held = [bolt.bolt_moe_workspace_bytes(bolt.moe_desc(n, 16, 4, 264, 136)) for n in range(0, 3000, 7)]
    assert held == sorted(held)


@pytest.mark.parametrize("N,K,group", [(1024, 8192, 128), (4096, 4096, 64), (256, 8192, 32), (72, 4104, 32), (12288, 520, 128)])
@pytest.mark.parametrize("act", ["relu", "silu"])
def test_workspace_of_the_4_bit_layer_does_not_fall_as_rows_grow(bolt, N, K, group, act):
    held = [bolt.bolt_gemm_w4_workspace_bytes(bolt.gemm_w4_desc(M, N, K, group, act=act)) for M in (*range(1, 9000, 13), 1 << 17, 1 << 20)]
    assert held == sorted(held) and held[0] == 0 and held[-1] == N * K * 2


def test_weights_of_2_gib_are_not_unpacked(bolt):
    assert bolt.bolt_gemm_w4_workspace_bytes(bolt.gemm_w4_desc(4096, 1 << 15, 1 << 15, 128)) == 0


def test_kernels_keep_their_working_set_in_registers():
    """The compiler's report of the build: no kernel of these operators spills, but for the persistent one of many rows, which may outside its k
    loop (44 to 84 bytes a lane).  Skipped where only the built library was shipped."""
    build = os.path.join(ROOT, "paper_2110_15238_amd", "csrc", "_build")
    if not os.path.exists(build):
        pytest.skip("no build directory (library shipped pre-built)")
    seen = set()
    for name in ("inst_few_rows_f16", "inst_few_rows_w4", "inst_shared_rows_f16", "inst_shared_rows_w4", "inst_moe_tile", "moe_api"):
        found = re.findall(r"Function Name: (\S+)\s+VGPRs: \d+\s+ScratchSize \[bytes/lane\]: (\d+)", open(os.path.join(build, name + ".usage")).read())
        assert found
        for kernel, scratch in found:
            seen.add(kernel)
            assert int(scratch) <= (128 if "moe_pp_kernel" in kernel else 0), (kernel, scratch)
    for family in ("few_rows_kernel", "few_rows_walk_kernel", "shared_rows_kernel", "moe_tile_kernel", "moe_pp_kernel", "moe_route_kernel"):
        assert any(family in k for k in seen), family
