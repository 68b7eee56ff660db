"""CPU-only: which kernels run 8-bit layers and projections with adapters, in a process whose HIP runtime is tests/hip_recorder.c."""
import os

import pytest

import rows_cases as cases
from test_host_launches import run  # noqa: F401  (the fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2110_15238_amd", "libbolt.so")),
                                reason="libbolt.so not built (run __graft_entry__.build())")

CALLS = """
import re
at = lambda i: 0x100000 * (i + 1)

def kernels():  # name<template arguments> of what was launched
    out = []
    for name in rec.recorder_launches().decode().split():
        m = re.match(r"_ZN4bolt(\\d+)", name)
        n, rest = int(m.group(1)), name[m.end():]
        if rest.startswith("_GLOBAL__N_1"): m = re.match(r"_GLOBAL__N_1(\\d+)", rest); n, rest = int(m.group(1)), rest[m.end():]
        args = re.match(r"I((?:L[ib]n?\\d+E)*)", rest[n:])
        out.append(rest[:n] + "<" + ",".join(re.findall(r"L[ib](n?\\d+)E", args.group(1) if args else "")) + ">")
    return out

def q8(M, N, K, **k):
    d = b.gemm_q8_desc(M, N, K, **k)
    s = lib.bolt_gemm_q8(C.byref(d), at(0), at(1), at(2), at(3), at(4), at(5), None, 0, None)
    return s, kernels()

def lora(M, N, K, n, rank, weights="f16", group=0, **k):
    d = b.gemm_lora_desc(M, N, K, n, rank, weights=weights, group=group, **k)
    s = lib.bolt_gemm_lora(C.byref(d), *map(at, range(9)), 1 << 60, None)
    return s, kernels()
"""


def test_projections_whose_share_goes_through_memory(run):  # noqa: F811
    run(CALLS + """
for size, kernel in %r:
    s, k = lora(*size)
    assert s == 0 and any(x.startswith("lora_up_kernel") for x in k) and kernel in k, (size, k)
    small = lora(*size[:3], 2, *size[4:])[1]
    assert any(x.startswith("lora_up_kernel") for x in small) == (size[5] == "w4" and ("w4_unpack_kernel" in str(k) or ",8,2,8,1,3,1>" in kernel)), (size, small)
""" % (cases.SHARE,))


def test_projections_whose_tiles_compute_the_share(run):  # noqa: F811
    run(CALLS + """
for size, kernel in %r:
    s, k = lora(*size)
    assert s == 0 and len(k) == 2 and k[1] == kernel, (size, k)
""" % (cases.IN_TILES,))


def test_every_kernel_that_adds_adapters_has_a_size():
    """None of the instances that csrc/inst_*lora.hip and csrc/inst_few_rows_*.hip hold for adapters is left out of the two lists."""
    named = {k for _, k in cases.SHARE + cases.IN_TILES}
    for tile in ("64,32,2,1,3,4", "64,64,2,2,3,2", "128,64,4,1,3,2", "128,128,2,2,3,1", "128,256,2,4,3,1"):
        assert {"rows_tile_kernel<0,1,%s>" % tile, "rows_tile_kernel<0,2,%s>" % tile} <= named
    assert {"moe_pp_kernel<0,0,0,1>", "moe_pp_kernel<0,0,0,2>"} <= named
    for family, least in (("few_rows_kernel<0", 2), ("few_rows_kernel<1", 6), ("shared_rows_kernel<1", 10)):
        assert len({k for k in named if k.startswith(family)}) >= least, family


def test_8_bit_layers_on_the_largest_tiles(run):  # noqa: F811
    run(CALLS + """
for size in %r:
    for alpha in (1.0, 0.0):
        assert q8(*size, alpha=alpha) == (0, ["moe_pp_kernel<0,0,2,0>"]), size
""" % (cases.Q8_LARGE,))


@pytest.mark.parametrize("M", [520, 4096])
def test_the_largest_tiles_give_way_where_weights_pass_31_bits(run, M):  # noqa: F811
    """Sixteen columns fewer and the estimate takes them: it is the limit that keeps them off the larger weights."""
    run(CALLS + """
M, (below, beyond), (f16_below, f16_beyond) = %d, %r, %r
assert below[0] * below[1] < 2 ** 31 <= beyond[0] * beyond[1] and f16_below[0] * f16_below[1] * 2 < 2 ** 31 <= f16_beyond[0] * f16_beyond[1] * 2
assert q8(M, *below) == (0, ["moe_pp_kernel<0,0,2,0>"]) and q8(M, *beyond) == (0, ["rows_tile_kernel<2,0,128,256,2,4,3,1>"])
for n, how in ((2, 2), (600, 1)):
    assert lora(M, *f16_below, n, 8)[1][-1] == "moe_pp_kernel<0,0,0,%%d>" %% how
    assert lora(M, *f16_beyond, n, 8)[1][-1] == "rows_tile_kernel<0,%%d,128,256,2,4,3,1>" %% how
""" % (M, cases.Q8_WEIGHTS, cases.F16_WEIGHTS))


@pytest.mark.parametrize("size", [2 ** 31, 2 ** 32 + 64])
def test_sizes_past_32_bits_are_refused(size):
    """What the C calls' 32 bits would cut short (2^32 + 64 to 64: other rows, or fewer) is refused, row strides of tensors among it."""
    torch = pytest.importorskip("torch")
    import paper_2110_15238_amd as bolt
    for make, names in ((bolt.rms_norm_desc, ("rows", "width", "ldx", "ldr", "lds", "ldy", "ldq")), (bolt.gemm_q8_desc, ("M", "N", "K", "lda", "ldd")),
                        (bolt.gemm_lora_desc, ("M", "N", "K", "lda", "ldd", "adapters", "rank"))):
        good = {n: 64 for n in names if not n.startswith("ld")}
        make(**good)
        for name in names:
            with pytest.raises(AssertionError, match="32 bits"):
                make(**{**good, name: size})
    rows = lambda n, ld, dtype: torch.empty_strided((n, 64), (ld, 1), dtype=dtype, device="meta")
    for x, q, n in ((size, 64, 2), (64, size, 2), (64, 64, size)):
        with pytest.raises(AssertionError, match="32 bits"):
            bolt.bolt_quantize_rows(rows(n, x, torch.float16), rows(n, q, torch.float8_e4m3fn), torch.empty(2, device="meta"))
