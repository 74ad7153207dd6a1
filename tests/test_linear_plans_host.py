"""CPU-only: the kernels that linear layers take, as the GPU tests that are named for them expect."""
import math
import random

import pytest

import linear_plan_util as lp
import paper_1706_00095_amd as cg

PASSES = (cg.CG_PASS_FWD, cg.CG_PASS_BWD_DATA, cg.CG_PASS_BWD_WEIGHT)


def desc(dtype, M, K, N):
    return cg.cg_linear_desc(cg.CG_TYPE_FP32 if dtype == "fp32" else cg.CG_TYPE_BF16, M, N, K, 0, 0)


@pytest.mark.parametrize("M,K,N", lp.LARGE)
def test_large_tiles_in_every_pass(M, K, N):
    d = desc("bf16", M, K, N)
    for which in PASSES:
        assert cg.cg_debug_linear_plan(d, which) == (256, 1, False), which
    # x in 8 bits is unpacked into the workspace, which the bias's sums have before
    assert cg.cg_debug_linear_plan(d, cg.CG_PASS_BWD_WEIGHT, packed=True) == (256, 1, False)
    assert cg.cg_linear_workspace_bytes(d, cg.CG_PASS_BWD_WEIGHT) == 2 * M * K
    # long enough for the loop between a product's first and last steps, and for a bias of several slices
    assert min(M, K, N) >= 64 * 8


def test_what_is_refused():
    L, d = cg.lib(), desc("bf16", 100, 24, 40)
    out = [cg.C.c_int() for _ in range(3)]
    refs = [cg.C.byref(i) for i in out]
    assert L.cg_debug_linear_plan(d, 0, 1, 0, *refs) == cg.CG_OK and out[0].value == 64
    assert L.cg_debug_linear_plan(None, 0, 1, 0, *refs) == cg.CG_EINVAL and L.cg_debug_linear_plan(d, 3, 1, 0, *refs) == cg.CG_EINVAL
    for i in range(3):
        assert L.cg_debug_linear_plan(d, 0, 1, 0, *[None if i == j else r for j, r in enumerate(refs)]) == cg.CG_EINVAL


@pytest.mark.parametrize("dtype,which,whole,packed,tile,cut,M,K,N", lp.CASES)
def test_every_product(dtype, which, whole, packed, tile, cut, M, K, N):
    got, parts, _ = cg.cg_debug_linear_plan(desc(dtype, M, K, N), which, whole, packed)
    assert (got, parts > 1) == (tile, cut)


def test_no_kernel_without_a_case():
    """Sizes by chance take no kernel that no case takes (up to 32 tokens forward and tiles of 256 apart, which have tests of their own)."""
    def kind(dtype, which, whole, packed, M, K, N):
        tile, parts, halves = cg.cg_debug_linear_plan(desc(dtype, M, K, N), which, whole, packed)
        return dtype, which, whole, packed, tile, parts > 1, halves

    have = {kind(*c[:4], *c[6:]) for c in lp.CASES}
    rng = random.Random(1)
    for _ in range(20000):
        M, K, N, whole, dtype = *(int(round(math.exp(rng.uniform(0, math.log(16384))))) for _ in range(3)), rng.random() < 0.5, rng.choice(["fp32", "bf16"])
        if whole:
            K, N, dtype = (K + 7) // 8 * 8, (N + 7) // 8 * 8, "bf16"
        for which in PASSES:
            for packed in (False, True) if which == cg.CG_PASS_BWD_WEIGHT else (False,):
                k = kind(dtype, which, whole, packed, M, K, N)
                assert k[4] in (16, 256) or k in have, (k, M, K, N)


def test_rows_too_far_apart_are_not_unpacked():
    """x in 8 bits becomes a dense tensor whose rows lie K apart: as far as tiles of 256 take them and no further."""
    M, N = 1024, 256
    for K, unpacked in ((1 << 21, True), ((1 << 21) + 8, False), (1 << 24, False)):
        d = desc("bf16", M, K, N)
        assert cg.cg_debug_linear_plan(d, cg.CG_PASS_BWD_WEIGHT) == (256, 1, False)
        assert (cg.cg_debug_linear_plan(d, cg.CG_PASS_BWD_WEIGHT, packed=True)[0] == 256) == unpacked, K
        n = cg.cg_linear_workspace_bytes(d, cg.CG_PASS_BWD_WEIGHT)
        assert n == 2 * M * K if unpacked else n < 1 << 20, K
