"""CPU-only: the kernels that linear layers take, as the GPU tests that are named for them expect."""
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
