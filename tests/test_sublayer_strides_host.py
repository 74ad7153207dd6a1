"""CPU-only checks of attention's strides: a tensor that is written has each of its elements in a place of its own."""
import itertools

import pytest

import paper_1706_00095_amd as cg
from test_sublayer_host import attn, bwd, fwd


def taken(call, d, which, **more):
    """Refused for its strides, or taken as far as the workspace, which is a byte too small."""
    rc = call(d, n=cg.cg_attn_workspace_bytes(d, which) - 1, **more)
    assert rc in (cg.CG_EINVAL, cg.CG_ENOSPC)
    return rc == cg.CG_ENOSPC


def forward(**strides):
    return taken(fwd, attn(buckets=8, far=9, **strides), cg.CG_PASS_FWD, bias=64)


def backward(**strides):
    return taken(bwd, attn(**strides), cg.CG_PASS_BWD_DATA)


def test_outputs_that_overlap_are_refused():
    assert forward() and backward()
    for bad in (dict(o_tok=0), dict(o_head=0), dict(o_head=63), dict(o_tok=511), dict(o_tok=64, o_head=64)):
        assert not forward(**bad), bad
    for bad in (dict(q_tok=0), dict(q_head=0), dict(k_head=0), dict(k_tok=0), dict(v_tok=127), dict(v_head=32), dict(q_tok=448), dict(k_tok=64, k_head=64 * 99)):
        assert not backward(**bad), bad


def test_inputs_may_be_broadcast():
    assert forward(k_head=0, v_head=0, q_tok=0, q_head=0, k_tok=0)
    assert backward(o_tok=0, o_head=0)


def test_other_orders_and_gaps_are_taken():
    assert forward(o_tok=64, o_head=6400) and forward(o_tok=3 * 512) and forward(o_tok=600, o_head=75)
    assert backward(k_tok=64, k_head=6400) and backward(q_tok=1536, k_tok=1536, v_tok=1536)
    big = 1 << 62
    assert backward(q_tok=big, k_head=big) and forward(o_tok=512, o_head=big) and forward(o_tok=big, o_head=big - 64)     # 64 elements apart
    assert not forward(o_tok=big, o_head=big - 63)
    assert forward(Tq=1, o_tok=0) and backward(Tk=1, k_tok=0, v_tok=0) and forward(Hq=1, Hkv=1, o_head=0, o_tok=64)


@pytest.mark.parametrize("T,H,D", [(2, 4, 3), (5, 3, 2), (4, 4, 1)])
def test_every_pair_of_small_strides(T, H, D):
    for tok, head in itertools.product(range(0, 14), repeat=2):
        places = [t * tok + h * head + e for t in range(T) for h in range(H) for e in range(D)]
        apart = len(set(places)) == len(places)
        assert forward(Tq=T, Hq=H, Hkv=1, D=D, o_tok=tok, o_head=head) == apart, (tok, head)
        assert backward(Tq=9, Tk=T, Hq=H, Hkv=H, D=D, v_tok=tok, v_head=head) == apart, (tok, head)
