"""CPU-only checks of the limits of attention's launches: what would need more blocks than a launch has room for is refused before
anything is launched, and nothing short of it is."""
import paper_1706_00095_amd as cg
from test_sublayer_host import attn, bwd, fwd

MOST = (1 << 24) - 1        # blocks


def accepted(d, which=cg.CG_PASS_BWD_DATA):
    return cg.cg_attn_workspace_bytes(d, which) > 0


def test_more_blocks_than_a_launch_has_room_for_are_refused():
    one = dict(Hq=1, Hkv=1, D=8)
    for d in (attn(B=MOST + 1, Tq=5, Tk=5, **one), attn(B=MOST, Tq=128, Tk=5, **one), attn(B=1 << 18, Hq=64, Hkv=64, D=8, Tq=5, Tk=5),
              attn(B=2, Hq=1, Hkv=1, D=1, Tq=(1 << 31) - (1 << 16), Tk=5, buckets=8, far=9, type=0), attn(B=1 << 19, Tq=5, Tk=5, Hq=32, Hkv=32, D=8)):
        blocks = d.Hq // (1 if d.buckets else d.Hq // d.Hkv) * (d.Tq * (1 if d.buckets else d.Hq // d.Hkv) // 128 + d.B)
        if blocks > MOST:
            assert fwd(d, bias=64) == cg.CG_EUNSUPPORTED and bwd(d, bias=64) == cg.CG_EUNSUPPORTED, blocks
            assert not accepted(d) and not accepted(d, cg.CG_PASS_FWD)
        else:
            assert accepted(d), blocks
    assert bwd(attn(B=MOST - 1, Tq=5, Tk=256, **one)) == cg.CG_EUNSUPPORTED                     # the kernel over the keys
    assert bwd(attn(B=MOST - 5, Tq=5, Tk=5, buckets=96, far=100, **one), bias=64) == cg.CG_EUNSUPPORTED      # with six blocks for dbias


def test_calls_within_the_limits_are_taken():
    assert accepted(attn(B=MOST, Tq=5, Tk=5, Hq=1, Hkv=1, D=8))
    assert accepted(attn(B=MOST - 6, Tq=5, Tk=5, Hq=1, Hkv=1, D=8, buckets=96, far=100))
    assert accepted(attn(B=2, Hq=128, Hkv=128, D=1, Tq=1 << 23, Tk=5))                           # Tq * Hq = 2^30
    assert accepted(attn(B=2, Hq=512, Hkv=4, D=1, Tq=1 << 21, Tk=1 << 20))
    assert accepted(attn(B=1 << 20, Hq=64, Hkv=8, D=64, Tq=1 << 20, Tk=1 << 24))                 # many sequences, grouped heads
    assert accepted(attn(B=1, Hq=1, Hkv=1, D=1, Tq=1, Tk=MOST, buckets=8, far=9), cg.CG_PASS_FWD)
