"""Attention at the limits of what a launch or a number holds, against its plain form in 64 bits."""
import pytest

from test_gpu_attention import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("far", [849, 850, 1024, 1025])
@pytest.mark.parametrize("D,shift", [(128, 0), (97, 1)])
def test_bias_of_far_distances_where_tiles_fill_the_lds(far, D, shift):
    """The widest fp32 kernel keeps distances up to 849 one by one, beside its tiles; the others do up to 1024."""
    run("fp32", [900, 130], [1400, 130], 2, 1, D, False, shift=shift, bias=32, far=far, both=True)


@pytest.mark.parametrize("dtype,D", [("fp32", 96), ("bf16", 128), ("fp32", 32)])
def test_bias_of_far_distances_of_other_widths(dtype, D):
    for far in (1024, 1025):
        run(dtype, [900], [1400], 2, 2, D, True, bias=32, far=far)
