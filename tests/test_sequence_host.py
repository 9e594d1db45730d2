"""What the host side of the operators on token sequences answers without a GPU: which kernel takes a size, and sizes that are too large."""
import pytest

from paper_2608_20725_b200 import binding


@pytest.mark.parametrize("dtype", [binding.F32, binding.F16, binding.BF16])
@pytest.mark.parametrize("group", [32, 64, 128, 256])
def test_rows_of_whole_blocks_go_through_the_ring(dtype, group):
    """Whatever the number of groups: odd multiples of 128 too."""
    for k in (128, 256, 384, 896, 1152, 4224, 4736, 8192):
        for m in (1, 7, 16):
            assert binding.im2win_matvec_int4_kernel_name(m, 48, k, group, dtype) == "ring"
    for k in (1, 127, 192, 1000):
        assert binding.im2win_matvec_int4_kernel_name(1, 48, k, group, dtype) == "registers"
    assert binding.im2win_matvec_int4_kernel_name(2, 48, 256, group, dtype, x_stride=257) == "registers"
    assert binding.im2win_matvec_int4_kernel_name(17, 48, 256, group, dtype) == "none"
    assert binding.im2win_matvec_int4_kernel_name(1, 48, 256, 96, dtype) == "none"
    assert binding.im2win_matvec_int4_kernel_name(0, 48, 256, group, dtype) == "none"
