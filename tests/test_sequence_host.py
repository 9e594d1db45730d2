"""What the host side of the operators on token sequences answers without a GPU: which kernel takes a size, and sizes that are too large."""
import ctypes

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


MOST = 2 ** 31 - 4096
A = 1 << 20                # an address, aligned; nothing is read from it


@pytest.mark.parametrize("tokens,sequences", [(2 ** 31 - 1, 1), (MOST + 1, 1), (2 ** 31 - 1, 2 ** 31 - 1), (0, 2 ** 31 - 1), (MOST + 1, MOST + 1)])
@pytest.mark.parametrize("packed", [False, True])
def test_row_numbers_that_32_bits_would_not_count_past(tokens, sequences, packed):
    """The kernels' row numbers run up to some chunks beyond the last row."""
    seqs = binding.Sequences(A if packed else None, None, None)
    conv = binding.Conv1dShape(tokens, sequences, 0, 64, 4, 0, 64, 64)
    assert binding.lib().im2win_causal_conv1d(A, A, None, A, None, None, ctypes.byref(seqs), ctypes.byref(conv), binding.BF16, None) == 5
    shape = binding.AttentionShape(tokens, sequences, 0, 0, 1, 1, 64, 64, 1.0, 64, 64, 64, 64, 1)
    assert binding.lib().im2win_linear_attention(A, A, A, A, A, None, None, ctypes.byref(seqs), A, 1 << 60, ctypes.byref(shape), binding.BF16, None) == 5
    with pytest.raises(binding.Im2winError) as e:
        binding.im2win_linear_attention_workspace_size(shape, binding.BF16)
    assert e.value.code == 5
