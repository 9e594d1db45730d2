"""im2win_gated_delta_rule on the ways a call can take: which one it is, and each against the recurrence in 64 bits."""
import pytest

from delta_helpers import run
from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES

pytestmark = pytest.mark.gpu

SHORT = [3, 0, 16, 7, 1]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("heads,dk,dv", [(80, 64, 128), (64, 128, 128), (80, 40, 100), (40, 64, 96), (30, 128, 128), (50, 200, 128), (39, 256, 98),
                                         (3, 64, 64), (3, 128, 33), (2, 200, 40)])
def test_short_prompts_of_every_width(dtype, heads, dk, dv):
    """Prompts of up to 16 tokens run token by token: four columns a lane (dv above 64, some 296 blocks of 128), two (296 of 64), and one."""
    run(dtype, SHORT, heads, heads // 2 if heads % 2 == 0 else heads, dk, dv, max_len=16, resume=[1, 0, 0, 1, 1], tail=2, kernel="tokens")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("heads,dk,dv", [(80, 64, 128), (160, 33, 100), (100, 64, 48), (80, 256, 128), (60, 100, 96)])
def test_single_tokens_of_every_width(dtype, heads, dk, dv):
    run(dtype, [1] * 4, heads, heads, dk, dv, mode="step")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("dk", [64, 128])
def test_a_max_len_that_is_too_small_keeps_the_results(dtype, dk):
    run(dtype, [5, 100, 0, 30], 2, 1, dk, 64, max_len=1, resume=[1, 0, 1, 1], kernel="tokens")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("max_len,kernel", [(0, "chunks"), (17, "chunks"), (16, "tokens")])
def test_which_way_is_taken(dtype, max_len, kernel):
    run(dtype, [17, 5] if max_len != 16 else [16, 5], 2, 2, 64, 64, max_len=max_len, kernel=kernel)
    shape = binding.make_delta_shape(100, 2, 2, 2, 129, 64, max_len)
    assert binding.im2win_gated_delta_rule_kernel_name(shape, binding._sequence_dtype(DTYPES[dtype])) == "tokens"


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_prompts_above_128_elements_of_a_key(dtype):
    run(dtype, [40, 3], 2, 1, 160, 64, kernel="tokens")
