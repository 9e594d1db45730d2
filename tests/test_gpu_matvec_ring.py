"""im2win_matvec_int4 through the ring of bulk copies, by name, where the number of groups is no multiple of four; and scales and zero
points that start anywhere."""
import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, close, matvec_64, rounding
from test_gpu_matvec_int4 import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("k", [128, 384, 896, 1152, 4224, 4736])
@pytest.mark.parametrize("m", [1, 3, 8, 16])
def test_odd_multiples_of_128_with_groups_of_64(dtype, k, m):
    code = binding._sequence_dtype(DTYPES[dtype])
    assert binding.im2win_matvec_int4_kernel_name(m, 50, k, 64, code) == "ring"
    run(dtype, m, 50, k, 64, zeros=m != 3)
    run(dtype, m, 148 * 16 + 37, k, 64, zeros=m == 3)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_scales_and_zero_points_that_start_anywhere(dtype, group, shift):
    n, k, tdt = 50, 896, DTYPES[dtype]
    gen = torch.Generator().manual_seed(shift)
    x = torch.randn(3, k, generator=gen).to(tdt)
    w = torch.randint(0, 256, (n, k // 2), generator=gen, dtype=torch.uint8)
    s = ((torch.rand(n, k // group, generator=gen) + 0.5) * 0.1).to(tdt)
    z = torch.randint(0, 16, (n, k // group), generator=gen, dtype=torch.uint8)
    def moved(t, by):
        return torch.cat([torch.zeros(by, dtype=t.dtype), t.flatten()]).cuda()[by:].view(t.shape)
    want, a = matvec_64(x, w, s, z, None, group)
    tol = (k / 8 + 16 + k // group) * 2.0 ** -23 * a + rounding(want, tdt)
    for by_s, by_z in ((shift, 0), (0, shift), (shift, shift)):
        y = torch.empty(3, n, dtype=tdt, device="cuda")
        binding.im2win_matvec_int4(x.cuda(), w.cuda(), moved(s, by_s), y, group, zeros=moved(z, by_z))
        close(y, want, tol, "y")
