"""im2win_rms_norm where fp32 does not hold a row's squares: too small, and too large."""
import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, Guarded, close, rounding
from test_gpu_rms_norm import OFF, norm_64

pytestmark = pytest.mark.gpu

TINY = {"f32": [1e-18, 1e-25, 1e-38, 3e-42], "bf16": [1e-18, 1e-25, 1e-37], "f16": [1e-4, 3e-7]}


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("channels", [64, 509, 1000, 4096, 40000])
@pytest.mark.parametrize("residual", [False, True])
def test_small_rows_without_eps(dtype, int8, channels, residual):
    """Rows of zeros come out as zeros, others as their direction, however small they are; a row of ordinary size lies between them."""
    gen, tdt = torch.Generator().manual_seed(channels), DTYPES[dtype]
    sizes = TINY[dtype] + [0.0, 1.0]
    x = (torch.randn(len(sizes), channels, generator=gen) * torch.tensor(sizes)[:, None]).to(tdt)
    r = (torch.randn(len(sizes), channels, generator=gen) * torch.tensor(sizes)[:, None]).to(tdt) if residual else None
    w = (1 + 0.3 * torch.randn(channels, generator=gen)).to(tdt)
    y = Guarded(x.shape, torch.int8 if int8 else tdt)
    scales = torch.full((len(sizes),), 5.0, device="cuda") if int8 else None
    total = None if r is None else torch.zeros_like(x).cuda()
    binding.im2win_rms_norm(x.cuda(), w.cuda(), y.view, scales=scales, residual=None if r is None else r.cuda(), residual_out=total, eps=0.0)
    h, z, rate = norm_64(x, r, w, 0.0)
    zeros = h.double().abs().amax(1) == 0
    assert bool(zeros[-2]) and not bool(zeros[[0, -1]].any())
    rate = torch.where(zeros, 0.0, rate)
    if int8:
        top = z.abs().amax(1)
        assert torch.equal(y.view.cpu().double(), torch.where(zeros[:, None], 0.0, z * 127 / top[:, None]).round())
        want = top * rate / 127
        close(scales, want, OFF * want + 2.0 ** -149, "scales")
    else:
        want = z * rate[:, None]
        close(y.view, want, OFF * want.abs() + rounding(want, tdt), "y")
    y.assert_untouched_outside()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_an_eps_as_small_as_the_squares(dtype):
    gen = torch.Generator().manual_seed(8)
    x = (torch.randn(3, 512, generator=gen) * torch.tensor([[1e-22], [1e-20], [1e-24]])).to(DTYPES[dtype])
    for eps in (1e-44, 1e-40, 1e-36):
        y = torch.zeros(3, 512, device="cuda", dtype=DTYPES[dtype])
        binding.im2win_rms_norm(x.cuda(), None, y, eps=eps)
        kept = torch.tensor(eps, dtype=torch.float32).double()           # (eps as the call takes it)
        want = x.double() / (x.double().square().mean(1, keepdim=True) + kept).sqrt()
        close(y, want, OFF * want.abs() + rounding(want, DTYPES[dtype]), "y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_squares_beyond_the_range_in_8_bits(dtype):
    """The numbers are as they would be, their scale is 0; into x's type y is 0."""
    x = torch.full((2, 100), 1e25).to(DTYPES[dtype])
    x[1, ::2] *= -0.5
    y, scales = torch.zeros(2, 100, dtype=torch.int8, device="cuda"), torch.ones(2, device="cuda")
    binding.im2win_rms_norm(x.cuda(), None, y, scales=scales)
    assert torch.equal(y.cpu().double(), (x.double() * 127 / x.double().amax(1, keepdim=True)).round()) and not scales.any()
