"""im2win_rms_norm against the definition in 64 bits.

Tolerances, relative: the sum of squares adds up positive numbers, up to 32 in a thread and ten levels of threads, each rounding by at most
2^-24 of it, of which the root takes half; its reciprocal (2 units), the division by the channels, the sum with eps and two products: 32 * 2^-24
in all, and the one rounding of y.  Whole numbers have to be equal."""
import math

import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, Guarded, close, rounding

pytestmark = pytest.mark.gpu

OFF = 32 * 2.0 ** -24


def norm_64(x, residual, weight, eps):
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    z = h.double() * (1.0 if weight is None else weight.double())
    return h, z, 1 / (h.double().square().mean(1) + eps).sqrt()


def int8_64(z, rate):
    top = z.abs().amax(1)
    fine = torch.isfinite(top) & (top <= torch.finfo(torch.float32).max)
    q = (z * 127 / torch.where(fine & (top > 0), top, 1.0)[:, None]).round()
    return torch.where(fine[:, None], q, 0.0), torch.where(fine, top * rate / 127, math.nan)


def run(dtype, rows, channels, residual=False, int8=False, weight=True, pitch=0, shift=0, eps=1e-6, edit=None, alias=None, seed=1):
    gen = torch.Generator().manual_seed(seed)
    tdt = DTYPES[dtype]
    x = torch.randn(rows, channels, generator=gen).to(tdt)
    r = (torch.randn(rows, channels, generator=gen) * 2).to(tdt) if residual else None
    w = (1 + 0.3 * torch.randn(channels, generator=gen)).to(tdt) if weight else None
    if edit:
        edit(x, r, w)
    xg = Guarded((rows, channels), tdt, pitch, shift=shift)
    xg.view.copy_(x)
    rg = hg = None
    if residual:
        rg = Guarded((rows, channels), tdt, 2 * pitch, shift=shift)
        rg.view.copy_(r)
        hg = {"x": xg, "residual": rg}.get(alias) or Guarded((rows, channels), tdt, 3 * pitch, shift=shift)
    yg = xg if alias == "y" else Guarded((rows, channels), torch.int8 if int8 else tdt, 3 * pitch, shift=shift)
    sg = Guarded((rows,), torch.float32) if int8 else None
    binding.im2win_rms_norm(xg.view, None if w is None else w.cuda(), yg.view, scales=sg.view if int8 else None,
                            residual=rg.view if residual else None, residual_out=hg.view if residual else None, eps=eps)
    torch.cuda.synchronize()
    h, z, rate = norm_64(x, r, w, eps)
    if residual:
        assert torch.equal(hg.view.cpu(), h)
        hg.assert_untouched_outside()
    if int8:
        q, scales = int8_64(z, rate)
        assert torch.equal(yg.view.cpu().double(), q)
        close(sg.view, scales, OFF * scales.abs() + 2.0 ** -149, "scales")
        sg.assert_untouched_outside()
    else:
        want = z * rate[:, None]
        close(yg.view, want, OFF * want.abs() + rounding(want, tdt), "y", same_infinities=False)
    yg.assert_untouched_outside()


CHANNELS = [1, 2, 7, 32, 64, 100, 128, 256, 512, 1000, 1001, 1024, 2048, 4096, 4099, 8192, 16384]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("channels", CHANNELS)
def test_channels(dtype, int8, channels):
    run(dtype, 5, channels, residual=channels % 2 == 0, int8=int8)
    run(dtype, 3, channels, residual=channels % 2 == 1, int8=int8, pitch=3, weight=channels % 3 == 0)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("channels", [17000, 32768, 40000, 70001])
def test_long_rows(dtype, int8, channels):
    run(dtype, 2, channels, residual=True, int8=int8)
    run(dtype, 2, channels, int8=int8)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("rows", [1, 4, 593, 2001])
def test_rows(dtype, int8, rows):
    run(dtype, rows, 1024, residual=True, int8=int8)
    run(dtype, rows, 2304, int8=int8)
    run(dtype, rows, 72, int8=int8)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("int8", [False, True])
def test_rows_that_start_anywhere(dtype, int8):
    for shift in (1, 2, 4, 8):
        run(dtype, 4, 512, residual=True, int8=int8, shift=shift)
    for pitch in (1, 4, 8, 64):
        run(dtype, 4, 512, residual=True, int8=int8, pitch=pitch)


@pytest.mark.parametrize("alias", ["x", "residual"])
@pytest.mark.parametrize("channels", [96, 4096, 40000])
def test_in_place(alias, channels):
    run("bf16", 3, channels, residual=True, alias=alias)
    run("f32", 3, channels, residual=True, alias=alias, int8=True)
    run("f16", 3, channels, alias="y")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("int8", [False, True])
def test_rows_of_zeros_and_of_values_that_are_not_finite(dtype, int8):
    def edit(x, r, w):
        x[0] = 0.0
        x[1, 7] = math.inf
        x[2, 300] = math.nan
        x[3] = 0.0
        x[3, 5] = -3.0
        x[4] *= 1e-3
    run(dtype, 6, 512, int8=int8, edit=edit)
    run(dtype, 6, 509, int8=int8, edit=edit, eps=0.125)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_numbers_halfway_between_two(dtype):
    """x = 254 top / 127 and smaller: quotients of every whole number and half, and next to them; ties go to the even number."""
    def halves(x, r, w):
        x[:] = torch.arange(512) - 255.0
        x[:, 0], x[:, 511] = 254.0, -254.0
        x.clamp_(-254, 254)
        x[1] *= 2.0 ** -12
        x[2] *= 64
    run(dtype, 4, 512, int8=True, weight=False, edit=halves)

    def near(x, r, w):
        halves(x, r, w)
        x[:] = torch.nextafter(x.float(), torch.tensor(1e9)).to(x.dtype) if dtype == "f32" else x
        w[:] = 3.0
    run(dtype, 4, 512, int8=True, edit=near)


def test_products_that_fp32_does_not_hold():
    """Rows so small that products lose bits, or vanish, in fp32, and so large that they pass its range."""
    def edit(x, r, w):
        x[0] *= 1e-30
        x[1] *= 1e-38
        w *= 1e-6
        x[2] *= 2.0 ** -66
    run("bf16", 4, 640, int8=True, edit=edit)
    run("f32", 4, 640, int8=True, edit=edit)

    def large(x, r, w):
        w *= 1e30
        x[1] *= 1e12
    run("bf16", 3, 640, int8=True, edit=large)
    run("f32", 3, 641, int8=True, edit=large)


def test_no_rows():
    x = torch.zeros(0, 64, device="cuda")
    binding.im2win_rms_norm(x, None, torch.zeros_like(x))


def test_captured_and_on_another_stream():
    x, w = torch.randn(70, 1024, device="cuda").bfloat16(), torch.ones(1024, device="cuda").bfloat16()
    y, other = torch.zeros_like(x), torch.zeros_like(x)
    binding.im2win_rms_norm(x, w, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.im2win_rms_norm(x, w, y)
    x.copy_(torch.randn(70, 1024))
    graph.replay()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    binding.im2win_rms_norm(x, w, other, stream=side)
    side.synchronize()
    assert torch.equal(y, other) and bool(y.any())


def test_rows_beyond_32_bits():
    """Elements whose number passes 2^31."""
    rows, channels = 33000, 65600
    x = torch.zeros(rows, channels, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn(3, channels, device="cuda").bfloat16()
    y, scales = torch.zeros(rows, channels, dtype=torch.int8, device="cuda"), torch.zeros(rows, device="cuda")
    binding.im2win_rms_norm(x, None, y, scales=scales)
    h, z, rate = norm_64(x[-3:].cpu(), None, None, 1e-6)
    q, want = int8_64(z, rate)
    assert torch.equal(y[-3:].cpu().double(), q)
    close(scales[-3:], want, OFF * want, "scales")
    assert not y[:-3].any() and not scales[:-3].any()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_zeros_without_eps_and_squares_beyond_the_range(dtype):
    """A row of zeros and eps of 0 has a scale of 0; rows whose squares pass fp32 come out as 0."""
    x = torch.zeros(2, 100, dtype=DTYPES[dtype], device="cuda")
    if dtype != "f16":
        x[1] = 1e25
    y, scales = torch.full((2, 100), 5, dtype=torch.int8, device="cuda"), torch.full((2,), 5.0, device="cuda")
    binding.im2win_rms_norm(x, None, y, scales=scales, eps=0.0)
    assert not y[0].any() and not scales.any()
    if dtype != "f16":
        out = torch.ones_like(x)
        binding.im2win_rms_norm(x, None, out)
        assert not out.any()
