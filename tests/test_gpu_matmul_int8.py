"""im2win_matmul_int8 against sums of whole numbers: the sum is exact, its conversion, two products and the bias's sum round by 2^-24 each, y once."""
import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, Guarded, close, rounding

pytestmark = pytest.mark.gpu


def run(dtype, m, n, k, bias=False, pitch=0, y_pitch=0, shift=0, extremes=False, seed=1, kernel=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tdt = DTYPES[dtype]
    x, w = (torch.randint(-128, 128, (rows, k), generator=gen, device="cuda", dtype=torch.int8) for rows in (m, n))
    if extremes:
        x.fill_(-128)
        w.fill_(-128)
        w[::2] = 127
    xs, ws = torch.rand(m, generator=gen, device="cuda") * 0.1, (torch.rand(n, generator=gen, device="cuda") + 0.5) * 0.01
    b = torch.randn(n, generator=gen, device="cuda") if bias else None
    xg, yg = Guarded((m, k), torch.int8, pitch, fill=99, shift=shift), Guarded((m, n), tdt, y_pitch)
    xg.view.copy_(x)
    if kernel:
        assert binding.im2win_matmul_int8_kernel_name(m, n, k, binding._sequence_dtype(tdt), k + pitch) == kernel
    binding.im2win_matmul_int8(xg.view, xs, w, ws, yg.view, bias=b)
    torch.cuda.synchronize()
    acc = x.double() @ w.double().T                  # (whole numbers below 2^53: exact)
    want = acc * xs.double()[:, None] * ws.double()
    off = 3 * 2.0 ** -24 * want.abs()
    if bias:
        want = want + b.double()
        off = off + 2.0 ** -24 * (want.abs() + off)
    want, off = want.cpu(), off.cpu()
    close(yg.view, want, off + rounding(want, tdt), "y")
    yg.assert_untouched_outside()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 64, 64), (1, 4096, 4096), (3, 100, 33), (8, 128, 128), (16, 1001, 2080), (17, 512, 1024),
                                   (64, 256, 4096), (65, 129, 144), (128, 128, 16), (200, 300, 257), (701, 1001, 2080), (300, 72, 15)])
def test_sizes(dtype, m, n, k):
    run(dtype, m, n, k, bias=m % 2 == 1)


@pytest.mark.parametrize("m", [1, 2, 5, 15, 16, 31, 33, 64, 100, 128, 129, 255, 256, 257, 511, 1000])
def test_rows(m):
    run("bf16", m, 384, 512)
    run("f32", m, 200, 208, bias=True)


@pytest.mark.parametrize("n", [8, 16, 63, 127, 128, 129, 255, 256, 257, 640, 1500])
def test_columns(n):
    for m in (4, 200):
        run("f16", m, n, 384)


@pytest.mark.parametrize("k", [16, 32, 48, 112, 128, 144, 240, 1040, 16384])
def test_reductions(k):
    for m in (4, 40, 200):
        run("f32", m, 264, k)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_strides_and_rows_that_start_anywhere(dtype):
    for m in (5, 300):
        run(dtype, m, 200, 256, pitch=16, y_pitch=8)
        run(dtype, m, 200, 256, pitch=3, y_pitch=1)
        run(dtype, m, 200, 256, shift=1)
        run(dtype, m, 201, 253, shift=2, pitch=5)
        run(dtype, m, 200, 256, shift=4, y_pitch=56)


@pytest.mark.parametrize("k", [4096, 131071, 131056])
def test_the_largest_sums(k):
    """2^31 - 2^14 and the like: as far as 32 bits go."""
    for m in (2, 130):
        run("f32", m, 130, k, extremes=True)


@pytest.mark.parametrize("m", [1, 2, 4, 5, 8, 15, 16, 17])
def test_few_rows_that_start_anywhere(m):
    for n, k in ((1, 1), (30, 17), (17, 31), (40, 2047), (33, 2049), (100, 4095), (1001, 8191)):
        run("f32", m, n, k, bias=n % 2 == 1)
    run("bf16", m, 64, 512, shift=3, pitch=1)


def test_many_tiles():
    run("bf16", 3000, 2100, 512, kernel=None)
    run("bf16", 40, 30000, 256)


def test_no_rows():
    y = torch.zeros(0, 8, device="cuda")
    binding.im2win_matmul_int8(torch.zeros(0, 16, dtype=torch.int8, device="cuda"), torch.zeros(0, device="cuda"),
                               torch.zeros(8, 16, dtype=torch.int8, device="cuda"), torch.zeros(8, device="cuda"), y)


@pytest.mark.parametrize("m", [4, 300])
def test_captured_and_on_another_stream(m):
    make = lambda rows: torch.randint(-127, 128, (rows, 512), device="cuda", dtype=torch.int8)
    x, w, xs, ws = make(m), make(640), torch.rand(m, device="cuda"), torch.rand(640, device="cuda")
    y, other = torch.zeros(m, 640, device="cuda"), torch.zeros(m, 640, device="cuda")
    binding.im2win_matmul_int8(x, xs, w, ws, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.im2win_matmul_int8(x, xs, w, ws, y)
    x.copy_(make(m))
    graph.replay()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    binding.im2win_matmul_int8(x, xs, w, ws, other, stream=side)
    side.synchronize()
    assert torch.equal(y, other) and bool(y.any())


@pytest.mark.parametrize("k", [16, 15])
def test_outputs_beyond_32_bits(k):
    """Elements of y whose number passes 2^31."""
    m, n = 70001, 32768
    x, w = (torch.randint(-127, 128, (rows, k), device="cuda", dtype=torch.int8) for rows in (m, n))
    xs, ws = torch.rand(m, device="cuda"), torch.rand(n, device="cuda")
    y = torch.zeros(m, n, dtype=torch.float16, device="cuda")
    binding.im2win_matmul_int8(x, xs, w, ws, y)
    for part in (slice(0, 3), slice(m - 3, m)):
        want = (x[part].double() @ w.double().T * xs[part].double()[:, None] * ws.double()).cpu()
        # (65520 and more lies nearer to 2^16, which fp16 does not have, than to its largest number, 65504: an infinity)
        want = torch.where(want.abs() >= 65520, want.sign() * torch.inf, want)
        close(y[part], want, 3 * 2.0 ** -24 * want.abs() + rounding(want, torch.float16), "y")


@pytest.mark.parametrize("m,n", [(300, 30000), (40, 40000)])
@pytest.mark.parametrize("drop", ["0", "1"])
def test_gives_up_and_says_so(m, n, drop, monkeypatch):
    """The first CTA (pair) does not say that a tile's sums are done: a testing aid, which also lowers the limit of looks; the kernel returns.  What comes of
    other CTAs is right, of this one's that tile and those behind it are NaN (of a pair all of them where its last waits ran out)."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, w = (torch.randint(-127, 128, (rows, 256), generator=gen, device="cuda", dtype=torch.int8) for rows in (m, n))
    xs, ws = torch.rand(m, generator=gen, device="cuda"), torch.rand(n, generator=gen, device="cuda")
    y = torch.zeros(m, n, device="cuda")
    monkeypatch.setenv("IM2WIN_MATMUL_DROP", drop)
    binding.im2win_matmul_int8(x, xs, w, ws, y)
    torch.cuda.synchronize()
    monkeypatch.delenv("IM2WIN_MATMUL_DROP")
    want = (x.double() @ w.double().T) * xs.double()[:, None] * ws.double()
    bad = ~((y.double() - want).abs() <= 4 * 2.0 ** -24 * want.abs() + 2.0 ** -140)
    assert bool(bad.any()) and bool(y[bad].isnan().all()) and float(bad.float().mean()) < 0.05
    again = torch.zeros_like(y)
    binding.im2win_matmul_int8(x, xs, w, ws, again)
    assert not bool(((again.double() - want).abs() > 4 * 2.0 ** -24 * want.abs()).any())


def test_more_rows_than_a_grid_has():
    """Rows that start anywhere, more than 65535 tiles of 64."""
    m = 65535 * 64 + 100
    x, w = torch.randint(-127, 128, (m, 3), device="cuda", dtype=torch.int8), torch.randint(-127, 128, (9, 3), device="cuda", dtype=torch.int8)
    xs, ws, y = torch.rand(m, device="cuda"), torch.rand(9, device="cuda"), torch.zeros(m, 9, device="cuda")
    binding.im2win_matmul_int8(x, xs, w, ws, y)
    want = x.double() @ w.double().T * xs.double()[:, None] * ws.double()
    assert not bool(((y.double() - want).abs() > 3 * 2.0 ** -24 * want.abs()).any())
