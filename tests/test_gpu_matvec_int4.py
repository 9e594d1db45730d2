"""im2win_matvec_int4 against its definition in 64 bits.

Tolerance: products are exact; fp32 sums of K terms, in eight parts and by groups, none of whose partial sums exceeds the sum of magnitudes,
are off by less than (K / 8 + 16 + groups) units of 2^-23 of it even where the tensor cores cut off every addend (K / 16 additions of a
group's sixteen-term products, one for each, and the group's product with its scale); y is rounded once."""
import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, Guarded, close, matvec_64, rounding

pytestmark = pytest.mark.gpu


def run(dtype, m, n, k, group, zeros=True, bias=True, pitch=0, shift=0, seed=1, edit=None):
    gen = torch.Generator().manual_seed(seed)
    tdt, groups = DTYPES[dtype], -(-k // group)
    x = torch.randn(m, k, generator=gen).to(tdt)
    w = torch.randint(0, 256, (n, (k + 1) // 2), generator=gen, dtype=torch.uint8)
    s = ((torch.rand(n, groups, generator=gen) + 0.5) * 0.1).to(tdt)
    z = torch.randint(0, 16, (n, groups), generator=gen, dtype=torch.uint8) if zeros else None
    b = torch.randn(n, generator=gen) if bias else None
    if edit:
        edit(x, w, s, z)
    xg, yg = Guarded((m, k), tdt, pitch, shift=shift, fill=float("nan") if pitch else -77.0), Guarded((m, n), tdt, pitch, shift=shift)
    xg.view.copy_(x)
    binding.im2win_matvec_int4(xg.view, w.cuda(), s.cuda(), yg.view, group, zeros=None if z is None else z.cuda(),
                               bias=None if b is None else b.cuda())
    torch.cuda.synchronize()
    y, a = matvec_64(x, w, s, z, b, group)
    close(yg.view, y, (k / 8 + 16 + groups) * 2.0 ** -23 * a + rounding(y, tdt), "y")
    yg.assert_untouched_outside()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("m", [1, 3, 8, 16])
def test_types_groups_and_rows(dtype, group, zeros, m):
    run(dtype, m, 48, 1280, group, zeros=zeros, bias=m % 2 == 1)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("m", range(1, 17))
def test_every_number_of_rows(dtype, m):
    run(dtype, m, 33, 256, 64, pitch=8)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("n,k,group", [(1, 1, 32), (5, 2, 64), (17, 31, 32), (15, 33, 32), (16, 129, 64), (100, 1000, 128), (31, 96, 32), (64, 1500, 384),
                                       (40, 100, 256), (9473, 160, 32), (9500, 224, 64), (9473, 300, 128)])
def test_ragged_sizes(dtype, n, k, group):
    run(dtype, 2, n, k, group)
    run(dtype, 5, n, k, group, pitch=1, shift=1, zeros=False)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_largest_tiles(dtype):
    run(dtype, 16, 9472 + 24, 512, 64)
    run(dtype, 1, 18944 + 1, 512, 128)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("m,k", [(16, 4224), (16, 12000), (9, 9000), (1, 16384 + 64), (5, 16384)])
def test_rows_longer_than_what_lies_in_shared_memory(dtype, m, k):
    run(dtype, m, 50, k, 64, zeros=m % 2 == 1)
    run(dtype, m, 148 * 32 * 9 + 5 if m == 16 and k < 5000 else 40, k, 128, zeros=False)


@pytest.mark.parametrize("dtype,group", [("f16", 64), ("bf16", 32), ("bf16", 128), ("f32", 64)])
def test_parts_of_the_rows_that_differ_over_several_passes(dtype, group):
    # blocks of an SM with an odd and an even number of 16 rows, the last one cut off; passes of up to 4096 elements, the last one shorter
    run(dtype, 2, 148 * 16 * 3 + 5 * 16 + 3, 4096 + 5 * 128, group, zeros=group != 32)
    run(dtype, 1, 148 * 16 * 17 + 16 + 5, 4096 + 2 * 128, group, zeros=group == 32)


def test_infinities_and_nans_stay_in_their_row_of_x():
    def edit(x, w, s, z):
        x[0, 5] = float("inf")
        x[1, 200] = float("nan")
    for dtype in DTYPES:
        run(dtype, 3, 40, 256, 64, edit=edit)


def test_fp32_values_of_every_size():
    def edit(x, w, s, z):
        x[0] *= 1e30
        x[1] *= 1e-30
        x[2, ::2] *= 1e8
    run("f32", 4, 40, 512, 128, edit=edit)


def test_captured_and_replayed():
    x = torch.randn(2, 512, device="cuda").half()
    w = torch.randint(0, 256, (64, 256), device="cuda", dtype=torch.uint8)
    s = torch.rand(64, 4, device="cuda").half()
    y = torch.zeros(2, 64, device="cuda").half()
    binding.im2win_matvec_int4(x, w, s, y, 128)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.im2win_matvec_int4(x, w, s, y, 128)
    for _ in range(2):
        x.copy_(torch.randn(2, 512))
        graph.replay()
        want, a = matvec_64(x.cpu(), w.cpu(), s.cpu(), None, None, 128)
        close(y, want, 84 * 2.0 ** -23 * a + rounding(want, torch.float16), "y")
