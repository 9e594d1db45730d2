"""im2win_matvec_int4 of fp32 rows, whose elements go through the tensor cores as three bf16 pieces: results that all three decide.

One element of x a row, 24 bits long: (w - z) times each piece is exact, each of the three is multiplied by its scale and added to the
others, five roundings in all of numbers no larger than y.  Without the third piece y would be off by up to 2^-16 of itself, 2^8 of those.
Two elements of opposite sign, equal but for their low pieces, before equal weights: the first pieces cancel exactly, and y comes from
what is left, exactly as before."""
import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import matvec_64

pytestmark = pytest.mark.gpu

MS = [1, 2, 3, 8, 11, 16]
SIZES = [(40, 128, 32), (33, 384, 64), (50, 4096, 64), (48, 8192 + 128, 128), (300, 2176, 64)]


def odd_mantissas(shape, gen):
    """Floats all of whose 24 bits count, of either sign, from 2^-20 to 2^20."""
    bits = torch.randint(0, 1 << 22, shape, generator=gen) * 2 + 1 + (1 << 23)
    return (bits.double() * 2.0 ** (torch.randint(-20, 21, shape, generator=gen) - 23).double()
            * (torch.randint(0, 2, shape, generator=gen) * 2 - 1)).float()


def check(x, w, s, z, group):
    y = torch.empty(x.shape[0], w.shape[0], device="cuda")
    binding.im2win_matvec_int4(x.cuda(), w.cuda(), s.cuda(), y, group, zeros=z.cuda())
    want, _ = matvec_64(x, w, s, z, None, group)
    off = (y.double().cpu() - want).abs() - 5 * 2.0 ** -24 * want.abs()
    assert float(off.max()) <= 0.0, float(off.max())


@pytest.mark.parametrize("m", MS)
@pytest.mark.parametrize("n,k,group", SIZES)
def test_one_element_a_row(m, n, k, group):
    gen = torch.Generator().manual_seed(m * k)
    x = torch.zeros(m, k)
    x[torch.arange(m), torch.randint(0, k, (m,), generator=gen)] = odd_mantissas((m,), gen)
    x[m - 1] = 0.0
    x[m - 1, k - 1] = odd_mantissas((1,), gen)[0]
    w = torch.randint(0, 256, (n, k // 2), generator=gen, dtype=torch.uint8)
    s = torch.rand(n, k // group, generator=gen) + 0.5
    z = torch.randint(0, 16, (n, k // group), generator=gen, dtype=torch.uint8)
    check(x, w, s, z, group)


@pytest.mark.parametrize("m", MS)
@pytest.mark.parametrize("n,k,group", SIZES)
def test_elements_that_cancel_but_for_their_low_pieces(m, n, k, group):
    gen = torch.Generator().manual_seed(m * k + 1)
    x = torch.zeros(m, k)
    at = torch.randint(0, k // group, (m,), generator=gen) * group
    a = odd_mantissas((m,), gen)
    first = (a.view(torch.int32) & -65536).view(torch.float32)
    r = torch.arange(m)
    x[r, at + 1], x[r, at + group - 2] = a, -first
    nibbles = torch.randint(0, 16, (n, 1), generator=gen, dtype=torch.uint8)
    w = (nibbles * 17).expand(n, k // 2).contiguous()
    s = torch.rand(n, k // group, generator=gen) + 0.5
    z = torch.randint(0, 16, (n, k // group), generator=gen, dtype=torch.uint8)
    check(x, w, s, z, group)
