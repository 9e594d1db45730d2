"""im2win_matmul_int8: the sum is exact, and what is done with it is the same steps whichever way a call is run."""
import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, Guarded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("m,n", [(3, 300), (8, 1000), (40, 500), (130, 640), (3000, 2100)])
def test_rows_that_start_anywhere_agree_bit_for_bit(dtype, m, n):
    """Few rows, tiles of 64 with and without clusters, of 128, against the tiles of rows on 16 bytes."""
    gen = torch.Generator(device="cuda").manual_seed(m)
    x, w = (torch.randint(-128, 128, (rows, 512), generator=gen, device="cuda", dtype=torch.int8) for rows in (m, n))
    xs, ws = torch.rand(m, generator=gen, device="cuda"), torch.rand(n, generator=gen, device="cuda") * 1e-3
    for bias in (torch.randn(n, generator=gen, device="cuda"), None):
        out = []
        for shift in (0, 1):
            at, y = Guarded((m, 512), torch.int8, 16, fill=99, shift=shift), torch.zeros(m, n, dtype=DTYPES[dtype], device="cuda")
            at.view.copy_(x)
            binding.im2win_matmul_int8(at.view, xs, w, ws, y, bias=bias)
            out.append(y)
        assert torch.equal(*out), int((out[0] != out[1]).sum())
