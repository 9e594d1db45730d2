"""o of the gated delta rule's chunks is rounded to its type once: what is rounded before, of rows of 16 bits too, is far below that."""
import math

import pytest
import torch

from delta_helpers import delta_64
from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, close, rounding, sequence_list

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("heads,dk,dv", [(2, 64, 64), (2, 128, 128), (3, 80, 40), (40, 128, 128), (80, 64, 64)])
def test_o_is_rounded_once(dtype, heads, dk, dv):
    """Tolerance: half a step of the type, and delta_64 with the sums in fp32 alone; of bf16 a term's weight and its new value are two bf16 pieces each, off by
    2^-18, and the product of the two small pieces is left out, 2^-18."""
    gen, tdt, n = torch.Generator().manual_seed(5), DTYPES[dtype], 200 if heads < 10 else 70
    q, k, v = (torch.randn(n, heads, d, generator=gen).to(tdt) for d in (dk, dk, dv))
    g, beta = -0.1 * torch.rand(n, heads, generator=gen), torch.rand(n, heads, generator=gen)
    o = torch.zeros(n, heads, dv, dtype=tdt, device="cuda")
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    binding.im2win_gated_delta_rule(*(x.cuda() for x in (q, k, v, g, beta)), o, scale=1 / math.sqrt(dk), normalize=True, cu_seqlens=cu)
    want, off = delta_64(q, k, v, g, beta, 1 / math.sqrt(dk), True, torch.zeros(n, heads, dv), None, None, sequence_list([n]), 1,
                         3 * 2.0 ** -18 if dtype == "bf16" else 0.0)[:2]
    close(o, want, off + rounding(want, tdt), "o")
