"""im2win_gated_delta_rule on values that lie far apart within 64 tokens, against the recurrence in 64 bits: what a token makes takes no bits from the
tokens before it, nor from those behind a decay that empties the state (tolerances: delta_64, which goes by each token's own sums, and one rounding)."""
import math

import pytest
import torch

from delta_helpers import delta_64, run
from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, close, rounding, sequence_list

pytestmark = pytest.mark.gpu


def check(dtype, lengths, **kw):
    run(dtype, lengths, 2, 1, 64, 64, kernel="chunks", **kw)
    run(dtype, lengths, 2, 2, 128, 48, kernel="chunks", **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("factor", [1e5, 1e7, 1e9, 1e12, 1e30])
def test_one_large_v(dtype, factor):
    """In the first, a middle and the last block of 16 tokens; rows before it, behind it, and of the next chunk."""
    for row in (5, 40, 63):
        def edit(q, k, v, g, beta, st):
            v[row] *= factor
        check(dtype, [100], edit=edit)
        check(dtype, [100], edit=edit, normalize=False, state=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("factor", [1e7, 1e12, 1e30])
@pytest.mark.parametrize("decay", [-math.inf, -60.0])
def test_decays_behind_a_large_v(dtype, factor, decay):
    """The decay leaves nothing of it, or a part that its size brings back to the others'."""
    def edit(q, k, v, g, beta, st):
        v[10] *= factor
        g[11:13] = decay
        v[30, 0] *= factor
        g[37, 0] = decay / 2
    check(dtype, [100], edit=edit)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decays_bring_a_large_state_down(dtype):
    """10 tokens of e^-3 each, from 1e13 to the size of v, in the middle of a block of 16."""
    def edit(q, k, v, g, beta, st):
        st *= 1e13
        v[:20] *= 1e13
        g[20:30] = -3.0
    check(dtype, [100], edit=edit)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", [1e7, 1e12, 1e25])
def test_a_large_state_that_is_emptied(dtype, size):
    """Rows behind it are the sequence's own (those before it ask for nothing, so that fp16 rows do not overflow)."""
    def edit(q, k, v, g, beta, st):
        st *= size
        g[35] = -math.inf
        q[:35] = 0.0
    check(dtype, [100], edit=edit)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-6, 1e-10, 1e-20])
def test_small_rows_before_ordinary_ones(dtype, size):
    def edit(q, k, v, g, beta, st):
        v[:21] *= size
        v[64:70] *= size
    check(dtype, [100], edit=edit, state=False)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("length", [1.9, 2.5, 3.0])
def test_alike_keys_that_are_longer_than_one(dtype, length):
    """beta |k|^2 of `length`: what is written grows from token to token by |1 - length|."""
    def edit(q, k, v, g, beta, st):
        k[:] = k[:1]
        beta.fill_(length)
        g *= 0.01
    check(dtype, [24 if dtype == "f16" else 40], edit=edit, normalize=False, scale=1e-3 if dtype == "f16" else None, state=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_keys(dtype):
    """|k|^2 of 64: what is written grows by many powers of ten."""
    def edit(q, k, v, g, beta, st):
        k *= 8.0
    check(dtype, [30], edit=edit, normalize=False, state=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_apart_in_wide_blocks(dtype):
    """More heads than give each SM a block of 32 columns."""
    def edit(q, k, v, g, beta, st):
        v[50, 3] *= 1e12
        v[9, 7] *= 1e20
        g[60, 7] = -math.inf
        st[0, 11] *= 1e15
        g[20, 11] = -math.inf
    for dk in (64, 128):
        run(dtype, [90], 80, 16, dk, 64, edit=edit, kernel="chunks")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-30, 1e-20, 1e20, 1e36])
def test_everything_small_or_large(dtype, size):
    def edit(q, k, v, g, beta, st):
        v.mul_(size)
        st.mul_(size)
    check(dtype, [100], edit=edit)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_growth_beyond_the_range(dtype):
    """Alike keys of beta |k|^2 of 20: a token's part in a later one grows by 19 a token and passes the range of floats some 30 tokens on.  Rows up to 15
    before that are right, of the others each is, or is not finite."""
    gen, tdt = torch.Generator().manual_seed(3), DTYPES[dtype]
    q, v = (torch.randn(40, 1, 64, generator=gen).to(tdt) for _ in range(2))
    k = (torch.ones(40, 1, 64) / 8).to(tdt)
    g, beta = torch.zeros(1), torch.full((1,), 20.0)
    o = torch.zeros(40, 1, 64, dtype=tdt, device="cuda")
    binding.im2win_gated_delta_rule(*(x.cuda() for x in (q, k, v, g, beta)), o, scale=0.125, cu_seqlens=torch.tensor([0, 40], dtype=torch.int32, device="cuda"))
    want, off = delta_64(q, k, v, g, beta, 0.125, False, torch.zeros(40, 1, 64), None, None, sequence_list([40]), 1,
                         0.0 if dtype == "f32" else 3 * 2.0 ** -18)[:2]
    off, got = off + rounding(want, tdt), o.double().cpu()
    close(got[:14], want[:14], off[:14], "o")
    assert bool((((got - want).abs() <= off) | ~torch.isfinite(got)).all())
