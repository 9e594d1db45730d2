"""The bounded waits of the operators on token sequences.  Nothing here faults, traps or hangs the GPU: a testing aid leaves one arrival
out and lowers the limit of polls, the waits for it give up, the kernel returns, and what it could not make is NaN."""
import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, close, half_step, linear_64, matvec_64, rounding, sequence_list

pytestmark = pytest.mark.gpu


def attention(dtype, lengths, dk, dv, seed=1, spread=1.0):
    gen = torch.Generator().manual_seed(seed)
    rows, b = sum(lengths), len(lengths)
    q, k = (torch.randn(rows, 2, dk, generator=gen).to(DTYPES[dtype]) for _ in range(2))
    v = torch.randn(rows, 2, dv, generator=gen).to(DTYPES[dtype])
    g, state = -0.1 * torch.rand(rows, 2, generator=gen), torch.randn(b, 2, dk, dv, generator=gen)
    cu = torch.tensor([sum(lengths[:i]) for i in range(b + 1)], dtype=torch.int32, device="cuda")
    o, new = torch.zeros(rows, 2, dv, dtype=DTYPES[dtype], device="cuda"), state.cuda()
    ws = binding.alloc_attention_workspace(binding.make_attention_shape(rows, b, 2, 2, dk, dv), DTYPES[dtype])
    binding.im2win_linear_attention(q.cuda(), k.cuda(), v.cuda(), g.cuda(), o, ws, scale=0.1, state=new, state_out=new, cu_seqlens=cu)
    want = linear_64(q, k, v, g, 0.1, torch.zeros(rows, 2, dv), state, state, sequence_list(lengths), b, half_step(DTYPES[dtype]))
    return ws, o, new, want


def compare(dtype, o, new, want, heads):
    ref, off, states, states_off = want
    close(o[:, heads], ref[:, heads], (off + rounding(ref, DTYPES[dtype]))[:, heads], "o")
    close(new[:, heads], states[:, heads], states_off[:, heads], "state_out")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 200), (100, 41)])
@pytest.mark.parametrize("segments,drop,lengths", [(1, "0", [300, 70]), (1, "2", [300, 135]), (1, "1", [128, 90]), (1, "4", [300, 290]),
                                                   (3, "0", [600]), (3, "1", [600])])
def test_attention_gives_up_and_says_so(dtype, dk, dv, segments, drop, lengths, monkeypatch):
    """Head 0's blocks do not hear of a chunk's products: its o and states are NaN, where a sequence has such a chunk; head 1's are right."""
    monkeypatch.setenv("IM2WIN_SEGMENTS", str(segments))
    monkeypatch.setenv("IM2WIN_ATTENTION_DROP", drop)
    ws, o, new, want = attention(dtype, lengths, dk, dv)
    with pytest.raises(binding.Im2winError) as err:
        binding.im2win_check_status(ws)
    assert err.value.code == 7
    compare(dtype, o, new, want, slice(1, 2))
    assert bool(o[:, 0].isnan().all()) and bool(new[:, 0].isnan().all())
    monkeypatch.delenv("IM2WIN_ATTENTION_DROP")
    for _ in range(2):                            # the tensor memory was given back: the same call, from the start
        ws, o, new, want = attention(dtype, lengths, dk, dv)
        binding.im2win_check_status(ws)
        compare(dtype, o, new, want, slice(0, 2))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 200)])
@pytest.mark.parametrize("drop", ["0", "1", "2"])
def test_attention_gives_up_in_the_sums_of_segments(dtype, dk, dv, drop, monkeypatch):
    """The first segment starts from the caller's state and is right; all behind it hang on sums that were not made."""
    monkeypatch.setenv("IM2WIN_SEGMENTS", "3")
    monkeypatch.setenv("IM2WIN_ATTENTION_DROP_SUMS", drop)
    ws, o, new, want = attention(dtype, [576], dk, dv)
    with pytest.raises(binding.Im2winError) as err:
        binding.im2win_check_status(ws)
    assert err.value.code == 7
    compare(dtype, o, new, want, slice(1, 2))
    ref, off, _, _ = want
    close(o[:192, 0], ref[:192, 0], (off + rounding(ref, DTYPES[dtype]))[:192, 0], "o of the first segment")
    assert bool(o[192:, 0].isnan().all()) and bool(new[:, 0].isnan().all())
    monkeypatch.delenv("IM2WIN_ATTENTION_DROP_SUMS")
    ws, o, new, want = attention(dtype, [576], dk, dv)
    binding.im2win_check_status(ws)
    compare(dtype, o, new, want, slice(0, 2))


@pytest.mark.parametrize("dtype,m,group", [("f16", 1, 128), ("bf16", 8, 64), ("bf16", 16, 32), ("f32", 2, 64), ("f32", 7, 128)])
@pytest.mark.parametrize("k", [2048, 4096])
def test_products_give_up_and_say_so(dtype, m, group, k, monkeypatch):
    """A warp of the first block does not free its slot after the first tile: the ring stops there.  The tiles that had come by then are
    right, the block's others NaN; those of the other blocks are right."""
    n, rows, tdt = 148 * 32 * 7, 32 * 7, DTYPES[dtype]
    gen = torch.Generator().manual_seed(m)
    x = torch.randn(m, k, generator=gen).to(tdt)
    w = torch.randint(0, 256, (n, k // 2), generator=gen, dtype=torch.uint8)
    s = ((torch.rand(n, k // group, generator=gen) + 0.5) * 0.1).to(tdt)
    xd, wd, sd, y = x.cuda(), w.cuda(), s.cuda(), torch.zeros(m, n, dtype=tdt, device="cuda")
    want, a = matvec_64(x, w[:2 * rows], s[:2 * rows], None, None, group)
    tol = (k / 8 + 16 + k // group) * 2.0 ** -23 * a + rounding(want, tdt)
    monkeypatch.setenv("IM2WIN_MATVEC_DROP", "0")
    binding.im2win_matvec_int4(xd, wd, sd, y, group)
    torch.cuda.synchronize()
    monkeypatch.delenv("IM2WIN_MATVEC_DROP")
    bad = y.isnan().cpu()
    assert bool(bad[:, 4 * 32:rows].all()) and not bool(bad[:, rows:].any()) and torch.equal(bad, bad[:1].expand_as(bad))
    right = ~bad[0, :2 * rows]
    close(y[:, :2 * rows][:, right.cuda()], want[:, right], tol[:, right], "y")
    again = torch.zeros_like(y)
    binding.im2win_matvec_int4(xd, wd, sd, again, group)
    close(again[:, :2 * rows], want, tol, "y")
    assert torch.equal(again[:, rows:], y[:, rows:])
