"""im2win_gated_delta_rule against the recurrence in 64 bits (tolerances: delta_64, and one rounding of o to its type)."""
import math

import pytest
import torch

from delta_helpers import close_columns, delta_64, run
from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, Guarded, close, half_step, rounding, sequence_list

pytestmark = pytest.mark.gpu

LENGTHS = [5, 0, 1, 70, 2, 33, 0, 130, 64, 65]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (64, 128), (16, 32), (1, 1), (7, 33), (80, 96), (100, 41), (200, 36), (128, 256)])
def test_packed_sequences_of_every_kind(dtype, normalize, dk, dv):
    run(dtype, LENGTHS, 2, 1, dk, dv, tail=3, resume=[1, 0, 1, 0, 1, 1, 1, 0, 1, 0], normalize=normalize)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("decay", ["heads", "expanded"])
def test_one_decay_for_each_head(dtype, decay):
    run(dtype, [3, 150], 4, 2, 64, 64, decay=decay)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("mode", ["packed", "dense", "step"])
def test_states_in_any_order_with_padding(mode, in_place):
    n = {"packed": [9, 100, 0, 1, 2], "dense": [77] * 5, "step": [1] * 5}[mode]
    run("bf16", n, 3, 3, 64, 128, slots=[6, -1, 3, 0, 9], pool=9, in_place=in_place, mode=mode,
        resume=None if mode == "step" else [1, 1, 0, 1, 1])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("heads,dk,dv", [(1, 128, 128), (16, 64, 64), (2, 256, 256), (3, 48, 80), (5, 33, 35), (80, 128, 128)])
def test_single_tokens(dtype, heads, dk, dv):
    run(dtype, [1] * 4, heads, heads, dk, dv, mode="step", pitch=3)


@pytest.mark.parametrize("mode", ["packed", "dense", "step"])
def test_without_states(mode):
    n = {"packed": [9, 100, 0, 1, 2], "dense": [3] * 5, "step": [1] * 5}[mode]
    run("f16", n, 2, 2, 64, 64, state=False, mode=mode)
    run("f16", n, 2, 2, 64, 64, state=False, mode=mode, slots=[0, 5, -2, 1, 3])


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_shared_heads_and_strides(dtype):
    run(dtype, [40, 90], 8, 2, 64, 64, pitch=8)
    run(dtype, [40, 90], 6, 2, 64, 128, pitch=5)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("normalize", [False, True])
def test_rows_that_are_alike(dtype, normalize):
    """The same k again and again, beta of 1: each token replaces what the one before wrote; and beta of 0, which writes nothing."""
    def edit(q, k, v, g, beta, st):
        k[:] = k[:1]
        beta[:90] = 1.0
        beta[100:110] = 0.0
        g[:50] = 0.0
    run(dtype, [64, 80, 20], 2, 2, 64, 64, edit=edit, normalize=normalize)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_beta_up_to_two(dtype):
    """Reflections: the state does not shrink."""
    def edit(q, k, v, g, beta, st):
        beta.mul_(2.0).clamp_(max=1.99)
        g.mul_(0.05)
    run(dtype, [200, 31], 2, 2, 64, 64, edit=edit)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("normalize", [False, True])
def test_rows_of_zeros_and_of_other_sizes(dtype, normalize):
    def edit(q, k, v, g, beta, st):
        q[3] = k[4] = 0.0
        k[5] *= 1e-3
        k[70:72] *= 2.0 ** -10
        q[20:30] *= 100
        v[10:20] *= 1000
        v[80:90] *= 1e-4
    run(dtype, [100, 30], 2, 1, 64, 64, edit=edit, normalize=normalize)


def test_large_and_small_values_in_fp16():
    """States beyond the type's range and far below its smallest normal number."""
    def large(q, k, v, g, beta, st):
        v.mul_(1e4)
        st.mul_(1e6)
        q.mul_(1e-2)
    def small(q, k, v, g, beta, st):
        v.mul_(1e-5)
        st.mul_(1e-9)
        q.mul_(100)
    run("f16", [150, 40], 2, 2, 64, 64, edit=large, scale=1e-6)
    run("f16", [150, 40], 2, 2, 64, 64, edit=small, scale=1e3, normalize=False)


def test_empty_calls_move_states():
    run("bf16", [0, 0, 0], 2, 2, 64, 64, resume=[1, 0, 1])
    run("f32", [0, 0], 1, 1, 64, 64, mode="dense")


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_decays_of_every_size(dtype):
    """No decay, one that empties the state (minus infinity, the type's lowest value), very strong and very weak ones, growth."""
    def edit(q, k, v, g, beta, st):
        g[:40] = 0.0
        g[40] = -math.inf
        g[50] = torch.finfo(torch.float32).min
        g[51:55] = -300.0
        g[55:70] = -20.0
        g[70:80] = -1e-6
        g[80:90] = 0.05
        g[100:102] = -math.inf
    run(dtype, [128, 30], 2, 2, 64, 64, edit=edit)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("which", ["v", "k", "q", "beta", "g"])
def test_values_stay_within_their_sequence_and_behind_their_row(dtype, which):
    """Infinities and NaNs of a row, of rows behind the last sequence and of states that are not resumed meet no other row before them."""
    def edit(q, k, v, g, beta, st):
        x = {"q": q, "k": k, "v": v}.get(which)
        if x is None:
            x = (beta if which == "beta" else g)[:, :, None]
        x[70, 0, 3 % x.shape[2]] = math.inf
        x[75, 1, 1 % x.shape[2]] = math.nan
        x[-2:] = math.nan
        st[0] = math.nan
        st[2] = math.inf
        st[2, 1] = math.nan
    run(dtype, [10, 100, 0, 30], 2, 2, 64, 64, tail=2, resume=[0, 1, 0, 1], edit=edit)


def test_columns_that_are_not_finite_stay_alone():
    """A state with an infinity in one column, a v with one in another, in chunks that are whole and one that is not."""
    def edit(q, k, v, g, beta, st):
        st[0, 0, 5, 17] = math.inf
        st[0, 1, 60, 2] = math.nan
        v[100, 0, 40] = -math.inf
        v[150, 1, 41] = math.nan
    for dtype in DTYPES:
        run(dtype, [170], 2, 2, 64, 64, edit=edit)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128)])
def test_states_are_32_bit_ones(dtype, dk, dv):
    """Over 600 tokens the whole state is off by no more than 2^-20 of its norm: 2^-22 for each of the sums that an error passes through (products
    of pieces of 22 bits and more), which are independent, and four times that on top."""
    gen = torch.Generator().manual_seed(7)
    q, k = (torch.randn(600, 2, dk, generator=gen).to(DTYPES[dtype]) for _ in range(2))
    v = torch.randn(600, 2, dv, generator=gen).to(DTYPES[dtype])
    g, beta = -0.02 * torch.rand(600, 2, generator=gen), torch.rand(600, 2, generator=gen)
    o, state = torch.zeros(1, 600, 2, dv, dtype=DTYPES[dtype], device="cuda"), torch.zeros(1, 2, dk, dv, device="cuda")
    binding.im2win_gated_delta_rule(*(x[None].cuda() for x in (q, k, v, g, beta)), o, normalize=True, state_out=state)
    want = delta_64(q, k, v, g, beta, 1.0, True, torch.zeros(600, 2, dv), None, torch.zeros(1, 2, dk, dv), sequence_list([600]), 1)[2]
    off = float((state.double().cpu() - want).norm() / want.norm())
    assert off < 2.0 ** -20, off


def test_prompt_and_single_tokens_agree():
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(1, 70, 2, 64, generator=gen, device="cuda") for _ in range(3))
    g, beta = -torch.rand(1, 70, 2, generator=gen, device="cuda"), torch.rand(1, 70, 2, generator=gen, device="cuda")
    whole, final = torch.empty_like(v), torch.empty(1, 2, 64, 64, device="cuda")
    binding.im2win_gated_delta_rule(q, k, v, g, beta, whole, normalize=True, state_out=final)
    o, state = torch.empty_like(v), torch.zeros(1, 2, 64, 64, device="cuda")
    for t in range(70):
        part = torch.empty(1, 1, 2, 64, device="cuda")
        binding.im2win_gated_delta_rule(q[:, t:t + 1], k[:, t:t + 1], v[:, t:t + 1], g[:, t:t + 1], beta[:, t:t + 1], part, normalize=True,
                                        state=state, state_out=state)
        o[:, t:t + 1] = part
    assert float((o - whole).norm() / whole.norm()) < 2.0 ** -20 and float((state - final).norm() / final.norm()) < 2.0 ** -20


def test_captured_step_replays_on_new_values_and_slots():
    q, k, v = (torch.randn(4, 2, 64, device="cuda").bfloat16() for _ in range(3))
    g, beta = -torch.rand(4, 2, device="cuda"), torch.rand(4, 2, device="cuda")
    o, pool = torch.zeros_like(v), torch.randn(6, 2, 64, 64, device="cuda")
    slots = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    call = lambda: binding.im2win_gated_delta_rule(q, k, v, g, beta, o, normalize=True, state=pool, state_out=pool, slots=slots)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for order in ([5, 2, -1, 0], [1, 4, 3, -1]):
        slots.copy_(torch.tensor(order, dtype=torch.int32))
        v.copy_(torch.randn(4, 2, 64))
        o.zero_()
        before = pool.cpu().clone()
        graph.replay()
        want, off, new, new_off = delta_64(q.cpu(), k.cpu(), v.cpu(), g.cpu(), beta.cpu(), 1.0, True, torch.zeros(4, 2, 64), before, before,
                                           sequence_list([1] * 4, order), 6)
        close(o, want, off + rounding(want, torch.bfloat16), "o")
        close_columns(pool, new, new_off, "pool")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_captured_prompt_replays_with_other_lengths(dtype):
    """A call captured for a batch of prompts, replayed on other rows, other cuts and another number of real sequences."""
    tdt = DTYPES[dtype]
    q, k, v = (torch.randn(300, 2, 64, device="cuda").to(tdt) for _ in range(3))
    g, beta = -torch.rand(300, 2, device="cuda"), torch.rand(300, 2, device="cuda")
    o, pool = torch.zeros_like(v), torch.randn(4, 2, 64, 64, device="cuda")
    cu = torch.tensor([0, 100, 200, 300], dtype=torch.int32, device="cuda")
    slots = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    call = lambda: binding.im2win_gated_delta_rule(q, k, v, g, beta, o, normalize=True, state=pool, state_out=pool, cu_seqlens=cu, slots=slots)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lengths, order in (([7, 0, 250], [3, 0, 1]), ([129, 64, 20], [2, -1, 0])):
        cu.copy_(torch.tensor([0] + [sum(lengths[:i + 1]) for i in range(3)], dtype=torch.int32))
        slots.copy_(torch.tensor(order, dtype=torch.int32))
        v.copy_(torch.randn(300, 2, 64))
        o.zero_()
        before = pool.cpu().clone()
        graph.replay()
        want, off, new, new_off = delta_64(q.cpu(), k.cpu(), v.cpu(), g.cpu(), beta.cpu(), 1.0, True, torch.zeros(300, 2, 64), before, before,
                                           sequence_list(lengths, order), 4, 2 * half_step(torch.float16))
        close(o, want, off + rounding(want, tdt), "o")
        close_columns(pool, new, new_off, "pool")


def test_the_same_call_gives_the_same_bits():
    a = run("bf16", LENGTHS, 3, 3, 64, 64).clone()
    assert torch.equal(a, run("bf16", LENGTHS, 3, 3, 64, 64))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_row_numbers_that_break_the_rules_stay_within_the_buffers(dtype):
    tdt = DTYPES[dtype]
    for cu in ([-5, 3, 900, 20], [10, 4, 2, 1], [0, 2 ** 31 - 1, -2 ** 31, 7], [300, 300, 300, 300]):
        for max_len in (0, 1):
            o, state = Guarded((300, 2, 64), tdt), Guarded((3, 2, 64, 64), torch.float32)
            x = torch.ones(300, 2, 64, dtype=tdt, device="cuda")
            binding.im2win_gated_delta_rule(x, x, x, torch.zeros(2, device="cuda"), torch.ones(2, device="cuda"), o.view, normalize=True,
                                            state=state.view, state_out=state.view, max_len=max_len,
                                            cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda"))
            torch.cuda.synchronize()
            for t in (o, state):
                t.assert_untouched_outside()


def test_on_another_stream():
    side = torch.cuda.Stream()
    q, k, v = (torch.randn(1, 200, 2, 64, device="cuda").bfloat16() for _ in range(3))
    g, beta = -torch.rand(2, device="cuda"), torch.rand(2, device="cuda")
    o, other = torch.zeros_like(v), torch.zeros_like(v)
    binding.im2win_gated_delta_rule(q, k, v, g, beta, o, normalize=True)
    torch.cuda.synchronize()
    binding.im2win_gated_delta_rule(q, k, v, g, beta, other, normalize=True, stream=side)
    side.synchronize()
    assert torch.equal(o, other) and bool(o.any())


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("heads,dk,dv", [(40, 64, 128), (75, 128, 64), (40, 100, 100), (52, 33, 96)])
def test_more_columns_than_blocks_of_32(dtype, heads, dk, dv):
    """Heads and columns beyond one block of 32 columns for each SM."""
    run(dtype, [65, 20], heads, heads // 5 if heads % 5 == 0 else heads, dk, dv, tail=1, resume=[1, 0])


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_columns_that_are_not_finite_in_wide_blocks(dtype):
    def edit(q, k, v, g, beta, st):
        v[30, 3, 100] = math.inf
        v[70, 39, 7] = math.nan
        st[0, 5, 3, 64] = math.nan
        k[80, 1, 0] = math.inf
    run(dtype, [100], 40, 8, 64, 128, edit=edit)


def test_pools_beyond_32_bits():
    """A state whose first element is number 2^31 and more of the pool."""
    pool = torch.empty(4200, 32, 128, 128, device="cuda")
    gen = torch.Generator().manual_seed(2)
    for n in (1, 40):
        q, k, v = (torch.randn(n, 32, 128, generator=gen).bfloat16() for _ in range(3))
        g, beta, st = -torch.rand(n, 32, generator=gen), torch.rand(n, 32, generator=gen), torch.randn(1, 32, 128, 128, generator=gen)
        pool[4199].copy_(st[0])
        o = torch.zeros(n, 32, 128, dtype=torch.bfloat16, device="cuda")
        binding.im2win_gated_delta_rule(*(x.cuda() for x in (q, k, v, g, beta)), o, normalize=True, state=pool, state_out=pool,
                                        cu_seqlens=torch.tensor([0, n], dtype=torch.int32, device="cuda"),
                                        slots=torch.tensor([4199], dtype=torch.int32, device="cuda"))
        want, off, new, new_off = delta_64(q, k, v, g, beta, 1.0, True, torch.zeros(n, 32, 128), st, st, sequence_list([n]), 1,
                                           2 * half_step(torch.float16))
        close(o, want, off + rounding(want, torch.bfloat16), "o")
        close_columns(pool[4199:], new, new_off, "pool")
