"""im2win_causal_conv1d against its definition in 64 bits.

Tolerance: the fp32 sum of taps + 1 terms, each term one fused multiply-add, is off by at most (taps + 1) 2^-24 sum|w x|; the slope of
z / (1 + exp(-z)) stays below 1.1; the 16-bit types' exp2, reciprocal, product and sum add 2^-22 + 2^-23 + 3 * 2^-24 + 2^-23 |z|
relative (the last from rounding z log2 e, up to its half step, in the exponent: |z| log2(e) 2^-24 ln 2), fp32's exp and division less; and one rounding to the type."""
import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, Guarded, close, conv1d_64, rounding, sequence_list

pytestmark = pytest.mark.gpu


def run(dtype, lengths, channels, taps, bias=True, silu=True, tail=0, slots=None, pool=None, resume=None, state=True, in_place=False,
        pitch=0, shift=0, mode="packed", seed=1, edit=None):
    """One call on guarded tensors, compared with the definition.  mode: packed (cu_seqlens), dense ([sequences, tokens, channels]) or step."""
    g = torch.Generator().manual_seed(seed)
    tdt, rows, b = DTYPES[dtype], sum(lengths) + tail, len(lengths)
    pool = pool or b
    x = torch.randn(rows, channels, generator=g).to(tdt)
    w = ((torch.rand(channels, taps, generator=g) * 2 - 1)).to(tdt)
    bs = torch.randn(channels, generator=g) if bias else None
    st = torch.randn(pool, taps - 1, channels, generator=g).to(tdt) if state else None
    if edit:
        edit(x, st)
    xg, yg = Guarded((rows, channels), tdt, pitch, shift=shift), Guarded((rows, channels), tdt, pitch, shift=shift)
    xg.view.copy_(x)
    y_before = yg.view.cpu().clone()
    sg = og = None
    if state:
        sg = Guarded((pool, taps - 1, channels), tdt)
        sg.view.copy_(st)
        og = sg if in_place else Guarded((pool, taps - 1, channels), tdt)
    out_before = og.view.cpu().clone() if state else None
    args = dict(bias=None if bs is None else bs.cuda(), silu=silu)
    xv, yv = xg.view, yg.view
    if mode == "packed":
        cu = [0]
        for n in lengths:
            cu.append(cu[-1] + n)
        args["cu_seqlens"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    elif mode == "dense":
        xv, yv = (v.unflatten(0, (b, lengths[0])) for v in (xv, yv))
    if slots is not None:
        args["slots"] = torch.tensor(slots, dtype=torch.int32, device="cuda")
    if resume is not None:
        args["resume"] = torch.tensor(resume, dtype=torch.bool, device="cuda")
    if state:
        args.update(state=sg.view, state_out=og.view)
    binding.im2win_causal_conv1d(xv, w.cuda(), yv, **args)
    torch.cuda.synchronize()
    bound_pool = pool if state or slots is None else 1 << 31
    want, new, a = conv1d_64(x, w, bs, silu, y_before, st, out_before, sequence_list(lengths, slots, resume), bound_pool)
    z = 2.0 ** -24
    tol = 1.1 * (taps + 1) * z * a + rounding(want, tdt)
    if silu:
        tol = tol + want.abs() * (2.0 ** -22 + 2.0 ** -23 + 3 * z + 2 * z * a)
    close(yg.view, want, tol, "y")
    yg.assert_untouched_outside()
    if state:
        close(og.view, new, torch.zeros_like(new), "state_out")
        og.assert_untouched_outside()
    return yg.view


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("taps", [1, 2, 3, 4, 5, 8])
def test_packed_sequences_of_every_kind(dtype, taps):
    run(dtype, [5, 0, 1, 70, 2, 33, 0, 3, 32, 64], 72, taps, tail=3, resume=[1, 0, 1, 0, 1, 1, 1, 0, 1, 0])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("channels,pitch,shift", [(1, 0, 0), (7, 0, 0), (64, 8, 0), (64, 3, 0), (64, 0, 1), (1024, 0, 0), (1032, 16, 0), (2049, 5, 3)])
def test_widths_strides_and_alignments(dtype, channels, pitch, shift):
    run(dtype, [3, 40, 0, 1], channels, 4, pitch=pitch, shift=shift, bias=channels % 2 == 0, silu=channels % 3 == 0)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("mode", ["packed", "dense", "step"])
def test_states_in_any_order_with_padding(mode, in_place):
    n = {"packed": [9, 100, 0, 1, 2], "dense": [37] * 5, "step": [1] * 5}[mode]
    run("bf16", n, 136, 4, slots=[6, -1, 3, 0, 9], pool=9, in_place=in_place, mode=mode, resume=None if mode == "step" else [1, 1, 0, 1, 1])


@pytest.mark.parametrize("mode", ["packed", "dense", "step"])
def test_without_states(mode):
    n = {"packed": [9, 100, 0, 1, 2], "dense": [3] * 5, "step": [1] * 5}[mode]
    run("f16", n, 40, 3, state=False, mode=mode)
    run("f16", n, 40, 3, state=False, mode=mode, slots=[0, 5, -2, 1, 3])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("taps", [1, 2, 4, 7, 8])
@pytest.mark.parametrize("channels", [33, 2048])
def test_single_tokens_of_many_sequences(dtype, taps, channels):
    b = 301
    slots = [(7 * i) % 320 if i % 5 else -1 for i in range(b)]
    run(dtype, [1] * b, channels, taps, mode="step", slots=slots, pool=320, in_place=True, resume=[i % 3 != 1 for i in range(b)])


def test_more_sequences_than_a_block_has_threads():
    run("f32", [i % 5 for i in range(700)], 8, 3, tail=1)


def test_empty_calls_move_states():
    run("bf16", [0, 0, 0], 24, 4, resume=[1, 0, 1])
    run("bf16", [0, 0, 0], 24, 4, resume=[1, 0, 1], mode="dense")


def test_values_stay_within_their_sequence_and_behind_their_row():
    """Infinities and NaNs of one sequence, of the rows behind the last one and of states that are not resumed."""
    def edit(x, st):
        x[20] = float("nan")
        x[21:24] = float("inf")
        x[-2:] = float("nan")
        st[0] = float("nan")
        st[3] = float("inf")
    run("bf16", [10, 30, 5, 6], 64, 4, silu=False, tail=2, resume=[0, 1, 1, 0], edit=edit)


def test_large_magnitudes_through_the_activation():
    def edit(x, st):
        x.mul_(200)
    run("f32", [50], 64, 4, edit=edit)
    run("bf16", [50], 64, 4, edit=edit)


def test_prompt_and_single_tokens_agree():
    """A prompt in one call, or in two, or token by token: the same bits."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(1, 45, 96, generator=g, device="cuda").half()
    w = torch.randn(96, 4, generator=g, device="cuda").half()
    whole = torch.empty_like(x)
    final = torch.empty(1, 3, 96, dtype=torch.float16, device="cuda")
    binding.im2win_causal_conv1d(x, w, whole, silu=True, state_out=final)
    for cuts in ([0, 20, 45], [0, 1, 2, 45], list(range(46))):
        y, state = torch.empty_like(x), torch.zeros(1, 3, 96, dtype=torch.float16, device="cuda")
        for s, e in zip(cuts, cuts[1:]):
            part = torch.empty(1, e - s, 96, dtype=torch.float16, device="cuda")
            binding.im2win_causal_conv1d(x[:, s:e], w, part, silu=True, state=state, state_out=state)
            y[:, s:e] = part
        assert torch.equal(y, whole) and torch.equal(state, final)


def test_captured_step_replays_on_new_values_and_slots():
    x = torch.randn(4, 64, device="cuda").bfloat16()
    w = torch.randn(64, 4, device="cuda").bfloat16()
    y = torch.zeros_like(x)
    pool = torch.randn(6, 3, 64, device="cuda").bfloat16()
    slots = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    keep = pool.clone()
    binding.im2win_causal_conv1d(x, w, y, state=pool, state_out=pool, slots=slots)
    pool.copy_(keep)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.im2win_causal_conv1d(x, w, y, state=pool, state_out=pool, slots=slots)
    for order in ([5, 2, -1, 0], [1, 4, 3, -1]):
        slots.copy_(torch.tensor(order, dtype=torch.int32))
        x.copy_(torch.randn(4, 64))
        y.zero_()
        before = pool.cpu().clone()
        graph.replay()
        want, new, a = conv1d_64(x.cpu(), w.cpu(), None, False, torch.zeros(4, 64), before, before, sequence_list([1] * 4, order), 6)
        close(y, want, 5 * 2.0 ** -24 * a + rounding(want, torch.bfloat16), "y")
        close(pool, new, torch.zeros_like(new), "pool")


def test_on_another_stream():
    stream = torch.cuda.Stream()
    x = torch.randn(2, 9, 64, device="cuda")
    w = torch.randn(64, 3, device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    binding.im2win_causal_conv1d(x, w, y)
    torch.cuda.synchronize()
    binding.im2win_causal_conv1d(x, w, z, stream=stream)
    stream.synchronize()
    assert torch.equal(y, z)


def test_row_numbers_that_break_the_rules_stay_within_the_buffers():
    """Values below zero, beyond the tokens and falling: whatever comes out, nothing outside is written (every value is clamped)."""
    for cu in ([-5, 3, 900, 20], [10, 4, 2, 1], [0, 2 ** 31 - 1, -2 ** 31, 7], [40, 40, 40, 40]):
        y = Guarded((40, 24), torch.float16)
        state = Guarded((3, 3, 24), torch.float16)
        x = torch.ones(40, 24, dtype=torch.float16, device="cuda")
        binding.im2win_causal_conv1d(x, torch.ones(24, 4, dtype=torch.float16, device="cuda"), y.view, state=state.view, state_out=state.view,
                                     cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        y.assert_untouched_outside()
        state.assert_untouched_outside()
