"""im2win_linear_attention against the recurrence in 64 bits (tolerances: linear_64, and one rounding of o to its type)."""
import math

import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, Guarded, close, half_step, linear_64, rounding, sequence_list

pytestmark = pytest.mark.gpu


def run(dtype, lengths, heads, qk_heads, dk, dv, tail=0, slots=None, pool=None, resume=None, state=True, in_place=False, pitch=0, decay="tokens",
        mode="packed", max_len=0, scale=None, seed=1, edit=None, kernel=None, spread=1.0):
    """One call on guarded tensors, compared with the recurrence.  mode: packed (cu_seqlens), dense or step."""
    gen = torch.Generator().manual_seed(seed)
    tdt, rows, b = DTYPES[dtype], sum(lengths) + tail, len(lengths)
    pool = pool or b
    scale = 1 / math.sqrt(dk) if scale is None else scale
    q, k = (torch.randn(rows, qk_heads, dk, generator=gen).mul(spread).to(tdt) for _ in range(2))
    v = torch.randn(rows, heads, dv, generator=gen).to(tdt)
    rate = torch.exp(torch.rand(heads, generator=gen) * math.log(300)) * 1e-3
    g = -rate if decay == "heads" else -rate * torch.nn.functional.softplus(torch.randn(rows, heads, generator=gen))
    st = torch.randn(pool, heads, dk, dv, generator=gen) * 2 if state else None
    if edit:
        edit(q, k, v, g, st)
    qg, kg = Guarded((rows, qk_heads, dk), tdt, pitch), Guarded((rows, qk_heads, dk), tdt, 2 * pitch)
    vg, og = Guarded((rows, heads, dv), tdt, pitch), Guarded((rows, heads, dv), tdt, pitch)
    for t, x in ((qg, q), (kg, k), (vg, v)):
        t.view.copy_(x)
    o_before = og.view.cpu().clone()
    sg = ng = None
    if state:
        sg = Guarded((pool, heads, dk, dv), torch.float32)
        sg.view.copy_(st)
        ng = sg if in_place else Guarded((pool, heads, dk, dv), torch.float32)
    new_before = ng.view.cpu().clone() if state else None
    gd = g.cuda()
    if decay == "expanded":
        g = g[0].clone()
        gd = g.cuda().expand(rows, heads)
    args, views = {}, [qg.view, kg.view, vg.view, gd, og.view]
    if mode == "packed":
        cu = [0]
        for n in lengths:
            cu.append(cu[-1] + n)
        args["cu_seqlens"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    elif mode == "dense":
        views = [t if t.dim() == 1 else t.unflatten(0, (b, lengths[0])) for t in views]
    if slots is not None:
        args["slots"] = torch.tensor(slots, dtype=torch.int32, device="cuda")
    if resume is not None:
        args["resume"] = torch.tensor(resume, dtype=torch.bool, device="cuda")
    if state:
        args.update(state=sg.view, state_out=ng.view)
    shape = binding.make_attention_shape(rows, b, heads, qk_heads, dk, dv, max_len)
    if kernel:
        assert binding.im2win_linear_attention_kernel_name(shape, binding._sequence_dtype(tdt)) == kernel
    need = binding.im2win_linear_attention_workspace_size(shape, binding._sequence_dtype(tdt))
    ws = Guarded((need,), torch.uint8, fill=0x5a)
    binding.im2win_linear_attention(*views, ws.view, scale=scale, max_len=max_len, **args)
    binding.im2win_check_status(ws.view)
    bound_pool = pool if state or slots is None else 1 << 31
    o, off, new, new_off = linear_64(q, k, v, g, scale, o_before, st, new_before, sequence_list(lengths, slots, resume), bound_pool,
                                     0.0 if dtype == "f32" else half_step(tdt))
    # By chunks an infinity of v meets q . k, one number: it comes out as an infinity.  In the recurrence it meets each element of k and then
    # of q, infinities of both signs, whose sum is a NaN.  Both are right readings of the formula; o is not finite in the same places.
    close(og.view, o, off + rounding(o, tdt), "o", same_infinities=dtype == "f32")
    for t in (og, ws):
        t.assert_untouched_outside()
    if state:
        close(ng.view, new, new_off, "state_out")
        ng.assert_untouched_outside()
    return og.view


LENGTHS = [5, 0, 1, 70, 2, 33, 0, 130, 64, 65]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (64, 128), (16, 32), (1, 1), (7, 33), (80, 96), (100, 41), (200, 36)])
def test_packed_sequences_of_every_kind(dtype, dk, dv):
    run(dtype, LENGTHS, 2, 1, dk, dv, tail=3, resume=[1, 0, 1, 0, 1, 1, 1, 0, 1, 0])


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


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("segments", [1, 2, 3, 7])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (37, 51), (128, 200)])
def test_sequences_in_segments(dtype, segments, dk, dv, monkeypatch):
    """Long sequences cut into any number of segments, beside short and empty ones, their states in place."""
    monkeypatch.setenv("IM2WIN_SEGMENTS", str(segments))
    run(dtype, [460, 3, 0, 200, 64, 129], 2, 1, dk, dv, tail=5, resume=[1, 1, 0, 0, 1, 1], in_place=True, slots=[3, 1, 0, 7, 2, 5], pool=8,
        kernel="chunks" if segments == 1 else "chunks+segments")
    run(dtype, [300, 300], 1, 1, dk, dv, mode="dense", decay="heads")


def test_a_decay_that_empties_the_state_in_the_middle_of_segments(monkeypatch):
    monkeypatch.setenv("IM2WIN_SEGMENTS", "4")
    def edit(q, k, v, g, st):
        g[100] = -math.inf
        g[64 * 4 + 5] = -500.0
        g[300:310] = -60.0
    for dtype in ("f16", "bf16"):
        run(dtype, [512], 2, 2, 64, 64, edit=edit)


def test_large_and_small_values_in_fp16():
    """States beyond the type's range and far below its smallest normal number."""
    def large(q, k, v, g, st):
        k.mul_(200)
        v.mul_(300)
        q.mul_(1e-2)
        st.mul_(1e6)
        g.mul_(0.1)
    def small(q, k, v, g, st):
        k.mul_(1e-3)
        v.mul_(1e-3)
        st.mul_(1e-7)
        q.mul_(100)
    run("f16", [150, 40], 2, 2, 64, 64, edit=large, scale=1e-6)
    run("f16", [150, 40], 2, 2, 64, 64, edit=small, scale=1e3)


def test_empty_calls_move_states():
    run("bf16", [0, 0, 0], 2, 2, 64, 64, resume=[1, 0, 1])
    run("f32", [0, 0], 1, 1, 64, 64, mode="dense")


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_decays_of_every_size(dtype):
    """No decay, one that empties the state (minus infinity, the type's lowest value), very strong and very weak ones, growth."""
    def edit(q, k, v, g, st):
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
@pytest.mark.parametrize("which", ["v", "k", "q"])
def test_values_stay_within_their_sequence_and_behind_their_row(dtype, which):
    """Infinities and NaNs of a row, of rows behind the last sequence and of states that are not resumed meet no other row before them."""
    def edit(q, k, v, g, st):
        x = {"q": q, "k": k, "v": v}[which]
        x[70, 0, 3] = math.inf
        x[75, 1, 1] = math.nan
        x[-2:] = math.nan
        st[0] = math.nan
        st[2] = math.inf
        st[2, 1] = math.nan
    run(dtype, [10, 100, 0, 30], 2, 2, 64, 64, tail=2, resume=[0, 1, 0, 1], edit=edit)


def test_long_memory_stays_exact():
    """A decay so near 1 that an error of exp in its last place, made at every token, would add up to more than the tolerance here."""
    def edit(q, k, v, g, st):
        g.fill_(-1.3e-4)
    run("f32", [1500], 1, 1, 16, 32, edit=edit, decay="heads")


def test_prompt_and_single_tokens_agree():
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(1, 70, 2, 64, generator=gen, device="cuda") for _ in range(3))
    g = -torch.rand(1, 70, 2, generator=gen, device="cuda")
    ws = binding.alloc_attention_workspace(binding.make_attention_shape(70, 1, 2, 2, 64, 64), torch.float32)
    whole, final = torch.empty_like(v), torch.empty(1, 2, 64, 64, device="cuda")
    binding.im2win_linear_attention(q, k, v, g, whole, ws, state_out=final)
    o, state = torch.empty_like(v), torch.zeros(1, 2, 64, 64, device="cuda")
    for t in range(70):
        part = torch.empty(1, 1, 2, 64, device="cuda")
        binding.im2win_linear_attention(q[:, t:t + 1], k[:, t:t + 1], v[:, t:t + 1], g[:, t:t + 1], part, ws, state=state, state_out=state)
        o[:, t:t + 1] = part
    assert float((o - whole).norm() / whole.norm()) < 70 * 2.0 ** -24 and float((state - final).norm() / final.norm()) < 70 * 2.0 ** -24


def test_captured_step_replays_on_new_values_and_slots():
    q, k, v = (torch.randn(4, 2, 64, device="cuda").bfloat16() for _ in range(3))
    g = -torch.rand(4, 2, device="cuda")
    o, pool = torch.zeros_like(v), torch.randn(6, 2, 64, 64, device="cuda")
    slots = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    ws = binding.alloc_attention_workspace(binding.make_attention_shape(4, 4, 2, 2, 64, 64), torch.bfloat16)
    call = lambda: binding.im2win_linear_attention(q, k, v, g, o, ws, state=pool, state_out=pool, slots=slots)
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
        want, off, new, new_off = linear_64(q.cpu(), k.cpu(), v.cpu(), g.cpu(), 1.0, torch.zeros(4, 2, 64), before, before,
                                            sequence_list([1] * 4, order), 6)
        close(o, want, off + rounding(want, torch.bfloat16), "o")
        close(pool, new, new_off, "pool")


def test_the_same_call_gives_the_same_bits():
    a = run("bf16", LENGTHS, 3, 3, 64, 64).clone()
    assert torch.equal(a, run("bf16", LENGTHS, 3, 3, 64, 64))


def test_row_numbers_that_break_the_rules_stay_within_the_buffers():
    for cu in ([-5, 3, 900, 20], [10, 4, 2, 1], [0, 2 ** 31 - 1, -2 ** 31, 7], [300, 300, 300, 300]):
        for max_len in (0, 1):
            o = Guarded((300, 2, 64), torch.float16)
            state = Guarded((3, 2, 64, 64), torch.float32)
            x = torch.ones(300, 2, 64, dtype=torch.float16, device="cuda")
            shape = binding.make_attention_shape(300, 3, 2, 2, 64, 64, max_len)
            ws = Guarded((binding.im2win_linear_attention_workspace_size(shape, binding.F16),), torch.uint8, fill=0x5a)
            binding.im2win_linear_attention(x, x, x, torch.zeros(2, device="cuda"), o.view, ws.view, state=state.view, state_out=state.view,
                                            cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda"), max_len=max_len)
            torch.cuda.synchronize()
            for t in (o, state, ws):
                t.assert_untouched_outside()
