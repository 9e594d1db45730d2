"""Calls of the operators on token sequences that their documentation allows, each for itself: streams, calls at once, states on one side
only, strides of one tensor only, very many sequences, values that are no numbers among the decays."""
import math

import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, close, half_step, linear_64, matvec_64, rounding, sequence_list
from test_gpu_linear_attention import run

pytestmark = pytest.mark.gpu


class Call:
    """One call of linear attention on packed sequences, and what it has to give."""

    def __init__(self, dtype, lengths, heads, dk, dv, seed, state=True):
        gen = torch.Generator().manual_seed(seed)
        self.dtype, self.lengths, self.tdt, rows, b = dtype, lengths, DTYPES[dtype], sum(lengths), len(lengths)
        q, k = (torch.randn(rows, heads, dk, generator=gen).to(self.tdt) for _ in range(2))
        v = torch.randn(rows, heads, dv, generator=gen).to(self.tdt)
        g = -0.3 * torch.rand(rows, heads, generator=gen)
        st = torch.randn(b, heads, dk, dv, generator=gen) if state else None
        self.cpu = q, k, v, g, st
        self.gpu = [None if t is None else t.cuda() for t in self.cpu]
        self.cu = torch.tensor([sum(lengths[:i]) for i in range(b + 1)], dtype=torch.int32, device="cuda")
        self.o = torch.zeros(rows, heads, dv, dtype=self.tdt, device="cuda")
        self.new = torch.zeros(b, heads, dk, dv, device="cuda")
        self.ws = binding.alloc_attention_workspace(binding.make_attention_shape(rows, b, heads, heads, dk, dv), self.tdt)

    def __call__(self, stream=None, o=None, state_out=True, **changed):
        q, k, v, g, st = self.gpu
        args = dict(q=q, k=k, v=v, log_decay=g)
        args.update(changed)
        binding.im2win_linear_attention(args["q"], args["k"], args["v"], args["log_decay"], self.o if o is None else o, self.ws, scale=0.1,
                                        state=st, state_out=self.new if state_out else None, cu_seqlens=self.cu, stream=stream)

    def check(self, o=None, state_out=True):
        q, k, v, g, st = self.cpu
        products_off = 0.0 if self.dtype == "f32" else half_step(self.tdt)
        ref, off, new, new_off = linear_64(q, k, v, g, 0.1, torch.zeros(v.shape), st, torch.zeros(self.new.shape), sequence_list(self.lengths),
                                           len(self.lengths), products_off)
        close(self.o if o is None else o, ref, off + rounding(ref, self.tdt), "o")
        if state_out:
            close(self.new, new, new_off, "state_out")


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_states_on_one_side_only(dtype):
    for state, state_out in ((False, True), (True, False)):
        call = Call(dtype, [70, 0, 1, 33], 2, 64, 64, 5, state=state)
        call(state_out=state_out)
        call.check(state_out=state_out)
        assert state_out or not call.new.any()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("which", ["q", "k", "v", "o", "log_decay"])
def test_one_tensor_whose_rows_start_anywhere(dtype, which):
    """The others' rows lie on 16-byte boundaries."""
    call = Call(dtype, [200, 64, 3], 2, 64, 128, 6)
    shape = call.o.shape if which == "o" else dict(zip(("q", "k", "v", "log_decay"), call.gpu))[which].shape
    width = math.prod(shape[1:])
    wide = torch.zeros(shape[0], width + 3, dtype=torch.float32 if which == "log_decay" else call.tdt, device="cuda")
    view = wide[:, 1:1 + width].unflatten(1, shape[1:])
    if which == "o":
        call(o=view)
        call.check(o=view)
        assert not wide[:, 0].any() and not wide[:, 1 + width:].any()
    else:
        view.copy_(dict(zip(("q", "k", "v", "log_decay"), call.gpu))[which])
        call(**{which: view})
        call.check()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_two_calls_at_once(dtype):
    """Each on a stream of its own, with its own workspace, more than once, while the others' run."""
    calls = [Call(dtype, [300, 100], 2, 64, 64, 7), Call(dtype, [17, 200, 64], 3, 128, 100, 8)]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(3):
        for call, stream in zip(calls, streams):
            call(stream=stream)
    torch.cuda.synchronize()
    for call in calls:
        call.check()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_products_on_streams_of_their_own(dtype):
    tdt, gen = DTYPES[dtype], torch.Generator().manual_seed(9)
    done = []
    streams = [torch.cuda.Stream() for _ in range(2)]
    for k in (1024, 1000):
        x, w = torch.randn(5, k, generator=gen).to(tdt), torch.randint(0, 256, (700, k // 2), generator=gen, dtype=torch.uint8)
        s = (torch.rand(700, -(-k // 64), generator=gen) * 0.1).to(tdt)
        done.append(([t.cuda() for t in (x, w, s)], torch.zeros(5, 700, dtype=tdt, device="cuda"), matvec_64(x, w, s, None, None, 64), k))
    torch.cuda.synchronize()
    for _ in range(3):
        for (t, y, _, _), stream in zip(done, streams):
            binding.im2win_matvec_int4(*t, y, 64, stream=stream)
    torch.cuda.synchronize()
    for _, y, (want, a), k in done:
        close(y, want, (k / 8 + 16 + k / 64 + 1) * 2.0 ** -23 * a + rounding(want, tdt), "y")


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_more_sequences_than_a_block_has_threads(dtype):
    run(dtype, [(7 * i) % 40 if i % 3 else i % 2 for i in range(1500)], 1, 1, 16, 8, tail=1, resume=[i % 5 != 0 for i in range(1500)])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("segments", [1, 3])
def test_a_decay_that_is_no_number_reaches_no_row_before_it(dtype, segments, monkeypatch):
    monkeypatch.setenv("IM2WIN_SEGMENTS", str(segments))
    def edit(q, k, v, g, st):
        g[100, 0] = math.nan
        g[320, 1] = math.nan
    run(dtype, [200, 256], 2, 1, 64, 64, edit=edit)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("scale", [0.0, -3.0, 1e-4])
def test_scales_of_every_kind(dtype, scale):
    run(dtype, [100, 20], 2, 2, 64, 64, scale=scale)


def test_captured_on_two_streams_and_replayed_together():
    """Two graphs, each with its own workspace, replayed at the same time."""
    calls = [Call("bf16", [300], 2, 64, 64, 10), Call("f16", [300, 90], 2, 128, 64, 11)]
    graphs, streams = [], [torch.cuda.Stream() for _ in calls]
    for call in calls:
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
        call.o.zero_()
        call.new.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for call in calls:
        call.check()
    del graphs


def test_elements_of_fp32_rows_near_the_smallest():
    """Products of fp32 rows are exact to 2^-133 of x for each of the 15 (w - z) at most (the smallest bf16), beside the sums' roundings."""
    gen = torch.Generator().manual_seed(12)
    x = torch.randn(4, 512, generator=gen) * torch.tensor([[2.0 ** -100], [2.0 ** -115], [2.0 ** -125], [2.0 ** -140]])
    w = torch.randint(0, 256, (40, 256), generator=gen, dtype=torch.uint8)
    s = torch.full((40, 4), 2.0 ** 100)
    y = torch.empty(4, 40, device="cuda")
    binding.im2win_matvec_int4(x.cuda(), w.cuda(), s.cuda(), y, 128)
    want, a = matvec_64(x, w, s, None, None, 128)
    close(y, want, (512 / 8 + 16 + 4) * 2.0 ** -23 * a + 512 * 15 * 2.0 ** -133 * 2.0 ** 100 + rounding(want, torch.float32), "y")
