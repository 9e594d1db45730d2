"""The operators on token sequences together, as a layer of a model that is served runs them: a 4-bit projection makes the rows of q, k
and v, the short convolution runs over them, linear attention over its rows, and a 4-bit projection brings them back.  Prompts of
several sequences in one call, then generation, a token of each at a time, replayed from a captured graph with some of them padding.

Compared with the same layer in 64 bits; tolerance, as a share of each row's norm: every operator rounds its rows to the type (half a
step each, four times, and one inside attention by chunks), and each of the later ones turns an error of its input into one of its output of the
same share, times the condition of its sums, taken as 4 for projections and 2 for attention here (uniform random signs: their square
root, as a rule)."""
import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import half_step

pytestmark = pytest.mark.gpu

HIDDEN, HEADS, DK, DV, TAPS, GROUP = 256, 4, 64, 64, 4, 64
QKV = 2 * HEADS * DK + HEADS * DV


class Layer:
    def __init__(self, dtype, seed):
        g = torch.Generator().manual_seed(seed)
        self.dtype = dtype
        self.into = self.matrix(QKV, HIDDEN, g)
        self.back = self.matrix(HIDDEN, HEADS * DV, g)
        self.filter = (torch.rand(QKV, TAPS, generator=g) - 0.3).to(dtype).cuda()
        self.rate = (-torch.rand(HEADS, generator=g) * 0.2).cuda()

    def matrix(self, n, k, g):
        w = torch.randint(0, 256, (n, k // 2), generator=g, dtype=torch.uint8).cuda()
        s = ((torch.rand(n, k // GROUP, generator=g) + 0.5) * 0.3 / k ** 0.5).to(self.dtype).cuda()
        return w, s

    def project(self, x, matrix):
        y = torch.empty(x.shape[0], matrix[0].shape[0], dtype=self.dtype, device="cuda")
        for i in range(0, x.shape[0], 16):              # (sixteen rows a call)
            binding.im2win_matvec_int4(x[i:i + 16], *matrix, y[i:i + 16], GROUP)
        return y

    def heads(self, rows):
        q, k, v = rows.split([HEADS * DK, HEADS * DK, HEADS * DV], 1)
        return q.unflatten(1, (HEADS, DK)), k.unflatten(1, (HEADS, DK)), v.unflatten(1, (HEADS, DV))

    def run(self, x, window, state, workspace, **sequences):
        rows = self.project(x, self.into)
        mixed = torch.zeros_like(rows)
        binding.im2win_causal_conv1d(rows, self.filter, mixed, silu=True, state=window, state_out=window, **sequences)
        o = torch.zeros(x.shape[0], HEADS, DV, dtype=self.dtype, device="cuda")
        binding.im2win_linear_attention(*self.heads(mixed), self.rate, o, workspace, scale=DK ** -0.5, state=state, state_out=state, **sequences)
        return self.project(o.flatten(1), self.back)

    def whole_64(self, x):
        """One sequence from its first row on."""
        def dense(w, s):
            w = torch.stack([w & 15, w >> 4], 2).flatten(1).double().cpu() - 8
            return w * s.double().cpu().repeat_interleave(GROUP, 1)
        rows = x.double().cpu() @ dense(*self.into).T
        f = self.filter.double().cpu()
        padded = torch.cat([torch.zeros(TAPS - 1, QKV, dtype=torch.float64), rows])
        z = sum(padded[i:i + len(x)] * f[:, i] for i in range(TAPS))
        q, k, v = self.heads(z / (1 + torch.exp(-z)))
        S, o, decay = torch.zeros(HEADS, DK, DV, dtype=torch.float64), [], self.rate.double().cpu().exp()[:, None, None]
        for t in range(len(x)):
            S = decay * S + k[t][:, :, None] * v[t][:, None, :]
            o.append((q[t][:, :, None] * S).sum(1) * DK ** -0.5)
        return torch.stack(o).flatten(1) @ dense(*self.back).T


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lengths", [[130, 1, 70], [5, 64, 200]])
def test_prompts_then_generation(dtype, lengths):
    layer, steps, pool = Layer(dtype, 5), 6, 5
    g = torch.Generator().manual_seed(6)
    xs = [torch.randn(n + steps, HIDDEN, generator=g).to(dtype).cuda() for n in lengths]
    want = [layer.whole_64(x) for x in xs]
    slots = torch.tensor([3, 0, 4], dtype=torch.int32, device="cuda")
    window = torch.full((pool, TAPS - 1, QKV), 7.0, dtype=dtype, device="cuda")       # (left there by others)
    state = torch.full((pool, HEADS, DK, DV), 7.0, device="cuda")
    cu = torch.tensor([0, lengths[0], sum(lengths[:2]), sum(lengths)], dtype=torch.int32, device="cuda")
    workspace = binding.alloc_attention_workspace(binding.make_attention_shape(sum(lengths), 3, HEADS, HEADS, DK, DV), dtype)
    fresh = torch.zeros(3, dtype=torch.bool, device="cuda")
    y = layer.run(torch.cat([x[:n] for x, n in zip(xs, lengths)]), window, state, workspace, cu_seqlens=cu, slots=slots, resume=fresh)
    binding.im2win_check_status(workspace)
    got = [list(part) for part in y.split(lengths)]

    x = torch.stack([x[n] for x, n in zip(xs, lengths)] + [torch.zeros_like(xs[0][0])])
    four = torch.cat([slots, torch.tensor([-1], dtype=torch.int32, device="cuda")])   # the batch it is captured for: one more, padding
    step_ws = binding.alloc_attention_workspace(binding.make_attention_shape(4, 4, HEADS, HEADS, DK, DV, 1), dtype)
    kept = window.clone(), state.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.run(x, window, state, step_ws, slots=four)
    torch.cuda.current_stream().wait_stream(side)
    window.copy_(kept[0])
    state.copy_(kept[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.run(x, window, state, step_ws, slots=four)
    for t in range(steps):
        x[:3].copy_(torch.stack([x[n + t] for x, n in zip(xs, lengths)]))
        graph.replay()
        assert not out[3].any()
        for rows, row in zip(got, out[:3].clone()):
            rows.append(row)
    assert bool((window[[1, 2]] == 7).all()) and bool((state[[1, 2]] == 7).all())
    tol = half_step(dtype) * (1 + 4 * (1 + 2 * (1 + 1 + 2 * (1 + 1)))) if dtype != torch.float32 else 2.0 ** -24 * 1000
    for rows, ref in zip(got, want):
        err = torch.stack(rows).double().cpu() - ref
        scale = ref.norm(dim=1).clamp(min=float(ref.norm(dim=1).mean()) / 10)
        assert float((err.norm(dim=1) / scale).max()) < tol, float((err.norm(dim=1) / scale).max())


def test_captured_prompt_in_segments(monkeypatch):
    """A prompt by chunks and segments, captured; replayed on new rows it gives what the call gives."""
    monkeypatch.setenv("IM2WIN_SEGMENTS", "3")
    make = lambda: torch.randn(400, 2, 64, device="cuda").bfloat16()
    q, k, v = make(), make(), make()
    g, cu = -torch.rand(400, 2, device="cuda") * 0.1, torch.tensor([0, 390], dtype=torch.int32, device="cuda")
    shape = binding.make_attention_shape(400, 1, 2, 2, 64, 64)
    ws = [binding.alloc_attention_workspace(shape, torch.bfloat16) for _ in range(2)]
    o, other = torch.zeros_like(v), torch.zeros_like(v)
    call = lambda out, w: binding.im2win_linear_attention(q, k, v, g, out, w, cu_seqlens=cu)
    call(o, ws[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(o, ws[0])
    for _ in range(2):
        for t in (q, k, v):
            t.copy_(make())
        graph.replay()
        call(other, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(o, other) and not o[390:].any() and o[:390].any()
