"""The norm, the 8-bit products, the short convolution and the gated delta rule together, as a layer of a model that is served runs them: the residual is
added and normed into 8 bits, a projection makes the rows of q, k and v, the convolution runs over them, the delta rule over its rows, its rows are normed into
8 bits and a projection brings them back.  Prompts of several sequences in one call, then generation from a captured graph with a row of padding.

Compared with the same layer in 64 bits, step by step on the layer's own 8-bit rows (which number is nearest is decided on rounded rows, and a number off
by one is no error of the next operator's).  Tolerances, as a share of each row's norm: each of convolution, delta rule and product rounds its rows to the
type (half a step each); an error of its input becomes one of its output of the same share times the condition of its sums, taken as 4
for the convolution (SiLU, and signs that cancel) and 4 for the delta rule, whose normalised q and k it moves by twice its share."""
import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import half_step

pytestmark = pytest.mark.gpu

HIDDEN, HEADS, QK, DK, DV, TAPS = 256, 4, 2, 64, 64, 4
QKV = 2 * QK * DK + HEADS * DV


class Layer:
    def __init__(self, dtype):
        g = torch.Generator().manual_seed(11)
        self.dtype = dtype
        self.into, self.back = self.matrix(QKV, HIDDEN, g), self.matrix(HIDDEN, HEADS * DV, g)
        self.before, self.behind = ((1 + 0.2 * torch.randn(n, generator=g)).to(dtype).cuda() for n in (HIDDEN, HEADS * DV))
        self.filter = (torch.rand(QKV, TAPS, generator=g) - 0.3).to(dtype).cuda()
        self.rate = (-torch.rand(HEADS, generator=g) * 0.2).cuda()
        self.beta = torch.rand(HEADS, generator=g).cuda()

    def matrix(self, n, k, g):
        return torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8).cuda(), ((torch.rand(n, generator=g) + 0.5) / (73 * k ** 0.5)).cuda()

    def projected(self, x, weight, matrix, residual=None):
        n = x.shape[0]
        rows, scales = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        total = None if residual is None else torch.empty_like(x)
        binding.im2win_rms_norm(x, weight, rows, scales=scales, residual=residual, residual_out=total)
        y = torch.empty(n, matrix[0].shape[0], dtype=self.dtype, device="cuda")
        binding.im2win_matmul_int8(rows, scales, *matrix, y)
        return rows, scales, total, y

    def heads(self, rows):
        q, k, v = rows.split([QK * DK, QK * DK, HEADS * DV], 1)
        return q.unflatten(1, (QK, DK)), k.unflatten(1, (QK, DK)), v.unflatten(1, (HEADS, DV))

    def run(self, x, residual, window, state, **sequences):
        rows, scales, total, y = self.projected(x, self.before, self.into, residual)
        mixed = torch.zeros_like(y)
        binding.im2win_causal_conv1d(y, self.filter, mixed, silu=True, state=window, state_out=window, **sequences)
        o = torch.zeros(x.shape[0], HEADS, DV, dtype=self.dtype, device="cuda")
        binding.im2win_gated_delta_rule(*self.heads(mixed), self.rate, self.beta, o, scale=DK ** -0.5, normalize=True, state=state, state_out=state,
                                        **sequences)
        rows2, scales2, _, out = self.projected(o.flatten(1), self.behind, self.back)
        return rows, scales, total, o, rows2, scales2, out

    def product(self, rows, scales, matrix):
        return rows.double() @ matrix[0].double().T * scales.double()[:, None] * matrix[1].double()

    def whole_64(self, rows, scales):
        """o of one sequence from its first row on, of the rows in 8 bits."""
        y = self.product(rows, scales, self.into)
        f = self.filter.double()
        padded = torch.cat([torch.zeros(TAPS - 1, QKV, dtype=torch.float64, device="cuda"), y])
        z = sum(padded[i:i + len(y)] * f[:, i] for i in range(TAPS))
        q, k, v = self.heads(z / (1 + torch.exp(-z)))
        q, k = ((x / (x.square().sum(2, keepdim=True) + 1e-6).sqrt()).repeat_interleave(HEADS // QK, 1) for x in (q, k))
        S, o, a = torch.zeros(HEADS, DK, DV, dtype=torch.float64, device="cuda"), [], self.rate.double().exp()[:, None, None]
        for t in range(len(y)):
            S = a * S
            S = S + k[t][:, :, None] * (self.beta.double()[:, None] * (v[t] - (k[t][:, :, None] * S).sum(1)))[:, None, :]
            o.append((q[t][:, :, None] * S).sum(1) * DK ** -0.5)
        return torch.stack(o)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lengths", [[130, 1, 70], [5, 64, 200]])
def test_prompts_then_generation(dtype, lengths):
    layer, steps, pool = Layer(dtype), 6, 5
    g = torch.Generator().manual_seed(6)
    xs, rs = ([torch.randn(n + steps, HIDDEN, generator=g).to(dtype).cuda() for n in lengths] for _ in range(2))
    slots = torch.tensor([3, 0, 4], dtype=torch.int32, device="cuda")
    window = torch.full((pool, TAPS - 1, QKV), 7.0, dtype=dtype, device="cuda")       # (left there by others)
    state = torch.full((pool, HEADS, DK, DV), 7.0, device="cuda")
    cu = torch.tensor([0, lengths[0], sum(lengths[:2]), sum(lengths)], dtype=torch.int32, device="cuda")
    fresh = torch.zeros(3, dtype=torch.bool, device="cuda")
    cut = lambda parts: torch.cat([x[:n] for x, n in zip(parts, lengths)])
    outs = layer.run(cut(xs), cut(rs), window, state, cu_seqlens=cu, slots=slots, resume=fresh)
    assert torch.equal(outs[2], (cut(xs).float() + cut(rs).float()).to(dtype))
    got = [[list(part) for part in t.split(lengths)] for t in outs]

    x, r = (torch.stack([p[n] for p, n in zip(parts, lengths)] + [torch.zeros_like(parts[0][0])]) for parts in (xs, rs))
    four = torch.cat([slots, torch.tensor([-1], dtype=torch.int32, device="cuda")])   # the batch it is captured for: one more, padding
    kept = window.clone(), state.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.run(x, r, window, state, slots=four)
    torch.cuda.current_stream().wait_stream(side)
    window.copy_(kept[0])
    state.copy_(kept[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step = layer.run(x, r, window, state, slots=four)
    for t in range(steps):
        x[:3].copy_(torch.stack([p[n + t] for p, n in zip(xs, lengths)]))
        r[:3].copy_(torch.stack([p[n + t] for p, n in zip(rs, lengths)]))
        graph.replay()
        assert not step[3][3].any() and not step[6][3].any()
        for rows, more in zip(got, step):
            for row, one in zip(rows, more[:3].clone()):
                row.append(one)
    assert bool((window[[1, 2]] == 7).all()) and bool((state[[1, 2]] == 7).all())
    half = half_step(dtype)
    tol = half * (1 + 4 * (1 + 4 * 1)) if dtype != torch.float32 else 2.0 ** -24 * 1000
    for b in range(3):
        rows, scales, _, o, rows2, scales2, out = (torch.stack(t[b]) for t in got)
        want = layer.whole_64(rows, scales).flatten(1)
        err, size = (o.double().flatten(1) - want).norm(dim=1), want.norm(dim=1)
        worst = float((err / size.clamp(min=float(size.mean()) / 10)).max())
        assert worst < tol, worst
        want = layer.product(rows2, scales2, layer.back)
        assert float(((out.double() - want).norm(dim=1) / want.norm(dim=1)).max()) < half + 2.0 ** -21
