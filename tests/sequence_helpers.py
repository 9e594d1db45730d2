"""Plain implementations, in 64 bits on the CPU, of the operators on token sequences, and what their tests share."""
import math

import torch

from gpu_helpers import GUARD

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def half_step(dtype):
    """The largest relative error of one rounding to nearest."""
    return torch.finfo(dtype).eps / 2


def rounding(y, dtype):
    """The largest error of rounding y (float64) once to dtype: relative, or half a subnormal step."""
    info = torch.finfo(dtype)
    return y.abs() * half_step(dtype) + info.tiny * info.eps / 2


def sequence_list(lengths, slots=None, resume=None):
    """(first row, length, slot or None for padding, whether it resumes) of each sequence."""
    at, out = 0, []
    for b, n in enumerate(lengths):
        slot = b if slots is None else slots[b]
        out.append((at, n, slot, True if resume is None else bool(resume[b])))
        at += n
    return out


def conv1d_64(x, weight, bias, silu, y, state, state_out, sequences, pool):
    """The definition, row by row; y and state_out: what lay there before.  Also returns the sums of magnitudes that bound fp32 sums."""
    x, w = x.double(), weight.double()
    y, bound = y.double().clone(), torch.zeros_like(y, dtype=torch.float64)
    state_out = None if state_out is None else state_out.double().clone()
    taps = w.shape[1]
    for first, n, slot, resumes in sequences:
        if not 0 <= slot < pool:
            continue
        old = state[slot].double() if state is not None and resumes else torch.zeros(taps - 1, x.shape[1], dtype=torch.float64)
        whole = torch.cat([old, x[first:first + n]])
        for t in range(n):
            window = whole[t:t + taps]
            z = (window * w.T).sum(0)
            a = (window.abs() * w.T.abs()).sum(0)
            if bias is not None:
                z, a = z + bias.double(), a + bias.double().abs()
            y[first + t] = z / (1 + torch.exp(-z)) if silu else z
            bound[first + t] = a
        if state_out is not None and taps > 1:
            state_out[slot] = whole[n:]
    return y, state_out, bound


class Guarded:
    """A device tensor with canaries before and behind it (values that no kernel computes), and rows as far apart as wanted."""

    def __init__(self, shape, dtype, pitch=0, fill=-77.0, shift=0):
        width = math.prod(shape[1:])
        self.shape, self.fill, self.shift = shape, fill, shift
        self.pitch = width + pitch
        self.whole = torch.full((2 * GUARD + shift + shape[0] * self.pitch,), fill, dtype=dtype, device="cuda")
        inner = [1]
        for n in reversed(shape[2:]):
            inner.insert(0, inner[0] * n)
        self.view = self.whole.as_strided(shape, [self.pitch] + inner if len(shape) > 1 else [1], GUARD + shift)

    def assert_untouched_outside(self):
        whole = self.whole.clone()
        whole.as_strided(self.view.shape, self.view.stride(), GUARD + self.shift).fill_(self.fill)
        assert bool((whole == self.fill).all()), "written outside the tensor"


def close(got, want, bound, what, same_infinities=True):
    """got within bound of want, element by element; NaN and infinities where want has them (without same_infinities: one or the other)."""
    got, want = got.double().cpu(), want.cpu()
    fine = torch.isfinite(want)
    if not same_infinities:
        assert torch.equal(torch.isfinite(got), fine), f"{what}: finite elsewhere"
        got, want = got.where(fine, 0.0), want.where(fine, 0.0)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaNs elsewhere"
    rest = ~fine & ~torch.isnan(want)
    assert torch.equal(got[rest], want[rest]), f"{what}: infinities elsewhere"
    err = (got - want).abs()[fine]
    over = err > bound.cpu()[fine]
    assert not bool(over.any()), f"{what}: {int(over.sum())} of {over.numel()} off, the largest error {float(err.max()):.3g}"


def linear_64(q, k, v, g, scale, o, state, state_out, sequences, pool, products_off=0.0):
    """The recurrence, token by token; o and state_out: what lay there before.  Also returns how far results may be off:
      the state   E <- exp(g) E + 8 * 2^-24 A with A <- exp(g) A + |k|^T |v|: eight roundings of a token's sums (the recurrence makes three)
      o           |scale| |q| (E + products_off A + (dk + 128) 2^-23 A): the sum over dk (and 128 terms of a chunk more, each cut off instead of
                  rounded) on top; products_off: the rounding of what enters the 16-bit products (a term's weight, an element of the state)"""
    q, k, v, g = q.double(), k.double(), v.double(), g.double()
    h, dk, dv = v.shape[1], q.shape[2], v.shape[2]
    of = torch.arange(h) // (h // q.shape[1])
    o, o_off = o.double().clone(), torch.zeros_like(o, dtype=torch.float64)
    new, new_off = (None, None) if state_out is None else (state_out.double().clone(), torch.zeros_like(state_out, dtype=torch.float64))
    for first, n, slot, resumes in sequences:
        if not 0 <= slot < pool:
            continue
        S = state[slot].double().clone() if state is not None and resumes else torch.zeros(h, dk, dv, dtype=torch.float64)
        A, E = S.abs(), torch.zeros_like(S)
        for t in range(first, first + n):
            a = torch.exp(g if g.dim() == 1 else g[t])[:, None, None]
            kk, qq = k[t][of], q[t][of]
            S = a * S + kk[:, :, None] * v[t][:, None, :]
            A = a * A + kk.abs()[:, :, None] * v[t].abs()[:, None, :]
            E = a * E + 8 * 2.0 ** -24 * A
            o[t] = scale * (qq[:, :, None] * S).sum(1)
            o_off[t] = abs(scale) * (qq.abs()[:, :, None] * (E + (products_off + (dk + 128) * 2.0 ** -23) * A)).sum(1)
        if new is not None:
            new[slot], new_off[slot] = S, E + 2.0 ** -149
    return o, o_off, new, new_off


def matvec_64(x, weight, scales, zeros, bias, group):
    """The definition, and the sum of the magnitudes of its terms."""
    x, k = x.double(), x.shape[1]
    w = torch.stack([weight & 15, weight >> 4], 2).flatten(1)[:, :k].double()
    of = torch.arange(k) // group
    w = (w - (8.0 if zeros is None else (zeros & 15).double()[:, of])) * scales.double()[:, of]
    y, a = x @ w.T, x.abs() @ w.abs().T
    return (y, a) if bias is None else (y + bias.double(), a + bias.double().abs())
