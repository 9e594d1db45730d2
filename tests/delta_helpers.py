"""The gated delta rule in 64 bits on the CPU, and one call of it on guarded tensors."""
import math

import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import DTYPES, Guarded, close, half_step, rounding, sequence_list

EPS = 1e-6


def delta_64(q, k, v, g, beta, scale, normalize, o, state, state_out, sequences, pool, products_off=0.0):
    """The recurrence, token by token; o and state_out: what lay there before.  Also returns how far results may be off.  With |.| the norm
    over dk of a column of the state, m = a |S| + |k| beta (|v| + |k| a |S|) what passes through a token's sums, and c = 2^-24 (8 + sqrt(dk + 64))
    what rounding sums of dk terms, and of 64 tokens, puts it off by (independent roundings of running sums, and eight more):
      the state   E^2 <- (a max(1, |1 - beta k k|))^2 E^2 + (c m)^2 adds these up as independent errors, which the rule does not let grow;
                  the norm of a column's error stays below 4 E
      o           |scale| |q| (4 E + c |S| + products_off Z): Z <- a Z + |k| |u| bounds the terms that enter the 16-bit products, products_off
                  is their rounding"""
    q, k, v, g, beta = (x.double() for x in (q, k, v, g, beta))
    if normalize:
        q, k = (x / (x.square().sum(-1, keepdim=True) + EPS).sqrt() for x in (q, k))
    h, dk, dv = v.shape[1], q.shape[2], v.shape[2]
    of = torch.arange(h) // (h // q.shape[1])
    c = 2.0 ** -24 * (8 + math.sqrt(dk + 64))
    o, o_off = o.double().clone(), torch.zeros_like(o, dtype=torch.float64)
    new, new_off = (None, None) if state_out is None else (state_out.double().clone(), torch.zeros(*state_out.shape[:2], dv, dtype=torch.float64))
    for first, n, slot, resumes in sequences:
        if not 0 <= slot < pool:
            continue
        S = state[slot].double().clone() if state is not None and resumes else torch.zeros(h, dk, dv, dtype=torch.float64)
        E, Z = torch.zeros(h, dv, dtype=torch.float64), S.norm(dim=1)
        for t in range(first, first + n):
            a = torch.exp(g if g.dim() == 1 else g[t])[:, None]
            bt = (beta if beta.dim() == 1 else beta[t])[:, None]
            kk, qq = k[t][of], q[t][of]
            old = a[:, :, None] * S
            size, kn, qn = old.norm(dim=1), kk.norm(dim=1)[:, None], qq.norm(dim=1)[:, None]
            u = bt * (v[t] - (kk[:, :, None] * old).sum(1))
            S = old + kk[:, :, None] * u[:, None, :]
            m = size + kn * bt.abs() * (v[t].abs() + kn * size)
            E = ((a * (1 - bt * kn * kn).abs().clamp(min=1.0) * E).square() + (c * m).square()).sqrt()
            Z = a * Z + kn * u.abs()
            o[t] = scale * (qq[:, :, None] * S).sum(1)
            o_off[t] = abs(scale) * qn * (4 * E + c * (S.norm(dim=1) + m) + products_off * Z)
        if new is not None:
            new[slot], new_off[slot] = S, 4 * E + 2.0 ** -140
    return o, o_off, new, new_off


def close_columns(got, want, bound, what):
    """The norm over dk of every column's error within bound; not finite where want is not."""
    got = got.double().cpu()
    fine = torch.isfinite(want).all(2)
    assert torch.equal(torch.isfinite(got).all(2), fine), f"{what}: finite elsewhere"
    err = torch.where(fine[:, :, None], got - want, 0.0).norm(dim=2)
    over = (err > bound) & fine
    assert not bool(over.any()), f"{what}: {int(over.sum())} of {over.numel()} columns off, the largest error {float(err.max()):.3g}"


def run(dtype, lengths, heads, qk_heads, dk, dv, tail=0, slots=None, pool=None, resume=None, state=True, in_place=False, pitch=0, decay="tokens",
        mode="packed", max_len=0, scale=None, seed=1, edit=None, kernel=None, normalize=True, spread=1.0):
    """One call on guarded tensors, compared with the recurrence.  mode: packed (cu_seqlens), dense or step."""
    gen = torch.Generator().manual_seed(seed)
    tdt, rows, b = DTYPES[dtype], sum(lengths) + tail, len(lengths)
    pool = pool or b
    scale = 1 / math.sqrt(dk) if scale is None else scale
    q, k = (torch.randn(rows, qk_heads, dk, generator=gen).mul(spread) for _ in range(2))
    if not normalize:
        q, k = (x / x.norm(dim=2, keepdim=True).clamp(min=1e-30) for x in (q, k))
    q, k = q.to(tdt), k.to(tdt)
    v = torch.randn(rows, heads, dv, generator=gen).to(tdt)
    rate = torch.exp(torch.rand(heads, generator=gen) * math.log(300)) * 1e-3
    g = -rate if decay == "heads" else -rate * torch.nn.functional.softplus(torch.randn(rows, heads, generator=gen))
    beta = torch.sigmoid(torch.randn(heads, generator=gen) if decay == "heads" else torch.randn(rows, heads, generator=gen))
    st = torch.randn(pool, heads, dk, dv, generator=gen) * 0.5 if state else None
    if edit:
        edit(q, k, v, g, beta, st)
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
    gd, bd = g.cuda(), beta.cuda()
    if decay == "expanded":
        g, beta = g[0].clone(), beta[0].clone()
        gd, bd = g.cuda().expand(rows, heads), beta.cuda().expand(rows, heads)
    args, views = {}, [qg.view, kg.view, vg.view, gd, bd, og.view]
    if mode == "packed":
        args["cu_seqlens"] = torch.tensor([sum(lengths[:i]) for i in range(b + 1)], dtype=torch.int32, device="cuda")
    elif mode == "dense":
        views = [t if t.dim() == 1 else t.unflatten(0, (b, lengths[0])) for t in views]
    if slots is not None:
        args["slots"] = torch.tensor(slots, dtype=torch.int32, device="cuda")
    if resume is not None:
        args["resume"] = torch.tensor(resume, dtype=torch.bool, device="cuda")
    if state:
        args.update(state=sg.view, state_out=ng.view)
    if kernel:
        shape = binding.make_delta_shape(rows, b, heads, qk_heads, dk, dv, max_len)
        assert binding.im2win_gated_delta_rule_kernel_name(shape, binding._sequence_dtype(tdt)) == kernel
    binding.im2win_gated_delta_rule(*views, scale=scale, normalize=normalize, max_len=max_len, **args)
    torch.cuda.synchronize()
    bound_pool = pool if state or slots is None else 1 << 31
    o, off, new, new_off = delta_64(q, k, v, g, beta, scale, normalize, o_before, st, new_before, sequence_list(lengths, slots, resume),
                                    bound_pool, 0.0 if dtype == "f32" else 2 * half_step(torch.float16))
    close(og.view, o, off + rounding(o, tdt), "o", same_infinities=False)
    og.assert_untouched_outside()
    if state:
        close_columns(ng.view, new, new_off, "state_out")
        ng.assert_untouched_outside()
    return og.view
