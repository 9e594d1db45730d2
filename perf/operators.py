"""The operators on token sequences that the library's speed is measured on, each case the way a program that serves a model calls it.

``conv``    im2win_causal_conv1d: depthwise causal convolution of packed sequences, its window carried from call to call
``linear``  im2win_linear_attention: S = exp(g) S + k^T v, o = scale q S for each head, S carried from call to call
``matvec``  im2win_matvec_int4: a few rows times a matrix of 4-bit weights with a scale (and a zero point) for each group

A case of the first two has ``tokens`` in ``sequences``: ``step`` one token a sequence (the decoding loop), ``packed`` ragged
sequences one behind the other, some of them empty or of one token, with ``tail`` allocated rows behind the last (left as they are).
``spare`` more states than sequences lie in the pool and the sequences take them in any order; ``padded`` of the step's sequences are
padding (slot -1: nothing of theirs is read or written).  Of packed sequences every third starts afresh, the others resume.

Each pass reads its states from one pool and writes them to another, so that every pass of a case does the same.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_CHUNK = 64


def _conv(name, form, dtype, tokens, sequences, channels, taps, **options):
    c = {"name": name, "op": "conv", "form": form, "dtype": dtype, "tokens": tokens, "sequences": sequences, "channels": channels,
         "taps": taps, "bias": True, "silu": True, "tail": 0, "spare": 0, "padded": 0, "pitch": 0}
    assert not set(options) - set(c)
    c.update(options)
    return c


def _linear(name, form, dtype, tokens, sequences, heads, qk_heads, dk, dv, **options):
    c = {"name": name, "op": "linear", "form": form, "dtype": dtype, "tokens": tokens, "sequences": sequences, "heads": heads,
         "qk_heads": qk_heads, "dk": dk, "dv": dv, "tail": 0, "spare": 0, "padded": 0, "fused": False, "by_head": False}
    assert not set(options) - set(c)
    c.update(options)
    return c


def _matvec(name, dtype, rows, n, k, group, zeros, bias):
    return {"name": name, "op": "matvec", "dtype": dtype, "rows": rows, "n": n, "k": k, "group": group, "zeros": zeros, "bias": bias}


def listed():
    return [
        # one user's next token through the window of a layer: launch and host time are all of it
        _conv("conv_step_one", "step", "bf16", 1, 1, 2048, 4),
        # a full decoding batch, states anywhere in the pool, the last rows padding up to a captured batch size
        _conv("conv_step_batch", "step", "bf16", 256, 256, 8192, 4, spare=40, padded=6),
        # prompts of a serving batch packed one behind the other
        _conv("conv_packed", "packed", "bf16", 16384, 11, 4096, 4, tail=37),
        # nothing is a round number, 32 bits, rows that are a slice of wider ones
        _conv("conv_packed_f32_odd", "packed", "f32", 4099, 3, 1001, 3, silu=False, pitch=7, spare=2),
        # one user's next token through the recurrence
        _linear("linear_step_one", "step", "bf16", 1, 1, 16, 16, 128, 128),
        # a full decoding batch: the states, 2 MB a sequence, are read and written
        _linear("linear_step_batch", "step", "bf16", 128, 128, 32, 32, 128, 128, spare=8, padded=3),
        # one long prompt: as many heads as there are and nothing else to spread over the GPU
        _linear("linear_long", "packed", "bf16", 16384, 1, 32, 32, 128, 128),
        # ragged prompts packed one behind the other, query and key heads shared, rows cut from one projection's
        _linear("linear_packed", "packed", "f16", 9001, 13, 24, 8, 64, 128, tail=23, fused=True),
        # 32 bits, odd head sizes, one decay for each head
        _linear("linear_packed_f32_odd", "packed", "f32", 701, 3, 6, 2, 48, 80, by_head=True),
        # one token through a projection
        _matvec("matvec_one", "f16", 1, 4096, 4096, 128, False, False),
        # the largest projection of a large layer for a small batch, with zero points
        _matvec("matvec_large", "bf16", 8, 28672, 8192, 64, True, False),
        # nothing is a round number, 32 bits
        _matvec("matvec_f32_odd", "f32", 3, 1001, 2080, 32, True, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["conv", "linear", "linear", "matvec"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if op == "matvec":
            n, k = _log_int(rng, 256, 32768), _log_int(rng, 256, 16384)
            if rng.random() < 0.7:
                n, k = -(-n // 64) * 64, -(-k // 128) * 128
            c = _matvec("", dtype, rng.choice([1, 1, 2, 4, 8, 16, rng.randint(1, 16)]), n, k, rng.choice([32, 64, 128]),
                        rng.random() < 0.5, rng.random() < 0.5)
            if n * k > 28672 * 8192:
                continue
        else:
            form = rng.choice(["step", "packed"])
            sequences = _log_int(rng, 1, 256) if form == "step" else _log_int(rng, 1, 24)
            tokens = sequences if form == "step" else _log_int(rng, max(sequences, 16), 32768)
            options = {"spare": rng.choice([0, rng.randint(0, 40)])}
            if form == "step":
                options["padded"] = rng.choice([0, rng.randint(0, sequences - 1)])
            else:
                options["tail"] = rng.choice([0, rng.randint(0, 64)])
            if op == "conv":
                channels = _log_int(rng, 64, 16384)
                if rng.random() < 0.7:
                    channels = -(-channels // 64) * 64
                options.update(bias=rng.random() < 0.5, silu=rng.random() < 0.5, pitch=rng.choice([0, 0, 64, rng.randint(1, 99)]))
                c = _conv("", form, dtype, tokens, sequences, channels, rng.choice([2, 3, 4, 4, 4, rng.randint(1, 8)]), **options)
                if tokens * channels > 1 << 26:
                    continue
            else:
                qk_heads = _log_int(rng, 1, 32)
                heads = qk_heads * rng.choice([1, 1, 1, 2, 4])
                dk = rng.choice([64, 64, 128, 128, rng.choice([16, 32, 80, 96, 256]), rng.randint(8, 128)])
                dv = rng.choice([dk, 64, 128, rng.choice([32, 96, 256]), rng.randint(8, 128)])
                options.update(fused=rng.random() < 0.5, by_head=rng.random() < 0.3)
                c = _linear("", form, dtype, tokens, sequences, heads, qk_heads, dk, dv, **options)
                if max(tokens, 64 * sequences if form == "packed" else 0) * heads * max(dk, dv) > 16384 * 32 * 128 \
                        or (sequences + options["spare"]) * heads * dk * dv > 136 * 32 * 128 * 128:
                    continue
        del c["name"]
        return c


def _lengths(c):
    """Tokens of each sequence, by the case alone: ragged, and where there are many an empty one and one of a single token."""
    n, b = c["tokens"], c["sequences"]
    if c["form"] == "step":
        return [1] * b
    rng = random.Random(n * 31 + b)
    cuts = sorted(rng.randint(0, n) for _ in range(b - 1))
    if b > 4:
        cuts[1] = cuts[0]
        cuts[3] = min(cuts[2] + 1, n)
        cuts.sort()
    return [e - s for s, e in zip([0] + cuts, cuts + [n])]


def _inputs(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = _TYPES[c["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    s = {"case": c}
    if c["op"] == "matvec":
        n, k, groups = c["n"], c["k"], -(-c["k"] // c["group"])
        s["x"] = normal(c["rows"], k).to(dtype)
        s["weight"] = torch.randint(0, 256, (n, (k + 1) // 2), generator=g, device="cuda", dtype=torch.uint8)
        s["scales"] = ((0.5 + uniform(n, groups)) * 0.2 / math.sqrt(k)).to(dtype)
        s["zeros"] = torch.randint(5, 11, (n, groups), generator=g, device="cuda", dtype=torch.uint8) if c["zeros"] else None
        s["bias"] = normal(n) * 0.1 if c["bias"] else None
        s["y"] = torch.zeros((c["rows"], n), dtype=dtype, device="cuda")
        return s
    lengths = _lengths(c)
    b, rows = c["sequences"], c["tokens"] + c["tail"]
    slots = torch.randperm(b + c["spare"], generator=g, device="cuda")[:b].to(torch.int32)
    if c["padded"]:
        slots[b - c["padded"]:] = -1
    s["slots"] = slots if c["spare"] or c["padded"] else None
    packed = c["form"] == "packed"
    s["cu"] = torch.tensor([sum(lengths[:i]) for i in range(b + 1)], dtype=torch.int32, device="cuda") if packed else None
    s["resume"] = (torch.arange(b, device="cuda") % 3 != 0) if packed else None
    pool = b + c["spare"]
    if c["op"] == "conv":
        n, taps = c["channels"], c["taps"]
        s["x"] = normal(rows, n + c["pitch"]).to(dtype)[:, :n]
        s["weight"] = ((uniform(n, taps) * 2 - 1) / math.sqrt(taps)).to(dtype)
        s["bias"] = normal(n) * 0.1 if c["bias"] else None
        s["y"] = torch.zeros((rows, n), dtype=dtype, device="cuda")
        s["state"] = normal(pool, taps - 1, n).to(dtype)
    else:
        h, hk, dk, dv = c["heads"], c["qk_heads"], c["dk"], c["dv"]
        if c["fused"]:
            qkv = normal(rows, 2 * hk * dk + h * dv).to(dtype)
            q, k, v = qkv[:, :hk * dk], qkv[:, hk * dk:2 * hk * dk], qkv[:, 2 * hk * dk:]
        else:
            q, k, v = (normal(rows, m).to(dtype) for m in (hk * dk, hk * dk, h * dv))
        s["q"], s["k"], s["v"] = q.unflatten(1, (hk, dk)), k.unflatten(1, (hk, dk)), v.unflatten(1, (h, dv))
        rate = torch.exp(uniform(h) * math.log(300.0)) * 1e-3
        s["g"] = -rate if c["by_head"] else -rate * torch.nn.functional.softplus(normal(rows, h))
        s["o"] = torch.zeros((rows, h, dv), dtype=dtype, device="cuda")
        s["state"] = normal(pool, h, dk, dv) * 3
        s["scale"] = 1.0 / math.sqrt(dk)
        s["most"] = max(lengths)
    s["state_out"] = torch.zeros_like(s["state"])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and case["op"] == "linear":      # the scratch buffer that the program keeps
        from paper_2608_20725_b200 import binding
        s["shape"] = binding.make_attention_shape(s["q"].shape[0], case["sequences"], case["heads"], case["qk_heads"], case["dk"], case["dv"],
                                                  s["most"])
        s["workspace"] = binding.alloc_attention_workspace(s["shape"], s["q"].dtype)
    return s


def run(s):
    case = s["case"]
    if not own:
        return {"conv": _plain_conv, "linear": _plain_linear, "matvec": _plain_matvec}[case["op"]](s)
    from paper_2608_20725_b200 import binding
    if case["op"] == "conv":
        binding.im2win_causal_conv1d(s["x"], s["weight"], s["y"], bias=s["bias"], silu=case["silu"], state=s["state"],
                                     state_out=s["state_out"], cu_seqlens=s["cu"], slots=s["slots"], resume=s["resume"])
        return s["y"], s["state_out"]
    if case["op"] == "linear":
        binding.im2win_linear_attention(s["q"], s["k"], s["v"], s["g"], s["o"], scale=s["scale"], state=s["state"],
                                        state_out=s["state_out"], cu_seqlens=s["cu"], slots=s["slots"], resume=s["resume"],
                                        max_len=s["most"], workspace=s["workspace"])
        return s["o"], s["state_out"]
    binding.im2win_matvec_int4(s["x"], s["weight"], s["scales"], s["y"], group=case["group"], zeros=s["zeros"], bias=s["bias"])
    return s["y"]


def _sequences(s):
    """(first row, length, slot, whether it is no padding, whether it resumes) of each sequence."""
    b, device = s["case"]["sequences"], s["state"].device
    one = torch.arange(b + 1, device=device)
    cu = one if s["cu"] is None else s["cu"].long()
    slot = one[:b] if s["slots"] is None else s["slots"].long()
    resume = torch.ones(b, dtype=torch.bool, device=device) if s["resume"] is None else s["resume"]
    return cu[:-1], cu[1:] - cu[:-1], slot, slot >= 0, resume


def _store_states(s, slot, real, new):
    """The new states in the pool; its other rows as they are."""
    out = s["state_out"]
    out[slot[real]] = new[real].to(out.dtype)
    return out


def _plain_conv(s):
    x, c = s["x"].float(), s["case"]
    taps, n = c["taps"], c["channels"]
    first, length, slot, real, resume = _sequences(s)
    old = s["state"].float()[slot.clamp(min=0)] * resume[:, None, None]
    rows = torch.arange(x.shape[0], device=x.device)
    of = torch.searchsorted(first + length, rows, right=True).clamp(max=len(slot) - 1)
    at = rows - first[of]
    ours = (at < length[of]) & real[of]
    # the rows, then each sequence's carried ones
    carried = x.shape[0] + of * (taps - 1) + taps - 1 + at
    x = torch.cat([x, old.reshape(-1, n)])
    z = sum(x[torch.where(at >= d, rows - d, (carried - d).clamp(max=x.shape[0] - 1))] * s["weight"].float()[:, taps - 1 - d]
            for d in range(taps))
    if s["bias"] is not None:
        z = z + s["bias"]
    if c["silu"]:
        z = z / (1 + torch.exp(-z))
    s["y"].copy_(torch.where(ours[:, None], z, s["y"].float()))
    r = torch.arange(taps - 1, device=x.device) - (taps - 1)
    behind = length[:, None] + r                                    # where the new state's rows lie in the sequence
    b = torch.arange(len(slot), device=x.device)[:, None]
    new = x[torch.where(behind >= 0, first[:, None] + behind, rows.numel() + b * (taps - 1) + taps - 1 + behind)]
    return s["y"], _store_states(s, slot, real, new)


def _plain_linear(s):
    c = s["case"]
    h, hk, dk, dv = c["heads"], c["qk_heads"], c["dk"], c["dv"]
    first, length, slot, real, resume = _sequences(s)
    b, most = len(slot), s["most"]
    chunk = min(_CHUNK, most)
    chunks = -(-most // chunk)
    at = torch.arange(chunks * chunk, device=first.device)
    inside = at < length[:, None]                                   # [b, positions]
    rows = torch.where(inside, first[:, None] + at, 0)

    def by_chunk(t, heads):                                         # -> [b, heads, chunks, chunk, ...] in 32 bits, 0 beyond the end
        t = t.float()[rows] * inside[..., None, None]
        t = t.unflatten(1, (chunks, chunk)).movedim(3, 1)
        return t.repeat_interleave(h // heads, 1) if heads != h else t

    q, k, v = by_chunk(s["q"], hk), by_chunk(s["k"], hk), by_chunk(s["v"], h)
    g = s["g"].double() if s["g"].dim() == 2 else s["g"].double().expand(s["q"].shape[0], h)
    g = (g[rows] * inside[..., None]).unflatten(1, (chunks, chunk)).movedim(3, 1).cumsum(3)         # [b, h, chunks, chunk]
    causal = torch.tril(torch.ones((chunk, chunk), dtype=torch.bool, device=g.device))
    decay = torch.exp((g[..., :, None] - g[..., None, :]).masked_fill(~causal, -math.inf).float())
    o = ((q @ k.transpose(3, 4)) * decay) @ v
    added = (k * torch.exp(g[..., -1:] - g).float()[..., None]).transpose(3, 4) @ v                 # [b, h, chunks, dk, dv]
    ends = torch.cat([torch.zeros_like(g[..., :1, -1]), g[..., -1].cumsum(2)], 2)                   # [b, h, chunks + 1]
    # the state before chunk j: the first one and what the chunks i < j added, each decayed up to there
    later = torch.tril(torch.ones((chunks + 1, chunks), dtype=torch.bool, device=g.device), -1)
    carry = torch.exp((ends[..., :, None] - ends[..., None, 1:]).masked_fill(~later, -math.inf).float())
    old = s["state"][slot.clamp(min=0)] * resume[:, None, None, None]
    states = (carry @ added.flatten(3)).unflatten(3, (dk, dv)) + torch.exp(ends.float())[..., None, None] * old[:, :, None]
    o = (o + (q * torch.exp(g.float())[..., None]) @ states[:, :, :-1]) * s["scale"]
    o = o.movedim(1, 3).flatten(1, 2)                               # [b, positions, h, dv]
    inside = inside & real[:, None]
    s["o"][rows[inside]] = o[inside].to(s["o"].dtype)
    return s["o"], _store_states(s, slot, real, states[:, :, -1])


def _plain_matvec(s):
    c = s["case"]
    w = torch.stack([s["weight"] & 15, s["weight"] >> 4], 2).flatten(1)[:, :c["k"]].float()
    groups = torch.arange(c["k"], device=w.device) // c["group"]
    zero = 8.0 if s["zeros"] is None else s["zeros"].float()[:, groups]
    y = s["x"].float() @ ((w - zero) * s["scales"].float()[:, groups]).T
    if s["bias"] is not None:
        y = y + s["bias"]
    s["y"].copy_(y)
    return s["y"]


def work(case):
    """Inputs once, outputs once; a state is read where it is resumed and written for every sequence that is none of the padding."""
    c, es = case, _BYTES[case["dtype"]]
    if c["op"] == "matvec":
        n, k, groups = c["n"], c["k"], -(-c["k"] // c["group"])
        moved = n * ((k + 1) // 2) + n * groups * (es + c["zeros"]) + c["rows"] * (n + k) * es + n * 4 * c["bias"]
        return {"bytes": moved, "flops": 2 * c["rows"] * n * k}
    tokens, b = c["tokens"] - c["padded"], c["sequences"] - c["padded"]
    read = b if c["form"] == "step" else b - (b + 2) // 3
    if c["op"] == "conv":
        state = (c["taps"] - 1) * c["channels"] * es
        weights = c["channels"] * (c["taps"] * es + 4 * c["bias"])
        return {"bytes": 2 * tokens * c["channels"] * es + (read + b) * state + weights, "flops": 2 * tokens * c["channels"] * c["taps"]}
    state = c["heads"] * c["dk"] * c["dv"] * 4
    rows = 2 * c["qk_heads"] * c["dk"] * es + 2 * c["heads"] * c["dv"] * es + c["heads"] * 4 * (not c["by_head"])
    return {"bytes": tokens * rows + (read + b) * state, "flops": 4 * tokens * c["heads"] * c["dk"] * c["dv"]}


def exact(case, seed):
    """The definitions, in 64 bits: a window for each position, a token after the other, a group after the other."""
    s = _inputs(case, seed)
    return {"conv": _exact_conv, "linear": _exact_linear, "matvec": _exact_matvec}[case["op"]](case, s)


def _exact_conv(c, s):
    taps, y, out = c["taps"], s["y"].double(), s["state_out"].double()
    slots = range(c["sequences"]) if s["slots"] is None else s["slots"].tolist()
    at = 0
    lengths = _lengths(c)
    if c["form"] == "step":                 # all at once: each window is the state and the one row behind it
        real = [i for i, slot in enumerate(slots) if slot >= 0]
        pool = torch.tensor([slots[i] for i in real], device="cuda")
        window = torch.cat([s["state"].double()[pool], s["x"].double()[real, None]], 1)
        y[real] = _activated(c, s, (window * s["weight"].double().T).sum(1))
        out[pool] = window[:, 1:]
        return y, out
    for i, (slot, n) in enumerate(zip(slots, lengths)):
        old = s["state"][slot].double() * (i % 3 != 0)
        whole = torch.cat([old, s["x"][at:at + n].double()])
        if n:
            y[at:at + n] = _activated(c, s, torch.einsum("tck,ck->tc", whole.unfold(0, taps, 1), s["weight"].double()))
        out[slot] = whole[n:]
        at += n
    return y, out


def _activated(c, s, z):
    z = z if s["bias"] is None else z + s["bias"].double()
    return z * torch.sigmoid(z) if c["silu"] else z


def _exact_linear(c, s):
    h, hk, lengths = c["heads"], c["qk_heads"], _lengths(c)
    b, of = c["sequences"], torch.arange(c["heads"], device="cuda") // (c["heads"] // c["qk_heads"])
    slots = list(range(b)) if s["slots"] is None else s["slots"].tolist()
    first = [sum(lengths[:i]) for i in range(b)]
    decay = s["g"].double().exp()
    state = s["state"].double()[[max(i, 0) for i in slots]]
    if c["form"] == "packed":
        state[0::3] = 0
    o, out = s["o"].double(), s["state_out"].double()
    order = sorted((i for i in range(b) if slots[i] >= 0), key=lambda i: -lengths[i])      # the longest ones first: the live ones lead
    state = state[order]
    for t in range(max(lengths)):
        live = sum(lengths[i] > t for i in order)
        if not live:
            break
        rows = torch.tensor([first[i] + t for i in order[:live]]).cuda()
        q, k, v = s["q"][rows].double()[:, of], s["k"][rows].double()[:, of], s["v"][rows].double()
        a = decay.expand(live, h) if c["by_head"] else decay[rows]
        state[:live] *= a[..., None, None]
        state[:live] += k[..., :, None] * v[..., None, :]
        o[rows] = (q[..., None, :] @ state[:live]).squeeze(2) * s["scale"]
    out[torch.tensor([slots[i] for i in order], device="cuda")] = state
    return o, out


def _exact_matvec(c, s):
    x, y = s["x"].double(), torch.zeros_like(s["y"], dtype=torch.float64)
    low, high = (s["weight"] % 16).double(), (s["weight"] // 16).double()
    for j in range(s["scales"].shape[1]):
        k0, k1 = j * c["group"], min((j + 1) * c["group"], c["k"])
        zero = torch.full_like(low[:, :1], 8.0) if s["zeros"] is None else s["zeros"][:, j:j + 1].double()
        even = x[:, k0:k1:2] @ (low[:, k0 // 2:(k1 + 1) // 2] - zero).T
        odd = x[:, k0 + 1:k1:2] @ (high[:, k0 // 2:k1 // 2] - zero).T
        y += (even + odd) * s["scales"][:, j].double()
    return y if s["bias"] is None else y + s["bias"].double()
