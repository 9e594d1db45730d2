"""More operators on token sequences that the library's speed is measured on, each case the way a program that serves a model calls it.

``delta``    im2win_gated_delta_rule: S = exp(g) S + k^T beta (v - k exp(g) S), o = scale q S for each head, S carried from call to call
``norm``     im2win_rms_norm: the residual's addition, the root-mean-square norm, rows in 8 bits with a scale each where wanted
``matmul``   im2win_matmul_int8: rows times a matrix, both in 8 bits, with scales for each row and each row of the matrix
``project``  the last two as a layer runs them: rows are normed into 8 bits and multiplied

A case of ``delta`` has ``tokens`` in ``sequences``: ``step`` one token a sequence (the decoding loop), ``packed`` ragged sequences
one behind the other, some of them empty or of one token, with ``tail`` allocated rows behind the last (left as they are).  ``spare``
more states than sequences lie in the pool and the sequences take them in any order; ``padded`` of the step's sequences are padding
(slot -1: nothing of theirs is read or written).  Of packed sequences every third starts afresh, the others resume.

Each pass reads its states from one pool and writes them to another, so that every pass of a case does the same.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_CHUNK = 64
_EPS = 1e-6


def _delta(name, form, dtype, tokens, sequences, heads, qk_heads, dk, dv, **options):
    c = {"name": name, "op": "delta", "form": form, "dtype": dtype, "tokens": tokens, "sequences": sequences, "heads": heads,
         "qk_heads": qk_heads, "dk": dk, "dv": dv, "tail": 0, "spare": 0, "padded": 0, "fused": False, "normalize": True}
    assert not set(options) - set(c)
    c.update(options)
    return c


def _norm(name, dtype, rows, channels, residual, int8, pitch=0):
    return {"name": name, "op": "norm", "dtype": dtype, "rows": rows, "channels": channels, "residual": residual, "int8": int8, "pitch": pitch}


def _matmul(name, dtype, rows, n, k, bias):
    return {"name": name, "op": "matmul", "dtype": dtype, "rows": rows, "n": n, "k": k, "bias": bias}


def _project(name, dtype, rows, n, k, residual):
    return {"name": name, "op": "project", "dtype": dtype, "rows": rows, "n": n, "k": k, "residual": residual, "bias": False}


def listed():
    return [
        # one user's next token through the recurrence: launch and host time are all of it
        _delta("delta_step_one", "step", "bf16", 1, 1, 16, 16, 128, 128),
        # a full decoding batch, states anywhere in the pool, the last rows padding up to a captured batch size
        _delta("delta_step_batch", "step", "bf16", 128, 128, 32, 16, 128, 128, spare=8, padded=3),
        # one long prompt: as many heads as there are and nothing else to spread over the GPU
        _delta("delta_long", "packed", "bf16", 16384, 1, 32, 16, 128, 128),
        # ragged prompts packed one behind the other, query and key heads shared, rows cut from one projection's
        _delta("delta_packed", "packed", "f16", 9001, 13, 24, 8, 64, 128, tail=23, fused=True),
        # 32 bits, odd head sizes, rows that come normalised
        _delta("delta_packed_f32_odd", "packed", "f32", 701, 3, 6, 2, 48, 80, normalize=False),
        # one user's next token between two layers
        _norm("norm_step", "bf16", 1, 4096, True, False),
        # a batch of prompts between two layers
        _norm("norm_prompt", "bf16", 16384, 4096, True, False),
        # nothing is a round number, rows that are a slice of wider ones, out in 8 bits
        _norm("norm_int8_odd", "f16", 701, 1001, False, True, pitch=7),
        # the next tokens of a small batch through a projection
        _matmul("matmul_step", "bf16", 8, 4096, 4096, False),
        # a batch of prompts through a projection
        _matmul("matmul_prompt", "bf16", 16384, 8192, 4096, False),
        # nothing is a round number, 32 bits
        _matmul("matmul_f32_odd", "f32", 701, 1001, 2080, True),
        # a prompt's rows into 8 bits and through the widest projection of a layer
        _project("project_prompt", "bf16", 2048, 28672, 4096, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["delta", "delta", "norm", "matmul", "project"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if op == "delta":
            form = rng.choice(["step", "packed", "packed"])
            sequences = _log_int(rng, 1, 256) if form == "step" else _log_int(rng, 1, 24)
            tokens = sequences if form == "step" else _log_int(rng, max(sequences, 16), 16384)
            qk_heads = _log_int(rng, 1, 32)
            heads = qk_heads * rng.choice([1, 1, 2, 2, 4])
            dk = rng.choice([64, 128, 128, rng.choice([16, 32, 80, 96]), rng.randint(8, 128)])
            dv = rng.choice([dk, 64, 128, rng.choice([32, 96, 256]), rng.randint(8, 128)])
            options = {"spare": rng.choice([0, rng.randint(0, 40)]), "fused": rng.random() < 0.5, "normalize": rng.random() < 0.7}
            if form == "step":
                options["padded"] = rng.choice([0, rng.randint(0, sequences - 1)])
            else:
                options["tail"] = rng.choice([0, rng.randint(0, 64)])
            c = _delta("", form, dtype, tokens, sequences, heads, qk_heads, dk, dv, **options)
            if max(tokens, 64 * sequences if form == "packed" else 0) * heads * max(dk, dv) > 16384 * 32 * 128 \
                    or (sequences + options["spare"]) * heads * dk * dv > 136 * 32 * 128 * 128:
                continue
        elif op == "norm":
            channels = _log_int(rng, 64, 16384)
            if rng.random() < 0.7:
                channels = -(-channels // 64) * 64
            c = _norm("", dtype, _log_int(rng, 1, 32768), channels, rng.random() < 0.6, rng.random() < 0.5,
                      rng.choice([0, 0, 64, rng.randint(1, 99)]))
            if c["rows"] * channels > 16384 * 4096:
                continue
        else:
            n, k = _log_int(rng, 64, 32768), _log_int(rng, 64, 16384)
            if rng.random() < 0.7:
                n, k = -(-n // 64) * 64, -(-k // 128) * 128
            rows = rng.choice([_log_int(rng, 1, 64), _log_int(rng, 1, 16384)])
            if op == "matmul":
                c = _matmul("", dtype, rows, n, k, rng.random() < 0.5)
            else:
                c = _project("", dtype, rows, n, k, rng.random() < 0.5)
            if rows * n * k > 16384 * 8192 * 4096 or n * k > 28672 * 8192:
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


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c, dtype = case, _TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    s = {"case": c}
    if c["op"] == "delta":
        lengths, b, rows = _lengths(c), c["sequences"], c["tokens"] + c["tail"]
        h, hk, dk, dv = c["heads"], c["qk_heads"], c["dk"], c["dv"]
        slots = torch.randperm(b + c["spare"], generator=g, device="cuda")[:b].to(torch.int32)
        if c["padded"]:
            slots[b - c["padded"]:] = -1
        s["slots"] = slots if c["spare"] or c["padded"] else None
        packed = c["form"] == "packed"
        s["cu"] = torch.tensor([sum(lengths[:i]) for i in range(b + 1)], dtype=torch.int32, device="cuda") if packed else None
        s["resume"] = (torch.arange(b, device="cuda") % 3 != 0) if packed else None
        q, k, v = normal(rows, hk, dk), normal(rows, hk, dk), normal(rows, h * dv)
        if not c["normalize"]:
            q, k = (x / x.norm(dim=2, keepdim=True) for x in (q, k))
        q, k = q.flatten(1), k.flatten(1)
        if c["fused"]:
            q, k, v = torch.cat([q, k, v], 1).to(dtype).split([hk * dk, hk * dk, h * dv], 1)
        else:
            q, k, v = (x.to(dtype) for x in (q, k, v))
        s["q"], s["k"], s["v"] = q.unflatten(1, (hk, dk)), k.unflatten(1, (hk, dk)), v.unflatten(1, (h, dv))
        s["g"] = -torch.exp(uniform(h) * math.log(300.0)) * 1e-3 * torch.nn.functional.softplus(normal(rows, h))
        s["beta"] = torch.sigmoid(normal(rows, h))
        s["o"] = torch.zeros((rows, h, dv), dtype=dtype, device="cuda")
        s["state"] = normal(b + c["spare"], h, dk, dv) * 0.3
        s["state_out"] = torch.zeros_like(s["state"])
        s["scale"], s["most"] = 1.0 / math.sqrt(dk), max(lengths)
    elif c["op"] == "norm":
        rows, n = c["rows"], c["channels"]
        s["x"] = normal(rows, n + c["pitch"]).to(dtype)[:, :n]
        s["residual"] = (normal(rows, n) * 2).to(dtype) if c["residual"] else None
        s["weight"] = (1 + 0.3 * normal(n)).to(dtype)
        s["sum"] = torch.zeros((rows, n), dtype=dtype, device="cuda") if c["residual"] else None
        s["y"] = torch.zeros((rows, n), dtype=torch.int8 if c["int8"] else dtype, device="cuda")
        s["scales"] = torch.zeros(rows, device="cuda") if c["int8"] else None
    else:
        m, n, k = c["rows"], c["n"], c["k"]
        s["matrix"] = torch.randint(-127, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
        s["matrix_scales"] = (0.5 + uniform(n)) / (73 * math.sqrt(k))
        s["bias"] = normal(n) * 0.1 if c["bias"] else None
        s["y"] = torch.zeros((m, n), dtype=dtype, device="cuda")
        if c["op"] == "matmul":
            s["x"] = (normal(m, k) * 32).round().clamp(-127, 127).to(torch.int8)
            s["x_scales"] = (0.5 + uniform(m)) / 32
        else:
            s["x"] = normal(m, k).to(dtype)
            s["residual"] = (normal(m, k) * 2).to(dtype) if c["residual"] else None
            s["weight"] = (1 + 0.3 * normal(k)).to(dtype)
            s["sum"] = torch.zeros((m, k), dtype=dtype, device="cuda") if c["residual"] else None
            s["rows8"], s["scales"] = torch.zeros((m, k), dtype=torch.int8, device="cuda"), torch.zeros(m, device="cuda")
    return s


def run(s):
    c = s["case"]
    if not own:
        return {"delta": _plain_delta, "norm": _plain_norm, "matmul": _plain_matmul, "project": _plain_project}[c["op"]](s)
    from paper_2608_20725_b200 import binding
    if c["op"] == "delta":
        binding.im2win_gated_delta_rule(s["q"], s["k"], s["v"], s["g"], s["beta"], s["o"], scale=s["scale"], normalize=c["normalize"],
                                        state=s["state"], state_out=s["state_out"], cu_seqlens=s["cu"], slots=s["slots"], resume=s["resume"],
                                        max_len=s["most"])
        return s["o"], s["state_out"]
    if c["op"] == "norm":
        binding.im2win_rms_norm(s["x"], s["weight"], s["y"], scales=s["scales"], residual=s["residual"], residual_out=s["sum"], eps=_EPS)
        return s["sum"], (s["y"].float() * s["scales"][:, None] if c["int8"] else s["y"])
    if c["op"] == "matmul":
        binding.im2win_matmul_int8(s["x"], s["x_scales"], s["matrix"], s["matrix_scales"], s["y"], bias=s["bias"])
        return s["y"]
    binding.im2win_rms_norm(s["x"], s["weight"], s["rows8"], scales=s["scales"], residual=s["residual"], residual_out=s["sum"], eps=_EPS)
    binding.im2win_matmul_int8(s["rows8"], s["scales"], s["matrix"], s["matrix_scales"], s["y"])
    return s["sum"], s["y"]


def _plain_delta(s):
    """By chunks of 64 tokens.  With G the sums of g within a chunk, A_ij = beta_i exp(G_i - G_j) k_i.k_j below the diagonal and
    T = (1 + A)^-1, a chunk's new values are U = T (beta V - beta exp(G) K S), its rows exp(G) Q S + (exp(G_i - G_j) q_i.k_j) U, and
    what it leaves exp(G_n) S + (exp(G_n - G) K)^T U."""
    c = s["case"]
    h, hk, dk, dv = c["heads"], c["qk_heads"], c["dk"], c["dv"]
    b, device = c["sequences"], s["state"].device
    cu = torch.arange(b + 1, device=device) if s["cu"] is None else s["cu"].long()
    first, length = cu[:-1], cu[1:] - cu[:-1]
    slot = torch.arange(b, device=device) if s["slots"] is None else s["slots"].long()
    real = slot >= 0
    resume = torch.ones(b, dtype=torch.bool, device=device) if s["resume"] is None else s["resume"]
    chunk = min(_CHUNK, s["most"])
    chunks = -(-s["most"] // chunk)
    at = torch.arange(chunks * chunk, device=device)
    inside = at < length[:, None]                                   # [b, positions]
    rows = torch.where(inside, first[:, None] + at, 0)

    def by_chunk(t, heads):                                         # -> [b, heads, chunks, chunk, ...], 0 beyond the end
        t = torch.where(inside.view(inside.shape + (1,) * (t.dim() - 1)), t[rows], 0)
        t = t.unflatten(1, (chunks, chunk)).movedim(3, 1)
        return t.repeat_interleave(h // heads, 1) if heads != h else t

    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    if c["normalize"]:
        q, k = (x * torch.rsqrt((x * x).sum(2, keepdim=True) + _EPS) for x in (q, k))
    q, k, v, beta = by_chunk(q, hk), by_chunk(k, hk), by_chunk(v, h), by_chunk(s["beta"], h)[..., None]
    g = by_chunk(s["g"].double(), h).cumsum(3)                      # [b, h, chunks, chunk]
    causal = torch.tril(torch.ones((chunk, chunk), dtype=torch.bool, device=device))
    decay = torch.exp((g[..., :, None] - g[..., None, :]).masked_fill(~causal, -math.inf).float())
    kt = k.transpose(3, 4)
    lower = ((k @ kt) * decay * beta).masked_fill(~torch.tril(causal, -1), 0.0)
    inverse = torch.eye(chunk, device=device).expand(lower.shape).clone()
    for i in range(1, chunk):
        inverse[..., i, :i] = -(lower[..., i:i + 1, :i] @ inverse[..., :i, :i]).squeeze(-2)
    from_start, to_end = torch.exp(g).float()[..., None], torch.exp(g[..., -1:] - g).float()[..., None]
    fresh, taken = inverse @ (v * beta), inverse @ (k * (beta * from_start))
    weights, q, kt = (q @ kt) * decay, q * from_start, kt * to_end.transpose(3, 4)
    total = torch.exp(g[..., -1]).float()[..., None, None]          # [b, h, chunks, 1, 1]
    state = s["state"][slot.clamp(min=0)] * resume[:, None, None, None]
    o = torch.empty_like(v)
    for i in range(chunks):
        new = fresh[:, :, i] - taken[:, :, i] @ state
        o[:, :, i] = (q[:, :, i] @ state + weights[:, :, i] @ new) * s["scale"]
        state = total[:, :, i] * state + kt[:, :, i] @ new
    o = o.movedim(1, 3).flatten(1, 2)                               # [b, positions, h, dv]
    inside = inside & real[:, None]
    s["o"][rows[inside]] = o[inside].to(s["o"].dtype)
    s["state_out"][slot[real]] = state[real]
    return s["o"], s["state_out"]


def _plain_sum(s):
    """What is normed: x, or x and the residual, added in 32 bits and rounded to their type."""
    if s["residual"] is None:
        return s["x"]
    s["sum"].copy_(s["x"].float() + s["residual"].float())
    return s["sum"]


def _plain_int8(h, weight):
    """Rows in 8 bits, the largest magnitude 127, and their scales.  Which whole number is nearest does not depend on the norm; it is
    looked for in 64 bits, ties to the even one."""
    p = h.double() * weight.double()
    top = p.abs().amax(1, keepdim=True)
    q = torch.where(top > 0, torch.round(p * 127 / top), 0.0).float()
    rate = torch.rsqrt(h.float().square().mean(1, keepdim=True) + _EPS)
    return q, top.float() * rate / 127


def _plain_norm(s):
    c, h = s["case"], _plain_sum(s)
    if c["int8"]:
        q, scales = _plain_int8(h, s["weight"])
        return s["sum"], q * scales
    x = h.float()
    s["y"].copy_(x * torch.rsqrt(x.square().mean(1, keepdim=True) + _EPS) * s["weight"].float())
    return s["sum"], s["y"]


def _plain_product(s, x, scales):
    y = (x @ s["matrix"].float().T) * scales * s["matrix_scales"]
    if s["bias"] is not None:
        y = y + s["bias"]
    s["y"].copy_(y)
    return s["y"]


def _plain_matmul(s):
    return _plain_product(s, s["x"].float(), s["x_scales"][:, None])


def _plain_project(s):
    q, scales = _plain_int8(_plain_sum(s), s["weight"])
    return s["sum"], _plain_product(s, q, scales)


def work(case):
    """Inputs once, outputs once; a state is read where it is resumed and written for every sequence that is none of the padding."""
    c, es = case, _BYTES[case["dtype"]]
    if c["op"] == "delta":
        tokens, b = c["tokens"] - c["padded"], c["sequences"] - c["padded"]
        read = b if c["form"] == "step" else b - (b + 2) // 3
        state = c["heads"] * c["dk"] * c["dv"] * 4
        rows = 2 * c["qk_heads"] * c["dk"] * es + 2 * c["heads"] * c["dv"] * es + c["heads"] * 8
        return {"bytes": tokens * rows + (read + b) * state, "flops": 6 * tokens * c["heads"] * c["dk"] * c["dv"]}
    if c["op"] == "norm":
        out = c["channels"] + 4 if c["int8"] else c["channels"] * es
        row = c["channels"] * es * (3 if c["residual"] else 1) + out
        return {"bytes": c["rows"] * row + c["channels"] * es, "flops": 4 * c["rows"] * c["channels"]}
    m, n, k = c["rows"], c["n"], c["k"]
    moved = n * k + n * 4 * (1 + c["bias"]) + m * n * es
    if c["op"] == "matmul":
        moved += m * (k + 4)
    else:
        moved += m * k * es * (3 if c["residual"] else 1) + k * es
    return {"bytes": moved, "flops": 2 * m * n * k}


def exact(case, seed):
    """The definitions, in 64 bits: a token after the other, a row's numbers from the row alone."""
    s = prepare(case, seed)
    if case["op"] == "delta":
        return _exact_delta(case, s)
    if case["op"] == "matmul":
        return _exact_product(s, s["x"].double(), s["x_scales"].double())
    h = s["x"].double()
    if s["residual"] is not None:
        h = (s["x"].float() + s["residual"].float()).to(s["x"].dtype).double()
    z = h * s["weight"].double()
    per_row = 1.0 / (h.pow(2).sum(1) / h.shape[1] + _EPS).sqrt()
    top = z.abs().max(1).values
    if case["op"] == "norm" and not case["int8"]:
        return (h if s["residual"] is not None else None), z * per_row[:, None]
    codes = (z * 127 / top.clamp(min=1e-300)[:, None]).round()
    scales = top * per_row / 127
    if case["op"] == "norm":
        return (h if s["residual"] is not None else None), codes * scales[:, None]
    return (h if s["residual"] is not None else None), _exact_product(s, codes, scales)


def _exact_product(s, x, scales):
    y = torch.empty(s["y"].shape, dtype=torch.float64, device="cuda")
    for n0 in range(0, y.shape[1], 4096):
        part = slice(n0, n0 + 4096)
        y[:, part] = x @ s["matrix"][part].double().T * scales[:, None] * s["matrix_scales"][part].double()
    return y if s["bias"] is None else y + s["bias"].double()


def _exact_delta(c, s):
    h, hk, lengths = c["heads"], c["qk_heads"], _lengths(c)
    b, of = c["sequences"], torch.arange(h, device="cuda") // (h // hk)
    slots = list(range(b)) if s["slots"] is None else s["slots"].tolist()
    first = [sum(lengths[:i]) for i in range(b)]
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
        q, k, v = s["q"][rows].double(), s["k"][rows].double(), s["v"][rows].double()
        if c["normalize"]:
            q, k = (x / torch.sqrt((x * x).sum(2, keepdim=True) + _EPS) for x in (q, k))
        q, k = q[:, of], k[:, of]
        state[:live] *= s["g"][rows].double().exp()[..., None, None]
        wrong = v - (k[..., None, :] @ state[:live]).squeeze(2)
        state[:live] += k[..., :, None] * (s["beta"][rows].double()[..., None] * wrong)[..., None, :]
        o[rows] = (q[..., None, :] @ state[:live]).squeeze(2) * s["scale"]
    out[torch.tensor([slots[i] for i in order], device="cuda")] = state
    return o, out
