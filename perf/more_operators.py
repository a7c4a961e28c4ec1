"""The operators of decoding over a growing cache: what is measured, and their plain forms.

Three operators around the paged prefix store:

  append     keys and values of a ragged batch written behind the tokens that prefixes hold already, the keys (and
             the queries of the same rows) rotated to their positions on the way, and read back
  window     attention of rows over a prefix's cached tokens: a sliding window and the first tokens, which stay
             visible; single tokens, blocks and prompts
  axes       rotary positions with several axes (time, height, width), and their table

`own` False: elementary torch operations.  `own` True: the library's entry points.
"""
import math

import torch

own = False

DEV = "cuda"
HEADS = {                       # query heads, KV heads, head dim: the shapes of the configurations
    "mha32": (32, 32, 128),
    "gqa28": (28, 4, 128),
    "gqa32": (32, 8, 128),
    "mha4": (4, 4, 64),
}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BASE = 10000.0


def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + salt) % (2 ** 62))
    return g


def _normal(shape, gen, dtype, std=1.0):
    return (torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32) * std).to(dtype)


# --------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------

def listed():
    return [
        # one block of a single request goes behind a long prompt: the smallest call of a step
        {"name": "append_block_step", "op": "append", "heads": "gqa28", "dtype": "bf16", "requests": 1, "rows_lo": 16,
         "rows_hi": 16, "offset_lo": 16384, "offset_hi": 16384, "rot": 128, "interleaved": False, "axes": 1,
         "queries": True},
        # one token of every request of a large batch
        {"name": "append_token_batch", "op": "append", "heads": "gqa32", "dtype": "bf16", "requests": 256, "rows_lo": 1,
         "rows_hi": 1, "offset_lo": 100, "offset_hi": 4096, "rot": 128, "interleaved": False, "axes": 1,
         "queries": True},
        # prompts of several requests, text and image patches, odd lengths and odd places inside a page
        {"name": "append_prompt_mix", "op": "append", "heads": "mha32", "dtype": "bf16", "requests": 12, "rows_lo": 1,
         "rows_hi": 4001, "offset_lo": 0, "offset_hi": 777, "rot": 128, "interleaved": False, "axes": 3,
         "queries": True},
        # 32-bit tensors, interleaved pairs over half of the head, keys alone
        {"name": "append_partial_f32", "op": "append", "heads": "mha4", "dtype": "f32", "requests": 9, "rows_lo": 3,
         "rows_hi": 1301, "offset_lo": 5, "offset_hi": 100, "rot": 32, "interleaved": True, "axes": 1,
         "queries": False},
        # the next token of a single request over its whole long cache
        {"name": "window_token", "op": "window", "heads": "gqa28", "dtype": "bf16", "requests": 1, "rows_lo": 1,
         "rows_hi": 1, "cached_lo": 16384, "cached_hi": 16384, "sinks": 0, "left": -1, "right": 0, "lse": False},
        # the next tokens of a batch of requests of all lengths, long window
        {"name": "window_token_batch", "op": "window", "heads": "gqa32", "dtype": "bf16", "requests": 64, "rows_lo": 1,
         "rows_hi": 1, "cached_lo": 700, "cached_hi": 16384, "sinks": 4, "left": 8191, "right": 0, "lse": False},
        # a block of every request in a block-diffusion step: the block sees itself and a window before it
        {"name": "window_block_batch", "op": "window", "heads": "gqa28", "dtype": "bf16", "requests": 32, "rows_lo": 16,
         "rows_hi": 16, "cached_lo": 1000, "cached_hi": 16384, "sinks": 4, "left": 1023, "right": -1, "lse": False},
        # a long prompt under a causal window: the largest call
        {"name": "window_prompt", "op": "window", "heads": "mha32", "dtype": "bf16", "requests": 1, "rows_lo": 16384,
         "rows_hi": 16384, "cached_lo": 16384, "cached_hi": 16384, "sinks": 4, "left": 4095, "right": 0, "lse": False},
        # ragged requests, a window on both sides, odd sizes, the log-sum-exp that accumulated weights take
        {"name": "window_both_sides", "op": "window", "heads": "gqa28", "dtype": "bf16", "requests": 5, "rows_lo": 31,
         "rows_hi": 2047, "cached_lo": 513, "cached_hi": 6001, "sinks": 0, "left": 500, "right": 201, "lse": True},
        # 32-bit tensors with a head dim of 64
        {"name": "window_f32", "op": "window", "heads": "mha4", "dtype": "f32", "requests": 3, "rows_lo": 77,
         "rows_hi": 1000, "cached_lo": 1500, "cached_hi": 3001, "sinks": 16, "left": 700, "right": 0, "lse": True},
        # queries and keys of image patches between text tokens
        {"name": "axes_patches", "op": "axes", "form": "rows", "heads": "gqa28", "dtype": "bf16", "rows": 32768,
         "rot": 128, "interleaved": False, "axes": 3, "layout": "blocks", "inverse": False},
        # the table of cosines and sines for the key projection of a prompt with images
        {"name": "axes_table", "op": "axes", "form": "table", "heads": "gqa28", "dtype": "f32", "rows": 4099,
         "rot": 128, "interleaved": False, "axes": 3, "layout": "cycle", "inverse": False},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _limit(op):
    costs = [work(c) for c in listed() if c["op"] == op]
    return max(c["bytes"] for c in costs), max(c["flops"] for c in costs)


def draw(rng):
    op = rng.choice(["append", "append", "window", "window", "window", "axes"])
    max_bytes, max_flops = _limit(op)
    while True:
        heads = rng.choice(list(HEADS))
        d = HEADS[heads][2]
        dtype = "f32" if heads == "mha4" else "bf16"
        if op == "append":
            hi = _log_int(rng, 1, 4001)
            far = _log_int(rng, 1, 8192)
            c = {"op": op, "heads": heads, "dtype": rng.choice([dtype, dtype, "f32"]), "requests": _log_int(rng, 1, 256),
                 "rows_lo": rng.choice([1, hi]), "rows_hi": hi, "offset_lo": rng.choice([0, far]), "offset_hi": far,
                 "rot": rng.choice([d, d, d // 2, d // 4, d - 20, 2]), "interleaved": rng.random() < 0.5,
                 "axes": rng.choice([1, 1, 2, 3]), "queries": rng.random() < 0.7}
            if c["requests"] * (c["offset_hi"] + c["rows_hi"]) > 1 << 20:       # a state of a few GB
                continue
        elif op == "window":
            kind = rng.choice(["token", "block", "prompt"])
            hi = 1 if kind == "token" else rng.randint(2, 64) if kind == "block" else _log_int(rng, 65, 16384)
            cached = _log_int(rng, 1, 16384)
            c = {"op": op, "heads": heads, "dtype": dtype,
                 "requests": _log_int(rng, 1, 4 if kind == "prompt" else 64), "rows_lo": rng.choice([1, hi]),
                 "rows_hi": hi, "cached_lo": rng.choice([1, cached]), "cached_hi": cached,
                 "sinks": rng.choice([0, 0, 1, 4, 16, 129]),
                 "left": rng.choice([-1, 0, _log_int(rng, 1, 8192), _log_int(rng, 64, 8192)]),
                 "right": rng.choice([0, 0, -1, _log_int(rng, 1, 1024)]), "lse": rng.random() < 0.5}
        else:
            form = rng.choice(["rows", "rows", "table"])
            c = {"op": op, "form": form, "heads": heads, "dtype": "f32" if form == "table" else
                 rng.choice([dtype, "f32"]), "rows": _log_int(rng, 1, 32768),
                 "rot": rng.choice([d, d, d // 2, d - 20, 6]), "interleaved": rng.random() < 0.5,
                 "axes": rng.choice([2, 3, 3, 4]), "layout": rng.choice(["blocks", "cycle"]),
                 "inverse": form == "rows" and rng.random() < 0.3}
        w = work(c)
        if w["bytes"] <= max_bytes and w["flops"] <= max_flops:
            return c


def _spread(lo, hi, count, step):
    """`count` whole numbers between lo and hi, the larger of the two among them."""
    return [hi - ((i * step) % 10007) * (hi - lo) // 10007 for i in range(count)]


def _append_shape(case):
    """rows and first token of every request"""
    n = case["requests"]
    return _spread(case["rows_lo"], case["rows_hi"], n, 7919), _spread(case["offset_lo"], case["offset_hi"], n, 6067)


def _window_shape(case):
    """rows, cached length and first position of every request: its rows are the last tokens of its cache"""
    n = case["requests"]
    rows = _spread(case["rows_lo"], case["rows_hi"], n, 7919)
    cached = [max(c, r) for c, r in zip(_spread(case["cached_lo"], case["cached_hi"], n, 6067), rows)]
    return rows, cached, [c - r for c, r in zip(cached, rows)]


def _bounds(case, cached, pos):
    """Of a row at `pos`: the first token of its window, and the end of what it sees."""
    first = 0 if case["left"] < 0 else max(0, pos - case["left"])
    end = cached if case["right"] < 0 else min(cached, pos + case["right"] + 1)
    return first, end


def _window_sizes(case):
    """tokens that some row of a request sees, and pairs of a row and a token it sees, over all requests"""
    seen = pairs = 0
    for n, cached, pos in zip(*_window_shape(case)):
        first, _ = _bounds(case, cached, pos)
        _, end = _bounds(case, cached, pos + n - 1)
        seen += end - first + min(case["sinks"], first)
        for p in range(pos, pos + n):
            f, e = _bounds(case, cached, p)
            pairs += e - f + min(case["sinks"], f)
    return seen, pairs


def work(case):
    op = case["op"]
    hq, hkv, d = HEADS[case["heads"]]
    es = 2 if case["dtype"] == "bf16" else 4
    if op == "append":
        n = sum(_append_shape(case)[0])
        turned = hkv + (hq if case["queries"] else 0)
        moved = 2 * hkv + (hq if case["queries"] else 0)
        # rows in and out once, and the store's pages written and read back
        return {"bytes": n * d * es * (2 * moved + 2 * 2 * hkv) + 4 * n * (case["axes"] if case["axes"] > 1 else 0),
                "flops": 3 * n * turned * case["rot"]}
    if op == "window":
        n = sum(_window_shape(case)[0])
        seen, pairs = _window_sizes(case)
        return {"bytes": 2 * n * hq * d * es + (4 * n * hq if case["lse"] else 0) + 2 * seen * hkv * d * es,
                "flops": (4 * d + 3) * pairs * hq}
    if case["form"] == "table":
        n = case["rows"] * case["rot"]
        return {"bytes": 4 * case["axes"] * case["rows"] + 4 * n, "flops": 10 * n}
    n = case["rows"] * (hq + hkv) * d
    return {"bytes": 4 * case["axes"] * case["rows"] + 2 * n * es, "flops": 3 * case["rows"] * (hq + hkv) * case["rot"]}


# --------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------

def _pair_axis(case):
    """The position axis that every rotated pair turns with."""
    pairs, axes = case["rot"] // 2, case["axes"]
    if case.get("layout", "blocks") == "cycle":
        return [i % axes for i in range(pairs)]
    return [i * axes // pairs for i in range(pairs)]


def _axis_positions(rows, axes, gen):
    """Positions of text tokens (the same on every axis) with pictures of 24 x 31 patches between them."""
    r = torch.arange(rows, device=DEV)
    start = torch.randint(0, 16384, (rows // 1024 + 1,), generator=gen, device=DEV)[r // 1024] + r % 1024
    patch = torch.rand((rows // 744 + 1,), generator=gen, device=DEV)[r // 744] < 0.6
    at = r % 744
    grid = [start - at, start - at + at // 31, start - at + at % 31, start - at + at // 372][:axes]
    return torch.stack([torch.where(patch, g.clamp(min=0), start) for g in grid]).to(torch.int32).contiguous()


def _append_inputs(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    gen, dtype = _gen(seed, 21), DTYPES[case["dtype"]]
    rows = sum(_append_shape(case)[0])
    k, v = _normal((rows, hkv, d), gen, dtype), _normal((rows, hkv, d), gen, dtype)
    q = _normal((rows, hq, d), gen, dtype) if case["queries"] else None
    positions = _axis_positions(rows, case["axes"], gen) if case["axes"] > 1 else None
    return q, k, v, positions


def _window_inputs(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    gen, dtype = _gen(seed, 22), DTYPES[case["dtype"]]
    rows, cached, _ = _window_shape(case)
    q = _normal((sum(rows), hq, d), gen, dtype, 1.5)      # scores of a trained model spread wider than N(0, 1)
    ks = [_normal((m, hkv, d), gen, dtype) for m in cached]
    vs = [_normal((m, hkv, d), gen, dtype) for m in cached]
    return q, ks, vs


def _axes_inputs(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    gen = _gen(seed, 23)
    positions = _axis_positions(case["rows"], case["axes"], gen)
    if case["form"] == "table":
        return positions, None, None
    dtype = DTYPES[case["dtype"]]
    return positions, _normal((case["rows"], hq, d), gen, dtype), _normal((case["rows"], hkv, d), gen, dtype)


def _offsets(lengths):
    out, at = [], 0
    for n in lengths:
        out.append(at)
        at += n
    return out


def _frequencies(case):
    """The angle per position of every pair, in 64 bits."""
    i = torch.arange(case["rot"] // 2, dtype=torch.float64)
    return BASE ** (-2.0 * i / case["rot"])


def _rotation(case):
    from paper_2606_07571_b200 import binding
    return binding.Rotation(binding.rope_frequencies(case["rot"], BASE), interleaved=case["interleaved"],
                            pair_axis=_pair_axis(case), num_axes=case["axes"])


def prepare(case, seed):
    op = case["op"]
    hq, hkv, d = HEADS[case["heads"]]
    dtype = DTYPES[case["dtype"]]
    state = {"case": case}
    if op == "append":
        q, k, v, positions = _append_inputs(case, seed)
        lengths, firsts = _append_shape(case)
        state.update(q=q, k=k, v=v, positions=positions)
        if not own:
            state["freq"] = _frequencies(case).to(DEV)
            base = _offsets([f + n for n, f in zip(lengths, firsts)])       # caches one after the other
            state["token"] = torch.cat([torch.arange(f, f + n, device=DEV) for n, f in zip(lengths, firsts)])
            state["place"] = torch.cat([torch.arange(b + f, b + f + n, device=DEV)
                                        for b, n, f in zip(base, lengths, firsts)])
            total = sum(lengths) + sum(firsts)
            state["k_cache"] = torch.zeros((total, hkv, d), dtype=dtype, device=DEV)
            state["v_cache"] = torch.zeros((total, hkv, d), dtype=dtype, device=DEV)
            return state
        from paper_2606_07571_b200 import binding
        pages = sum((f + n + 15) // 16 for n, f in zip(lengths, firsts))
        bc = binding.BiCache(1, hq, hkv, d, pages, dtype, k.shape[0], len(lengths))
        state.update(bc=bc, rotation=_rotation(case), lengths=lengths, firsts=firsts, offs=_offsets(lengths),
                     ids=[bc.reserve_prefix(i + 1, f + n)[0] for i, (n, f) in enumerate(zip(lengths, firsts))],
                     q_out=None if q is None else torch.empty_like(q), k_out=torch.empty_like(k),
                     v_out=torch.empty_like(v))
        return state
    if op == "window":
        q, ks, vs = _window_inputs(case, seed)
        state["q"] = q
        if not own:
            state.update(ks=ks, vs=vs)
            return state
        from paper_2606_07571_b200 import binding
        rows, cached, pos = _window_shape(case)
        bc = binding.BiCache(1, hq, hkv, d, sum((m + 15) // 16 for m in cached), dtype, q.shape[0], len(rows))
        state.update(bc=bc, rows=rows, cached=cached, pos=pos, offs=_offsets(rows),
                     ids=[bc.put_prefix(i + 1, k[None], v[None])[0] for i, (k, v) in enumerate(zip(ks, vs))],
                     out=torch.empty_like(q),
                     lse=torch.empty(q.shape[:2], dtype=torch.float32, device=DEV) if case["lse"] else None)
        return state
    positions, q, k = _axes_inputs(case, seed)
    state.update(positions=positions, q=q, k=k)
    if not own:
        state["freq"] = _frequencies(case).to(DEV)
        return state
    from paper_2606_07571_b200 import binding
    state["rotation"] = _rotation(case)
    state["bc"] = binding.BiCache(1, hq, hkv, d, 16, dtype, 16, 1)
    if case["form"] == "table":
        state["table"] = torch.empty((case["rows"], case["rot"] // 2, 2), dtype=torch.float32, device=DEV)
    else:
        state["q_out"], state["k_out"] = torch.empty_like(q), torch.empty_like(k)
    return state


# --------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    return (_run_own if own else _run_plain)[case["op"]](case, state)


def _append_own(case, st):
    bc = st["bc"]
    bc.append_tokens(0, st["ids"], st["firsts"], st["offs"], st["lengths"], st["k"], st["v"], st["q"], st["q_out"],
                     rotation=st["rotation"], positions=st["positions"])
    bc.read_tokens(0, st["ids"], st["firsts"], st["offs"], st["lengths"], st["k_out"], st["v_out"])
    return (st["k_out"], st["v_out"]) if st["q"] is None else (st["k_out"], st["v_out"], st["q_out"])


def _window_own(case, st):
    st["bc"].attend_window(0, st["ids"], st["cached"], st["pos"], st["offs"], st["rows"], st["q"], st["out"], st["lse"],
                           sinks=case["sinks"], left=case["left"], right=case["right"])
    return (st["out"], st["lse"]) if case["lse"] else st["out"]


def _axes_own(case, st):
    if case["form"] == "table":
        st["bc"].rope_axes_table(st["rotation"], st["positions"], st["table"])
        return st["table"]
    st["bc"].rope_axes(st["rotation"], st["positions"], st["q"], st["q_out"], st["k"], st["k_out"],
                       inverse=case["inverse"])
    return st["q_out"], st["k_out"]


def _angles(case, positions, freq):
    """[rows, pairs], 64 bits; positions [axes, rows]"""
    axis = torch.tensor(_pair_axis(case), device=DEV)
    return positions.double()[axis].t() * freq


def _turn(case, x, cos, sin):
    rot = case["rot"]
    xf = x.float()
    r = xf[..., :rot]
    if case["interleaved"]:
        a, b = r[..., 0::2], r[..., 1::2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([y, xf[..., rot:]], dim=-1).to(x.dtype)


def _append_plain(case, st):
    positions = st["token"][None] if st["positions"] is None else st["positions"]
    angle = _angles(case, positions, st["freq"])
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    st["k_cache"][st["place"]] = _turn(case, st["k"], cos, sin)
    st["v_cache"][st["place"]] = st["v"]
    out = (st["k_cache"][st["place"]], st["v_cache"][st["place"]])
    return out if st["q"] is None else out + (_turn(case, st["q"], cos, sin),)


def _window_plain(case, st):
    hq, hkv, d = HEADS[case["heads"]]
    gq, scale = hq // hkv, d ** -0.5
    q = st["q"]
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=DEV)
    row = 0
    for (n, cached, pos), k, v in zip(zip(*_window_shape(case)), st["ks"], st["vs"]):
        step = max(1, min(n, (1 << 28) // (cached * hq), 1024))
        for a in range(0, n, step):
            b = min(n, a + step)
            first, _ = _bounds(case, cached, pos + a)
            _, end = _bounds(case, cached, pos + b - 1)
            if first <= case["sinks"]:
                first = 0
            token = torch.arange(first, end, device=DEV)
            kk, vv = k[first:end], v[first:end]
            if first > 0 and case["sinks"] > 0:               # the first tokens before the window's
                token = torch.cat([torch.arange(case["sinks"], device=DEV), token])
                kk, vv = torch.cat([k[:case["sinks"]], kk]), torch.cat([v[:case["sinks"]], vv])
            p = torch.arange(pos + a, pos + b, device=DEV)[:, None]
            seen = token < cached
            if case["right"] >= 0:
                seen = seen & (token <= p + case["right"])
            if case["left"] >= 0:
                seen = seen & ((token < case["sinks"]) | (token >= p - case["left"]))
            seen = seen.expand(b - a, -1).repeat_interleave(gq, dim=0)          # one row per token and head of a group
            x = q[row + a:row + b].float().view(b - a, hkv, gq, d).permute(1, 0, 2, 3).reshape(hkv, -1, d)
            s = torch.matmul(x, kk.float().permute(1, 2, 0)) * scale
            s = torch.where(seen, s, torch.full_like(s, -math.inf))
            top = s.amax(dim=2, keepdim=True)
            e = torch.exp(s - top)
            total = e.sum(dim=2, keepdim=True)
            o = torch.matmul(e, vv.float().permute(1, 0, 2)) / total
            out[row + a:row + b] = o.view(hkv, b - a, gq, d).permute(1, 0, 2, 3).reshape(b - a, hq, d).to(q.dtype)
            lse[row + a:row + b] = (top + torch.log(total)).view(hkv, b - a, gq).permute(1, 0, 2).reshape(b - a, hq)
        row += n
    return (out, lse) if case["lse"] else out


def _axes_plain(case, st):
    angle = _angles(case, st["positions"], st["freq"])
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if case["form"] == "table":
        return torch.stack([cos, sin], dim=-1)
    if case["inverse"]:
        sin = -sin
    cos, sin = cos[:, None, :], sin[:, None, :]
    return _turn(case, st["q"], cos, sin), _turn(case, st["k"], cos, sin)


_run_own = {"append": _append_own, "window": _window_own, "axes": _axes_own}
_run_plain = {"append": _append_plain, "window": _window_plain, "axes": _axes_plain}


# --------------------------------------------------------------------------------------------
# the definition in 64 bits
# --------------------------------------------------------------------------------------------

def _phases(case, positions):
    """Every pair of every row as a complex number of length one: [rows, pairs]."""
    turn = torch.empty((positions.shape[1], case["rot"] // 2), dtype=torch.float64, device=DEV)
    for i, axis in enumerate(_pair_axis(case)):
        turn[:, i] = positions[axis].double() * BASE ** (-2.0 * i / case["rot"])
    return torch.polar(torch.ones_like(turn), turn)


def _turn64(case, x, phase):
    rot, y = case["rot"], x.double()
    if case["interleaved"]:
        z = torch.view_as_complex(y[..., :rot].reshape(*y.shape[:2], rot // 2, 2).contiguous()) * phase[:, None]
        y[..., :rot] = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * phase[:, None]
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    return y


def exact(case, seed):
    op = case["op"]
    if op == "append":
        q, k, v, positions = _append_inputs(case, seed)
        if positions is None:
            positions = torch.tensor([t for n, f in zip(*_append_shape(case)) for t in range(f, f + n)], device=DEV)[None]
        phase = _phases(case, positions)
        out = (_turn64(case, k, phase), v.double())
        return out if q is None else out + (_turn64(case, q, phase),)
    if op == "window":
        hq, hkv, d = HEADS[case["heads"]]
        q, ks, vs = _window_inputs(case, seed)
        out = torch.empty(q.shape, dtype=torch.float64, device=DEV)
        lse = torch.empty(q.shape[:2], dtype=torch.float64, device=DEV)
        row = 0
        for (n, cached, pos), k, v in zip(zip(*_window_shape(case)), ks, vs):
            t = torch.arange(cached, device=DEV)
            step = max(1, (1 << 27) // cached)
            for head in range(hq):                            # head by head, every cached token
                kh, vh = k[:, head // (hq // hkv)].double(), v[:, head // (hq // hkv)].double()
                for a in range(0, n, step):
                    b = min(n, a + step)
                    ahead = t[None] - torch.arange(pos + a, pos + b, device=DEV)[:, None]
                    hidden = torch.zeros_like(ahead, dtype=torch.bool)
                    if case["right"] >= 0:
                        hidden |= ahead > case["right"]
                    if case["left"] >= 0:
                        hidden |= (ahead < -case["left"]) & (t >= case["sinks"])
                    s = torch.einsum("rd,td->rt", q[row + a:row + b, head].double(), kh).div_(math.sqrt(d))
                    s.masked_fill_(hidden, -math.inf)
                    lse[row + a:row + b, head] = torch.logsumexp(s, dim=1)
                    out[row + a:row + b, head] = s.sub_(lse[row + a:row + b, head, None]).exp_() @ vh
            row += n
        return (out, lse) if case["lse"] else out
    positions, q, k = _axes_inputs(case, seed)
    phase = _phases(case, positions)
    if case["form"] == "table":
        return torch.view_as_real(phase)
    phase = phase.conj() if case["inverse"] else phase
    return _turn64(case, q, phase), _turn64(case, k, phase)
