"""The token-eviction and rotary operators: what is measured, and their plain forms.

Four operators around the paged prefix cache:

  weights   accumulated attention weight of every cached key (what an eviction decides by)
  select    the tokens to keep: largest weights, protected ends, ties to the lowest index
  compact   a stored prefix reduced to its kept tokens, inside the store
  rope      rotary positions of queries and keys, and the table the key projection takes

`own` False: elementary torch operations.  `own` True: the library's entry points.
"""
import math

import numpy as np
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
        # one block of a single request against a long shared prefix: the smallest call of a step
        {"name": "weights_block_step", "op": "weights", "heads": "gqa28", "dtype": "bf16", "prefixes": "16384",
         "suffixes": "16", "decay": 0.9, "padded": False},
        # a layer of 16 requests sharing a prompt, first accumulation (nothing to add to)
        {"name": "weights_layer", "op": "weights", "heads": "mha32", "dtype": "bf16", "prefixes": "1024",
         "suffixes": ",".join(["256"] * 16), "decay": 0.0, "padded": False},
        # a mixed serving batch: several prefixes, ragged suffixes, some rows padding, running sum
        {"name": "weights_ragged_mix", "op": "weights", "heads": "mha32", "dtype": "bf16",
         "prefixes": "513,2047,1300,4001", "suffixes": "33,700,129,1|1024,77,512,300,96|250|31,640,200",
         "decay": 1.0, "padded": True},
        # the long-prefix stack: 32 requests of 1024 rows over 16384 cached keys, the largest call
        {"name": "weights_long_prefix", "op": "weights", "heads": "gqa28", "dtype": "bf16", "prefixes": "16384",
         "suffixes": ",".join(["1024"] * 32), "decay": 1.0, "padded": False},
        # one layer's choice for four KV heads: a quarter of a long prefix stays
        {"name": "select_layer", "op": "select", "rows": 4, "n": 16384, "keep": 4096, "first": 4, "last": 64,
         "ties": False},
        # every layer and head of a 28-layer stack at once, odd length, many equal weights
        {"name": "select_stack", "op": "select", "rows": 896, "n": 40001, "keep": 9999, "first": 4, "last": 33,
         "ties": True},
        # one layer after a step: an odd number of tokens kept of a short prefix
        {"name": "compact_layer", "op": "compact", "heads": "gqa28", "dtype": "bf16", "layers": 1, "m": 2047,
         "keep": 1001, "per_head": True},
        # four layers of a long prefix with 32 KV heads, half of it kept
        {"name": "compact_stack", "op": "compact", "heads": "mha32", "dtype": "bf16", "layers": 4, "m": 16384,
         "keep": 8192, "per_head": True},
        # the rows of one block of a block-diffusion step
        {"name": "rope_block_step", "op": "rope", "form": "rows", "heads": "gqa28", "dtype": "bf16", "rows": 16,
         "rot": 128, "interleaved": False, "scaling": "none", "inverse": False, "far": False},
        # the suffix rows of 32 requests, frequencies scaled for a long context
        {"name": "rope_suffix_rows", "op": "rope", "form": "rows", "heads": "gqa28", "dtype": "bf16", "rows": 32768,
         "rot": 128, "interleaved": False, "scaling": "yarn", "inverse": False, "far": False},
        # interleaved pairs over part of the head, 32-bit tensors, far positions, taken back
        {"name": "rope_partial_f32", "op": "rope", "form": "rows", "heads": "mha4", "dtype": "f32", "rows": 9973,
         "rot": 32, "interleaved": True, "scaling": "ntk", "inverse": True, "far": True},
        # the cosines and sines of a long prefix, as the key projection takes them
        {"name": "rope_table_prefix", "op": "rope", "form": "table", "heads": "gqa28", "dtype": "f32", "rows": 16384,
         "rot": 128, "interleaved": False, "scaling": "bands", "inverse": False, "far": False},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _limit(op):
    costs = [work(c) for c in listed() if c["op"] == op]
    return max(c["bytes"] for c in costs), max(c["flops"] for c in costs)


def draw(rng):
    op = rng.choice(["weights", "weights", "select", "compact", "rope", "rope"])
    max_bytes, max_flops = _limit(op)
    while True:
        if op == "weights":
            heads = rng.choice(list(HEADS))
            groups = rng.choice([1, 1, 1, 2, 3, 5, 8])
            prefixes = [_log_int(rng, 1, 16384) for _ in range(groups)]
            suffixes = ["%s" % ",".join(str(_log_int(rng, 1, 1024)) for _ in range(rng.randint(1, 12)))
                        for _ in range(groups)]
            c = {"op": op, "heads": heads, "dtype": "f32" if heads == "mha4" else "bf16",
                 "prefixes": ",".join(map(str, prefixes)), "suffixes": "|".join(suffixes),
                 "decay": rng.choice([0.0, 0.5, 0.9, 1.0]), "padded": rng.random() < 0.5}
        elif op == "select":
            n = _log_int(rng, 1, 131072)
            first, last = rng.choice([0, 1, 4]), rng.choice([0, 1, 32, 100])
            floor = max(1, min(n, first + last))
            c = {"op": op, "rows": _log_int(rng, 1, 896), "n": n, "keep": rng.randint(floor, n), "first": first,
                 "last": last, "ties": rng.random() < 0.5}
        elif op == "compact":
            heads = rng.choice(list(HEADS))
            m = _log_int(rng, 1, 16384)
            c = {"op": op, "heads": heads, "dtype": rng.choice(["bf16", "bf16", "f32"]),
                 "layers": rng.randint(1, 4), "m": m, "keep": rng.randint(1, m), "per_head": rng.random() < 0.7}
        else:
            heads = rng.choice(list(HEADS))
            d = HEADS[heads][2]
            form = rng.choice(["rows", "rows", "rows", "table"])
            c = {"op": op, "form": form, "heads": heads, "dtype": rng.choice(["bf16", "bf16", "f32"]),
                 "rows": _log_int(rng, 1, 32768), "rot": rng.choice([d, d, d // 2, d // 4, d - 20, 2]),
                 "interleaved": rng.random() < 0.5,
                 "scaling": rng.choice(["none", "linear", "ntk", "yarn", "bands"]),
                 "inverse": form == "rows" and rng.random() < 0.3, "far": rng.random() < 0.3}
            if form == "table":
                c["dtype"] = "f32"
        w = work(c)
        if w["bytes"] <= max_bytes and w["flops"] <= max_flops:
            return c


def _lengths(case):
    """prefix length and request lengths of every group"""
    return [(int(m), [int(n) for n in s.split(",")])
            for m, s in zip(case["prefixes"].split(","), case["suffixes"].split("|"))]


def work(case):
    op = case["op"]
    if op == "select":
        n = case["rows"] * case["n"]
        return {"bytes": 4 * n + 4 * case["rows"] * case["keep"], "flops": n}
    hq, hkv, d = HEADS[case["heads"]]
    es = 2 if case["dtype"] == "bf16" else 4
    if op == "weights":
        b = f = 0
        for m, ns in _lengths(case):
            b += m * hkv * d * es + sum(ns) * hq * (d * es + 4) + m * hkv * 4 * (2 if case["decay"] else 1)
            f += (2 * d + 3) * m * sum(ns) * hq             # the product, then scale, exponential and sum
        return {"bytes": b, "flops": f}
    if op == "compact":
        kept = 2 * case["layers"] * case["keep"] * hkv * d * es
        lists = 4 * case["layers"] * case["keep"] * (hkv if case["per_head"] else 1)
        return {"bytes": 3 * kept + lists, "flops": 0}      # read, the shortened prefix, its rows handed back
    if case["form"] == "table":
        n = case["rows"] * case["rot"]
        return {"bytes": 4 * case["rows"] + 4 * n, "flops": 10 * n}
    n = case["rows"] * (hq + hkv) * d
    return {"bytes": 4 * case["rows"] + 2 * n * es,
            "flops": 3 * case["rows"] * (hq + hkv) * case["rot"]}


# --------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------

SCALINGS = {        # kind -> (factor, original length, low, high) as the library's call takes them
    "none": (1.0, 0, 0.0, 0.0),
    "linear": (4.0, 0, 0.0, 0.0),
    "ntk": (8.0, 0, 0.0, 0.0),
    "yarn": (16.0, 4096, 1.0, 32.0),
    "bands": (8.0, 8192, 1.0, 4.0),
}
BASE = 10000.0


def _attention_scale(case):
    return 0.1 * math.log(SCALINGS["yarn"][0]) + 1.0 if case["scaling"] == "yarn" else 1.0


def _weights_inputs(case, seed):
    """K per group, queries of all requests, their log-sum-exps and the running scores."""
    hq, hkv, d = HEADS[case["heads"]]
    dtype = DTYPES[case["dtype"]]
    gen = _gen(seed, 11)
    groups = _lengths(case)
    gq, scale, std = hq // hkv, d ** -0.5, 1.5        # scores of a trained model spread wider than N(0, 1)
    total = sum(sum(ns) for _, ns in groups)
    q = _normal((total, hq, d), gen, dtype, std)
    ks = [_normal((m, hkv, d), gen, dtype) for m, _ in groups]
    lse = torch.empty((total, hq), dtype=torch.float32, device=DEV)
    row = 0
    for (m, ns), k in zip(groups, ks):
        n_rows = sum(ns)
        own_part = torch.log(torch.tensor([float(n) for n in ns for _ in range(n)], device=DEV)) + std * std / 2
        for h in range(hkv):
            kt = k[:, h].float().t().contiguous()
            step = max(1, (1 << 27) // (m * gq))
            for a in range(0, n_rows, step):
                b = min(n_rows, a + step)
                s = q[row + a:row + b, h * gq:(h + 1) * gq].float().reshape(-1, d) @ kt
                part = torch.logsumexp(s * scale, dim=1).view(b - a, gq)
                lse[row + a:row + b, h * gq:(h + 1) * gq] = torch.logaddexp(part, own_part[a:b, None])
        row += n_rows
    if case["padded"]:                                # rows that a batch carries along without a request's token
        pad = torch.rand(total, generator=gen, device=DEV) < 0.05
        lse[pad] = math.inf
    m_max = max(m for m, _ in groups)
    scores = torch.rand((len(groups), hkv, m_max), generator=gen, device=DEV) * 3.0
    return groups, q, ks, lse, scores, scale


def _select_inputs(case, seed):
    gen = _gen(seed, 12)
    # accumulated weights are positive and heavy-tailed; with `ties` many tokens were never attended to
    s = torch.exp(torch.randn((case["rows"], case["n"]), generator=gen, device=DEV) * 2.0 - 5.0)
    if case["ties"]:
        s = torch.where(s < 0.008, torch.zeros_like(s), (s * 256).round() / 256)
    return s


def _compact_inputs(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    gen = _gen(seed, 13)
    dtype = DTYPES[case["dtype"]]
    layers, m, keep = case["layers"], case["m"], case["keep"]
    k = _normal((layers, m, hkv, d), gen, dtype)
    v = _normal((layers, m, hkv, d), gen, dtype)
    order = torch.rand((layers, hkv if case["per_head"] else 1, m), generator=gen, device=DEV).argsort(dim=-1)
    idx = order[..., :keep].sort(dim=-1).values.to(torch.int32).contiguous()
    return k, v, idx


def _rope_inputs(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    gen = _gen(seed, 14)
    rows = case["rows"]
    if case["far"]:
        pos = torch.randint(0, 1 << 20, (rows,), generator=gen, device=DEV, dtype=torch.int32)
    else:                                             # runs of positions, as a batch of requests has them
        start = torch.randint(0, 16384, (rows // 1024 + 1,), generator=gen, device=DEV)
        i = torch.arange(rows, device=DEV)
        pos = (start[i // 1024] + i % 1024).to(torch.int32)
    if case["form"] == "table":
        return pos, None, None
    dtype = DTYPES[case["dtype"]]
    return pos, _normal((rows, hq, d), gen, dtype), _normal((rows, hkv, d), gen, dtype)


def prepare(case, seed):
    op = case["op"]
    state = {"case": case}
    if op == "select":
        state["scores"] = _select_inputs(case, seed)
        if own:
            from paper_2606_07571_b200 import binding
            state["bc"] = binding.BiCache(1, 1, 1, 128, 16, torch.bfloat16, 16, 1)
            state["idx"] = torch.empty((case["rows"], case["keep"]), dtype=torch.int32, device=DEV)
        return state
    hq, hkv, d = HEADS[case["heads"]]
    dtype = DTYPES[case["dtype"]]
    if op == "weights":
        groups, q, ks, lse, scores, scale = _weights_inputs(case, seed)
        state.update(groups=groups, q=q, lse=lse, scores=scores, scale=scale)
        if not own:
            state["ks"] = ks
            return state
        from paper_2606_07571_b200 import binding
        pages = sum((m + 15) // 16 for m, _ in groups)
        bc = binding.BiCache(1, hq, hkv, d, pages, dtype, q.shape[0], sum(len(ns) for _, ns in groups))
        ids, offs, lens, score_off, row = [], [], [], [], 0
        for g, ((m, ns), k) in enumerate(zip(groups, ks)):
            pid, _, _ = bc.put_prefix(g + 1, k[None], k[None])
            for n in ns:
                ids.append(pid)
                offs.append(row)
                lens.append(n)
                score_off.append(g * scores.stride(0))
                row += n
        out = torch.zeros_like(scores)
        state.update(bc=bc, ids=ids, offs=offs, lens=lens, score_off=score_off, out=out)
        return state
    if op == "compact":
        k, v, idx = _compact_inputs(case, seed)
        state.update(idx=idx)
        if not own:
            state.update(k=k, v=v)
            return state
        from paper_2606_07571_b200 import binding
        m, keep = case["m"], case["keep"]
        pages = (m + 15) // 16 + (keep + 15) // 16
        bc = binding.BiCache(case["layers"], hq, hkv, d, pages, dtype, 16, 1)
        src, _, _ = bc.put_prefix(1, k, v)
        dst, _, _ = bc.reserve_prefix(2, keep)
        state.update(bc=bc, src=src, dst=dst,
                     k_out=torch.empty((case["layers"], keep, hkv, d), dtype=dtype, device=DEV),
                     v_out=torch.empty((case["layers"], keep, hkv, d), dtype=dtype, device=DEV))
        return state
    pos, q, k = _rope_inputs(case, seed)
    state.update(pos=pos, q=q, k=k)
    if not own:
        state["freq"] = _frequencies(case).to(DEV)
        return state
    from paper_2606_07571_b200 import binding
    factor, length, low, high = SCALINGS[case["scaling"]]
    state["freq"] = binding.rope_frequencies(case["rot"], BASE, case["scaling"], factor, length, low, high)
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


def _weights_views(groups, scores):
    return [scores[g, :, :m] for g, (m, _) in enumerate(groups)]


def _weights_own(case, st):
    st["bc"].prefix_weights(0, st["ids"], st["offs"], st["lens"], st["q"], st["lse"], st["out"], st["score_off"],
                            scores_in=st["scores"] if case["decay"] else None, decay=case["decay"],
                            scale=st["scale"])
    return _weights_views(st["groups"], st["out"])


def _select_own(case, st):
    st["bc"].select_tokens(st["scores"], case["keep"], st["idx"], protect_first=case["first"],
                           protect_last=case["last"])
    return st["idx"]


def _compact_own(case, st):
    st["bc"].compact_prefix(st["src"], st["dst"], st["idx"])
    for layer in range(case["layers"]):
        st["bc"].read_prefix_layer(st["dst"], layer, st["k_out"][layer], st["v_out"][layer])
    return st["k_out"], st["v_out"]


def _rope_own(case, st):
    scale = _attention_scale(case)
    if case["form"] == "table":
        st["bc"].rope_table(st["freq"], st["table"], positions=st["pos"], attention_scale=scale)
        return st["table"]
    st["bc"].rope(st["freq"], st["q"], st["q_out"], st["k"], st["k_out"], positions=st["pos"],
                  interleaved=case["interleaved"], attention_scale=scale, inverse=case["inverse"])
    return st["q_out"], st["k_out"]


def _weights_plain(case, st):
    hq, hkv, d = HEADS[case["heads"]]
    gq = hq // hkv
    out = []
    row = 0
    for g, ((m, ns), k) in enumerate(zip(st["groups"], st["ks"])):
        n_rows = sum(ns)
        acc = torch.zeros((hkv, m), dtype=torch.float64, device=DEV)
        for h in range(hkv):
            kt = k[:, h].float().t().contiguous()
            step = max(1, (1 << 27) // (m * gq))
            for a in range(row, row + n_rows, step):
                b = min(row + n_rows, a + step)
                s = (st["q"][a:b, h * gq:(h + 1) * gq].float().reshape(-1, d) @ kt) * st["scale"]
                l = st["lse"][a:b, h * gq:(h + 1) * gq].reshape(-1, 1)
                w = torch.exp(s - l)
                acc[h] += torch.where(torch.isinf(l), torch.zeros_like(w), w).sum(dim=0)
        if case["decay"]:
            acc += case["decay"] * st["scores"][g, :, :m].double()
        out.append(acc.float())
        row += n_rows
    return out


def _select_plain(case, st):
    s = torch.where(torch.isnan(st["scores"]), torch.full_like(st["scores"], -math.inf), st["scores"])
    n = case["n"]
    first = min(case["first"], n)
    last = min(case["last"], n - first)
    inner = s[:, first:n - last]
    order = torch.sort(inner, dim=1, descending=True, stable=True).indices[:, :case["keep"] - first - last] + first
    ends = torch.cat([torch.arange(first, device=DEV), torch.arange(n - last, n, device=DEV)])
    kept = torch.cat([order, ends.expand(s.shape[0], -1)], dim=1)
    return kept.sort(dim=1).values.to(torch.int32)


def _compact_plain(case, st):
    idx = st["idx"].long().transpose(1, 2)[..., None]           # [layers][keep][heads or 1][1]
    idx = idx.expand(-1, -1, st["k"].shape[2], st["k"].shape[3])
    return torch.gather(st["k"], 1, idx), torch.gather(st["v"], 1, idx)


def _frequencies(case):
    """The angle per position of every pair, in 64 bits."""
    rot = case["rot"]
    factor, length, low, high = SCALINGS[case["scaling"]]
    i = torch.arange(rot // 2, dtype=torch.float64)
    base = BASE
    if case["scaling"] == "ntk" and rot > 2:                    # one pair alone is left as it is
        base = BASE * factor ** (rot / (rot - 2))
    f = base ** (-2.0 * i / rot)
    if case["scaling"] == "linear":
        f = f / factor
    elif case["scaling"] == "yarn":
        # the share of interpolation rises linearly with the pair's index, between the pairs that turn
        # `high` and `low` times over the original length
        def index(turns):
            return rot * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(BASE))
        lo = max(math.floor(index(high)), 0)
        hi = min(math.ceil(index(low)), rot - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f = f / factor * ramp + f * (1 - ramp)
    elif case["scaling"] == "bands":
        # the same, linear in the number of turns
        turns = length * f / (2 * math.pi)
        kept = ((turns - low) / (high - low)).clamp(0, 1)
        f = f / factor * (1 - kept) + f * kept
    return f


def _rope_plain(case, st):
    angle = st["pos"].double()[:, None] * st["freq"]
    scale = _attention_scale(case)
    cos, sin = torch.cos(angle), torch.sin(angle)
    if case["form"] == "table":
        return (torch.stack([cos, sin], dim=-1) * scale).float()
    if case["inverse"]:
        cos, sin = cos / scale, -sin / scale
    else:
        cos, sin = cos * scale, sin * scale
    cos, sin = cos.float()[:, None, :], sin.float()[:, None, :]
    rot = case["rot"]
    outs = []
    for x in (st["q"], st["k"]):
        xf = x.float()
        r = xf[..., :rot]
        if case["interleaved"]:
            a, b = r[..., 0::2], r[..., 1::2]
            y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
        else:
            a, b = r[..., :rot // 2], r[..., rot // 2:]
            y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
        outs.append(torch.cat([y, xf[..., rot:]], dim=-1).to(x.dtype))
    return tuple(outs)


_run_own = {"weights": _weights_own, "select": _select_own, "compact": _compact_own, "rope": _rope_own}
_run_plain = {"weights": _weights_plain, "select": _select_plain, "compact": _compact_plain, "rope": _rope_plain}


# --------------------------------------------------------------------------------------------
# the definition in 64 bits
# --------------------------------------------------------------------------------------------

def exact(case, seed):
    op = case["op"]
    if op == "weights":
        hq, hkv, d = HEADS[case["heads"]]
        groups, q, ks, lse, scores, scale = _weights_inputs(case, seed)
        out, row = [], 0
        for g, ((m, ns), k) in enumerate(zip(groups, ks)):
            total = case["decay"] * scores[g, :, :m].double() if case["decay"] else \
                torch.zeros((hkv, m), dtype=torch.float64, device=DEV)
            k64 = k.double()
            for head in range(hq):                              # head by head, a run of rows at a time
                kv = head // (hq // hkv)
                for a in range(row, row + sum(ns), 4096):
                    b = min(a + 4096, row + sum(ns))
                    s = torch.einsum("td,rd->tr", k64[:, kv], q[a:b, head].double()).mul_(scale)
                    l = lse[a:b, head].double()
                    s.sub_(torch.where(torch.isinf(l), torch.full_like(l, math.inf), l)).exp_()
                    total[kv] += s.sum(dim=1)
            out.append(total)
            row += sum(ns)
        return out
    if op == "select":
        s = _select_inputs(case, seed).cpu().numpy().astype(np.float64)
        n, keep = case["n"], case["keep"]
        s[np.isnan(s)] = -np.inf
        protected = np.zeros(n, dtype=bool)
        protected[:case["first"]] = True
        if case["last"]:
            protected[max(0, n - case["last"]):] = True
        res = np.empty((case["rows"], keep), dtype=np.int32)
        for r in range(case["rows"]):
            res[r] = np.sort(np.lexsort((np.arange(n), -s[r], ~protected))[:keep])
        return torch.from_numpy(res)
    if op == "compact":
        k, v, idx = _compact_inputs(case, seed)
        out_k, out_v = [], []
        for layer in range(case["layers"]):
            heads = range(k.shape[2])
            rows = [idx[layer, h if case["per_head"] else 0].long() for h in heads]
            out_k.append(torch.stack([k[layer, rows[h], h] for h in heads], dim=1))
            out_v.append(torch.stack([v[layer, rows[h], h] for h in heads], dim=1))
        return torch.stack(out_k).double(), torch.stack(out_v).double()
    pos, q, k = _rope_inputs(case, seed)
    turn = pos.double()[:, None] * _frequencies(case).to(DEV)
    phase = torch.polar(torch.ones_like(turn), turn)            # the pair as a complex number
    scale = _attention_scale(case)
    if case["form"] == "table":
        return torch.view_as_real(phase * scale)
    phase = phase.conj() / scale if case["inverse"] else phase * scale
    rot, res = case["rot"], []
    for x in (q, k):
        y = x.double()
        if case["interleaved"]:
            z = torch.view_as_complex(y[..., :rot].reshape(*y.shape[:2], rot // 2, 2).contiguous()) * phase[:, None]
            y[..., :rot] = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * phase[:, None]
            y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
        res.append(y)
    return tuple(res)
