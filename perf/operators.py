"""The 8-bit cache operators as they are timed: what each call is in use, its inputs, its bytes and flops, its exact result.

Four operators work on one cache of keys and values that is held in 8 bits with a 32-bit scale for each token and head:

  rope    rotary positions of query and key rows (halves or interleaved pairs, all or part of a head, frequencies scaled
          for long contexts), forward and as the gradient;
  cache   new rows are quantised into the cache and read back: what a step has appended, as the values it stands for;
  read    a prefix of the cache back in the model's type;
  attend  attention of new rows over the cache: single tokens, candidates to verify, prompts; shared heads; causal, with
          a sliding window behind a few first tokens, or over a cache that the rows are not part of.

The cache is four plain tensors, [kv_heads][tokens][head_dim] codes and [kv_heads][tokens] scales for K and V; sequence j
owns the rows off[j] .. off[j] + cap[j] of every head, and `length[j]` says how many tokens it held before the new rows.
"""
from __future__ import annotations

import math

import torch

own = False

SCALE_MIN = 2.0 ** -60
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one conversation's candidates (five and the pending token): q and k of 32 heads inside the packed projection
        {"name": "rope_step", "op": "rope", "dtype": "bf16", "rows": 6, "heads": 64, "packed": 96, "dim": 128, "rot": 128,
         "interleaved": False, "inverse": False, "scaling": "none", "far": 2048},
        # a long prompt's queries and keys at positions beyond the trained length
        {"name": "rope_prompt", "op": "rope", "dtype": "bf16", "rows": 8192, "heads": 40, "packed": 48, "dim": 128, "rot": 128,
         "interleaved": False, "inverse": False, "scaling": "bands", "far": 131072},
        # a training step's gradient through rotations of half of each head
        {"name": "rope_grad_part", "op": "rope", "dtype": "fp32", "rows": 1003, "heads": 24, "packed": 24, "dim": 64, "rot": 32,
         "interleaved": True, "inverse": True, "scaling": "ramp", "far": 16384},
        # the candidates of 32 conversations enter the cache of one layer of the 32-head target
        {"name": "cache_step", "op": "cache", "dtype": "bf16", "n": 32, "rows": 6, "ragged": False, "kv": 32, "dim": 128,
         "len": 2048},
        # five prompts of unequal length enter it
        {"name": "cache_prompt", "op": "cache", "dtype": "fp32", "n": 5, "rows": 8191, "ragged": True, "kv": 32, "dim": 128,
         "len": 513},
        # one conversation's short prefix of a 12-head draft, for a look at what the cache holds
        {"name": "read_prefix", "op": "read", "dtype": "fp32", "n": 1, "kv": 12, "dim": 64, "len": 777},
        # two long prefixes leave the cache for a path that works in 16 bits
        {"name": "read_long", "op": "read", "dtype": "bf16", "n": 2, "kv": 8, "dim": 128, "len": 32768},
        # a 12-head draft's next token over a short context: the smallest call, latency counts
        {"name": "attend_token", "op": "attend", "dtype": "fp32", "n": 1, "rows": 1, "ragged": False, "heads": 12, "kv": 12,
         "dim": 64, "len": 100, "causal": True, "window": 0, "sinks": 0},
        # the ordinary serving batch: the target verifies five candidates of each of 32 conversations
        {"name": "attend_verify", "op": "attend", "dtype": "bf16", "n": 32, "rows": 6, "ragged": False, "heads": 32, "kv": 32,
         "dim": 128, "len": 4096, "causal": True, "window": 0, "sinks": 0},
        # few conversations with very long contexts, four query heads to a key head
        {"name": "attend_long", "op": "attend", "dtype": "bf16", "n": 4, "rows": 6, "ragged": False, "heads": 32, "kv": 8,
         "dim": 128, "len": 65536, "causal": True, "window": 0, "sinks": 0},
        # drafts that look at the last 1024 tokens and the first four
        {"name": "attend_window", "op": "attend", "dtype": "fp32", "n": 16, "rows": 2, "ragged": False, "heads": 16, "kv": 16,
         "dim": 64, "len": 8192, "causal": True, "window": 1024, "sinks": 4},
        # pieces of three prompts, some with a context in front of them
        {"name": "attend_prompt", "op": "attend", "dtype": "bf16", "n": 3, "rows": 4095, "ragged": True, "heads": 32, "kv": 8,
         "dim": 128, "len": 4000, "causal": True, "window": 0, "sinks": 0},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["rope", "cache", "read", "attend", "attend", "attend"])
    dtype = rng.choice(["fp32", "bf16"])
    dim = rng.choice([64, 128])
    if op == "rope":
        heads = rng.randint(1, 64)
        most = 8192 * 40 * 128 // (heads * dim) // (2 if dtype == "fp32" else 1)
        return {"op": op, "dtype": dtype, "rows": _log(rng, 1, min(8192, most)), "heads": heads,
                "packed": heads + rng.choice([0, 0, 8, heads]), "dim": dim, "rot": rng.choice([dim, dim, dim // 2, dim // 4]),
                "interleaved": rng.random() < 0.5, "inverse": rng.random() < 0.5,
                "scaling": rng.choice(["none", "linear", "bands", "ramp"]), "far": _log(rng, 64, 1 << 20)}
    kv = rng.choice([1, 2, 4, 8, 12, 16, 32])
    if op == "cache":
        n = _log(rng, 1, 48)
        ragged = rng.random() < 0.5
        most = 8191 * 32 * 128 // (kv * dim)
        rows = _log(rng, n, min(most, 8191)) if ragged else _log(rng, 1, 16)
        return {"op": op, "dtype": dtype, "n": n, "rows": rows, "ragged": ragged, "kv": kv, "dim": dim, "len": _log(rng, 1, 2048)}
    if op == "read":
        n = _log(rng, 1, 32)
        most = 2 * 32768 * 8 * 128 // (n * kv * dim) // (2 if dtype == "fp32" else 1)
        return {"op": op, "dtype": dtype, "n": n, "kv": kv, "dim": dim, "len": _log(rng, 1, min(most, 32768))}
    group = rng.choice([1, 1, 2, 4, 5, 8])
    if kv * group > 40:
        group = 1
    causal = rng.random() < 0.85
    window = _log(rng, 1, 4096) if causal and rng.random() < 0.35 else 0
    sinks = rng.choice([0, 1, 4, 16]) if window else 0
    if causal and rng.random() < 0.3:  # prompts
        n = rng.randint(1, 4)
        rows = _log(rng, 17 * n, 4095 if dtype == "bf16" else 1024)
        return {"op": op, "dtype": dtype, "n": n, "rows": rows, "ragged": True, "heads": min(kv * group, 32) // kv * kv, "kv": kv,
                "dim": dim, "len": _log(rng, 1, 4000), "causal": True, "window": window, "sinks": sinks}
    n = _log(rng, 1, 48)
    most = 4 * 65536 * 8 * 128 // (n * kv * dim) // 2
    return {"op": op, "dtype": dtype, "n": n, "rows": _log(rng, 1, 16), "ragged": False, "heads": kv * group, "kv": kv, "dim": dim,
            "len": _log(rng, 1, max(1, min(most, 65536))), "causal": causal, "window": window, "sinks": sinks}


# ---------------------------------------------------------------- what a case says about its sequences
def _lengths(case):
    """Tokens that each sequence holds before the call: spread between an eighth of `len` and `len`, odd ones among them."""
    n, top = case["n"], case["len"]
    return [max(1, top - (j * 5 % n) * top * 7 // (8 * n)) for j in range(n)]


def _rows(case):
    """New rows of each sequence: `rows` of each, or (ragged) `rows` of all together, the first with the most."""
    n, rows = case["n"], case["rows"]
    if not case["ragged"]:
        return [rows] * n
    w = [n - j for j in range(n)]
    got = [max(1, rows * x // sum(w)) for x in w]
    got[0] += max(0, rows - sum(got))
    return got


def _frequencies(case):
    """Angle per position of each pair, after scaling by a factor of 8 from 8192 trained positions."""
    rot, base, factor, trained = case["rot"], 10000.0, 8.0, 8192.0
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if case["scaling"] == "linear":  # every position moves closer
        return [x / factor for x in f]
    if case["scaling"] == "bands":  # waves shorter than the trained length keep their frequency, longer ones are slowed
        low, high = 1.0, 4.0
        out = []
        for x in f:
            turns = trained * x / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - low) / (high - low)))
            out.append(keep * x + (1 - keep) * x / factor)
        return out
    if case["scaling"] == "ramp":  # the same by the pair's index, between the pairs that turn 32 times and once
        at = [rot * math.log(trained / (2 * math.pi * r)) / (2 * math.log(base)) for r in (32.0, 1.0)]
        lo, hi = max(0.0, math.floor(at[0])), min(rot - 1.0, math.ceil(at[1]))
        return [x * (1 - g) + x / factor * g for x, g in
                ((x, min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3)))) for i, x in enumerate(f))]
    return f


def _gain(case):
    return 0.1 * math.log(8.0) + 1.0 if case["scaling"] == "ramp" else 1.0


# ---------------------------------------------------------------- inputs
def _quantised(x):
    """Codes and scales of rows x [..., dim]: s = max|x| / 127 in 32 bits, the code is the integer nearest to x / s."""
    s = (x.float().abs().amax(-1) / 127.0).clamp_min(SCALE_MIN)
    return torch.round(x.double() / s.double().unsqueeze(-1)).to(torch.int8), s


def _rows_like(g, shape, dtype):
    """Key or value rows: a few channels are larger than the rest, and so are some tokens."""
    dev = g.device
    channel = torch.exp(0.5 * torch.randn(shape[-1], generator=g, device=dev))
    token = torch.exp(0.3 * torch.randn(shape[0], 1, 1, generator=g, device=dev))
    return (torch.randn(shape, generator=g, device=dev) * channel * token).to(dtype)


def _cache(case, g, lens, rows):
    """A cache whose sequences hold `lens` tokens and have room for `rows` more; the rows behind them hold old data."""
    kv, dim, dev = case["kv"], case["dim"], g.device
    cap = [a + b + 3 for a, b in zip(lens, rows)]
    off = [sum(cap[:j]) for j in range(len(cap))]
    st = {"tokens": sum(cap), "off": torch.tensor(off, dtype=torch.int64, device=dev),
          "cap": torch.tensor(cap, dtype=torch.int32, device=dev), "length": torch.tensor(lens, dtype=torch.int32, device=dev),
          "max_len": max(lens)}
    for name in ("k", "v"):
        codes = torch.empty(kv, st["tokens"], dim, dtype=torch.int8, device=dev)
        scales = torch.empty(kv, st["tokens"], device=dev)
        for h in range(kv):
            codes[h], s = _quantised(_rows_like(g, (st["tokens"], 1, dim), torch.float32)[:, 0])
            scales[h] = s
        st[name], st[name + "_scale"] = codes, scales
    return st


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    if case["op"] == "rope":
        rows, heads, dim = case["rows"], case["heads"], case["dim"]
        packed = torch.randn(rows, case["packed"], dim, generator=g, device=dev).to(dtype)
        first = max(0, case["far"] - rows - seed % 7)
        return {"case": case, "x": packed[:, :heads], "y": torch.empty(rows, heads, dim, dtype=dtype, device=dev),
                "pos": torch.arange(first, first + rows, dtype=torch.int32, device=dev),
                "freq": torch.tensor(_frequencies(case), dtype=torch.float64, device=dev), "gain": _gain(case)}
    lens, rows = _lengths(case), [0] * case["n"] if case["op"] == "read" else _rows(case)
    st = _cache(case, g, lens, rows)
    st["case"] = case
    kv, dim = case["kv"], case["dim"]
    if case["op"] == "read":
        rows = lens
    start = [sum(rows[:j]) for j in range(len(rows) + 1)]
    st["max_rows"], st["total"] = max(rows), start[-1]
    st["row_start"] = torch.tensor(start, dtype=torch.int32, device=dev)
    st["uniform"] = case["op"] != "read" and not case["ragged"]
    if case["op"] == "cache":
        st["new_k"], st["new_v"] = (_rows_like(g, (st["total"], kv, dim), dtype) for _ in range(2))
    if case["op"] in ("cache", "read"):
        st["out_k"], st["out_v"] = (torch.empty(st["total"], kv, dim, dtype=dtype, device=dev) for _ in range(2))
        st["zero"] = torch.zeros(case["n"], dtype=torch.int32, device=dev)
    else:
        heads = case["heads"]
        st["q"] = (1.3 * torch.randn(st["total"], heads, dim, generator=g, device=dev)).to(dtype)
        st["out"] = torch.empty(st["total"], heads, dim, dtype=dtype, device=dev)
        st["lse"] = torch.empty(st["total"], heads, device=dev)
        st["scale"] = dim ** -0.5
    return st


# ---------------------------------------------------------------- the operators
def _plain_rope(st):
    case, x = st["case"], st["x"].float()
    rot = case["rot"]
    angle = st["pos"].double()[:, None] * st["freq"]
    c, s = (st["gain"] * torch.cos(angle)).float()[:, None], (st["gain"] * torch.sin(angle)).float()[:, None]
    if case["inverse"]:
        s = -s
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack((a, b), -1).flatten(-2) if case["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., rot:]), -1).to(st["x"].dtype)


def _owner(st):
    """Of each row: the sequence it belongs to, and its place among that sequence's rows."""
    r = torch.arange(st["total"], device=st["row_start"].device)
    j = torch.searchsorted(st["row_start"], r.to(torch.int32), right=True) - 1
    return j, r - st["row_start"].long()[j]


def _plain_cache(st):
    out = {}
    for name in ("k", "v"):
        codes, s = _quantised(st["new_" + name])
        out[name] = (codes.float() * s.unsqueeze(-1)).to(st["new_" + name].dtype)
    return out


def _plain_read(st):
    j, i = _owner(st)
    at = st["off"][j] + i
    return {n: (st[n][:, at].float() * st[n + "_scale"][:, at].unsqueeze(-1)).to(st["out_k"].dtype).transpose(0, 1) for n in ("k", "v")}


def _plain_attend(st):
    case, dev = st["case"], st["q"].device
    n, heads, kv, dim = case["n"], case["heads"], case["kv"], case["dim"]
    r_max, t_max, grp = st["max_rows"], st["max_len"] + (st["max_rows"] if case["causal"] else 0), heads // kv
    t = torch.arange(t_max, device=dev)
    at = torch.minimum(st["off"][:, None] + t, (st["off"] + st["cap"] - 1)[:, None])
    k, v = (st[x][:, at].float() * st[x + "_scale"][:, at].unsqueeze(-1) for x in ("k", "v"))  # [kv][n][t][dim]
    i = torch.arange(r_max, device=dev)
    rows = torch.clamp(st["row_start"].long()[:-1, None] + i, max=st["total"] - 1)
    q = st["q"][rows].float().view(n, r_max, kv, grp, dim).permute(2, 0, 3, 1, 4).reshape(kv, n, grp * r_max, dim)
    pos = st["length"].long()[:, None] + (i if case["causal"] else -1 + 0 * i)  # last token that a row sees
    seen = t <= pos[..., None]
    if case["window"]:
        seen &= (t > pos[..., None] - case["window"]) | (t < case["sinks"])
    s = torch.matmul(q, k.transpose(-1, -2)).view(kv, n, grp, r_max, t_max) * st["scale"]
    s = torch.where(seen[:, None], s, -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(kv, n, grp * r_max, t_max), v).view(kv, n, grp, r_max, dim) / torch.where(total == 0, 1.0, total)
    j, i = _owner(st)
    out = o.permute(1, 3, 0, 2, 4).reshape(n, r_max, heads, dim)[j, i]
    lse = (m + torch.log(total)).squeeze(-1).permute(1, 3, 0, 2).reshape(n, r_max, heads)[j, i]
    return {"out": out.to(st["q"].dtype), "lse": lse}


def run(st):
    case = st["case"]
    if not own:
        return {"rope": _plain_rope, "cache": _plain_cache, "read": _plain_read, "attend": _plain_attend}[case["op"]](st)
    from paper_2505_08600_amd import api
    if case["op"] == "rope":
        return api.sd_rope(st["x"], st["pos"], st["freq"], out=st["y"], interleaved=case["interleaved"],
                           inverse=case["inverse"], gain=st["gain"])
    cache = api.Kv8Cache(st["k"], st["v"], st["k_scale"], st["v_scale"], st["off"], st["cap"])
    row_start = None if st["uniform"] else st["row_start"]
    if case["op"] == "cache":
        api.sd_kv8_append(cache, st["length"], st["new_k"], st["new_v"], row_start=row_start)
        api.sd_kv8_read(cache, st["length"], st["out_k"], st["out_v"], row_start=row_start)
        return {"k": st["out_k"], "v": st["out_v"]}
    if case["op"] == "read":
        api.sd_kv8_read(cache, st["zero"], st["out_k"], st["out_v"], row_start=row_start)
        return {"k": st["out_k"], "v": st["out_v"]}
    api.sd_kv8_attend(cache, st["length"], st["q"], st["out"], st["scale"], row_start=row_start, max_rows=st["max_rows"],
                      max_len=st["max_len"], causal=case["causal"], window=case["window"], sinks=case["sinks"], lse=st["lse"])
    return {"out": st["out"], "lse": st["lse"]}


# ---------------------------------------------------------------- bytes and flops
def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    dim = case["dim"]
    if case["op"] == "rope":
        values = case["rows"] * case["heads"] * dim
        return {"bytes": 2 * values * size + 4 * case["rows"] + 4 * case["rot"], "flops": 3 * case["rows"] * case["heads"] * case["rot"]}
    kv = case["kv"]
    if case["op"] == "cache":  # rows in, codes and scales out and in again, values out
        vectors = 2 * sum(_rows(case)) * kv
        return {"bytes": vectors * (2 * dim * size + 2 * (dim + 4)), "flops": vectors * dim * 4}
    if case["op"] == "read":
        vectors = 2 * sum(_lengths(case)) * kv
        return {"bytes": vectors * (dim * size + dim + 4), "flops": vectors * dim}
    tokens = pairs = 0
    for length, rows in zip(_lengths(case), _rows(case)):
        held = length + (rows if case["causal"] else 0)
        seen = [min(length + i + 1, held) if case["causal"] else length for i in range(rows)]
        w, s = case["window"], case["sinks"]
        if w:  # the tokens that any row sees: the first ones, and those from the first row's window on
            first = max(0, seen[0] - w)
            tokens += held - first + min(s, first)
            seen = [min(x, w) + min(s, max(0, x - w)) for x in seen]
        else:
            tokens += held
        pairs += sum(seen)
    values = sum(_rows(case)) * case["heads"]
    return {"bytes": 2 * tokens * kv * (dim + 4) + 2 * values * dim * size + 4 * values, "flops": 4 * pairs * case["heads"] * dim}


# ---------------------------------------------------------------- the same from the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        rot, x = case["rot"], st["x"].double()
        turn = torch.polar(torch.full_like(st["freq"], st["gain"]).expand(case["rows"], -1).contiguous(),
                           (-1.0 if case["inverse"] else 1.0) * st["pos"].double()[:, None] * st["freq"])
        pair = x[..., :rot].unflatten(-1, (-1, 2) if case["interleaved"] else (2, -1))
        if not case["interleaved"]:
            pair = pair.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn[:, None])
        if not case["interleaved"]:
            z = z.transpose(-1, -2)
        y = x.clone()
        y[..., :rot] = z.reshape(x[..., :rot].shape)
        return y
    if case["op"] == "cache":
        out = {}
        for name in ("k", "v"):
            x = st["new_" + name].double()
            s = (x.abs().max(-1, keepdim=True).values.float() / 127).clamp_min(SCALE_MIN).double()
            out[name] = (x / s).round() * s
        return out
    parts = {"k": [], "v": []} if case["op"] == "read" else {"out": [], "lse": []}
    lens = _lengths(case)
    rows = lens if case["op"] == "read" else _rows(case)
    off, first = 0, 0
    for length, r, cap in zip(lens, rows, st["cap"].tolist()):
        def held(name, h, upto):
            return st[name][h, off:off + upto].double() * st[name + "_scale"][h, off:off + upto].double()[..., None]
        if case["op"] == "read":
            for name in parts:
                parts[name].append(held(name, slice(None), length).transpose(0, 1))
        else:
            upto = length + (r if case["causal"] else 0)
            token = torch.arange(upto, device=st["q"].device)[None]
            last = (torch.arange(r, device=st["q"].device)[:, None] + length) if case["causal"] else torch.full_like(token[:1, :1], length - 1)
            hidden = token > last
            if case["window"]:
                hidden |= (token <= last - case["window"]) & (token >= case["sinks"])
            grp = case["heads"] // case["kv"]
            out = torch.empty(r, case["heads"], case["dim"], dtype=torch.float64, device=st["q"].device)
            lse = torch.empty(r, case["heads"], dtype=torch.float64, device=st["q"].device)
            for h in range(case["heads"]):
                if h % grp == 0:
                    k, v = held("k", h // grp, upto), held("v", h // grp, upto)
                z = (st["q"][first:first + r, h].double() @ k.T * st["scale"]).masked_fill(hidden, -math.inf)
                out[:, h] = torch.softmax(z, -1) @ v
                lse[:, h] = torch.logsumexp(z, -1)
            parts["out"].append(out)
            parts["lse"].append(lse)
        off, first = off + cap, first + r
    return {name: torch.cat(x) for name, x in parts.items()}
