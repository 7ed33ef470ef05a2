"""Performance cases of the operators that stand between and behind the products of a decode step: rotary positions of q and k, the
cache of keys and values held in 4 bits (new tokens written and read back), the attention over it, and the choice of the next token
from the logits.

Sizes are those of the 7B-, 8B- and 70B-shaped layers and generic ones.  Queries, keys and values are synthetic: N(0, 1), keys with a few
channels much larger than the others, as trained models have them; logits are N(0, 1) times a spread with a handful of likely tokens on top.

The 4-bit format: for every token and head, groups of 32 channels share m = fp16(smallest value) and s = fp16((largest - smallest) / 15,
computed in fp32); a channel's code is (x - m) / s rounded to the nearest whole number (ties to even), 0..15, and stands for s * code + m.
A framework's program keeps such a cache in pages, a plain one as rows of packed codes: that is what prepare() goes by `own` in.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_GROUP = 32


# ------------------------------------------------------------------------------------------------ cases

def _attend(name, seqs, heads, kv_heads, dim, cached, new=1, ragged=True, window=0, sinks=0, page=64, dtype="bf16"):
    return {"name": name, "op": "attend", "seqs": seqs, "heads": heads, "kv_heads": kv_heads, "dim": dim, "cached": cached, "new": new,
            "ragged": ragged, "window": window, "sinks": sinks, "page": page, "dtype": dtype}


def _cache(name, seqs, kv_heads, dim, cached, new, ragged=True, page=64, dtype="bf16"):
    return {"name": name, "op": "cache", "seqs": seqs, "kv_heads": kv_heads, "dim": dim, "cached": cached, "new": new, "ragged": ragged,
            "page": page, "dtype": dtype}


def _rotary(name, tokens, heads, kv_heads, dim, rot, sections, pairing="halves", in_turn=False, far=4096, dtype="bf16"):
    return {"name": name, "op": "rotary", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rot, "sections": sections,
            "pairing": pairing, "in_turn": in_turn, "far": far, "dtype": dtype}


def _sample(name, rows, vocab, kind, temperature, top_k, top_p, min_p):
    return {"name": name, "op": "sample", "rows": rows, "vocab": vocab, "kind": kind, "temperature": temperature, "top_k": top_k,
            "top_p": top_p, "min_p": min_p}


def listed():
    return [
        # one user's token in an 8B-shaped layer with 4096 tokens behind it: latency counts
        _attend("attend_8b_b1", 1, 32, 8, 128, 4095, ragged=False),
        # a full 70B-shaped decode batch, contexts of many lengths up to 8192: the largest read of a cache
        _attend("attend_70b_b40", 40, 64, 8, 128, 8191),
        # 7B-shaped layer (a key head for every query head) with a window of 1024 and four first tokens that stay visible, small pages
        _attend("attend_7b_window_b16", 16, 32, 32, 128, 6000, window=1024, sinks=4, page=16, dtype="fp16"),
        # prompts of eight users that go through the layer in pieces of 48 tokens, 8B-shaped
        _attend("attend_8b_pieces_b8", 8, 32, 8, 128, 2000, new=48),
        # three drafted tokens to be checked at once, odd group of heads and head size, odd lengths, pages that are no power of two
        _attend("attend_drafts_b5", 5, 28, 4, 96, 774, new=3, page=48, dtype="fp16"),
        # the new token of each of 64 users goes into the cache, 8B-shaped
        _cache("cache_8b_b64", 64, 8, 128, 1500, 1),
        # three prompts of some thousand tokens go into the cache, 70B-shaped
        _cache("cache_prompts", 3, 8, 128, 100, 3500),
        # q and k of one token far into a long text, 8B-shaped
        _rotary("rotary_8b_b1", 1, 32, 8, 128, 128, "64", far=100000),
        # image and video tokens with positions in time, height and width
        _rotary("rotary_video", 5003, 28, 4, 128, 128, "24,20,20", in_turn=True, far=2000),
        # one user, a small vocabulary, the usual top-k and top-p
        _sample("sample_32k_b1", 1, 32000, "f32", 0.8, 50, 0.9, 0.0),
        # a decode batch, a large vocabulary, top-p alone on a flat distribution
        _sample("sample_128k_b64", 64, 128000, "f32", 1.0, 0, 0.95, 0.0),
        # many users, logits in 16 bits with their many ties, odd vocabulary, all the cuts at once
        _sample("sample_150k_bf16_b200", 200, 150001, "bf16", 1.3, 400, 0.97, 0.02),
    ]


def _log_size(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choices(["attend", "cache", "rotary", "sample"], [45, 15, 20, 20])[0]
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if op == "sample":
        rows = _log_size(rng, 1, 256)
        vocab = _log_size(rng, 1000, min(200000, 200 * 150001 // rows))
        return {"op": op, "rows": rows, "vocab": vocab, "kind": rng.choice(["f32", "f32", "bf16", "fp16"]), "temperature": rng.choice([0.6, 0.8, 1.0, 1.3]),
                "top_k": rng.choice([0, _log_size(rng, 1, 1000)]), "top_p": rng.choice([1.0, round(rng.uniform(0.3, 0.99), 3)]),
                "min_p": rng.choice([0.0, 0.0, round(rng.uniform(0.005, 0.2), 3)])}
    dim = rng.choice([64, 96, 128, 128, 128, 192, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
    group = rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
    group = min(group, 64 // kv_heads)
    if op == "rotary":
        rot = rng.choice([dim, dim, dim // 2])
        tokens = _log_size(rng, 1, min(16384, 2 * 10 ** 8 // (kv_heads * (group + 1) * dim) // 4))
        axes = rng.choice([1, 1, 2, 3])
        cuts = sorted(rng.randint(1, rot // 2 - 1) for _ in range(axes - 1))
        sections = [b - a for a, b in zip([0] + cuts, cuts + [rot // 2])]
        return {"op": op, "tokens": tokens, "heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim, "rot": rot,
                "sections": ",".join(str(max(0, s)) for s in sections), "pairing": rng.choice(["halves", "halves", "neighbours"]),
                "in_turn": axes > 1 and rng.random() < 0.5, "far": _log_size(rng, 100, 1000000), "dtype": dtype}
    page = rng.choice([16, 16, 32, 48, 64, 64, 128, 256])
    if op == "cache":
        seqs = _log_size(rng, 1, 128)
        most = 3 * 3500 * 8 * 128 // (seqs * kv_heads * dim)
        new = rng.choice([1, _log_size(rng, 1, max(2, min(4000, most)))])
        return {"op": op, "seqs": seqs, "kv_heads": kv_heads, "dim": dim, "cached": _log_size(rng, 1, 2000), "new": new, "ragged": rng.random() < 0.8,
                "page": page, "dtype": dtype}
    seqs = _log_size(rng, 1, 64)
    most = 40 * 8192 * 8 * 128 * 2 // 3 // (seqs * kv_heads * dim)            # what one sequence may hold: no draw reads more than the largest listed case
    cached = _log_size(rng, 1, max(16, min(16384, most)))
    new = 1
    if rng.random() < 0.35:                                                  # nor computes more than the listed pieces of prompts
        new = _log_size(rng, 2, max(2, min(160, 8 * 32 * 128 * 48 * 2048 // (seqs * kv_heads * group * dim * (cached + 100)))))
    window = rng.choice([0, 0, _log_size(rng, 16, 4096)])
    return {"op": op, "seqs": seqs, "heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim, "cached": cached, "new": new,
            "ragged": rng.random() < 0.8, "window": window, "sinks": rng.choice([0, 1, 4, 64]) if window else 0, "page": page, "dtype": dtype}


def _spans(case):
    """(tokens in the cache before, new tokens) of every sequence."""
    if not case["ragged"]:
        return [(case["cached"], case["new"])] * case["seqs"]
    rng = random.Random(case["seqs"] * 1000003 + case["cached"] * 31 + case["new"])
    spans = []
    for i in range(case["seqs"]):
        cached = case["cached"] if i == 0 else int(case["cached"] * rng.uniform(0.1, 1.0))
        new = case["new"] if i == 0 or case["op"] == "attend" and case["new"] == 1 else max(1, int(case["new"] * rng.uniform(0.3, 1.0)))
        spans.append((cached, new))
    return spans


def _axes(case):
    """The axis of every pair."""
    sections = [int(s) for s in case["sections"].split(",")]
    if not case["in_turn"]:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    left, axes = list(sections), []
    while any(left):
        for a in range(len(left)):
            if left[a]:
                axes.append(a)
                left[a] -= 1
    return axes


# ------------------------------------------------------------------------------------------------ inputs

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    half = _TYPES[case.get("dtype", "bf16")]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    if case["op"] == "sample":
        x = randn(case["rows"], case["vocab"]) * 2.0
        likely = torch.randint(case["vocab"], (case["rows"], 8), generator=gen, device="cuda")
        x.scatter_add_(1, likely, randn(case["rows"], 8) * 3.0 + 6.0)
        d = {"logits": x.to(_TYPES[case["kind"]]), "uniform": torch.rand(case["rows"], generator=gen, device="cuda", dtype=torch.float32)}
        for name, dtype in (("temperature", torch.float32), ("top_k", torch.int32), ("top_p", torch.float32), ("min_p", torch.float32)):
            d[name] = torch.full((case["rows"],), case[name], dtype=dtype, device="cuda")
        return d
    if case["op"] == "rotary":
        n, axes = case["tokens"], len(case["sections"].split(","))
        d = {"q": randn(n, case["heads"], case["dim"]).to(half), "k": randn(n, case["kv_heads"], case["dim"]).to(half)}
        d["positions"] = torch.randint(case["far"], (axes, n), generator=gen, device="cuda", dtype=torch.int32)
        pairs = torch.arange(case["rot"] // 2, device="cuda", dtype=torch.float64)
        d["frequencies"] = (500000.0 ** (-2.0 * pairs / case["rot"])).float()
        return d
    spans = _spans(case)
    total = sum(c + n for c, n in spans)
    fresh = sum(n for _, n in spans)
    shape = (fresh if case["op"] == "cache" else total, case["kv_heads"], case["dim"])
    k = randn(*shape)
    k[:, :, :: case["dim"] // 4] *= 4
    d = {"k": k.to(half), "v": randn(*shape).to(half)}
    if case["op"] == "attend":
        q = randn(fresh, case["heads"], case["dim"]) * 1.5
        q[:, :, :: case["dim"] // 4] *= 0.5
        d["q"] = q.to(half)
    return d


# ------------------------------------------------------------------------------------------------ what a program of the framework keeps

def _starts(counts):
    starts = [0]
    for n in counts:
        starts.append(starts[-1] + n)
    return torch.tensor(starts, dtype=torch.int32, device="cuda")


def _own_state(case, d, seed):
    import paper_2502_00922_b200 as hl
    if case["op"] == "sample":
        tokens = torch.empty(case["rows"], dtype=torch.int32, device="cuda")
        kind, dtype = (hl.ELEM_F32, hl.BF16) if case["kind"] == "f32" else (hl.ELEM_16, hl.BF16 if case["kind"] == "bf16" else hl.FP16)
        call = hl.PreparedSampling(hl.Sampling(d["logits"], kind, case["rows"], case["vocab"], d["uniform"], tokens, dtype=dtype,
                                               temperature=d["temperature"], top_k=d["top_k"], top_p=d["top_p"], min_p=d["min_p"]))
        return {"calls": [call], "outs": [tokens]}
    dtype = hl.BF16 if case["dtype"] == "bf16" else hl.FP16
    if case["op"] == "rotary":
        outs = [torch.empty_like(d["q"]), torch.empty_like(d["k"])]
        call = hl.PreparedRotary(hl.Rotary(dtype, case["tokens"], case["dim"], d["positions"], d["frequencies"], d["q"], case["heads"], outs[0],
                                           d["k"], case["kv_heads"], outs[1], rotary_dim=case["rot"],
                                           sections=[int(s) for s in case["sections"].split(",")],
                                           in_turn=case["in_turn"], pairing=hl.PAIR_HALVES if case["pairing"] == "halves" else hl.PAIR_NEIGHBOURS))
        return {"calls": [call], "outs": outs}
    spans = _spans(case)
    used = [-(-(c + n) // case["page"]) for c, n in spans]
    order = list(range(sum(used) + 3))                                # pages come from the pool in any order
    random.Random(seed).shuffle(order)
    table = torch.full((len(spans), max(used)), -1, dtype=torch.int32)
    for i, n in enumerate(used):
        table[i, :n] = torch.tensor(order[:n], dtype=torch.int32)
        order = order[n:]
    table = table.cuda()
    lengths = torch.tensor([c + n for c, n in spans], dtype=torch.int32, device="cuda")
    cache = hl.Cache(dtype, case["kv_heads"], case["dim"], case["page"], sum(used) + 3, None, table, lengths)
    pool = torch.zeros(hl.cache_bytes(cache), dtype=torch.uint8, device="cuda")
    cache = hl.Cache(dtype, case["kv_heads"], case["dim"], case["page"], sum(used) + 3, pool, table, lengths)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    fresh = _starts([n for _, n in spans])
    rows = sum(n for _, n in spans)
    if case["op"] == "cache":
        outs = [torch.empty_like(d["k"]), torch.empty_like(d["v"])]
        calls = [hl.PreparedAppend(cache, d["k"], d["v"], rows, starts=fresh, err_flag_dev=err),
                 hl.PreparedRead(cache, outs[0], outs[1], hl.ELEM_16, rows, starts=fresh, err_flag_dev=err)]
        return {"calls": calls, "outs": outs}
    everything = _starts([c + n for c, n in spans])
    hl.cache_append(cache, d["k"], d["v"], d["k"].shape[0], starts=everything, err_flag_dev=err)
    out = torch.empty_like(d["q"])
    attention = hl.Attention(d["q"], case["heads"], out, rows, scale=case["dim"] ** -0.5, starts=None if case["new"] == 1 else fresh,
                             window=case["window"], sinks=case["sinks"])
    n = hl.attention_workspace_bytes(cache, attention)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    return {"calls": [hl.PreparedAttention(cache, attention, ws, n, err)], "outs": [out]}


def prepare(case, seed):
    d = _inputs(case, seed)
    if own:
        return _own_state(case, d, seed)
    if case["op"] == "attend":                                        # the cache as rows of packed codes
        d = {"q": d["q"], "k": _pack(*_quantise(d["k"])), "v": _pack(*_quantise(d["v"]))}
    return {"case": case, "in": d}


# ------------------------------------------------------------------------------------------------ one pass

def _quantise(x):
    """Codes, scales and offsets of rows [tokens][heads][dim]."""
    x = x.float().unflatten(-1, (-1, _GROUP))
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    m, s = low.half(), ((high - low) / 15).half()
    codes = []
    for part, pm, ps in zip(x.split(4096), m.split(4096), s.split(4096)):    # in 64 bits: next to a border 32 would take either code
        c = torch.round((part.double() - pm.double()) / torch.where(ps == 0, 1.0, ps.double()))
        codes.append(torch.where(ps == 0, 0.0, c).clamp(0, 15).to(torch.uint8))
    return torch.cat(codes), s, m


def _pack(codes, s, m):
    return codes[..., 0::2] | codes[..., 1::2] << 4, s, m


def _unpack(packed, s, m):
    codes = torch.stack([packed & 15, packed >> 4], -1).flatten(-2)
    return (codes.float() * s.float() + m.float()).flatten(-2)


def _rotate(x, cos, sin, case):
    x, r = x.float(), case["rot"]
    if case["pairing"] == "halves":
        a, b = x[..., : r // 2], x[..., r // 2: r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., r:]], -1).to(_TYPES[case["dtype"]])


def _choose(d):
    x = d["logits"].float()
    x, index = torch.sort(x, dim=1, descending=True, stable=True)
    w = torch.exp(((x - x[:, :1]) / d["temperature"][:, None]).double())     # sums over a vocabulary: in 64 bits
    place = torch.arange(x.shape[1], device=x.device)[None]
    top_k = d["top_k"][:, None]
    keep = (place < top_k) | (top_k <= 0)
    w = w * keep
    mass = torch.cumsum(w, 1)
    top_p = d["top_p"].double()[:, None]
    keep &= (mass - w < top_p * mass[:, -1:]) | (top_p >= 1)
    keep &= w >= d["min_p"].double()[:, None]
    back = torch.zeros_like(w).scatter_(1, index, w * keep)                  # in the vocabulary's order again
    mass = torch.cumsum(back, 1)
    return torch.argmax((mass > d["uniform"].double()[:, None] * mass[:, -1:]).byte(), 1).int()


def run(state):
    if own:
        stream = torch.cuda.current_stream().cuda_stream
        for call in state["calls"]:
            call.run(stream)
        return state["outs"]
    case, d = state["case"], state["in"]
    if case["op"] == "sample":
        return [_choose(d)]
    if case["op"] == "rotary":
        axes = torch.tensor(_axes(case), device="cuda")
        angle = d["positions"].double()[axes].T * d["frequencies"].double()   # far positions: in 64 bits
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        return [_rotate(d["q"], cos, sin, case), _rotate(d["k"], cos, sin, case)]
    half = _TYPES[case["dtype"]]
    if case["op"] == "cache":
        return [_unpack(*_pack(*_quantise(x))).to(half) for x in (d["k"], d["v"])]
    outs, at, row = [], 0, 0
    group = case["heads"] // case["kv_heads"]
    for cached, new in _spans(case):
        n = cached + new
        first = max(0, cached - case["window"] + 1) if case["window"] else 0
        first = 0 if first <= case["sinks"] else first
        seen = torch.arange(n, device="cuda")                                # tokens that some row sees
        if first:
            seen = torch.cat([seen[: case["sinks"]], seen[first:]])
        parts = [slice(at, at + n)] if not first else [slice(at, at + case["sinks"]), slice(at + first, at + n)]
        k, v = (torch.cat([_unpack(*(t[p] for t in d[x])) for p in parts]) for x in ("k", "v"))
        q = d["q"][row: row + new].float().unflatten(1, (case["kv_heads"], group))
        scores = torch.matmul(q.permute(1, 2, 0, 3).flatten(1, 2), k.permute(1, 2, 0)) * case["dim"] ** -0.5
        pos = torch.arange(cached, n, device="cuda")[:, None]
        visible = seen <= pos
        if case["window"]:
            visible &= (seen > pos - case["window"]) | (seen < case["sinks"])
        scores = scores.unflatten(1, (group, new)).masked_fill(~visible, float("-inf"))
        p = torch.exp(scores - scores.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        o = torch.matmul(p.flatten(1, 2), v.permute(1, 0, 2)).unflatten(1, (group, new))
        outs.append(o.permute(2, 0, 1, 3).flatten(1, 2).to(half))
        at, row = at + n, row + new
    return [torch.cat(outs)]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    op = case["op"]
    if op == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (4 if case["kind"] == "f32" else 2) + 24 * case["rows"], "flops": 4 * n}
    if op == "rotary":
        n = case["tokens"] * (case["heads"] + case["kv_heads"])
        return {"bytes": 4 * n * case["dim"] + 4 * case["tokens"] * len(case["sections"].split(",")) + 2 * case["rot"], "flops": 3 * n * case["rot"]}
    spans = _spans(case)
    if op == "cache":
        n = 2 * sum(new for _, new in spans) * case["kv_heads"] * case["dim"]
        return {"bytes": 4 * n + n * 5 // 8, "flops": 6 * n}
    read = pairs = 0
    for cached, new in spans:
        first = max(0, cached - case["window"] + 1) if case["window"] else 0
        read += cached + new - max(0, first - case["sinks"])
        for i in range(new):
            first = max(0, cached + i - case["window"] + 1) if case["window"] else 0
            pairs += cached + i + 1 - max(0, first - case["sinks"])
    rows = sum(new for _, new in spans)
    return {"bytes": 2 * read * case["kv_heads"] * case["dim"] * 5 // 8 + 4 * rows * case["heads"] * case["dim"],
            "flops": 4 * pairs * case["heads"] * case["dim"]}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits

def _stands_for(x):
    """What the cache's codes of x stand for, in 64 bits."""
    groups = x.float().reshape(-1, _GROUP)
    out = torch.empty(groups.shape, dtype=torch.float64, device=x.device)
    for at in range(0, groups.shape[0], 1 << 20):
        g = groups[at: at + (1 << 20)]
        low = g.min(1).values
        offset = low.to(torch.float16).double()[:, None]
        scale = ((g.max(1).values - low) / 15.0).to(torch.float16).double()[:, None]
        code = ((g.double() - offset) / scale).nan_to_num(0.0, 0.0, 0.0).round().clamp(0.0, 15.0)
        out[at: at + (1 << 20)] = scale * code + offset
    return out.reshape(x.shape)


def _exact_token(x, t, k, p, least, u):
    x = x.double()
    weight = torch.exp((x - x.max()) / t)
    order = torch.sort(x, descending=True, stable=True).indices
    if k > 0:
        order = order[:k]
    if p < 1:
        before = torch.cumsum(weight[order], 0) - weight[order]
        order = order[before < p * weight[order].sum()]
    order = order[weight[order] >= least]
    kept = order.sort().values
    running = torch.cumsum(weight[kept], 0)
    return kept[min(int((running <= u * running[-1]).sum()), kept.numel() - 1)]


def exact(case, seed):
    """What run() returns for these inputs, in 64 bits."""
    d, op = _inputs(case, seed), case["op"]
    if op == "sample":
        row = [_exact_token(x, *(d[n][i].double().item() for n in ("temperature",)), int(d["top_k"][i]), d["top_p"][i].double().item(),
                            d["min_p"][i].double().item(), d["uniform"][i].double().item()) for i, x in enumerate(d["logits"])]
        return [torch.stack(row).int()]
    if op == "cache":
        return [_stands_for(d["k"]), _stands_for(d["v"])]
    if op == "rotary":
        which, half = _axes(case), case["rot"] // 2
        outs = [d["q"].double(), d["k"].double()]
        for x in outs:
            for i in range(half):
                angle = (d["positions"][which[i]].double() * d["frequencies"][i].double())[:, None]
                at = (i, i + half) if case["pairing"] == "halves" else (2 * i, 2 * i + 1)
                z = torch.complex(x[..., at[0]], x[..., at[1]]) * torch.complex(torch.cos(angle), torch.sin(angle))
                x[..., at[0]], x[..., at[1]] = z.real, z.imag
        return outs
    out = torch.zeros(d["q"].shape, dtype=torch.float64, device="cuda")
    group, at, row = case["heads"] // case["kv_heads"], 0, 0
    for cached, new in _spans(case):
        n = cached + new
        pos, key = torch.arange(cached, n, device="cuda").view(1, -1, 1), torch.arange(n, device="cuda").view(1, 1, -1)
        hidden = key > pos
        if case["window"]:
            hidden = hidden | ((pos - key >= case["window"]) & (key >= case["sinks"]))
        for h in range(case["kv_heads"]):
            k, v = _stands_for(d["k"][at: at + n, h]), _stands_for(d["v"][at: at + n, h])
            q = d["q"][row: row + new, h * group: (h + 1) * group].double().transpose(0, 1)
            logit = (q @ k.T) / math.sqrt(case["dim"])
            logit[hidden.expand_as(logit)] = -math.inf
            out[row: row + new, h * group: (h + 1) * group] = (torch.softmax(logit, -1) @ v).transpose(0, 1)
        at, row = at + n, row + new
    return [out]
