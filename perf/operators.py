"""Performance cases of the operators around the products from compressed weights: what a decoder layer's projections take and
hand on.

Four operators: a projection with bias, activation and residual in its epilogue (alone, or q, k and v in one launch), the gated
feed-forward projections (gate and up with their activation and product), the residual's addition with the root-mean-square norm,
and the feed-forward sub-layer that is made of them.

Weights and activations are synthetic (no checkpoints here): weights N(0, std^2) times a per-row scale U(0.5, 2), which compress like
trained LLM weights do; down projections have the smaller std that training from a depth-scaled start leaves them with, so that a
sub-layer's update is a fraction of the residual stream, as in a trained model.  The residual stream has a few large channels.
"fp16_from_bf16" are BF16-trained weights stored as FP16 (low mantissa bits mostly zero), "fp16" FP16-trained ones.

A framework's program keeps its weights compressed, a plain one keeps them as they are: that is all in which prepare() goes by `own`.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")
_EPS = 1e-5


# ------------------------------------------------------------------------------------------------ cases

def _proj(name, rows, cols, batch, act="none", bias=False, residual=False, out="16", dtype="bf16", chunk=4096, limit=0):
    return {"name": name, "op": "proj", "rows": rows, "cols": cols, "batch": batch, "act": act, "bias": bias, "residual": residual,
            "out": out, "dtype": dtype, "chunk": chunk, "limit": limit}


def _gated(name, ffn, cols, batch, act="silu", bias=False, dtype="bf16", chunk=4096, limit=0):
    return {"name": name, "op": "gated", "ffn": ffn, "cols": cols, "batch": batch, "act": act, "bias": bias, "out": "16", "dtype": dtype,
            "chunk": chunk, "limit": limit}


def _norm(name, vectors, cols, stream, delta, dtype="bf16"):
    return {"name": name, "op": "norm", "vectors": vectors, "cols": cols, "stream": stream, "delta": delta, "dtype": dtype}


def _ffn(name, hidden, ffn, batch, act="silu", dtype="bf16", chunk=4096):
    return {"name": name, "op": "ffn", "hidden": hidden, "ffn": ffn, "batch": batch, "act": act, "dtype": dtype, "chunk": chunk, "limit": 0}


def listed():
    return [
        # one k or v projection with its bias, 8B-shaped, one token: the smallest product, where latency counts
        _proj("proj_kv_bias_b1", 1024, 4096, 1, bias=True),
        # the 7B-shaped down projection added to an fp32 residual stream, one token
        _proj("proj_down_7b_residual_b1", 4096, 11008, 1, residual=True, out="f32"),
        # the first half of an MLP without a gate (bias, GELU), FP16-trained weights, 24 sequences
        _proj("proj_up_gelu_fp16_b24", 11008, 4096, 24, act="gelu", bias=True, dtype="fp16", chunk=2048),
        # the 70B-shaped down projection added to the residual stream, the widest batch
        _proj("proj_down_70b_residual_b64", 8192, 28672, 64, residual=True),
        # q, k and v with biases in one launch, 8B-shaped grouped-query attention, 12 sequences
        {"name": "qkv_bias_8b_b12", "op": "qkv", "hidden": 4096, "kv": 1024, "batch": 12, "dtype": "bf16", "chunk": 4096, "limit": 0},
        # gate and up of the 7B-shaped layer, one token
        _gated("gated_7b_b1", 11008, 4096, 1),
        # odd numbers of gates and ragged columns, a handful of sequences, tanh GELU
        _gated("gated_odd_b5", 10003, 2720, 5, act="gelu_tanh", bias=True, chunk=2048),
        # gate and up of the 70B-shaped layer at the widest batch: the largest call
        _gated("gated_70b_b64", 28672, 8192, 64),
        # between two sub-layers of a 7B-shaped layer, one token, fp32 stream
        _norm("norm_4096_b1", 1, 4096, "f32", "f32"),
        # the same for the tokens of a prompt, 70B-shaped
        _norm("norm_8192_b2048", 2048, 8192, "16", "16"),
        # the feed-forward sub-layer, 8B-shaped, one token
        _ffn("ffn_8b_b1", 4096, 14336, 1),
        # the same, 7B-shaped, 32 sequences
        _ffn("ffn_7b_b32", 4096, 11008, 32),
    ]


def _log_size(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choices(["proj", "qkv", "gated", "norm", "ffn"], [30, 10, 30, 15, 15])[0]
    dtype = rng.choices(["bf16", "fp16", "fp16_from_bf16"], [70, 15, 15])[0]
    if op == "norm":
        cols = _log_size(rng, 250, 16384)                             # odd as often as not
        vectors = _log_size(rng, 1, 4096)
        return {"op": op, "vectors": vectors, "cols": cols, "stream": rng.choice(["f32", "16"]), "delta": rng.choice(["f32", "16", "none"]),
                "dtype": dtype}
    chunk = rng.choice([2048, 4096, 4096, 4096, 8192]) if dtype == "bf16" else rng.choice([1024, 2048, 2048, 4096])
    limit = rng.choice([0, 0, 0, 0, 9, 10, 12]) if dtype == "bf16" and chunk <= 4096 else rng.choice([0, 0, 0, 7]) if dtype != "bf16" else 0
    batch = rng.choice([1, _log_size(rng, 1, 64)])
    most = 24000 * 8192                                               # weights of a gate: FP16 ones compress less than the largest listed case's
    cols = 32 * _log_size(rng, 30, 448)                               # 960 .. 14336: what the fused products take
    if op == "qkv":
        if dtype != "bf16" and 8 < batch <= 16:                       # launches over several FP16 matrices take 1..8 and 17..64
            batch = 8
        kv = cols // rng.choice([1, 2, 4])
        return {"op": op, "hidden": min(cols, 8192), "kv": min(kv, 8192), "batch": batch, "dtype": dtype, "chunk": chunk, "limit": 0}
    if op == "ffn":
        hidden = min(cols, 8192)
        ffn = 32 * int(min(hidden * rng.uniform(2.0, 3.5), most * 2 / 3 / hidden) / 32)
        return {"op": op, "hidden": hidden, "ffn": ffn, "batch": batch, "act": rng.choice(_ACTS[2:]), "dtype": dtype, "chunk": chunk, "limit": limit}
    if op == "gated":
        ffn = _log_size(rng, 200, min(28672, most // cols))
        return {"op": op, "ffn": ffn, "cols": cols, "batch": batch, "act": rng.choice(_ACTS[1:]), "bias": rng.random() < 0.3, "out": "16",
                "dtype": dtype, "chunk": chunk, "limit": limit}
    rows = _log_size(rng, 200, 28672)
    residual = rng.random() < 0.5
    return {"op": op, "rows": rows, "cols": cols, "batch": batch, "act": rng.choice(_ACTS), "bias": rng.random() < 0.5, "residual": residual,
            "out": rng.choice(["f32", "16"]) if residual or batch == 1 else "16", "dtype": dtype, "chunk": chunk, "limit": limit}


# ------------------------------------------------------------------------------------------------ inputs

def _half(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


class _Maker:
    """Inputs of one state, in the order in which they are asked for."""

    def __init__(self, case, seed):
        self.case, self.gen = case, torch.Generator(device="cuda").manual_seed(seed)

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda", dtype=torch.float32)

    def weights(self, rows, cols, std=0.02):
        w = self.randn(rows, cols)
        w *= (torch.rand((rows, 1), generator=self.gen, device="cuda", dtype=torch.float32) * 1.5 + 0.5) * std
        return w.to(torch.bfloat16).to(torch.float16) if self.case["dtype"] == "fp16_from_bf16" else w.to(_half(self.case))

    def vector(self, n, mean=0.0, std=0.5):
        return (self.randn(n) * std + mean).to(_half(self.case))

    def activations(self, batch, cols):
        return self.randn(batch, cols).to(_half(self.case))

    def stream(self, batch, cols, kind):
        """The residual stream: a few channels much larger than the others."""
        h = self.randn(batch, cols) * 4
        h[:, :: max(1, cols // 5)] *= 12
        return h if kind == "f32" else h.to(_half(self.case))


def _inputs(case, seed):
    m, op = _Maker(case, seed), case["op"]
    if op == "proj":
        d = {"w": [m.weights(case["rows"], case["cols"], 0.02 if case["act"] != "none" else 0.005)], "x": m.activations(case["batch"], case["cols"])}
        d["bias"] = [m.vector(case["rows"]) if case["bias"] else None]
        d["residual"] = m.stream(case["batch"], case["rows"], case["out"]) if case["residual"] else None
    elif op == "qkv":
        rows = (case["hidden"], case["kv"], case["kv"])
        d = {"w": [m.weights(r, case["hidden"]) for r in rows], "x": m.activations(case["batch"], case["hidden"])}
        d["bias"] = [m.vector(r) for r in rows]
    elif op == "gated":
        d = {"gate": m.weights(case["ffn"], case["cols"]), "up": m.weights(case["ffn"], case["cols"]), "x": m.activations(case["batch"], case["cols"])}
        d["gate_bias"], d["up_bias"] = (m.vector(case["ffn"]), m.vector(case["ffn"])) if case["bias"] else (None, None)
    elif op == "norm":
        d = {"x": m.stream(case["vectors"], case["cols"], case["stream"]), "gain": m.vector(case["cols"], 1.0, 0.2), "delta": None}
        if case["delta"] != "none":
            d["delta"] = m.randn(case["vectors"], case["cols"])
            if case["delta"] == "16":
                d["delta"] = d["delta"].to(_half(case))
    else:
        h, f = case["hidden"], case["ffn"]
        d = {"gate": m.weights(f, h), "up": m.weights(f, h), "down": m.weights(h, f, 0.0025), "gain": m.vector(h, 1.0, 0.2),
             "h": m.stream(case["batch"], h, "16")}
    return d


# ------------------------------------------------------------------------------------------------ what a program of the framework keeps

def _compress(w, case):
    """(descriptor, blob) of one matrix, compressed where it sits."""
    import paper_2502_00922_b200 as hl
    rows, cols = w.shape
    dtype, widths = (hl.BF16, [1, 8, 7]) if case["dtype"] == "bf16" else (hl.FP16, [1, 5, 5, 5])
    counts = torch.zeros(hl.split_counts_size(widths), dtype=torch.int64, device="cuda")
    hl.split_histogram(w, rows * cols, widths, counts)
    c = counts.cpu().numpy().view(np.uint64)
    cb = hl.build_codebook_from_counts(c[2:258] if dtype == hl.BF16 else c[2:], dtype, case["limit"])
    blob = torch.zeros(hl.encode_bound(rows, cols, dtype, case["chunk"]), dtype=torch.uint8, device="cuda")
    scratch = torch.zeros(hl.encode_device_scratch_bytes(rows, cols, case["chunk"]), dtype=torch.uint8, device="cuda")
    desc = hl.encode_device(cb, w, rows, cols, case["chunk"], blob, blob.numel(), scratch, scratch.numel())
    cb.free()
    return desc, blob[:desc.blob_bytes].clone()


def _stack(gate, up, ffn, cols):
    import paper_2502_00922_b200 as hl
    stacked = torch.empty((hl.stacked_rows(ffn), cols), dtype=gate.dtype, device="cuda")
    hl.stack_gate_up_device(gate, up, ffn, cols, stacked)
    return stacked


def _own_state(case, d):
    import paper_2502_00922_b200 as hl
    op, half = case["op"], _half(case)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    dtype = hl.BF16 if case["dtype"] == "bf16" else hl.FP16
    if op == "norm":
        total = torch.empty_like(d["x"])
        out = torch.empty(d["x"].shape, dtype=half, device="cuda")
        elem = {"f32": hl.ELEM_F32, "16": hl.ELEM_16, "none": hl.ELEM_16}
        norm = hl.Norm(dtype, case["vectors"], case["cols"], d["x"], elem[case["stream"]], d["gain"], _EPS, out, delta=d["delta"],
                       delta_type=elem[case["delta"]], sum=total)
        return {"call": hl.PreparedNorm(norm), "outs": [total, out]}
    act = getattr(hl, "ACT_" + case.get("act", "none").upper())
    if op == "ffn":
        gate_up = _compress(_stack(d["gate"], d["up"], case["ffn"], case["hidden"]), case)
        down = _compress(d["down"], case)
        out = torch.empty_like(d["h"])
        ffn = hl.Ffn(gate_up[0], gate_up[1], down[0], down[1], case["ffn"], d["gain"], _EPS, act)
        n = hl.ffn_workspace_bytes(ffn, case["batch"])
        ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
        call = hl.PreparedFfn(ffn, d["h"], case["batch"], out, hl.ELEM_16, ws, n, err)
        return {"call": call, "outs": [out]}
    if op == "gated":
        bias = _stack(d["gate_bias"].view(-1, 1), d["up_bias"].view(-1, 1), case["ffn"], 1) if case["bias"] else None
        mats = [_compress(_stack(d["gate"], d["up"], case["ffn"], case["cols"]), case)]
        outs = [torch.empty((case["batch"], case["ffn"]), dtype=half, device="cuda")]
        eps = [hl.Epilogue(act, hl.ELEM_16, bias=bias, gated_rows=case["ffn"])]
    else:
        mats = [_compress(w, case) for w in d["w"]]
        f32 = case.get("out") == "f32"
        outs = [torch.empty((case["batch"], w.shape[0]), dtype=torch.float32 if f32 else half, device="cuda") for w in d["w"]]
        eps = [hl.Epilogue(act, hl.ELEM_F32 if f32 else hl.ELEM_16, bias=b, residual=d.get("residual")) for b in d["bias"]]
    n = max(hl.workspace_bytes(m[0], case["batch"]) for m in mats)
    wss = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in mats]
    call = hl.PreparedEpilogue([m[0] for m in mats], [m[1] for m in mats], [d["x"]] * len(mats), case["batch"], eps, outs, wss, n, err)
    return {"call": call, "outs": outs}


def prepare(case, seed):
    d = _inputs(case, seed)
    if own:
        return _own_state(case, d)
    return {"case": case, "in": d}


# ------------------------------------------------------------------------------------------------ one pass

def _act(v, act):
    if act == "relu":
        return v.clamp_min(0)
    if act == "silu":
        return v / (1 + torch.exp(-v))
    if act == "gelu":
        return 0.5 * v * torch.erfc(v * -math.sqrt(0.5))
    if act == "gelu_tanh":                                            # v / 2 (1 + tanh u) = v / (1 + exp(-2 u))
        return v / (1 + torch.exp(v * (-2 * math.sqrt(2 / math.pi)) * (1 + 0.044715 * v * v)))
    return v


def _affine(x, w, bias):
    v = x.float() @ w.float().T
    return v if bias is None else v + bias.float()


def _rms_norm(h, gain):
    return h * torch.rsqrt((h * h).mean(-1, keepdim=True) + _EPS) * gain.float()


def run(state):
    if own:
        state["call"].run(torch.cuda.current_stream().cuda_stream)
        return state["outs"]
    case, d = state["case"], state["in"]
    op, half = case["op"], _half(case)
    if op == "norm":
        h = d["x"].float()
        if d["delta"] is not None:
            h = h + d["delta"].float()
        return [h.to(d["x"].dtype), _rms_norm(h, d["gain"]).to(half)]
    if op == "ffn":
        h = d["h"].float()
        n = _rms_norm(h, d["gain"])
        mid = _act(_affine(n, d["gate"], None), case["act"]) * _affine(n, d["up"], None)
        return [(h + _affine(mid, d["down"], None)).to(half)]
    if op == "gated":
        return [(_act(_affine(d["x"], d["gate"], d["gate_bias"]), case["act"]) * _affine(d["x"], d["up"], d["up_bias"])).to(half)]
    if op == "qkv":
        return [_affine(d["x"], w, b).to(half) for w, b in zip(d["w"], d["bias"])]
    y = _act(_affine(d["x"], d["w"][0], d["bias"][0]), case["act"])
    if d["residual"] is not None:
        y = y + d["residual"].float()
    return [y if case["out"] == "f32" else y.to(half)]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    op, size = case["op"], {"f32": 4, "16": 2, "none": 0}
    if op == "norm":
        n = case["vectors"] * case["cols"]
        return {"bytes": n * (2 * size[case["stream"]] + size[case["delta"]] + 2) + 2 * case["cols"], "flops": 6 * n}
    # raw and coded bits of such a weight (payload without padding, index and table)
    per = {"fp16": 13.72, "fp16_from_bf16": 10.98, "bf16": 11.75}[case["dtype"]] / 8
    b = case["batch"]
    if op == "ffn":
        n, moved = 3 * case["hidden"] * case["ffn"], b * 4 * case["hidden"] + 2 * case["hidden"]
    elif op == "gated":
        n, moved = 2 * case["ffn"] * case["cols"], b * 2 * (case["cols"] + case["ffn"]) + 4 * case["ffn"] * case["bias"]
    elif op == "qkv":
        rows = case["hidden"] + 2 * case["kv"]
        n, moved = rows * case["hidden"], b * 2 * (case["hidden"] + rows) + 2 * rows
    else:
        n = case["rows"] * case["cols"]
        moved = b * (2 * case["cols"] + case["rows"] * size[case["out"]] * (1 + case["residual"])) + 2 * case["rows"] * case["bias"]
    return {"bytes": n * per + moved, "flops": 2 * n * b}


def exact(case, seed):
    """What run() returns for these inputs, in 64 bits."""
    d, act = _inputs(case, seed), case.get("act", "none")

    def product(v, w):                                               # row blocks: a large matrix need not be there in 64 bits at once
        return torch.cat([v @ part.double().T for part in w.split(4096)], dim=1)

    def acted(v):
        if act == "gelu":
            return v * 0.5 * (1 + torch.erf(v / math.sqrt(2.0)))
        if act == "gelu_tanh":
            return v * 0.5 * (1 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
        return {"none": v, "relu": v * (v > 0), "silu": v * torch.sigmoid(v)}[act]

    def normed(h):
        return h / torch.sqrt(torch.sum(h ** 2, dim=1, keepdim=True) / h.shape[1] + _EPS) * d["gain"].double()

    def bias_of(v):
        return 0 if v is None else v.double()

    if case["op"] == "norm":
        h = d["x"].double() + bias_of(d["delta"])
        return [h, normed(h)]
    if case["op"] == "ffn":
        h = d["h"].double()
        n = normed(h)
        return [h + product(acted(product(n, d["gate"])) * product(n, d["up"]), d["down"])]
    x = d["x"].double()
    if case["op"] == "gated":
        return [acted(product(x, d["gate"]) + bias_of(d["gate_bias"])) * (product(x, d["up"]) + bias_of(d["up_bias"]))]
    ys = [acted(product(x, w) + bias_of(b)) for w, b in zip(d["w"], d["bias"])]
    return [y + bias_of(d.get("residual")) for y in ys]
