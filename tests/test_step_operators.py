"""What stands between and behind the products of a decode step: rotary positions, the cache of keys and values in 4 bits with its
attention, the choice of the next token.  Against plain implementations in 64 bits.

Tolerances.  16-bit results are rounded once: half a step, finfo.eps / 2 of the value (fp16: or half of 2^-24).
Rotary: the angle, as half turns in fp32, is off by pi 2^-25, sine and cosine by 2^-23 more, products and their sum by 2^-24 each:
4e-7 of |a| + |b|.
Cache: nothing; codes, scales and offsets are exactly the format's, and s c + m is rounded once.
Attention: a score is a sum of fp32 products (exact factors) over `dim` channels, two products a channel (code and offset): off by
(2 dim + 64) 2^-23 of the sum of their magnitudes, and by 2^-19 of the offsets' part, whose factor is a number of two fp16 halves.
A weight is then off by twice that (its own and the largest's), by 2^-21 for the exponential, and by half a step of fp16 twice: as a factor of
the sum, and times its scale.  What is too small for a full fp16 number (below 2^-14) is off by half of 2^-24: n such at most, where the
largest weight is 2^11 or more, or 2^9 over the largest scale of the values (weights are held at most 2^15, their products with scales at
most 2^14, and a larger weight than any before starts out sixteen times smaller than that).  The sums over n tokens are off by (n + 64) 2^-23 of the sum of
magnitudes."""
import math

import numpy as np
import pytest

import workloads as wl

HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}      # finfo.eps / 2


@pytest.fixture(scope="module")
def hl():
    import paper_2502_00922_b200 as m
    m.lib()
    return m


@pytest.fixture(scope="module")
def torch():
    import torch as t
    return t


def to_bits(a, dtype):
    a = np.ascontiguousarray(a, dtype=np.float32)
    with np.errstate(over="ignore"):
        return wl.f32_to_bf16_bits(a) if dtype == "bf16" else a.astype(np.float16).view(np.uint16)


def to_f64(bits, dtype):
    bits = np.ascontiguousarray(bits, dtype=np.uint16)
    return (wl.bf16_bits_to_f32(bits) if dtype == "bf16" else bits.view(np.float16).astype(np.float32)).astype(np.float64)


def half(torch, dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float16


def up(torch, bits, dtype):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(half(torch, dtype))


def ints(torch, a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def values(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rounding(y, dtype):
    return np.abs(y) * HALF_STEP[dtype] + (2.0 ** -25 if dtype == "fp16" else 0.0)


def check(got, want, tol, dtype):
    tol = tol + rounding(np.abs(want) + tol, dtype)
    assert np.array_equal(np.isnan(got), np.isnan(want)), "NaN in other places"
    bad = ~((np.abs(got - want) <= tol) | np.isnan(want))
    assert not bad.any(), f"{bad.sum()} of {bad.size} outside, worst {np.nanmax(np.abs(got - want) / tol)} of the tolerance at {np.argwhere(bad)[0]}"


# ------------------------------------------------------------------------------------------------ rotary

def axes_of(sections, in_turn):
    if not in_turn:
        return np.repeat(np.arange(len(sections)), sections)
    left, out = list(sections), []
    while any(left):
        for a in range(len(left)):
            if left[a]:
                left[a] -= 1
                out.append(a)
    return np.array(out)


def rotary64(x, positions, frequencies, rot, sections, in_turn, neighbours):
    """x [tokens][heads][dim]; also the sum of magnitudes of every output."""
    angle = positions.astype(np.float64)[axes_of(sections, in_turn)].T * frequencies.astype(np.float64)
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if neighbours else (slice(0, rot // 2), slice(rot // 2, rot))
    y, mag = x.copy(), np.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    mag[..., a] = mag[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, mag


ROTARY = [  # tokens, heads, kv_heads, dim, rot, sections, in_turn, neighbours, far, dtype, strides beyond the packed row
    (1, 32, 8, 128, 128, [64], False, False, 1000, "bf16", 0),
    (1, 1, 1, 2, 2, [1], False, True, 10, "fp16", 0),
    (7, 5, 1, 64, 32, [16], False, True, 1000000, "bf16", 0),
    (33, 4, 4, 128, 128, [16, 24, 24], False, False, 5000, "fp16", 0),
    (33, 28, 4, 128, 128, [24, 20, 20], True, False, 300, "bf16", 24),
    (130, 3, 2, 96, 80, [5, 0, 35], True, True, 2 ** 31 - 1, "bf16", 5),
    (64, 2, 0, 256, 256, [1, 2, 3, 122], True, False, 100000, "fp16", 3),
    (300, 9, 3, 80, 80, [40], False, False, 2 ** 20, "bf16", 8),
    (17, 6, 2, 72, 20, [10], False, False, 4096, "bf16", 0),
    (1000, 16, 16, 192, 192, [96], False, True, 4096, "fp16", 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", ROTARY, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_rotary(hl, torch, case, in_place):
    tokens, heads, kv, dim, rot, sections, in_turn, neighbours, far, dtype, extra = case
    rng = np.random.default_rng(1)
    pos = rng.integers(0, far, (len(sections), tokens)).astype(np.int32)
    pos[:, 0] = far - 1
    if far > 1000:
        pos[-1, -1] = -far // 2
    freq = (10000.0 ** (-2.0 * np.arange(rot // 2) / rot)).astype(np.float32)
    bufs, outs, wants = [], [], []
    for n in (heads, kv):
        stride = n * dim + extra
        bits = to_bits(rng.standard_normal((tokens, max(stride, 1))), dtype)
        bufs.append((bits, stride))
    dev = [up(torch, b, dtype) for b, _ in bufs]
    outs = dev if in_place else [torch.full_like(d, 7.0) for d in dev]
    r = hl.Rotary(hl.BF16 if dtype == "bf16" else hl.FP16, tokens, dim, ints(torch, pos), torch.from_numpy(freq).cuda(), dev[0], heads, outs[0],
                  dev[1] if kv else None, kv, outs[1] if kv else None, rotary_dim=rot, sections=sections, in_turn=in_turn,
                  pairing=hl.PAIR_NEIGHBOURS if neighbours else hl.PAIR_HALVES, q_stride=bufs[0][1], k_stride=bufs[1][1] if kv else 0,
                  q_out_stride=bufs[0][1], k_out_stride=bufs[1][1] if kv else 0)
    hl.apply_rotary(r)
    for (bits, stride), out, n in zip(bufs, outs, (heads, kv)):
        if n == 0:
            continue
        got = values(out).reshape(tokens, -1)
        x = to_f64(bits, dtype).reshape(tokens, -1)
        want, mag = rotary64(x[:, :n * dim].reshape(tokens, n, dim), pos, freq, rot, sections, in_turn, neighbours)
        check(got[:, :n * dim].reshape(want.shape), want, 4e-7 * mag, dtype)
        assert np.array_equal(got[:, :n * dim].reshape(want.shape)[..., rot:], want[..., rot:]), "channels behind the turned ones"
        rest = x[:, n * dim:] if in_place else np.full_like(x[:, n * dim:], 7.0)
        assert np.array_equal(got[:, n * dim:], rest), "between the tokens"


@pytest.mark.gpu
def test_rotary_unaligned(hl, torch):
    """Pointers on every multiple of two bytes."""
    rng = np.random.default_rng(3)
    for shift in range(1, 8):
        bits = to_bits(rng.standard_normal(5 * 3 * 64 + 8), "bf16")
        dev, out = up(torch, bits, "bf16"), torch.zeros(5 * 3 * 64 + 8, dtype=torch.bfloat16, device="cuda")
        pos, freq = np.arange(5, dtype=np.int32)[None] * 77, np.linspace(1, 0.001, 32).astype(np.float32)
        hl.apply_rotary(hl.Rotary(hl.BF16, 5, 64, ints(torch, pos), torch.from_numpy(freq).cuda(), dev[shift:], 3, out[8 - shift:]))
        want, mag = rotary64(to_f64(bits, "bf16")[shift: shift + 960].reshape(5, 3, 64), pos, freq, 64, [32], False, False)
        check(values(out)[8 - shift: 8 - shift + 960].reshape(want.shape), want, 4e-7 * mag, "bf16")


# ------------------------------------------------------------------------------------------------ the cache

def quantise64(x):
    """[..., dim] in 64 bits (16-bit values) -> codes, scales, offsets; NaN where a group stands for NaN."""
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    with np.errstate(over="ignore", invalid="ignore"):
        low, high = g.min(-1), g.max(-1)
        s = ((high.astype(np.float32) - low.astype(np.float32)) / np.float32(15)).astype(np.float16).astype(np.float64)
        m = low.astype(np.float32).astype(np.float16).astype(np.float64)
        bad = ~np.isfinite(s) | ~np.isfinite(m) | ~np.isfinite(g).all(-1)
        s, m = np.where(bad, np.nan, s), np.where(bad, 0.0, m)
        c = np.where(s[..., None] == 0, 0.0, np.clip(np.rint((g - m[..., None]) / np.where(s == 0, 1.0, s)[..., None]), 0, 15))
    return np.where(bad[..., None], 0.0, c), s, m


def stands_for(x):
    c, s, m = quantise64(x)
    return (s[..., None] * c + m[..., None]).reshape(x.shape)


class Pages:
    """A cache with its pages in any order in a pool that starts as garbage (every scale a NaN)."""

    def __init__(self, hl, torch, dtype, kv, dim, page, lengths, rng, spare=2, stride=None):
        self.hl, self.torch, self.dtype, self.kv, self.dim, self.page = hl, torch, dtype, kv, dim, page
        used = [-(-n // page) for n in lengths]
        self.pages = sum(used) + spare
        order = rng.permutation(self.pages)
        table = np.full((len(lengths), stride or max(1, max(used))), 2 ** 30, np.int32)
        at = 0
        for i, n in enumerate(used):
            table[i, :n] = order[at: at + n]
            at += n
        self.host_table, self.table, self.lengths = table, ints(torch, table), ints(torch, lengths)
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.pool = torch.full((hl.cache_bytes(self._cache(None)),), 255, dtype=torch.uint8, device="cuda")
        self.cache = self._cache(self.pool)

    def _cache(self, pool):
        return self.hl.Cache(self.hl.BF16 if self.dtype == "bf16" else self.hl.FP16, self.kv, self.dim, self.page, self.pages, pool, self.table, self.lengths)

    def starts(self, counts, first=0):
        return ints(self.torch, np.concatenate([[0], np.cumsum(counts)]) + first)

    def error(self):
        return int(self.err.item())


def kv_values(rng, shape, kind):
    x = rng.standard_normal(shape)
    if kind == "outliers":
        x[..., ::17] *= 40
    elif kind == "far":                                  # far from zero: the offset is most of the value
        x = x * 0.3 + 50
    elif kind == "flat":
        x = np.full(shape, 0.75) * (1 + np.arange(shape[-1]) // 32)
    elif kind == "grid":                                 # many quotients next to a border
        x = rng.integers(0, 31, shape) / 2.0
    elif kind == "tiny":
        x = x * 1e-6
    return x


CACHE = [(d, kv, page, dt, kind) for d, kv, page, dt, kind in [
    (64, 1, 16, "bf16", "normal"), (96, 3, 48, "fp16", "outliers"), (128, 8, 64, "bf16", "far"), (192, 2, 32, "fp16", "grid"),
    (256, 1, 16, "bf16", "grid"), (128, 2, 16, "fp16", "tiny"), (128, 2, 16, "bf16", "tiny"), (64, 5, 80, "bf16", "flat"), (128, 4, 256, "fp16", "normal")]]


@pytest.mark.gpu
@pytest.mark.parametrize("dim,kv,page,dtype,kind", CACHE)
def test_cache_holds_the_format(hl, torch, dim, kv, page, dtype, kind):
    """Prompts, then a token each, then nothing new for some; read back as fp32, exactly, and as 16 bits."""
    rng = np.random.default_rng(5)
    first = [37, 1, 0, 16, 130, 64]
    n = len(first)
    p = Pages(hl, torch, dtype, kv, dim, page, [x + 3 for x in first], rng)
    held = [np.zeros((0, kv, dim)) for _ in first], [np.zeros((0, kv, dim)) for _ in first]
    total = np.zeros(n, int)
    for counts in (first, [1] * n, [2, 0, 0, 1, 0, 2]):
        total += counts
        p.lengths.copy_(ints(torch, total))
        rows = sum(counts) + 5                            # five rows behind the last sequence
        pad = {"normal": 8, "far": 3, "flat": 4}.get(kind, 0)      # between the rows
        new = [to_bits(kv_values(rng, (rows, kv * dim + pad), "normal" if kind == "flat" else kind), dtype) for _ in range(2)]
        hl.cache_append(p.cache, up(torch, new[0], dtype), up(torch, new[1], dtype), rows, starts=p.starts(counts), k_stride=kv * dim + pad,
                        v_stride=kv * dim + pad, err_flag_dev=p.err)
        at = 0
        for b, c in enumerate(counts):
            for side in range(2):
                held[side][b] = np.concatenate([held[side][b], to_f64(new[side], dtype)[at: at + c, :kv * dim].reshape(c, kv, dim)])
            at += c
    for elem in (hl.ELEM_F32, hl.ELEM_16):
        rows = int(total.sum()) + 3
        out = [torch.full((rows, kv * dim), 5.0, dtype=torch.float32 if elem == hl.ELEM_F32 else half(torch, dtype), device="cuda") for _ in range(2)]
        hl.cache_read(p.cache, out[0], out[1], elem, rows, starts=p.starts(total), err_flag_dev=p.err)
        assert p.error() == 0
        for side in range(2):
            want = stands_for(np.concatenate(held[side]))
            got = values(out[side])
            assert np.all(got[rows - 3:] == 5.0), "rows behind the last sequence"
            got = got[: rows - 3].reshape(want.shape)
            if elem == hl.ELEM_F32:
                assert np.array_equal(got, want.astype(np.float32).astype(np.float64))
            else:
                assert np.array_equal(got, to_f64(to_bits(want.astype(np.float32), dtype), dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_cache_groups_that_are_not_finite(hl, torch, dtype):
    rng = np.random.default_rng(6)
    p = Pages(hl, torch, dtype, 1, 128, 16, [9], rng)
    x = rng.standard_normal((9, 128))
    x[0, 3], x[1, 40], x[2, 70] = np.nan, np.inf, -np.inf
    x[3, :] = np.nan
    x[4, 5], x[4, 6] = 60000.0, -60000.0                  # finite, and the span is too
    x[5, 64] = 70000.0 if dtype == "bf16" else 65504.0    # bf16: the scale is finite still
    x[6, 9] = -70000.0 if dtype == "bf16" else -65504.0   # bf16: the offset is not
    bits = to_bits(x, dtype)
    hl.cache_append(p.cache, up(torch, bits, dtype), up(torch, bits[::-1].copy(), dtype), 9, starts=p.starts([9]), err_flag_dev=p.err)
    out = torch.zeros((2, 9, 128), device="cuda")
    hl.cache_read(p.cache, out[0], out[1], hl.ELEM_F32, 9, starts=p.starts([9]))
    want = stands_for(to_f64(bits, dtype)).astype(np.float32)
    got = out.cpu().numpy()
    assert np.array_equal(got[0], want, equal_nan=True) and np.array_equal(got[1], want[::-1], equal_nan=True)
    only = torch.zeros((9, 128), device="cuda")           # one side alone
    hl.cache_read(p.cache, None, only, hl.ELEM_F32, 9, starts=p.starts([9]))
    assert np.array_equal(only.cpu().numpy(), want[::-1], equal_nan=True)


# ------------------------------------------------------------------------------------------------ attention

def attention64(q, k, v, cached, scale, window, sinks):
    """q [new][heads][dim], k and v [tokens][kv][dim] as the cache's (codes, scales, offsets); result and tolerance without the final rounding."""
    def parts(t):
        c, s, m = quantise64(t)
        sc = s[..., None] * c
        return (sc + m[..., None]).reshape(t.shape), (np.abs(sc) + np.abs(m)[..., None]).reshape(t.shape), np.repeat(np.abs(m), 32, -1).reshape(t.shape), s
    (kx, kmag, koff, _), (vx, vmag, _, vs) = parts(k), parts(v)
    new, heads, dim = q.shape
    n, group = k.shape[0], heads // k.shape[1]
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(new):
        at = cached + i
        j = np.arange(n)
        seen = (j <= at) & ((j > at - window) | (j < sinks) if window else True)
        if not seen.any():
            continue
        for h in range(heads):
            kk, vv, mag = kx[seen, h // group], vx[seen, h // group], vmag[seen, h // group]
            with np.errstate(invalid="ignore"):
                x = scale * (kk @ q[i, h])
                off = abs(scale) * ((2 * dim + 64) * 2.0 ** -23 * (kmag[seen, h // group] @ np.abs(q[i, h])) + 2.0 ** -19 * (koff[seen, h // group] @ np.abs(q[i, h])))
                w = np.exp(x - x.max())
                p = w / w.sum()
                most = np.nanmax(np.concatenate([[0.0], vs[seen, h // group].ravel()]))
                small = 2.0 ** -25 / min(2.0 ** 11, 2.0 ** 9 / max(most, 2.0 ** -20))
                rel = np.exp(off + np.nanmax(np.concatenate([[0.0], off]))) * (1 + 2.0 ** -21) * (1 + 2.0 ** -11) ** 2 - 1 + (n + 64) * 2.0 ** -23
                out[i, h] = p @ vv
                # the weights' errors move the sum, and (over the sum of weights) the mean
                moved = ((p * rel) @ mag) + (p @ rel) * np.abs(out[i, h]) + small / w.sum() * (mag.sum(0) + n * np.abs(out[i, h]))
                tol[i, h] = 1.1 * moved
    return out, tol


def run_attention(p, q, heads, rows, scale, starts, window, sinks, q_stride=0, out_stride=0, stream=None, out=None):
    hl, torch = p.hl, p.torch
    width = out_stride or heads * p.dim
    out = torch.full((rows, width), 3.0, dtype=half(torch, p.dtype), device="cuda") if out is None else out
    a = hl.Attention(q, heads, out, rows, scale, starts=starts, window=window, sinks=sinks, q_stride=q_stride, out_stride=out_stride)
    nbytes = hl.attention_workspace_bytes(p.cache, a)
    ws = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")
    hl.cache_attention(p.cache, a, ws, nbytes, p.err, stream)
    hl.cache_attention(p.cache, a, ws, nbytes, p.err, stream)      # the workspace is as it was
    control = hl.attention_control_bytes(p.cache, a)
    assert not ws[:control].any().item(), "counters are left zero"
    return out


def attention_case(hl, torch, dim, heads, kv, page, dtype, lengths, counts, window=0, sinks=0, kind="normal", seed=7, scale=None, sharp=1.0, extra=0):
    """Appends, attends, compares; lengths count the new rows."""
    rng = np.random.default_rng(seed)
    p = Pages(hl, torch, dtype, kv, dim, page, lengths, rng)
    k = to_bits(kv_values(rng, (sum(lengths), kv, dim), kind), dtype)
    v = to_bits(kv_values(rng, (sum(lengths), kv, dim), kind), dtype)
    if sum(lengths):
        hl.cache_append(p.cache, up(torch, k, dtype), up(torch, v, dtype), sum(lengths), starts=p.starts(lengths), err_flag_dev=p.err)
    first, rows = (0, len(lengths)) if counts is None else (2, sum(counts) + 5)
    q_stride, out_stride = heads * dim + extra, heads * dim + 2 * extra
    q = to_bits(rng.standard_normal((rows, q_stride)) * sharp, dtype)
    starts = None if counts is None else p.starts(counts, first)
    scale = dim ** -0.5 if scale is None else scale
    got = values(run_attention(p, up(torch, q, dtype), heads, rows, scale, starts, window, sinks, q_stride, out_stride))
    assert p.error() == 0
    at, row = 0, first
    for n, c in zip(lengths, [1] * len(lengths) if counts is None else counts):
        qb = to_f64(q[row: row + c, :heads * dim].reshape(-1), dtype).reshape(c, heads, dim)
        kb, vb = (to_f64(t[at: at + n].reshape(-1), dtype).reshape(n, kv, dim) for t in (k, v))
        want, tol = attention64(qb, kb, vb, n - c, scale, window, sinks)
        check(got[row: row + c, :heads * dim].reshape(want.shape), want, tol, dtype)
        assert np.all(got[row: row + c, heads * dim:] == 3.0), "between the rows"
        at, row = at + n, row + c
    assert np.all(got[:first] == 3.0) and np.all(got[row:] == 3.0), "rows that are no sequence's"


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim,heads,kv,page", [(64, 4, 4, 16), (96, 10, 2, 48), (128, 8, 1, 32), (128, 8, 2, 64), (192, 14, 2, 16), (256, 16, 1, 128)])
def test_attention_single_tokens(hl, torch, dim, heads, kv, page, dtype):
    attention_case(hl, torch, dim, heads, kv, page, dtype, [1, 15, 16, 17, 0, 31, 32, 33, 64, 65, 300], None)


@pytest.mark.gpu
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 7, 8, 9, 12, 16, 17, 32, 40])
def test_attention_groups_of_heads(hl, torch, group):
    attention_case(hl, torch, 128, 2 * group, 2, 32, "bf16", [77, 5, 130], None, extra=24)


@pytest.mark.gpu
@pytest.mark.parametrize("dim,group,dtype", [(64, 4, "bf16"), (128, 4, "fp16"), (96, 7, "bf16"), (256, 2, "fp16"), (192, 1, "bf16"), (128, 16, "bf16")])
def test_attention_several_tokens(hl, torch, dim, group, dtype):
    """Pieces of prompts and drafts: rows see the tokens up to their own; one sequence has more rows than tokens."""
    attention_case(hl, torch, dim, 2 * group, 2, 48, dtype, [70, 3, 129, 40, 200, 0, 5], [70, 3, 1, 0, 33, 0, 9], extra=8)


@pytest.mark.gpu
@pytest.mark.parametrize("extra", [1, 2, 3, 5, 7])
def test_attention_strides_off_every_boundary(hl, torch, extra):
    attention_case(hl, torch, 96, 6, 2, 16, "fp16", [40, 3, 700], [3, 1, 2], extra=extra)
    attention_case(hl, torch, 128, 4, 4, 32, "bf16", [2000, 3], None, extra=extra)


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 4), (33, 0), (33, 40), (64, 16), (100, 1), (1000, 4), (2 ** 32 - 1, 2 ** 32 - 1)])
@pytest.mark.parametrize("counts", [None, [1, 7, 50, 128]])
def test_attention_window_and_first_tokens(hl, torch, window, sinks, counts):
    attention_case(hl, torch, 128, 8, 2, 16, "bf16", [1, 65, 250, 600], counts, window=window, sinks=sinks)


@pytest.mark.gpu
@pytest.mark.parametrize("lengths,heads,kv", [([3000], 4, 1), ([2500, 40, 3100], 16, 2), ([700] * 20, 8, 4), ([20] * 90, 4, 2), ([5000], 8, 8)])
def test_attention_split_over_long_caches(hl, torch, lengths, heads, kv):
    attention_case(hl, torch, 128, heads, kv, 64, "bf16", lengths, None, sharp=2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["outliers", "far", "flat", "grid", "tiny"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attention_values(hl, torch, kind, dtype):
    attention_case(hl, torch, 128, 8, 2, 32, dtype, [200, 33], [5, 1], kind=kind, sharp={"outliers": 0.1, "far": 0.3}.get(kind, 1.0))


@pytest.mark.gpu
@pytest.mark.parametrize("scale,sharp", [(0.0, 1.0), (-0.1, 1.0), (3.0, 4.0), (0.1, 1e-4), (1e-3, 1000.0)])
def test_attention_scales(hl, torch, scale, sharp):
    attention_case(hl, torch, 128, 8, 2, 32, "bf16", [300, 33], [3, 1], scale=scale, sharp=sharp)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("window,sinks,bad", [(0, 0, [90]), (0, 0, [99]), (20, 3, [3, 40, 79]), (20, 3, [2]), (20, 3, [85])])
def test_attention_nan_is_seen_only_where_it_is_visible(hl, torch, dtype, window, sinks, bad):
    """Keys or values of some tokens are NaN: rows that do not see them are as if they were not there, rows that do are NaN."""
    rng = np.random.default_rng(8)
    for side in (0, 1):
        p = Pages(hl, torch, dtype, 2, 128, 16, [100], rng)
        kv = [rng.standard_normal((100, 2, 128)) for _ in range(2)]
        kv[side][bad, :, 5] = np.nan                       # the group of channel 5 is
        bits = [to_bits(t, dtype) for t in kv]
        hl.cache_append(p.cache, up(torch, bits[0], dtype), up(torch, bits[1], dtype), 100, starts=p.starts([100]))
        q = to_bits(rng.standard_normal((12, 8 * 128)), dtype)
        got = values(run_attention(p, up(torch, q, dtype), 8, 12, 128 ** -0.5, p.starts([12]), window, sinks))
        kb, vb = (to_f64(t.reshape(-1), dtype).reshape(100, 2, 128) for t in bits)
        want, tol = attention64(to_f64(q.reshape(-1), dtype).reshape(12, 8, 128), kb, vb, 88, 128 ** -0.5, window, sinks)
        check(got.reshape(want.shape), want, np.nan_to_num(tol), dtype)


@pytest.mark.gpu
def test_attention_infinite_queries(hl, torch):
    rng = np.random.default_rng(9)
    p = Pages(hl, torch, "bf16", 1, 64, 16, [40], rng)
    bits = [to_bits(rng.standard_normal((40, 1, 64)), "bf16") for _ in range(2)]
    hl.cache_append(p.cache, up(torch, bits[0], "bf16"), up(torch, bits[1], "bf16"), 40, starts=p.starts([40]))
    q = rng.standard_normal((3, 2, 64))
    q[0, 0, 7], q[1, 1, 9] = np.nan, np.inf
    q = to_bits(q, "bf16")
    got = values(run_attention(p, up(torch, q.reshape(3, -1), "bf16"), 2, 3, 0.125, p.starts([3]), 0, 0)).reshape(3, 2, 64)
    assert np.isnan(got[0, 0]).all() and np.isnan(got[1, 1]).all()
    for i, h in ((0, 1), (1, 0), (2, 0), (2, 1)):
        assert np.isfinite(got[i, h]).all()


# ------------------------------------------------------------------------------------------------ bad pages and lengths

@pytest.mark.gpu
def test_cache_bad_pages_lengths_and_starts(hl, torch):
    """Sequence 1 is at fault in some way: it is named, the others are served, and nothing outside of their own pages is written."""
    rng = np.random.default_rng(10)
    lengths, kv, dim, heads = [40, 50, 20], 2, 64, 4
    for fault in ("page -1", "page beyond", "length", "negative", "start beyond", "start back"):
        p = Pages(hl, torch, "bf16", kv, dim, 16, lengths, rng, spare=1)
        table, ls, starts = p.host_table.copy(), list(lengths), [0, 40, 90, 110]
        if fault == "page -1":
            table[1, 1] = -1
        elif fault == "page beyond":
            table[1, 3] = p.pages
        elif fault == "length":
            ls[1] = table.shape[1] * 16 + 1
        elif fault == "negative":
            ls[1] = -3
        elif fault == "start beyond":
            starts = [0, 40, 2000, 2020]
        else:
            starts = [0, 40, 30, 50]
        p.table.copy_(ints(torch, table))
        p.lengths.copy_(ints(torch, ls))
        k, v = (to_bits(rng.standard_normal((110, kv, dim)), "bf16") for _ in range(2))
        before = p.pool.clone()
        hl.cache_append(p.cache, up(torch, k, "bf16"), up(torch, v, "bf16"), 110, starts=ints(torch, starts), err_flag_dev=p.err)
        torch.cuda.synchronize()
        named = (2, 3) if fault == "start beyond" else (2,)
        assert p.error() in named, fault
        changed = (p.pool != before).cpu().numpy().reshape(p.pages, -1).any(1)
        owned = set(p.host_table[0, :3].tolist()) | set(p.host_table[2, :2].tolist()) | set(t for t in table[1].tolist() if 0 <= t < p.pages)
        assert set(np.nonzero(changed)[0].tolist()) <= owned, fault
        p.err.zero_()
        q = to_bits(rng.standard_normal((3, heads * dim)), "bf16")
        got = values(run_attention(p, up(torch, q, "bf16"), heads, 3, 0.125, None, 0, 0)).reshape(3, heads, dim)
        if not fault.startswith("start"):
            assert p.error() == 2, fault
            if fault in ("length", "negative"):
                assert np.all(got[1] == 0.0), "a length that is none is no tokens"
        kb, vb = (to_f64(t[:40].reshape(-1), "bf16").reshape(40, kv, dim) for t in (k, v))
        want, tol = attention64(to_f64(q[:1].reshape(-1), "bf16").reshape(1, heads, dim), kb, vb, 39, 0.125, 0, 0)
        check(got[:1], want, tol, "bf16")


# ------------------------------------------------------------------------------------------------ sampling

def weights64(x, t):
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == np.inf:
        return x, (x == np.inf).astype(np.float64)
    if not t > 0:
        return x, (x == top).astype(np.float64)
    return x, np.exp((x - top) / t)


def sample64(x, t, k, p, least, u):
    """The token, and how near (relative to the mass) the draw came to a border; the kept tokens."""
    x, w = weights64(x, t)
    if x.max() == -np.inf:
        return -1, 1.0, []
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    if not t > 0:
        order = order[:1]
    if k > 0:
        order = order[:k]
    if p < 1:
        mass = np.cumsum(w[order])
        n = max(1, int(np.searchsorted(mass, max(p, 0) * mass[-1], "left")) + 1) if p > 0 else 1
        near = np.min(np.abs(mass - p * mass[-1])) / mass[-1] if p > 0 else 1.0
        order = order[:n]
    else:
        near = 1.0
    order = order[w[order] >= min(least, 1.0)]
    kept = np.sort(order)
    run = np.cumsum(w[kept])
    total = run[-1]
    aim = min(max(u, 0.0), 1.0) * total
    i = int(np.searchsorted(run, aim, "right"))
    last = kept[w[kept] > 0][-1]
    token = kept[i] if i < len(kept) else last
    near = min(near, np.min(np.abs(run - aim)) / total)
    return int(token), near, kept


def run_sample(hl, torch, x, dtype, settings, u, vocab=None, stride=0):
    rows, vocab = len(u), vocab or x.shape[1]
    dev = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()
    if dtype != "f32":
        dev = up(torch, to_bits(x, dtype), dtype)
    tokens = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    arrays = {n: None if v is None else torch.tensor(v, dtype=torch.int32 if n == "top_k" else torch.float32, device="cuda") for n, v in settings.items()}
    s = hl.Sampling(dev, hl.ELEM_F32 if dtype == "f32" else hl.ELEM_16, rows, vocab, torch.tensor(u, dtype=torch.float32, device="cuda"), tokens,
                    dtype=hl.FP16 if dtype == "fp16" else hl.BF16, stride=stride, **arrays)
    hl.sample(s)
    seen = values(dev.reshape(-1)).reshape(x.shape)[:, :vocab]
    return tokens.cpu().numpy(), seen


def check_samples(tokens, seen, settings, u):
    """Equal, but where the draw or a cut by mass is within 1e-5 of a border (fp32 weights are off by 2e-6)."""
    rows = len(tokens)
    get = lambda n, i, none: none if settings.get(n) is None else float(np.float32(settings[n][i]))
    exact = 0
    for i in range(rows):
        want, near, kept = sample64(seen[i], get("temperature", i, 1.0), int(get("top_k", i, 0)), get("top_p", i, 1.0), get("min_p", i, 0.0), float(np.float32(u[i])))
        if near > 1e-5:
            assert tokens[i] == want, (i, tokens[i], want, near)
            exact += 1
        else:
            assert tokens[i] in kept
    return exact


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 31, 33, 1000, 1025, 4099, 32000, 50257])
def test_sample(hl, torch, vocab, dtype):
    rng = np.random.default_rng(vocab)
    rows = 24
    x = rng.standard_normal((rows, vocab)) * rng.choice([0.5, 2.0, 6.0], (rows, 1))
    settings = {"temperature": rng.choice([0.3, 0.7, 1.0, 1.5, 0.0], rows), "top_k": rng.choice([0, 1, 2, 5, 40, 500, 10 ** 9, -3], rows),
                "top_p": rng.choice([1.0, 0.95, 0.5, 0.1, 0.999, 2.0, 0.0], rows), "min_p": rng.choice([0.0, 0.0, 0.01, 0.3, 1.0, 2.0], rows)}
    u = rng.random(rows).astype(np.float32)
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -24
    tokens, seen = run_sample(hl, torch, x, dtype, settings, u)
    # (a flat row of n tokens has borders 1 / n apart: from some ten thousand tokens on a draw is within 1e-5 of one more often than not)
    assert check_samples(tokens, seen, settings, u) >= (rows - 3 if vocab < 10000 else 12)


@pytest.mark.gpu
@pytest.mark.parametrize("only", ["temperature", "top_k", "top_p", "min_p", None])
def test_sample_settings_alone(hl, torch, only):
    rng = np.random.default_rng(11)
    x = rng.standard_normal((40, 5003)) * 3
    value = {"temperature": [0.7] * 40, "top_k": list(range(1, 41)), "top_p": list(np.linspace(0.02, 0.99, 40)), "min_p": list(np.linspace(0.0, 0.9, 40))}
    settings = {n: (value[n] if n == only else None) for n in value}
    u = rng.random(40)
    tokens, seen = run_sample(hl, torch, x, "f32", settings, u)
    assert check_samples(tokens, seen, settings, u) >= 37


@pytest.mark.gpu
def test_sample_ties_go_to_the_lowest_index(hl, torch):
    """Equal logits across every cut: all alike, two values, a tie at the edge of top-k and of top-p."""
    rng = np.random.default_rng(12)
    rows, vocab = 32, 3001
    x = np.zeros((rows, vocab))
    x[8:16] = rng.integers(0, 2, (8, vocab))
    x[16:24] = rng.integers(0, 6, (8, vocab)) / 2.0
    x[24:] = np.where(rng.random((8, vocab)) < 0.01, 3.0, -1.0)
    x[28:] *= -0.0
    settings = {"temperature": [1.0] * rows, "top_k": [0, 10, 100, 2999] * 8, "top_p": [0.503, 1.0, 0.303, 0.777, 0.9003, 1.0, 1.0, 0.0103] * 4,
                "min_p": [0.0] * rows}
    u = rng.random(rows)
    tokens, seen = run_sample(hl, torch, x, "f32", settings, u)
    assert check_samples(tokens, seen, settings, u) >= rows - 8
    greedy = run_sample(hl, torch, x, "f32", {"temperature": [0.0] * rows}, u)[0]
    assert np.array_equal(greedy, x.argmax(1))


@pytest.mark.gpu
@pytest.mark.parametrize("vocab,rows", [(30011, 3), (150001, 2), (9001, 160), (140001, 24)])
def test_sample_crowded_logits(hl, torch, vocab, rows):
    """Thousands of tokens next to each other in their logits, a few distinct values of them or many; very high and very low temperatures."""
    rng = np.random.default_rng(vocab)
    for kind in range(4):
        x = [rng.integers(0, 3, (rows, vocab)) * 1e-3, 5 + rng.random((rows, vocab)) * 1e-3, np.full((rows, vocab), -2.5),
             np.where(rng.random((rows, vocab)) < 0.5, 1.0, rng.standard_normal((rows, vocab)))][kind]
        x[:, vocab // 2] = 5.5
        for t in (1.0, 1e-4, 50.0):
            # (cuts by mass between the borders of whole groups of equals, where 1e-5 of the mass is less than a token)
            settings = {"temperature": [t] * rows, "top_k": [[vocab // 3, 0, 7000][i % 3] for i in range(rows)],
                        "top_p": [[0.61234, 0.5, 1.0, 0.87654][i % 4] for i in range(rows)], "min_p": [0.0] * rows}
            u = rng.random(rows)
            tokens, seen = run_sample(hl, torch, x, "f32", settings, u)
            for i in range(rows):
                want, near, kept = sample64(seen[i], np.float64(np.float32(t)), settings["top_k"][i], float(np.float32(settings["top_p"][i])), 0.0, float(np.float32(u[i])))
                # weights of up to 150000 like tokens lie 7e-6 of the mass apart: a draw lands within a few tokens of the exact one
                place, got = np.searchsorted(kept, want), np.searchsorted(kept, tokens[i])
                assert 0 <= got < len(kept) + 1 and abs(int(got) - int(place)) <= 2 + 1e-5 * len(kept) * 2, (kind, t, i, tokens[i], want)


@pytest.mark.gpu
def test_sample_one_crowded_bin_of_a_large_part(hl, torch):
    """All of a large vocabulary at the far end of one bin (1/64 in the exponent wide, as one token is masked)."""
    rng = np.random.default_rng(16)
    rows, vocab = 190, 150001
    x = np.full((rows, vocab), 5.46875, np.float32)
    x[:, 77], x[:, 5] = 5.5, -np.inf
    settings = {"temperature": [1.01] * rows, "top_p": [0.61234] * rows}
    u = rng.random(rows)
    tokens, seen = run_sample(hl, torch, x, "bf16", settings, u)
    for i in range(0, rows, 40):
        want, near, kept = sample64(seen[i], np.float64(np.float32(1.01)), 0, float(np.float32(0.61234)), 0.0, float(np.float32(u[i])))
        place, got = np.searchsorted(kept, want), np.searchsorted(kept, tokens[i])
        assert abs(int(got) - int(place)) <= 2 + 1e-5 * len(kept) * 2, (i, tokens[i], want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp16"])
def test_sample_masked_logits(hl, torch, dtype):
    """Minus infinity, the type's lowest value, NaN, plus infinity; rows with one token left, and with none."""
    rng = np.random.default_rng(13)
    low = {"f32": np.finfo(np.float32).min, "bf16": -3.38953139e38, "fp16": -65504.0}[dtype]
    x = rng.standard_normal((12, 2000))
    x[0, :] = -np.inf
    x[1, :] = np.nan
    x[2, :] = -np.inf
    x[2, 777] = 1.0
    x[3, ::2] = -np.inf
    x[4, 5:] = low
    x[5, :] = low
    x[6, 100:1900] = np.nan
    x[7, [3, 900, 1999]] = np.inf
    x[8, :] = -np.inf
    x[8, [1, 2]] = low
    x[9, :1999] = -np.inf
    x[10, 1:] = low
    settings = {"temperature": [1.0] * 11 + [0.0], "top_k": [0, 5, 3, 0, 0, 4, 50, 2, 0, 0, 0, 0], "top_p": [0.9, 0.9, 0.9, 0.9, 1.0, 0.503, 0.9, 1.0, 1.0, 0.9, 0.9, 1.0],
                "min_p": [0.0] * 12}
    for trial in range(4):
        u = rng.random(12)
        tokens, seen = run_sample(hl, torch, x, dtype, dict(settings), u)
        assert tokens[0] == -1 and tokens[1] == -1 and tokens[2] == 777 and tokens[9] == 1999
        assert check_samples(tokens, seen, settings, u) >= 11


@pytest.mark.gpu
def test_sample_numbers_outside_the_unit_interval(hl, torch):
    x = np.array([[0.0, 1.0, -np.inf, 2.0, -np.inf]] * 6)
    u = np.array([-1.0, 1.0, 2.0, np.nan, 0.0, np.inf])
    tokens, _ = run_sample(hl, torch, x, "f32", {}, u)
    assert tokens.tolist() == [0, 3, 3, 0, 0, 3]


@pytest.mark.gpu
def test_sample_settings_that_are_no_numbers(hl, torch):
    """NaN: temperature is greedy, the cuts are off."""
    rng = np.random.default_rng(14)
    x, u, nan = rng.standard_normal((3, 500)), [0.3, 0.6, 0.9], [float("nan")] * 3
    plain = run_sample(hl, torch, x, "f32", {}, u)[0]
    assert np.array_equal(run_sample(hl, torch, x, "f32", {"top_p": nan, "min_p": nan}, u)[0], plain)
    assert np.array_equal(run_sample(hl, torch, x, "f32", {"temperature": nan}, u)[0], x.astype(np.float32).argmax(1))


@pytest.mark.gpu
def test_sample_strides_and_alignment(hl, torch):
    rng = np.random.default_rng(15)
    x = rng.standard_normal((5, 1003)) * 2
    u = rng.random(5)
    for dtype in ("f32", "bf16", "fp16"):
        settings = {"top_k": [50] * 5, "top_p": [0.9] * 5}
        tokens, seen = run_sample(hl, torch, x, dtype, settings, u, vocab=997, stride=1003)
        assert check_samples(tokens, seen, settings, u) >= 4


@pytest.mark.gpu
def test_sample_frequencies(hl, torch):
    """4096 evenly spread numbers give every token its share, to within one of them at either border."""
    x = np.log(np.array([0.1, 0.2, 0.3, 0.15, 0.25]))
    u = (np.arange(4096) + 0.5) / 4096
    tokens, _ = run_sample(hl, torch, np.tile(x, (4096, 1)), "f32", {}, u)
    assert np.all(np.abs(np.bincount(tokens, minlength=5) / 4096 - np.exp(x)) <= 2 / 4096)


# ------------------------------------------------------------------------------------------------ refusals (no device needed)

FAKE = 1 << 20        # an address that is never looked at


def refused(hl, name, call):
    with pytest.raises(hl.HuffllmError) as e:
        call()
    assert e.value.status_name == name, (e.value.status_name, str(e.value))


def test_refusals_of_rotary(hl):
    def call(**kw):
        a = dict(dtype=hl.BF16, tokens=4, head_dim=64, positions=FAKE, frequencies=FAKE, q=FAKE, q_heads=2, q_out=FAKE)
        a.update(kw)
        return lambda: hl.apply_rotary(hl.Rotary(**a), stream=0)
    for kw in (dict(q=None), dict(q_out=None), dict(positions=None), dict(frequencies=None), dict(k=FAKE, k_heads=1), dict(k_out=FAKE), dict(tokens=0),
               dict(q_heads=0), dict(k=FAKE, k_out=FAKE, k_heads=0), dict(dtype=2), dict(pairing=2), dict(rotary_dim=63), dict(rotary_dim=66),
               dict(sections=[16, 15]), dict(sections=[2 ** 31, 2 ** 31, 32 + 1]), dict(q=FAKE + 1), dict(positions=FAKE + 2), dict(q_stride=127),
               dict(q_out_stride=127), dict(q_stride=256), dict(k=FAKE, k_out=FAKE + 64, k_heads=1, k_stride=63)):
        refused(hl, "INVALID_ARG", call(**kw))
    refused(hl, "UNSUPPORTED", call(head_dim=1026, q_stride=1 << 20, q_out_stride=1 << 20))
    refused(hl, "UNSUPPORTED", call(tokens=(1 << 24) + 1))
    with pytest.raises(ValueError):
        hl.Rotary(hl.BF16, 1, 64, FAKE, FAKE, FAKE, 1, FAKE, sections=[8, 8, 8, 4, 4])


def a_cache(hl, **kw):
    a = dict(dtype=hl.BF16, kv_heads=2, head_dim=64, page_tokens=32, pages=9, pool=FAKE, table=FAKE, lengths=FAKE, sequences=3, table_stride=4)
    a.update(kw)
    return hl.Cache(**a)


CACHE_FAULTS = [("INVALID_ARG", dict(dtype=2)), ("INVALID_ARG", dict(kv_heads=0)), ("INVALID_ARG", dict(pages=0)), ("UNSUPPORTED", dict(head_dim=80)),
                ("UNSUPPORTED", dict(head_dim=0)), ("INVALID_ARG", dict(page_tokens=0)), ("INVALID_ARG", dict(page_tokens=24)),
                ("INVALID_ARG", dict(page_tokens=65552)), ("UNSUPPORTED", dict(pages=2 ** 31)), ("UNSUPPORTED", dict(kv_heads=5000))]
POOL_FAULTS = [("INVALID_ARG", dict(pool=None)), ("INVALID_ARG", dict(table=None)), ("INVALID_ARG", dict(lengths=None)), ("INVALID_ARG", dict(pool=FAKE + 128)),
               ("INVALID_ARG", dict(table=FAKE + 2)), ("INVALID_ARG", dict(sequences=0)), ("INVALID_ARG", dict(table_stride=0)),
               ("UNSUPPORTED", dict(sequences=2 ** 20 + 1))]


def test_refusals_of_the_cache(hl):
    assert hl.cache_bytes(a_cache(hl, pool=None, table=None, lengths=None)) == 9 * 2 * 2 * 1280
    assert hl.cache_bytes(a_cache(hl, head_dim=128, page_tokens=16, kv_heads=1, pages=1)) == 16 * 2 * 128 * 5 // 8
    assert hl.cache_bytes(a_cache(hl, pages=2 ** 31 - 1, kv_heads=4096, page_tokens=16)) == (2 ** 31 - 1) * 4096 * 1280
    refused(hl, "UNSUPPORTED", lambda: hl.cache_bytes(a_cache(hl, pages=2 ** 31 - 1, kv_heads=4096, page_tokens=65536)))
    for name, kw in CACHE_FAULTS:
        refused(hl, name, lambda: hl.cache_bytes(a_cache(hl, **kw)))
    for call in (lambda c, **kw: hl.cache_append(c, **{**dict(k_dev=FAKE, v_dev=FAKE, rows=7, starts=FAKE, stream=0), **kw}),
                 lambda c, **kw: hl.cache_read(c, **{**dict(k_dev=FAKE, v_dev=FAKE, elem_type=1, rows=7, starts=FAKE, stream=0), **kw})):
        for name, kw in CACHE_FAULTS + POOL_FAULTS:
            refused(hl, name, lambda: call(a_cache(hl, **kw)))
        for kw in (dict(rows=0), dict(rows=7, starts=None), dict(starts=FAKE + 2), dict(k_dev=None, v_dev=None), dict(k_dev=FAKE + 1), dict(v_dev=FAKE + 1),
                   dict(k_stride=127), dict(v_stride=127), dict(err_flag_dev=FAKE + 1)):
            refused(hl, "INVALID_ARG", lambda: call(a_cache(hl), **kw))
        refused(hl, "UNSUPPORTED", lambda: call(a_cache(hl), rows=2 ** 24 + 1))
    refused(hl, "INVALID_ARG", lambda: hl.cache_append(a_cache(hl), FAKE, None, 7, starts=FAKE, stream=0))
    refused(hl, "INVALID_ARG", lambda: hl.cache_read(a_cache(hl), FAKE, FAKE, 2, 7, starts=FAKE, stream=0))
    refused(hl, "INVALID_ARG", lambda: hl.cache_read(a_cache(hl), FAKE + 2, FAKE, hl.ELEM_F32, 7, starts=FAKE, stream=0))


def test_refusals_of_attention(hl):
    def attention(**kw):
        a = dict(q=FAKE, heads=8, out=FAKE + 4096, rows=7, scale=0.1, starts=FAKE)
        a.update(kw)
        return hl.Attention(**a)
    run = lambda c, a, ws=FAKE, n=1 << 40, err=None: hl.cache_attention(c, a, ws, n, err, stream=0)
    for name, kw in CACHE_FAULTS + POOL_FAULTS:
        refused(hl, name, lambda: run(a_cache(hl, **kw), attention()))
    for kw in (dict(q=None), dict(out=None), dict(out=FAKE), dict(heads=0), dict(heads=7), dict(rows=0), dict(starts=None), dict(starts=FAKE + 2),
               dict(q=FAKE + 1), dict(out=FAKE + 1), dict(q_stride=511), dict(out_stride=511)):
        refused(hl, "INVALID_ARG", lambda: run(a_cache(hl), attention(**kw)))
    refused(hl, "UNSUPPORTED", lambda: run(a_cache(hl), attention(heads=4098)))
    refused(hl, "UNSUPPORTED", lambda: run(a_cache(hl), attention(rows=2 ** 24 + 1)))
    refused(hl, "INVALID_ARG", lambda: run(a_cache(hl), attention(), ws=None))
    refused(hl, "INVALID_ARG", lambda: run(a_cache(hl), attention(), ws=FAKE + 64))
    refused(hl, "INVALID_ARG", lambda: run(a_cache(hl), attention(), err=FAKE + 1))
    n = hl.attention_workspace_bytes(a_cache(hl), attention())
    assert 0 < hl.attention_control_bytes(a_cache(hl), attention()) <= n
    refused(hl, "BUFFER_TOO_SMALL", lambda: run(a_cache(hl), attention(), n=n - 1))


def test_refusals_of_sampling(hl):
    def call(**kw):
        a = dict(logits=FAKE, logits_type=hl.ELEM_F32, rows=3, vocab=100, uniform=FAKE, tokens=FAKE)
        a.update(kw)
        return lambda: hl.sample(hl.Sampling(**a), stream=0)
    for kw in (dict(logits=None), dict(uniform=None), dict(tokens=None), dict(logits_type=2), dict(dtype=2), dict(rows=0), dict(vocab=0), dict(logits=FAKE + 2),
               dict(logits=FAKE + 1, logits_type=hl.ELEM_16), dict(stride=99), dict(temperature=FAKE + 1), dict(top_k=FAKE + 2), dict(top_p=FAKE + 2),
               dict(min_p=FAKE + 2), dict(tokens=FAKE + 2), dict(uniform=FAKE + 1)):
        refused(hl, "INVALID_ARG", call(**kw))
    refused(hl, "UNSUPPORTED", call(rows=2 ** 24 + 1))
    refused(hl, "UNSUPPORTED", call(vocab=2 ** 31))
