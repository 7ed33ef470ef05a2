"""Attention over the 4-bit cache where its numbers end: queries next to the largest BF16 value, results in FP16, whose weights have to be better
than FP16.  Against 64 bits; helpers are those of the operators' other tests."""
import numpy as np
import pytest

from test_step_operators import Pages, attention_case, check, hl, quantise64, rounding, run_attention, stands_for, to_bits, to_f64, torch, up, values  # noqa: F401


@pytest.mark.gpu
@pytest.mark.parametrize("dim,heads,kv", [(64, 4, 1), (128, 8, 2), (128, 12, 1), (256, 3, 3)])
@pytest.mark.parametrize("power,scale", [(100, 2.0 ** -102), (108, 2.0 ** -110), (120, 2.0 ** -123), (124, 2.0 ** -126)])
def test_queries_next_to_the_largest(hl, torch, dim, heads, kv, power, scale):  # noqa: F811
    """BF16 queries of 2^100 to 2^126, with scales that bring the scores back."""
    attention_case(hl, torch, dim, heads, kv, 16, "bf16", [200, 33, 1], [5, 1, 1], sharp=2.0 ** power, scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("power", [90, 104, 107, 114, 119, 121])
def test_large_queries_with_an_ordinary_scale(hl, torch, power):  # noqa: F811
    """The scores lie so far apart that one token has all of the weight."""
    rng = np.random.default_rng(31)
    n, heads, dim = 100, 4, 128
    p = Pages(hl, torch, "bf16", 1, dim, 32, [n], rng)
    k, v = (to_bits(rng.standard_normal((n, 1, dim)), "bf16") for _ in range(2))
    hl.cache_append(p.cache, up(torch, k, "bf16"), up(torch, v, "bf16"), n, starts=p.starts([n]), err_flag_dev=p.err)
    q = to_bits(rng.standard_normal((1, heads * dim)) * 2.0 ** power, "bf16")
    got = values(run_attention(p, up(torch, q, "bf16"), heads, 1, dim ** -0.5, None, 0, 0)).reshape(heads, dim)
    kx, vx = (stands_for(to_f64(t.reshape(-1), "bf16").reshape(n, dim)) for t in (k, v))
    score = kx @ to_f64(q[0], "bf16").reshape(heads, dim).T
    first = score.argmax(0)
    apart = score.max(0) - np.sort(score, 0)[-2]
    assert np.all(apart > 2.0 ** -10 * score.max(0)), "one token is far ahead of the next"
    want = vx[first]
    # (its weight is 1 exactly; the two products of a channel and their sum: 2^-22 of their magnitudes, which the offsets bound)
    check(got, want, 2.0 ** -21 * 10 * np.ones_like(want), "bf16")


def alike(rng, n, dim):
    """Values of 50 and of -50 in turn, and a little of their own: weights that are nearly equal leave next to nothing of them."""
    return np.where(np.arange(n)[:, None, None] % 2, -50.0, 50.0) + rng.standard_normal((n, 1, dim))


@pytest.mark.gpu
@pytest.mark.parametrize("dim,heads", [(64, 4), (96, 12), (128, 8), (128, 16), (192, 5), (256, 8)])
@pytest.mark.parametrize("n", [4, 8, 30])
def test_fp16_results_have_weights_of_more_than_fp16(hl, torch, dim, heads, n):  # noqa: F811
    """Weights and their products with scales are two fp16 numbers each, 22 bits, where results are FP16.  (With one number each what is left
    of these values is off by up to 50 * 2^-11, many times the bound.)

    Scores: as in the operators' other tests, of queries of one small channel, so that theirs is a small part.  A weight is off by twice its score's error, by 2^-21
    for the exponential and 2^-22 as two numbers, and 2^-22 more times a scale; sums over n by (n + 64) 2^-23.  The second numbers end at 2^-25
    of numbers that are 2^11 at the largest weight or 2^9 over the largest scale."""
    rng = np.random.default_rng(32)
    p = Pages(hl, torch, "fp16", 1, dim, 16, [n], rng)
    k, v = to_bits(rng.standard_normal((n, 1, dim)), "fp16"), to_bits(alike(rng, n, dim), "fp16")
    hl.cache_append(p.cache, up(torch, k, "fp16"), up(torch, v, "fp16"), n, starts=p.starts([n]), err_flag_dev=p.err)
    scale = dim ** -0.5
    q = to_bits(one_channel(rng, heads, dim).reshape(1, -1), "fp16")
    got = values(run_attention(p, up(torch, q, "fp16"), heads, 1, scale, None, 0, 0)).reshape(heads, dim)
    q64 = to_f64(q[0], "fp16").reshape(heads, dim)
    (kx, kmag, koff), (vx, vmag, _), vs = *[parts(to_f64(t.reshape(-1), "fp16").reshape(n, dim)) for t in (k, v)], quantise64(to_f64(v.reshape(-1), "fp16").reshape(n, dim))[1]
    for h in range(heads):
        want, tol = fine64(q64[h], kx, kmag, koff, vx, vmag, vs.max(), scale)
        check(got[h], want, tol, "fp16")


def one_channel(rng, heads, dim):
    q = np.zeros((heads, dim))
    q[np.arange(heads), rng.integers(0, dim, heads)] = 0.004 * dim ** 0.5 * (1 + rng.random(heads))
    return q


def parts(x):
    c, s, m = quantise64(x)
    return (s[..., None] * c + m[..., None]).reshape(x.shape), (s[..., None] * c + np.abs(m)[..., None]).reshape(x.shape), np.repeat(np.abs(m), 32, -1)


def fine64(q, kx, kmag, koff, vx, vmag, most, scale, bits=22):
    n, dim = kx.shape
    x = scale * (kx @ q)
    off = scale * ((2 * dim + 64) * 2.0 ** -23 * (kmag @ np.abs(q)) + 2.0 ** -19 * (koff @ np.abs(q)))
    w = np.exp(x - x.max())
    p = w / w.sum()
    out = p @ vx
    small = 2 * 2.0 ** -25 / min(2.0 ** 11, 2.0 ** 9 / max(most, 2.0 ** -20))
    rel = np.exp(off + off.max()) * (1 + 2.0 ** -21) * (1 + 2.0 ** -bits) ** 2 - 1 + (n + 64) * 2.0 ** -23
    return out, 1.1 * ((p * rel) @ vmag + (p @ rel) * np.abs(out) + small / w.sum() * (vmag.sum(0) + n * np.abs(out)))


def test_the_bound_of_fp16_results_tells_one_number_from_two():
    """(On the CPU: the same with weights, and products with scales, of 11 bits lies outside of it for some of twelve heads.)"""
    rng = np.random.default_rng(32)
    for dim, n in ((64, 4), (96, 8), (128, 8), (128, 30), (256, 8)):
        k, v = (to_f64(to_bits(t, "fp16").reshape(-1), "fp16").reshape(n, dim) for t in (rng.standard_normal((n, 1, dim)), alike(rng, n, dim)))
        (kx, kmag, koff), (vx, vmag, _), (c, s, m) = parts(k), parts(v), quantise64(v)
        outside = []
        for q in one_channel(rng, 12, dim):
            want, tol = fine64(q, kx, kmag, koff, vx, vmag, s.max(), dim ** -0.5)
            x = dim ** -0.5 * (kx @ q)
            w = (np.exp(x - x.max()) * 2.0 ** 11).astype(np.float16).astype(np.float64)
            ws = (w[:, None] * s).astype(np.float16).astype(np.float64)
            got = ((ws[..., None] * c).reshape(n, dim).sum(0) + (w[:, None] * m).repeat(32, 1).sum(0)) / w.sum()
            outside.append(np.max(np.abs(got - want) / (tol + rounding(np.abs(want) + tol, "fp16"))) > 1.5)
        assert sum(outside) >= 2, (dim, n, outside)


@pytest.mark.gpu
@pytest.mark.parametrize("dim,heads,kv,dtype,lengths,counts,window,sinks", [
    (64, 4, 2, "bf16", [600, 257], [600, 257], 0, 0), (128, 8, 2, "fp16", [700], [650], 0, 0), (96, 9, 1, "bf16", [300, 5, 400], [300, 5, 129], 100, 4),
    (128, 5, 1, "bf16", [40, 513], [40, 513], 33, 0), (256, 2, 2, "fp16", [350], [350], 0, 0), (192, 3, 1, "bf16", [0, 270], [7, 270], 64, 20)])
def test_whole_prompts(hl, torch, dim, heads, kv, dtype, lengths, counts, window, sinks):  # noqa: F811
    """Hundreds of new tokens in a call, their own keys among those that they see."""
    attention_case(hl, torch, dim, heads, kv, 64, dtype, lengths, counts, window=window, sinks=sinks)
