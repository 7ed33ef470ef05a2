"""Attention over the 4-bit cache where its numbers end: queries next to the largest BF16 value.  Against 64 bits; helpers are those of the
operators' other tests."""
import numpy as np
import pytest

from test_step_operators import Pages, attention_case, check, hl, run_attention, stands_for, to_bits, to_f64, torch, up, values  # noqa: F401


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
