"""The choice of the next token at its borders: cuts far below the largest logit, logits next to a cut by min_p, masses of very many tokens,
temperatures at the ends of fp32.  Against 64 bits; helpers are those of the operators' other tests."""
import numpy as np
import pytest

from test_step_operators import hl, run_sample, torch  # noqa: F401


def kept64(x, t, k):
    """The tokens that top_k leaves, in the order of indexes, and their weights in 64 bits."""
    order = np.argsort(-x, kind="stable")[:k]
    kept = np.sort(order)
    return kept, np.exp((x[kept] - x.max()) / t)


@pytest.mark.gpu
def test_top_k_of_three_logits_at_a_low_temperature(hl, torch):  # noqa: F811
    """Places 48 and 70 in the exponent below the largest: the first token is not among the two that stay."""
    x = np.array([[3.0, 10.0, 5.0]] * 4)
    settings = {"temperature": [0.1] * 4, "top_k": [2, 2, 1, 3]}
    assert run_sample(hl, torch, x, "f32", settings, [0.0, 1e-30, 0.0, 0.0])[0].tolist() == [1, 1, 1, 0]
    x = np.array([[-1.0, 0.0, 0.0, 50.0]] * 3)                             # equals at the cut: the first of them stays
    assert run_sample(hl, torch, x, "f32", {"top_k": [2] * 3}, [0.0, 0.5, 1.0])[0].tolist() == [1, 3, 3]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab", [7, 300, 5003, 40009, 140001])
def test_top_k_far_below_the_largest_logit(hl, torch, vocab, dtype):  # noqa: F811
    """The last logits that stay lie 32 to 80 in the exponent below the largest; those that do not lie in front of and behind them.  A draw of 0
    or of next to it takes the first token that stays, one of 1 or more the last.  Weights are above 2^-126, and off by 2e-6 of themselves: a
    draw is held to its token unless the masses up to some token come as near as 1e-5 of the draw."""
    rng = np.random.default_rng(vocab)
    u = np.array([0.0, 1e-30, 1e-20, 1e-13, 1e-10, 1e-9, 1e-5, 0.5, 1.0 - 2.0 ** -24, 1.0, 2.0, 0.0] * 2, np.float32)
    rows = len(u)
    t = rng.choice([0.1, 0.05, 0.3], rows).astype(np.float32)
    k = np.minimum(rng.choice([2, 5, 40, 100, 500], rows), vocab - 1)
    x = np.empty((rows, vocab))
    for i in range(rows):
        x[i] = 10.0 - t[i] * rng.uniform(33, 80, vocab)
        near = rng.choice(vocab, max(1, int(k[i]) // 3), replace=False)
        x[i, near] = 10.0 - t[i] * rng.uniform(0, 31, len(near)) * (np.arange(len(near)) > 0)
        if i % 3 == 0:                                                     # many equals at the cut
            x[i] = np.round(x[i] * 4) / 4
    tokens, seen = run_sample(hl, torch, x, dtype, {"temperature": t.tolist(), "top_k": k.tolist()}, u)
    held = 0
    for i in range(rows):
        kept, w = kept64(seen[i], float(t[i]), int(k[i]))
        assert tokens[i] in kept, (i, u[i], tokens[i])
        run = np.cumsum(w)
        aim = float(u[i]) * run[-1]
        if u[i] >= 1:
            want = kept[-1]
        else:
            at = int(np.searchsorted(run, aim, "right"))
            if u[i] > 0 and np.min(np.abs(run - aim)) < 1e-5 * aim:
                continue
            want = kept[at]
        assert tokens[i] == want, (i, u[i], tokens[i], want)
        held += 1
    assert held >= rows - 6


@pytest.mark.gpu
def test_top_k_that_the_row_cannot_fill(hl, torch):  # noqa: F811
    """top_k of as many as are above minus infinity, of more, and next to the vocabulary: all of them stay, however small."""
    x = np.full((6, 3000), -np.inf)
    x[:, 100:140] = np.linspace(-60, -40, 40)
    x[:, 2000] = 0.0
    k = [41, 42, 500, 2999, 40, 30]
    for u, want in ((0.0, [100] * 4 + [101, 111]), (1.0, [2000] * 6)):
        assert run_sample(hl, torch, x, "f32", {"top_k": k}, [u] * 6)[0].tolist() == want
    x[:, 2500:2510] = np.linspace(-70, -61, 10)                            # behind the largest
    assert run_sample(hl, torch, x, "f32", {"top_k": [51, 60, 50, 2999, 41, 49]}, [1.0] * 6)[0].tolist() == [2509, 2509, 2509, 2509, 2000, 2509]


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [5, 3001, 60001])
def test_min_p_next_to_a_logit(hl, torch, vocab):  # noqa: F811
    """min_p of 1 leaves the largest and its equals, however near the others come; below 1, logits one step of fp32 to either side of the cut."""
    rng = np.random.default_rng(vocab)
    x = np.float32(1.0) - rng.integers(1, 4, (8, vocab)) * np.float32(2.0 ** -24)
    x[:, vocab // 3] = x[:, vocab // 2] = 1.0
    for t in (1.0, 50.0, 1e4):
        for least in (1.0, 2.0):
            got = run_sample(hl, torch, x, "f32", {"temperature": [t] * 8, "min_p": [least] * 8}, [0.0, 0.2, 0.4, 0.49, 0.51, 0.7, 0.99, 1.0])[0]
            assert got.tolist() == [vocab // 3] * 4 + [vocab // 2] * 4, (t, least)
    cases = []
    for least in (0.9, 0.5, 0.1, 0.013):
        for t in (0.7, 1.0, 3.0):
            least32, t32 = float(np.float32(least)), float(np.float32(t))
            cut = np.float32(t32 * np.log(least32))                        # largest logit 0: what is at or above it stays
            if float(cut) < t32 * np.log(least32):
                cut = np.nextafter(cut, np.float32(np.inf))
            cases.append((t32, least32, cut, np.nextafter(cut, np.float32(-np.inf))))
    x = np.full((len(cases), vocab), -np.inf, np.float32)
    for i, (_, _, stays, goes) in enumerate(cases):
        x[i, vocab // 2], x[i, 1], x[i, 0] = 0.0, stays, goes
        x[i, vocab - 1] = goes
    settings = {"temperature": [c[0] for c in cases], "min_p": [c[1] for c in cases]}
    assert run_sample(hl, torch, x, "f32", settings, [0.0] * len(cases))[0].tolist() == [1] * len(cases)
    assert run_sample(hl, torch, x, "f32", settings, [1.0] * len(cases))[0].tolist() == [vocab // 2] * len(cases)


def last_that_stays(n_top, below, n_below, p):
    """n_top tokens of weight 1 and n_below of exp(-below), which lie behind them: how many of those stay, in 64 bits and before rounding up."""
    w = np.exp(-np.float64(below))
    return (p * (n_top + n_below * w) - n_top) / w


@pytest.mark.gpu
@pytest.mark.parametrize("counted", [False, True])
@pytest.mark.parametrize("rows,vocab", [(70, 480000), (300, 60000), (3, 8000000), (1, 1 << 25)])
def test_cuts_by_mass_among_very_many_tokens(hl, torch, rows, vocab, counted):  # noqa: F811
    """Nearly all tokens alike, at the place of a bin of 1/64 in the exponent where weights held in few bits round worst: the number that top_p
    leaves shows what their masses came to.  Weights and their sums are good to 1e-6.  With top_k in front, which leaves out some thousandth of them, too."""
    n_top = vocab // 10
    scan = np.arange(1, 1024, dtype=np.float32) / np.float32(65536.0)
    held = 65536.0 * np.exp(-scan.astype(np.float64))
    below = scan[np.argmin(np.abs(held - np.floor(held) - 0.4999))] + np.float32(7 / 64)
    x = torch.full((rows, vocab), float(-below), device="cuda")
    x[:, :n_top] = 0.0
    x[:, vocab - 1] = -float("inf")                                        # (bins of 1/64)
    p = float(np.float32(0.61234))
    tokens = torch.zeros(rows, dtype=torch.int32, device="cuda")
    top_k = vocab - vocab // 1000
    hl.sample(hl.Sampling(x, hl.ELEM_F32, rows, vocab, torch.ones(rows, device="cuda"), tokens, top_p=torch.full((rows,), p, device="cuda"),
                          top_k=torch.full((rows,), top_k, dtype=torch.int32, device="cuda") if counted else None))
    want = n_top + last_that_stays(n_top, float(below), (top_k if counted else vocab - 1) - n_top, p) - 1
    got = tokens.cpu().numpy()
    assert np.all(np.abs(got - want) <= 1 + 1e-6 * vocab), (got[0], want)


@pytest.mark.gpu
@pytest.mark.parametrize("by", [0.3, 0.7, 1.1])
def test_draws_among_very_many_tokens(hl, torch, by):  # noqa: F811
    """Half of a row has weight 1, the other half exp(-by): where a draw falls shows what either half came to.  Good to 2e-6 of the row."""
    vocab = 1 << 25
    x = torch.zeros((1, vocab), device="cuda")
    x[:, vocab // 2:] = -by
    w = np.exp(-float(np.float32(by)))
    for u in (0.25, 0.5, 0.9):
        tokens = torch.zeros(1, dtype=torch.int32, device="cuda")
        hl.sample(hl.Sampling(x, hl.ELEM_F32, 1, vocab, torch.tensor([u], device="cuda"), tokens))
        aim = float(np.float32(u)) * (1 + w) * (vocab // 2)
        want = aim if aim < vocab // 2 else vocab // 2 + (aim - vocab // 2) / w
        assert abs(int(tokens) - want) <= 2 + 2e-6 * vocab, (u, int(tokens), want)


@pytest.mark.gpu
def test_temperatures_at_the_ends_of_fp32(hl, torch):  # noqa: F811
    """Next to 0 equals at the top share the mass still, and nothing else has any; without bound every token above minus infinity has the same."""
    x = np.array([[1.0, 5.0, 5.0, -2.0, 5.0, -np.inf]] * 3)
    for t in (1e-25, 1e-33, 1e-40):
        assert run_sample(hl, torch, x, "f32", {"temperature": [t] * 3}, [0.1, 0.5, 0.9])[0].tolist() == [1, 2, 4], t
    for t in (1e25, 3e38, float("inf")):
        for extra in ({}, {"top_k": [6] * 3}, {"min_p": [0.5] * 3}, {"top_p": [0.9999] * 3}):
            assert run_sample(hl, torch, x, "f32", {"temperature": [t] * 3, **extra}, [0.1, 0.5, 0.99])[0].tolist() == [0, 2, 4], (t, extra)
