"""Calls of the cache as programs make them: page tables that are part of a larger tensor, arrays of other types,
outputs over queries, starts that do not ascend."""
import numpy as np
import pytest

from test_step_operators import FAKE, Pages, a_cache, attention64, check, hl, ints, refused, run_attention, stands_for, to_bits, to_f64, torch, up, values  # noqa: F401


def test_tables_that_are_part_of_a_larger_tensor(hl, torch):  # noqa: F811
    """The stride is the tensor's; what the call cannot read as it lies, or would read as something else, is refused."""
    whole = torch.zeros((6, 20), dtype=torch.int32)
    lengths = torch.zeros(6, dtype=torch.int32)
    make = lambda table, n=lengths: hl.Cache(hl.BF16, 2, 64, 32, 9, FAKE, table, n)
    for table, sequences, stride in ((whole, 6, 20), (whole[:, :5], 6, 20), (whole[1:4, 3:9], 3, 20), (whole[::2], 3, 40), (whole[:1], 1, 20)):
        c = make(table, lengths[:sequences])
        assert (c.sequences, c.table_stride, c.table) == (sequences, stride, table.data_ptr())
    assert make(np.zeros((3, 8), np.int32)[:, :4], None).table_stride == 8
    for table in (whole.T, whole[:, ::2], whole.long(), whole.float(), np.zeros((3, 8), np.int64)):
        with pytest.raises(ValueError):
            make(table, None)
    for n in (lengths.long(), torch.zeros(12, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            make(whole, n)


def test_arrays_of_other_types_or_with_strides(hl, torch):  # noqa: F811
    i32, f32 = torch.zeros(8, dtype=torch.int32), torch.zeros(8)
    rotary = lambda positions, frequencies: hl.Rotary(hl.BF16, 8, 16, positions, frequencies, FAKE, 1, FAKE)
    attention = lambda starts: hl.Attention(FAKE, 4, FAKE, 7, 0.1, starts=starts)
    sampling = lambda **kw: hl.Sampling(**{**dict(logits=FAKE, logits_type=hl.ELEM_F32, rows=8, vocab=9, uniform=f32, tokens=i32), **kw})
    append = lambda starts, err=None: hl.PreparedAppend(a_cache(hl), FAKE, FAKE, 7, starts=starts, err_flag_dev=err)
    read = lambda starts, err=None: hl.PreparedRead(a_cache(hl), FAKE, FAKE, hl.ELEM_16, 7, starts=starts, err_flag_dev=err)
    rotary(i32[None], f32), attention(i32), sampling(top_k=i32, top_p=f32), append(i32, i32[:1]), read(i32)
    whole = torch.zeros((3, 16), dtype=torch.int32)
    for call in (lambda: rotary(i32.long(), f32), lambda: rotary(whole[:, :8], f32), lambda: rotary(i32, f32.double()), lambda: rotary(i32, f32.half()),
                 lambda: rotary(i32, torch.zeros(16)[::2]), lambda: attention(i32.long()), lambda: attention(np.zeros(8, np.int64)), lambda: append(i32.long()),
                 lambda: append(i32, i32.long()), lambda: read(whole[:, 0]), lambda: sampling(top_k=i32.long()), lambda: sampling(top_k=f32), lambda: sampling(top_p=f32.double()),
                 lambda: sampling(temperature=f32.half()), lambda: sampling(min_p=torch.zeros(16)[::2]), lambda: sampling(uniform=f32.double()), lambda: sampling(tokens=i32.long())):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_a_table_that_is_part_of_a_larger_tensor(hl, torch):  # noqa: F811
    rng = np.random.default_rng(61)
    lengths, kv, dim, heads = [40, 3, 70], 2, 64, 4
    p = Pages(hl, torch, "bf16", kv, dim, 16, lengths, rng)
    whole = torch.full((3, 40), 2 ** 30, dtype=torch.int32, device="cuda")
    whole[:, 4:4 + p.table.shape[1]] = p.table
    p.table = whole[:, 4:4 + p.table.shape[1]]
    p.cache = p._cache(p.pool)
    k, v = (to_bits(rng.standard_normal((113, kv, dim)), "bf16") for _ in range(2))
    hl.cache_append(p.cache, up(torch, k, "bf16"), up(torch, v, "bf16"), 113, starts=p.starts(lengths), err_flag_dev=p.err)
    q = to_bits(rng.standard_normal((3, heads * dim)), "bf16")
    got = values(run_attention(p, up(torch, q, "bf16"), heads, 3, 0.125, None, 0, 0)).reshape(3, 1, heads, dim)
    assert p.error() == 0
    at = 0
    for b, n in enumerate(lengths):
        kb, vb = (to_f64(t[at: at + n].reshape(-1), "bf16").reshape(n, kv, dim) for t in (k, v))
        want, tol = attention64(to_f64(q[b], "bf16").reshape(1, heads, dim), kb, vb, n - 1, 0.125, 0, 0)
        check(got[b], want, tol, "bf16")
        at += n


def test_outputs_over_queries_are_refused(hl):  # noqa: F811
    """Where the strides are alike every overlap shows: rows of 512 values (1024 bytes), 7 of them."""
    run = lambda **kw: hl.cache_attention(a_cache(hl), hl.Attention(**{**dict(heads=8, rows=7, scale=0.1, starts=FAKE), **kw}), FAKE, 1 << 40, stream=0)
    q = 1 << 24
    for out, stride in ((q + 2, 0), (q - 2, 0), (q + 1022, 0), (q + 7 * 1024 - 2, 0), (q - 7 * 1024 + 2, 0), (q + 1022, 2048), (q - 1022, 2048), (q + 4096 + 2, 2048),
                        (q + 4096 - 1022, 2048), (q, 2048), (q + 6 * 4096 + 1022, 2048)):
        refused(hl, "INVALID_ARG", lambda: run(q=q, out=out, q_stride=stride, out_stride=stride))


@pytest.mark.gpu
def test_outputs_between_queries(hl, torch):  # noqa: F811
    """Rows of a tensor that have queries and outputs side by side."""
    rng = np.random.default_rng(62)
    lengths, kv, dim, heads = [40, 3, 70], 2, 64, 4
    p = Pages(hl, torch, "bf16", kv, dim, 16, lengths, rng)
    k, v = (to_bits(rng.standard_normal((113, kv, dim)), "bf16") for _ in range(2))
    hl.cache_append(p.cache, up(torch, k, "bf16"), up(torch, v, "bf16"), 113, starts=p.starts(lengths), err_flag_dev=p.err)
    q = to_bits(rng.standard_normal((3, 2 * heads * dim)), "bf16")
    both = up(torch, q, "bf16")
    apart = values(run_attention(p, up(torch, q, "bf16"), heads, 3, 0.125, None, 0, 0, q_stride=512)).reshape(3, -1)
    for first in (0, 256):
        both.copy_(up(torch, q if first == 0 else np.roll(q, 256, 1), "bf16"))
        run_attention(p, both[:, first:], heads, 3, 0.125, None, 0, 0, 512, 512, out=both[:, 256 - first:])
        assert p.error() == 0 and np.array_equal(values(both)[:, 256 - first: 512 - first], apart)


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [[0, 40, 30, 50], [0, 40, 20, 10], [50, 40, 30, 50], [0, 110, 90, 110], [100, 0, 90, 110], [-5, 40, 90, 110], [0, 40, 90, 111]])
def test_starts_that_do_not_ascend(hl, torch, bad):  # noqa: F811
    """A sequence whose starts are no rows is named.  Every token is what it was, or what its own row says; what is read goes to rows of its own."""
    rng = np.random.default_rng(63)
    lengths, kv, dim = [40, 50, 20], 2, 64
    p = Pages(hl, torch, "bf16", kv, dim, 16, lengths, rng)
    old, new = ([to_bits(rng.standard_normal((110, kv, dim)), "bf16") for _ in range(2)] for _ in range(2))
    stands = lambda bits: stands_for(to_f64(bits.reshape(-1), "bf16").reshape(110, kv, dim))

    def cache_read(starts):
        out = [torch.full((110, kv * dim), 7.0, device="cuda") for _ in range(2)]
        p.err.zero_()
        hl.cache_read(p.cache, out[0], out[1], hl.ELEM_F32, 110, starts=ints(torch, starts), err_flag_dev=p.err)
        return [values(t).reshape(110, kv, dim) for t in out], p.error()
    good = [0, 40, 90, 110]
    at_fault = [b + 1 for b in range(3) if not 0 <= bad[b] <= bad[b + 1] <= 110]
    hl.cache_append(p.cache, up(torch, old[0], "bf16"), up(torch, old[1], "bf16"), 110, starts=ints(torch, good), err_flag_dev=p.err)
    assert p.error() == 0
    got, err = cache_read(bad)
    assert err in at_fault
    for side in range(2):
        want = stands(old[side])
        for r in range(110):                               # the tokens that row r may be
            may = [want[good[b] + lengths[b] - bad[b + 1] + r] for b in range(3)
                   if b + 1 not in at_fault and bad[b] <= r < bad[b + 1] and lengths[b] - bad[b + 1] + r >= 0]
            assert np.all(got[side][r] == 7.0) or any(np.array_equal(got[side][r], m) for m in may), r
    p.err.zero_()
    hl.cache_append(p.cache, up(torch, new[0], "bf16"), up(torch, new[1], "bf16"), 110, starts=ints(torch, bad), err_flag_dev=p.err)
    assert p.error() in at_fault
    got, err = cache_read(good)
    assert err == 0
    for side in range(2):
        was, now = stands(old[side]), stands(new[side])
        for b in range(3):
            for i in range(lengths[b]):
                row = bad[b + 1] - lengths[b] + i
                may = [was[good[b] + i]] + ([now[row]] if b + 1 not in at_fault and bad[b] <= row < bad[b + 1] else [])
                assert any(np.array_equal(got[side][good[b] + i], m) for m in may), (b, i)
