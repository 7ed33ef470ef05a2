"""A decode step made of the library's calls, as a program runs it: q, k and v from compressed weights, rotary positions, the cache and its
attention, the o projection added to the stream, the feed-forward sub-layer, norm, LM head, the next token.  Also calls of the cache and its
attention in captured graphs, on other streams, and in caches of more than 4 GB.

Tolerances of the step: every 16-bit rounding is off by half a step (2^-8 of the value in BF16), and what follows carries it on; each call is
therefore held against 64 bits of its own inputs as the device has them, with the roundings of that call alone."""
import numpy as np
import pytest

import workloads as wl
from test_step_operators import (Pages, attention64, check, half, ints, rotary64, sample64, stands_for, to_bits, to_f64, up, values)


@pytest.fixture(scope="module")
def hl():
    import paper_2502_00922_b200 as m
    m.lib()
    return m


@pytest.fixture(scope="module")
def torch():
    import torch as t
    return t


def blob(hl, torch, w):
    cb = hl.build_codebook(w)
    host, desc = hl.encode(cb, w, 1024)
    cb.free()
    return desc, torch.from_numpy(host).cuda()


class Layer:
    """One layer's weights, compressed, and what its calls need."""

    def __init__(self, hl, torch, hidden, heads, kv, dim, ffn, vocab, seed):
        gen = lambda r, c, i, std=0.05: wl.gaussian_weights(r, c, std, seed + i)
        self.w = {"q": gen(heads * dim, hidden, 0), "k": gen(kv * dim, hidden, 1), "v": gen(kv * dim, hidden, 2), "o": gen(hidden, heads * dim, 3),
                  "gate": gen(ffn, hidden, 4), "up": gen(ffn, hidden, 5), "down": gen(hidden, ffn, 6), "head": gen(vocab, hidden, 7, 0.1)}
        self.blobs = {n: blob(hl, torch, w) for n, w in self.w.items() if n not in ("gate", "up")}
        self.blobs["gate_up"] = blob(hl, torch, hl.stack_gate_up(self.w["gate"], self.w["up"]))
        self.f64 = {n: to_f64(w, "bf16") for n, w in self.w.items()}


HIDDEN, HEADS, KV, DIM, FFN, VOCAB, PAGE = 256, 4, 2, 64, 512, 4096, 32


def test_decode_steps_refuse_what_the_calls_refuse(hl):
    """(No device: the calls of a step share their checks with the calls alone.)"""
    cache = hl.Cache(hl.BF16, KV, DIM, PAGE, 4, 1 << 20, 1 << 20, 1 << 20, sequences=2, table_stride=4)
    with pytest.raises(hl.HuffllmError):
        hl.cache_attention(cache, hl.Attention(1 << 20, HEADS, 1 << 21, 3, 0.1), 1 << 20, 1 << 30, stream=0)
    with pytest.raises(hl.HuffllmError) as e:
        hl.attention_workspace_bytes(cache, hl.Attention(1 << 20, 4096, 1 << 21, 1 << 20, 0.1, starts=1 << 20))
    assert e.value.status_name == "UNSUPPORTED"


@pytest.mark.gpu
@pytest.mark.parametrize("captured", [False, True])
def test_decode_steps_from_compressed_weights(hl, torch, captured):
    """Three sequences with prompts of their own, then four tokens each; eagerly, and as one captured graph that is replayed while lengths,
    positions and random numbers change in place."""
    rng = np.random.default_rng(21)
    L = Layer(hl, torch, HIDDEN, HEADS, KV, DIM, FFN, VOCAB, 100)
    batch, prompts, steps = 3, [40, 7, 0], 4
    p = Pages(hl, torch, "bf16", KV, DIM, PAGE, [n + steps for n in prompts], rng)
    k0, v0 = (to_bits(rng.standard_normal((sum(prompts), KV, DIM)), "bf16") for _ in range(2))
    p.lengths.copy_(ints(torch, prompts))
    hl.cache_append(p.cache, up(torch, k0, "bf16"), up(torch, v0, "bf16"), sum(prompts), starts=p.starts(prompts), err_flag_dev=p.err)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    stream = torch.zeros((batch, HIDDEN), **bf)                            # the residual stream
    x, att, n = torch.empty((batch, HIDDEN), **bf), torch.empty((batch, HEADS * DIM), **bf), torch.empty((batch, HIDDEN), **bf)
    qkv = torch.empty((batch, (HEADS + 2 * KV) * DIM), **bf)               # side by side, as one row
    q, k, v = qkv[:, :HEADS * DIM], qkv[:, HEADS * DIM:(HEADS + KV) * DIM], qkv[:, (HEADS + KV) * DIM:]
    turned = torch.empty((batch, (HEADS + KV) * DIM), **bf)
    logits, tokens, u = torch.empty((batch, VOCAB), device="cuda"), torch.zeros(batch, dtype=torch.int32, device="cuda"), torch.zeros(batch, device="cuda")
    positions = torch.zeros((1, batch), dtype=torch.int32, device="cuda")
    freq = torch.from_numpy((10000.0 ** (-2.0 * np.arange(DIM // 2) / DIM)).astype(np.float32)).cuda()
    gain = up(torch, to_bits(1 + 0.1 * rng.standard_normal(HIDDEN), "bf16"), "bf16")
    err, row = p.err, (HEADS + 2 * KV) * DIM
    ws = {m: torch.zeros(hl.workspace_bytes(d, batch), dtype=torch.uint8, device="cuda") for m, (d, _) in L.blobs.items()}
    norm0 = hl.PreparedNorm(hl.Norm(hl.BF16, batch, HIDDEN, stream, hl.ELEM_16, gain, 1e-5, x))
    eps = [hl.Epilogue(out_type=hl.ELEM_16, out_stride=row) for _ in range(3)]
    proj = hl.PreparedEpilogue([L.blobs[m][0] for m in "qkv"], [L.blobs[m][1] for m in "qkv"], [x] * 3, batch, eps, [q, k, v], [ws[m] for m in "qkv"],
                               min(ws[m].numel() for m in "qkv"), err)
    rot = hl.PreparedRotary(hl.Rotary(hl.BF16, batch, DIM, positions, freq, q, HEADS, turned, k, KV, turned[:, HEADS * DIM:], q_stride=row, k_stride=row,
                                      q_out_stride=(HEADS + KV) * DIM, k_out_stride=(HEADS + KV) * DIM))
    app = hl.PreparedAppend(p.cache, turned[:, HEADS * DIM:], v, batch, k_stride=(HEADS + KV) * DIM, v_stride=row, err_flag_dev=err)
    attention = hl.Attention(turned, HEADS, att, batch, DIM ** -0.5, window=24, sinks=2, q_stride=(HEADS + KV) * DIM)
    att_ws = torch.zeros(hl.attention_workspace_bytes(p.cache, attention), dtype=torch.uint8, device="cuda")
    attend = hl.PreparedAttention(p.cache, attention, att_ws, att_ws.numel(), err)
    o = hl.PreparedEpilogue([L.blobs["o"][0]], [L.blobs["o"][1]], [att], batch, [hl.Epilogue(out_type=hl.ELEM_16, residual=stream)], [stream], [ws["o"]],
                            ws["o"].numel(), err)
    ffn = hl.Ffn(*L.blobs["gate_up"], *L.blobs["down"], FFN, gain)
    ffn_ws = torch.zeros(hl.ffn_workspace_bytes(ffn, batch), dtype=torch.uint8, device="cuda")
    feed = hl.PreparedFfn(ffn, stream, batch, stream, hl.ELEM_16, ffn_ws, ffn_ws.numel(), err)
    norm1 = hl.PreparedNorm(hl.Norm(hl.BF16, batch, HIDDEN, stream, hl.ELEM_16, gain, 1e-5, n))
    head = hl.PreparedEpilogue([L.blobs["head"][0]], [L.blobs["head"][1]], [n], batch, [hl.Epilogue(out_type=hl.ELEM_F32)], [logits], [ws["head"]],
                               ws["head"].numel(), err)
    top_k, top_p = ints(torch, [50] * batch), torch.full((batch,), 0.9, device="cuda")
    draw = hl.PreparedSampling(hl.Sampling(logits, hl.ELEM_F32, batch, VOCAB, u, tokens, top_k=top_k, top_p=top_p))
    calls = [norm0, proj, rot, app, attend, o, feed, norm1, head, draw]

    def run():
        for call in calls:
            call.run(torch.cuda.current_stream().cuda_stream)

    graph = None
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            keep = [t.clone() for t in (stream, p.pool)]
            p.lengths.copy_(ints(torch, [m + 1 for m in prompts]))
            run()                                                          # (warm)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        stream.copy_(keep[0])
        p.pool.copy_(keep[1])
    held = [[to_f64(t[sum(prompts[:b]): sum(prompts[:b + 1])].reshape(-1), "bf16").reshape(-1, KV, DIM) for b in range(batch)] for t in (k0, v0)]
    for step in range(steps):
        at = [m + step for m in prompts]
        p.lengths.copy_(ints(torch, [m + 1 for m in at]))
        positions.copy_(ints(torch, [at]))
        uu = rng.random(batch).astype(np.float32)
        u.copy_(torch.from_numpy(uu))
        stream.copy_(up(torch, to_bits(rng.standard_normal((batch, HIDDEN)), "bf16"), "bf16"))
        before = values(stream)
        run() if graph is None else graph.replay()
        torch.cuda.synchronize()
        assert p.error() == 0
        xs = values(x)
        for name, t in (("q", q), ("k", k), ("v", v)):
            want = xs @ L.f64[name].T
            check(values(t), want, (HIDDEN + 64) * 2.0 ** -23 * (np.abs(xs) @ np.abs(L.f64[name]).T), "bf16")
        for part, n_heads, t in ((q, HEADS, turned[:, :HEADS * DIM]), (k, KV, turned[:, HEADS * DIM:])):
            want, mag = rotary64(values(part).reshape(batch, n_heads, DIM), np.array([at]), values(freq), DIM, [DIM // 2], False, False)
            check(values(t).reshape(want.shape), want, 4e-7 * mag, "bf16")
        tk, tv, tq = values(turned[:, HEADS * DIM:]).reshape(batch, KV, DIM), values(v).reshape(batch, KV, DIM), values(turned[:, :HEADS * DIM]).reshape(batch, 1, HEADS, DIM)
        for b in range(batch):
            held[0][b], held[1][b] = np.concatenate([held[0][b], tk[b:b + 1]]), np.concatenate([held[1][b], tv[b:b + 1]])
            want, tol = attention64(tq[b], held[0][b], held[1][b], at[b], DIM ** -0.5, 24, 2)
            check(values(att[b]).reshape(want.shape), want, tol, "bf16")
        stream64 = before + values(att) @ L.f64["o"].T                     # (updated in place since: the norm's input is what the feed-forward left)
        assert np.isfinite(values(stream)).all() and not np.array_equal(values(stream), stream64)
        ns = values(n)
        want = ns @ L.f64["head"].T
        tol = (HIDDEN + 64) * 2.0 ** -23 * (np.abs(ns) @ np.abs(L.f64["head"]).T) + 2.0 ** -24 * np.abs(want)
        assert np.all(np.abs(values(logits) - want) <= tol)
        for b in range(batch):
            token, near, kept = sample64(values(logits)[b], 1.0, 50, float(np.float32(0.9)), 0.0, float(uu[b]))
            assert int(tokens[b]) == token or (near < 1e-5 and int(tokens[b]) in kept)


@pytest.mark.gpu
def test_one_workspace_for_captured_graphs_and_eager_calls(hl, torch):
    """Two graphs of different calls and eager calls, one after the other on one workspace, on a stream of their own."""
    rng = np.random.default_rng(22)
    stream = torch.cuda.Stream()
    cases = []
    ws = None
    with torch.cuda.stream(stream):
        for lengths, heads, kv, dim in (([900, 3, 450], 8, 2, 128), ([33] * 40, 12, 4, 64)):
            p = Pages(hl, torch, "bf16", kv, dim, 16, lengths, rng)
            k, v = (to_bits(rng.standard_normal((sum(lengths), kv, dim)), "bf16") for _ in range(2))
            hl.cache_append(p.cache, up(torch, k, "bf16"), up(torch, v, "bf16"), sum(lengths), starts=p.starts(lengths), err_flag_dev=p.err)
            q = up(torch, to_bits(rng.standard_normal((len(lengths), heads * dim)), "bf16"), "bf16")
            a = hl.Attention(q, heads, torch.empty_like(q), len(lengths), dim ** -0.5)
            n = hl.attention_workspace_bytes(p.cache, a)
            ws = torch.zeros(n, dtype=torch.uint8, device="cuda") if ws is None else ws
            assert ws.numel() >= n
            call = hl.PreparedAttention(p.cache, a, ws, n, p.err)
            call.run(stream.cuda_stream)
            stream.synchronize()
            cases.append((p, a._keep[1], call, a._keep[1].clone()))
        graphs = []
        for _, _, call, _ in cases:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                call.run(torch.cuda.current_stream().cuda_stream)
                call.run(torch.cuda.current_stream().cuda_stream)
            graphs.append(g)
        for turn in range(12):
            p, out, call, first = cases[turn % 2]
            out.zero_()
            graphs[turn % 2].replay() if turn % 3 else call.run(stream.cuda_stream)
            cases[(turn + 1) % 2][2].run(stream.cuda_stream)
            stream.synchronize()
            assert p.error() == 0 and torch.equal(out, first), "the same from run to run"


@pytest.mark.gpu
def test_calls_on_two_streams_at_once(hl, torch):
    """Every operator on two streams that run side by side, with buffers of their own."""
    rng = np.random.default_rng(23)
    work = []
    for s in range(2):
        p = Pages(hl, torch, "fp16", 4, 96, 48, [700, 90], rng)
        k, v = (to_bits(rng.standard_normal((790, 4, 96)), "fp16") for _ in range(2))
        x = rng.standard_normal((8, 20001)) * 2
        lg, u, tok = torch.from_numpy(x.astype(np.float32)).cuda(), torch.from_numpy(rng.random(8).astype(np.float32)).cuda(), torch.zeros(8, dtype=torch.int32, device="cuda")
        q = up(torch, to_bits(rng.standard_normal((2, 8 * 96)), "fp16"), "fp16")
        a = hl.Attention(q, 8, torch.empty_like(q), 2, 0.1)
        n = hl.attention_workspace_bytes(p.cache, a)
        pos, freq = ints(torch, [[5, 9000]]), torch.linspace(1, 0.01, 48, device="cuda")
        turned = torch.empty_like(q)
        work.append([hl.PreparedAppend(p.cache, up(torch, k, "fp16"), up(torch, v, "fp16"), 790, starts=p.starts([700, 90]), err_flag_dev=p.err),
                     hl.PreparedAttention(p.cache, a, torch.zeros(n, dtype=torch.uint8, device="cuda"), n, p.err),
                     hl.PreparedRotary(hl.Rotary(hl.FP16, 2, 96, pos, freq, q, 8, turned)),
                     hl.PreparedSampling(hl.Sampling(lg, hl.ELEM_F32, 8, 20001, u, tok, top_p=torch.full((8,), 0.9, device="cuda"))), (a._keep[1], turned, tok)])
    torch.cuda.synchronize()
    main = torch.cuda.current_stream().cuda_stream
    want = []
    for w in work:
        for call in w[:4]:
            call.run(main)
        torch.cuda.synchronize()
        want.append([t.clone() for t in w[4]])
        for t in w[4]:
            t.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(20):
        for w, s in zip(work, streams):
            for call in w[:4]:
                call.run(s.cuda_stream)
    torch.cuda.synchronize()
    for w, expect in zip(work, want):
        assert all(torch.equal(t, e) for t, e in zip(w[4], expect))


@pytest.mark.gpu
def test_cache_of_more_than_four_gigabytes(hl, torch):
    rng = np.random.default_rng(24)
    kv, dim, page, pages, n = 8, 128, 256, 13500, 300
    table, lengths = ints(torch, [[pages - 1, pages - 2]]), ints(torch, [n])
    pool = torch.empty(hl.cache_bytes(hl.Cache(hl.BF16, kv, dim, page, pages)), dtype=torch.uint8, device="cuda")
    assert pool.numel() > 1 << 32
    cache = hl.Cache(hl.BF16, kv, dim, page, pages, pool, table, lengths)
    k, v = (to_bits(rng.standard_normal((n, kv, dim)), "bf16") for _ in range(2))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    hl.cache_append(cache, up(torch, k, "bf16"), up(torch, v, "bf16"), n, starts=ints(torch, [0, n]), err_flag_dev=err)
    back = torch.empty((2, n, kv * dim), device="cuda")
    hl.cache_read(cache, back[0], back[1], hl.ELEM_F32, n, starts=ints(torch, [0, n]), err_flag_dev=err)
    for got, bits in zip(back, (k, v)):
        assert np.array_equal(values(got).reshape(n, kv, dim), stands_for(to_f64(bits.reshape(-1), "bf16").reshape(n, kv, dim)).astype(np.float32))
    q = to_bits(rng.standard_normal((1, 16 * dim)), "bf16")
    out = torch.empty((1, 16 * dim), dtype=torch.bfloat16, device="cuda")
    a = hl.Attention(up(torch, q, "bf16"), 16, out, 1, dim ** -0.5)
    nb = hl.attention_workspace_bytes(cache, a)
    hl.cache_attention(cache, a, torch.zeros(nb, dtype=torch.uint8, device="cuda"), nb, err)
    want, tol = attention64(to_f64(q.reshape(-1), "bf16").reshape(1, 16, dim), *(to_f64(t.reshape(-1), "bf16").reshape(n, kv, dim) for t in (k, v)), n - 1, dim ** -0.5, 0, 0)
    check(values(out).reshape(want.shape), want, tol, "bf16")
    assert int(err.item()) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", [(50, 3), (16, 0), (100, 20)])
def test_pages_that_no_row_sees_may_be_given_away(hl, torch, window, sinks):
    rng = np.random.default_rng(25)
    p = Pages(hl, torch, "bf16", 2, 64, 16, [400], rng)
    k, v = (to_bits(rng.standard_normal((400, 2, 64)), "bf16") for _ in range(2))
    hl.cache_append(p.cache, up(torch, k, "bf16"), up(torch, v, "bf16"), 400, starts=p.starts([400]))
    table = p.host_table.copy()
    gone = [i for i in range(25) if i * 16 >= sinks and i * 16 + 15 <= 397 - window]         # rows are tokens 397, 398 and 399
    table[0, gone] = -1
    p.table.copy_(ints(torch, table))
    q = to_bits(rng.standard_normal((3, 4 * 64)), "bf16")
    out = torch.empty((3, 256), dtype=torch.bfloat16, device="cuda")
    a = hl.Attention(up(torch, q, "bf16"), 4, out, 3, 0.125, starts=ints(torch, [0, 3]), window=window, sinks=sinks)
    n = hl.attention_workspace_bytes(p.cache, a)
    hl.cache_attention(p.cache, a, torch.zeros(n, dtype=torch.uint8, device="cuda"), n, p.err)
    want, tol = attention64(to_f64(q.reshape(-1), "bf16").reshape(3, 4, 64), *(to_f64(t.reshape(-1), "bf16").reshape(400, 2, 64) for t in (k, v)), 397, 0.125, window, sinks)
    assert p.error() == 0 and len(gone) > 10
    check(values(out).reshape(want.shape), want, tol, "bf16")


@pytest.mark.gpu
def test_sequences_that_share_pages_and_many_sequences(hl, torch):
    """1500 sequences, every one with the same first page (a common beginning) and a page of its own."""
    rng = np.random.default_rng(26)
    n, kv, dim, page = 1500, 1, 64, 16
    table = np.stack([np.zeros(n, np.int64), 1 + rng.permutation(n)], 1)
    lengths = rng.integers(17, 33, n)
    pool = torch.full((hl.cache_bytes(hl.Cache(hl.BF16, kv, dim, page, n + 1)),), 255, dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    common = [to_bits(rng.standard_normal((16, kv, dim)), "bf16") for _ in range(2)]
    first = hl.Cache(hl.BF16, kv, dim, page, n + 1, pool, ints(torch, [[0]]), ints(torch, [16]))
    hl.cache_append(first, up(torch, common[0], "bf16"), up(torch, common[1], "bf16"), 16, starts=ints(torch, [0, 16]), err_flag_dev=err)
    cache = hl.Cache(hl.BF16, kv, dim, page, n + 1, pool, ints(torch, table), ints(torch, lengths))
    counts = lengths - 16
    starts = np.concatenate([[0], np.cumsum(counts)])
    own = [to_bits(rng.standard_normal((int(starts[-1]), kv, dim)), "bf16") for _ in range(2)]
    hl.cache_append(cache, up(torch, own[0], "bf16"), up(torch, own[1], "bf16"), int(starts[-1]), starts=ints(torch, starts), err_flag_dev=err)
    q = to_bits(rng.standard_normal((n, 2 * dim)), "bf16")
    out = torch.empty((n, 2 * dim), dtype=torch.bfloat16, device="cuda")
    a = hl.Attention(up(torch, q, "bf16"), 2, out, n, 0.125)
    nb = hl.attention_workspace_bytes(cache, a)
    hl.cache_attention(cache, a, torch.zeros(nb, dtype=torch.uint8, device="cuda"), nb, err)
    assert int(err.item()) == 0
    got = values(out).reshape(n, 1, 2, dim)
    for b in range(0, n, 37):
        k, v = (np.concatenate([to_f64(c.reshape(-1), "bf16"), to_f64(o[starts[b]: starts[b + 1]].reshape(-1), "bf16")]).reshape(-1, kv, dim) for c, o in zip(common, own))
        want, tol = attention64(to_f64(q[b], "bf16").reshape(1, 2, dim), k, v, lengths[b] - 1, 0.125, 0, 0)
        check(got[b], want, tol, "bf16")
