"""Ways to make the calls of the layer operators: prepared, one matrix as a list, one blob twice in a launch, captured graphs and
eager calls that take turns on a workspace."""
import numpy as np
import pytest

import workloads as wl
from test_layer_operators import Blob, FfnCase, assert_clean, f_to_bits, hl, norm_case, torch, up, workspace, x_of  # noqa: F401


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 6, 12, 40])
def test_prepared_calls_are_the_calls(hl, torch, batch):  # noqa: F811
    """Over one matrix and over several, the norm and the sub-layer; on a stream of their own, run more than once; in-place updates go on from what
    they find."""
    cols, rows = 512, (300, 77)
    blobs = [Blob(hl, torch, wl.gaussian_weights(r, cols, 0.05, r), "bf16") for r in rows]
    n, wss = workspace(hl, torch, blobs, batch)
    x = up(torch, x_of(batch, cols, 1, "bf16"), "bf16")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    bias = up(torch, f_to_bits(np.random.default_rng(2).standard_normal(rows[0]), "bf16"), "bf16")
    stream = torch.cuda.Stream()
    hs = [torch.randn((batch, r), device="cuda") for r in rows]

    def epilogues(outs):
        return [hl.Epilogue(hl.ACT_SILU, bias=bias, residual=outs[0]), hl.Epilogue(residual=outs[1])]

    def called():
        outs = [h.clone() for h in hs]
        eps = epilogues(outs)
        for _ in range(2):
            hl.decode_gemm_epilogue(blobs[0].desc, blobs[0].dev, x, batch, eps[0], outs[0], wss[0], n, err)
        one = outs[0].clone()
        outs[0].copy_(hs[0])
        for _ in range(2):
            hl.decode_gemm_multi_epilogue([b.desc for b in blobs], [b.dev for b in blobs], [x] * 2, batch, eps, outs, wss, n, err)
        torch.cuda.synchronize()
        return one, outs

    def prepared():
        outs = [h.clone() for h in hs]
        eps = epilogues(outs)
        alone = hl.PreparedEpilogue([blobs[0].desc], [blobs[0].dev], [x], batch, eps[:1], outs[:1], wss[:1], n, err)
        both = hl.PreparedEpilogue([b.desc for b in blobs], [b.dev for b in blobs], [x] * 2, batch, eps, outs, wss, n, err)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for _ in range(2):
                alone.run(stream.cuda_stream)
            one = outs[0].clone()
            outs[0].copy_(hs[0])
            for _ in range(2):
                both.run(stream.cuda_stream)
        stream.synchronize()
        return one, outs
    (one, outs), (one2, outs2) = called(), prepared()
    assert torch.equal(one, one2) and all(torch.equal(a, b) for a, b in zip(outs, outs2)) and int(err.item()) == 0
    for b, ws in zip(blobs, wss):
        assert_clean(hl, b, ws, err)

    c = FfnCase(hl, torch, 96, 160, "bf16", seed=4)
    size = hl.ffn_workspace_bytes(c.ffn, batch)
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    h = torch.randn((batch, 96), device="cuda")
    a, b, na, nb = torch.empty_like(h), torch.empty_like(h), *(torch.empty((batch, 96), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    hl.decode_ffn(c.ffn, h, batch, a, hl.ELEM_F32, ws, size, err)
    hl.add_rms_norm(hl.Norm(hl.BF16, batch, 96, a, hl.ELEM_F32, c.dev[0], 1e-5, na))
    torch.cuda.synchronize()
    ffn = hl.PreparedFfn(c.ffn, h, batch, b, hl.ELEM_F32, ws, size, err)
    norm = hl.PreparedNorm(hl.Norm(hl.BF16, batch, 96, b, hl.ELEM_F32, c.dev[0], 1e-5, nb))
    for _ in range(3):
        ffn.run(stream.cuda_stream)
        norm.run(stream.cuda_stream)
    stream.synchronize()
    assert torch.equal(a, b) and torch.equal(na, nb) and int(err.item()) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 8, 12, 33])
def test_one_matrix_as_a_list_and_one_blob_twice(hl, torch, batch):  # noqa: F811
    cols, rows = 1024, 500
    blob = Blob(hl, torch, wl.gaussian_weights(rows, cols, 0.05, 1), "bf16")
    n, wss = workspace(hl, torch, [blob] * 2, batch)
    xs = [up(torch, x_of(batch, cols, s, "bf16"), "bf16") for s in (1, 2)]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ep = hl.Epilogue(hl.ACT_GELU_TANH)
    new = lambda: torch.full((batch, rows), float("nan"), device="cuda")
    alone, twice, single = [new(), new()], [new(), new()], new()
    for x, out in zip(xs, alone):
        hl.decode_gemm_epilogue(blob.desc, blob.dev, x, batch, ep, out, wss[0], n, err)
    hl.decode_gemm_multi_epilogue([blob.desc] * 2, [blob.dev] * 2, xs, batch, [ep] * 2, twice, wss, n, err)
    hl.decode_gemm_multi_epilogue([blob.desc], [blob.dev], xs[:1], batch, [ep], [single], wss[:1], n, err)
    torch.cuda.synchronize()
    # (sums may be taken in another order: 1024 products of some 0.05, 2^-23 of each at most)
    scale = 1024 * 2.0 ** -23 * 1024 * 0.05
    for got, want in [(single, alone[0])] + list(zip(twice, alone)):
        assert torch.all(torch.abs(got - want) <= scale)
    for ws in wss:
        assert_clean(hl, blob, ws, err)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 12, 40])
def test_captured_graphs_and_calls_take_turns_on_a_workspace(hl, torch, batch):  # noqa: F811
    """A matrix whose items outnumber the CTAs and one of fewer: graphs replayed between eager calls on the same workspaces, one after the other."""
    mats = [(700, 1024, 1024), (40000, 256, 512)]
    blobs = [Blob(hl, torch, wl.gaussian_weights(r, c, 0.05, r), "bf16", chunk) for r, c, chunk in mats]
    n = max(hl.workspace_bytes(b.desc, batch) for b in blobs)
    wss = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in mats]
    xs = [up(torch, x_of(batch, c, r, "bf16"), "bf16") for r, c, _ in mats]
    outs = [torch.zeros((batch, r), device="cuda") for r, _, _ in mats]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()

    def call(i):
        hl.decode_gemm_epilogue(blobs[i].desc, blobs[i].dev, xs[i], batch, hl.Epilogue(hl.ACT_RELU, residual=outs[i]), outs[i], wss[i], n, err, stream)
    want = []
    for i in (0, 1):
        call(i)
        stream.synchronize()
        want.append(outs[i].clone())
    graphs = []
    for i in (0, 1):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            call(i)
        graphs.append(g)
    for i in (0, 1, 1, 0, 1, 0, 0):
        outs[i].zero_()
        torch.cuda.synchronize()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i], want[i])
        outs[i].zero_()
        torch.cuda.synchronize()
        call(i)
        stream.synchronize()
        assert torch.equal(outs[i], want[i])
    for b, w in zip(blobs, wss):
        assert_clean(hl, b, w, err)


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [32769, 40001, 65536])
@pytest.mark.parametrize("over", ["x", "delta"])
def test_long_vectors_updated_in_place(hl, torch, cols, over):  # noqa: F811
    """Vectors that a CTA goes through twice: the second time every value is read by the thread that then writes it."""
    g = torch.Generator(device="cuda").manual_seed(cols)
    for t, elem in ((torch.bfloat16, hl.ELEM_16), (torch.float32, hl.ELEM_F32)):
        x, d = (torch.randn((3, cols), generator=g, device="cuda").to(t) for _ in range(2))
        results = []
        for place in (None, over):
            a, b = x.clone(), d.clone()
            s = torch.empty_like(a) if place is None else a if place == "x" else b
            o = torch.empty((3, cols), dtype=torch.bfloat16, device="cuda")
            hl.add_rms_norm(hl.Norm(hl.BF16, 3, cols, a, elem, None, 1e-6, o, b, elem, s))
            torch.cuda.synchronize()
            results.append((s.clone(), o))
        assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])


@pytest.mark.gpu
@pytest.mark.parametrize("x16,delta", [(True, "16"), (False, "f32"), (False, None)])
def test_very_long_vectors(hl, torch, x16, delta):  # noqa: F811
    norm_case(hl, torch, 2, 1_000_003, "bf16", x16, delta, True, True, pad=5, seed=1)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 5, 12, 40])
@pytest.mark.parametrize("out16", [True, False])
def test_outs_side_by_side_in_one_buffer(hl, torch, batch, out16):  # noqa: F811
    """q, k and v of a token next to each other, as attention wants them: three outs with the buffer's stride; the same values as in buffers of their own."""
    cols, rows = 512, (512, 128, 130)
    blobs = [Blob(hl, torch, wl.gaussian_weights(r, cols, 0.05, i), "bf16") for i, r in enumerate(rows)]
    n, wss = workspace(hl, torch, blobs, batch)
    x = up(torch, x_of(batch, cols, 1, "bf16"), "bf16")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    t, elem = (torch.bfloat16, hl.ELEM_16) if out16 else (torch.float32, hl.ELEM_F32)
    ld = sum(rows) + 6
    buf = torch.full((batch, ld), 77.0, dtype=t, device="cuda")
    at = [0, rows[0], rows[0] + rows[1]]
    own = [torch.empty((batch, r), dtype=t, device="cuda") for r in rows]
    for eps, outs in (([hl.Epilogue(hl.ACT_SILU, elem, out_stride=ld)] * 3, [buf[:, a:] for a in at]), ([hl.Epilogue(hl.ACT_SILU, elem)] * 3, own)):
        hl.decode_gemm_multi_epilogue([b.desc for b in blobs], [b.dev for b in blobs], [x] * 3, batch, eps, outs, wss, n, err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    for a, r, o in zip(at, rows, own):
        assert torch.equal(buf[:, a:a + r], o)
    assert torch.all(buf[:, sum(rows):] == 77.0)
