"""The products of a decode step behind its attention, each against 64 bits of its own inputs: the o projection added to the stream, and the
feed-forward sub-layer on what that leaves."""
import numpy as np
import pytest

from test_decode_step import DIM, FFN, HEADS, HIDDEN, KV, PAGE, VOCAB, Layer
from test_layer_operators import F32, Sums, norm64
from test_step_operators import Pages, check, hl, rounding, to_bits, to_f64, torch, up, values  # noqa: F401


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 3])
def test_o_projection_and_feed_forward_behind_attention(hl, torch, batch):  # noqa: F811
    rng = np.random.default_rng(51)
    L = Layer(hl, torch, HIDDEN, HEADS, KV, DIM, FFN, VOCAB, 300)
    lengths = [60, 9, 33][:batch]
    p = Pages(hl, torch, "bf16", KV, DIM, PAGE, lengths, rng)
    k, v = (to_bits(rng.standard_normal((sum(lengths), KV, DIM)), "bf16") for _ in range(2))
    hl.cache_append(p.cache, up(torch, k, "bf16"), up(torch, v, "bf16"), sum(lengths), starts=p.starts(lengths), err_flag_dev=p.err)
    q = up(torch, to_bits(rng.standard_normal((batch, HEADS * DIM)), "bf16"), "bf16")
    att, gain = torch.empty_like(q), up(torch, to_bits(1 + 0.1 * rng.standard_normal(HIDDEN), "bf16"), "bf16")
    stream = up(torch, to_bits(rng.standard_normal((batch, HIDDEN)), "bf16"), "bf16")
    a = hl.Attention(q, HEADS, att, batch, DIM ** -0.5)
    n = hl.attention_workspace_bytes(p.cache, a)
    hl.cache_attention(p.cache, a, torch.zeros(n, dtype=torch.uint8, device="cuda"), n, p.err)
    ws = torch.zeros(hl.workspace_bytes(L.blobs["o"][0], batch), dtype=torch.uint8, device="cuda")
    before = values(stream)
    hl.PreparedEpilogue([L.blobs["o"][0]], [L.blobs["o"][1]], [att], batch, [hl.Epilogue(out_type=hl.ELEM_16, residual=stream)], [stream], [ws], ws.numel(),
                        p.err).run(torch.cuda.current_stream().cuda_stream)
    s = Sums(L.f64["o"], values(att).reshape(batch, -1))
    want = before + s.v
    assert np.abs(s.v).max() > 20 * (s.tol + rounding(want, "bf16")).max(), "what the projection adds is far above the tolerance"
    h = values(stream)
    check(h, want, s.tol + F32 * np.abs(want), "bf16")

    # the sub-layer, and its three steps one by one
    ffn = hl.Ffn(*L.blobs["gate_up"], *L.blobs["down"], FFN, gain)
    size = hl.ffn_workspace_bytes(ffn, batch)
    after, steps = torch.empty_like(stream), torch.empty_like(stream)
    hl.decode_ffn(ffn, stream, batch, after, hl.ELEM_16, torch.zeros(size, dtype=torch.uint8, device="cuda"), size, p.err)
    nrm, mid = torch.empty_like(stream), torch.empty((batch, FFN), dtype=torch.bfloat16, device="cuda")
    hl.add_rms_norm(hl.Norm(hl.BF16, batch, HIDDEN, stream, hl.ELEM_16, gain, 1e-5, nrm))
    for name, x, epilogue, out in (("gate_up", nrm, hl.Epilogue(hl.ACT_SILU, hl.ELEM_16, gated_rows=FFN), mid), ("down", mid, hl.Epilogue(out_type=hl.ELEM_16, residual=stream), steps)):
        ws = torch.zeros(hl.workspace_bytes(L.blobs[name][0], batch), dtype=torch.uint8, device="cuda")
        hl.decode_gemm_epilogue(*L.blobs[name], x, batch, epilogue, out, ws, ws.numel(), p.err)
    assert p.error() == 0 and torch.equal(after, steps)
    n64 = norm64(h, to_f64(gain.view(torch.int16).cpu().numpy().view(np.uint16), "bf16"), 1e-5)
    check(values(nrm), n64, np.abs(n64) * ((HIDDEN + 16) * F32 + 2.0 ** -22), "bf16")
    gate, g = Sums(L.f64["gate"], values(nrm)).through("silu"), Sums(L.f64["up"], values(nrm))
    want = gate[0] * g.v
    check(values(mid), want, np.abs(gate[0]) * g.tol + np.abs(g.v) * gate[1] + gate[1] * g.tol + F32 * np.abs(want), "bf16")
    d = Sums(L.f64["down"], values(mid))
    assert np.abs(d.v).max() > 20 * (d.tol + rounding(h + d.v, "bf16")).max()
    check(values(after), h + d.v, d.tol + F32 * np.abs(h + d.v), "bf16")
