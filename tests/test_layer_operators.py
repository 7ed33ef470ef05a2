"""What a decoder layer does around its products from compressed weights: epilogues (bias, activation, residual, rounding), gated
products, residual addition and norm, the feed-forward sub-layer.  Against plain implementations in 64 bits.

Tolerances.  A sum of n products taken in fp32 in any order is off by at most n steps of 2^-24 of the sum of the products' magnitudes,
or of 2^-23 where the tensor cores' accumulators cut off instead of rounding: (cols + 64) 2^-23 sum |w x| (Sums).  The activations'
slopes are at most 1.13, and the functions are computed within 2e-6 (1 + |v|) of v's value: a few units in the last place of exp, erfc and
the quotient, and exponents off by a few parts in 2^24 where the result falls off faster than they grow.  The additions of bias and
residual round once each (2^-24), and 16-bit results once more: half a step, finfo.eps / 2 of the value (fp16: or half of 2^-24)."""
import math

import numpy as np
import pytest

import workloads as wl

SLOPE, FUNC, F32 = 1.13, 2e-6, 2.0 ** -24
HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}      # finfo.eps / 2
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


@pytest.fixture(scope="module")
def hl():
    import paper_2502_00922_b200 as m
    m.lib()
    return m


@pytest.fixture(scope="module")
def torch():
    import torch as t
    return t


def bits_to_f64(b, dtype):
    b = np.ascontiguousarray(b, dtype=np.uint16)
    return (wl.bf16_bits_to_f32(b) if dtype == "bf16" else b.view(np.float16).astype(np.float32)).astype(np.float64)


def f_to_bits(a, dtype):
    a = np.ascontiguousarray(a, dtype=np.float32)
    return wl.f32_to_bf16_bits(a) if dtype == "bf16" else a.astype(np.float16).view(np.uint16)


def half(torch, dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float16


def up(torch, bits, dtype):
    """Bit patterns -> tensor of the 16-bit type on the device."""
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(half(torch, dtype))


erf64 = np.vectorize(math.erf, otypes=[np.float64])


def act64(v, act):
    with np.errstate(over="ignore", invalid="ignore"):
        if act == "relu":
            return np.where(v < 0, 0.0, v)
        if act == "silu":
            return v / (1 + np.exp(-v))
        if act == "gelu":
            return 0.5 * v * (1 + erf64(v / np.sqrt(2.0)))
        if act == "gelu_tanh":
            return 0.5 * v * (1 + np.tanh(np.sqrt(2 / np.pi) * (v + 0.044715 * v ** 3)))
    return v


def rounding(y, out):
    """Largest error of the final rounding of values y (|y| given) to `out` ("f32", "bf16", "fp16")."""
    y = np.abs(y)
    return y * F32 if out == "f32" else y * HALF_STEP[out] + (2.0 ** -25 if out == "fp16" else 0.0)


class Sums:
    """W x in 64 bits and how far an fp32 sum may be from it."""

    def __init__(self, w, x):                       # [rows][cols], [batch][cols] in 64 bits
        self.v = x @ w.T
        self.tol = (w.shape[1] + 64) * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T)

    def plus(self, bias):
        if bias is not None:
            self.v = self.v + bias
            self.tol = self.tol + F32 * np.abs(self.v) + F32 * self.tol
        return self

    def through(self, act):
        if act == "none":
            return self.v, self.tol
        return act64(self.v, act), SLOPE * self.tol + FUNC * (1 + np.abs(self.v))


def check(got, want, tol, out):
    tol = tol + rounding(np.abs(want) + tol, out)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} outside, worst {np.nanmax(np.abs(got - want) / tol)} of the tolerance at {np.argwhere(bad)[0]}"


def values(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Blob:
    def __init__(self, hl, torch, w, dtype, chunk=1024, limit=0):
        cb = hl.build_codebook(w, hl.BF16 if dtype == "bf16" else hl.FP16, limit)
        host, self.desc = hl.encode(cb, w, chunk)
        cb.free()
        self.host = host
        self.dev = torch.from_numpy(host).cuda() if torch is not None else None


def workspace(hl, torch, blobs, batch):
    n = max(hl.workspace_bytes(b.desc, batch) for b in blobs)
    return n, [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in blobs]


def assert_clean(hl, blob, ws, err):
    assert int(err.item()) == 0
    assert int(ws[:hl.workspace_control_bytes(blob.desc)].count_nonzero().item()) == 0, "the control words must be left zero"


def x_of(batch, cols, seed, dtype):
    return wl.activations(batch, cols, seed, dtype)


# ------------------------------------------------------------------------------------------------ no GPU needed

@pytest.mark.parametrize("n,cols", [(1, 1), (1, 5), (7, 3), (8, 4), (9, 4), (16, 1), (23, 32), (64, 33)])
def test_stacking_puts_eight_gate_rows_before_the_eight_up_rows_of_the_same_outputs(hl, n, cols):
    rng = np.random.default_rng(n * 100 + cols)
    gate, up_ = (rng.integers(0, 65536, (n, cols), dtype=np.uint16) for _ in range(2))
    got = hl.stack_gate_up(gate, up_)
    assert got.shape == (hl.stacked_rows(n), cols) and hl.stacked_rows(n) == -(-n // 8) * 16
    for r in range(got.shape[0]):
        i = min(r // 16 * 8 + r % 8, n - 1)
        assert np.array_equal(got[r], (up_ if r % 16 >= 8 else gate)[i])


def test_stacking_is_refused(hl):
    g = np.zeros((8, 4), np.uint16)
    buf = np.zeros(8 * 4 * 4, np.uint16)
    L = hl.lib()
    for args in [(None, g.ctypes.data, 8, 4, buf.ctypes.data), (g.ctypes.data, g.ctypes.data, 0, 4, buf.ctypes.data),
                 (g.ctypes.data, g.ctypes.data, 8, 0, buf.ctypes.data), (g.ctypes.data, g.ctypes.data, (1 << 30) + 1, 4, buf.ctypes.data),
                 (buf.ctypes.data + 32, g.ctypes.data, 8, 4, buf.ctypes.data), (g.ctypes.data, buf.ctypes.data + 126, 8, 4, buf.ctypes.data)]:
        assert L.huffllm_stack_gate_up(*args) == 1
        assert L.huffllm_stack_gate_up_device(*args, None) == 1
    assert L.huffllm_stacked_rows(8, None) == 1
    with pytest.raises(ValueError):
        hl.stack_gate_up(g, g[:4])


def test_remembered_plans_are_those_worked_out_anew(hl):
    """Launch plans are kept per thread by the numbers that they follow from: more questions than are kept, in several orders, against threads
    that have kept nothing."""
    import threading
    descs = []
    for dtype, limit, chunk in (("bf16", 0, 1024), ("bf16", 9, 512), ("fp16", 0, 1024)):
        for rows, cols in ((64, 512), (700, 512), (64, 4096)):
            descs.append(Blob(hl, None, wl.gaussian_weights(rows, cols, 0.02, rows, dtype), dtype, chunk, limit).desc)
    questions = [(d, b, w) for d in descs for b in (9, 17, 64) for w in (0, hl.workspace_bytes(d, b), hl.workspace_bytes(d, b) + (1 << 22))]
    ask = lambda q: hl.gemm_launch_plan([q[0]], q[1], q[2])
    anew = []
    for q in questions:
        t = threading.Thread(target=lambda: anew.append(ask(q)))
        t.start()
        t.join()
    assert len(anew) == len(questions)
    order = list(range(len(questions)))
    for seed in range(3):
        np.random.default_rng(seed).shuffle(order)
        for i in order + order[::-1]:
            assert ask(questions[i]) == anew[i]


def status(call):
    from paper_2502_00922_b200 import HuffllmError
    try:
        call()
    except HuffllmError as e:
        return e.status_name
    return "OK"


def refusals(hl, desc, ws_bytes):
    """(what, arguments of decode_gemm_epilogue after desc, expected status); addresses are never followed."""
    A = 1 << 20                                            # some aligned address
    good = dict(blob_dev=A, x_dev=A, batch=2, epilogue=hl.Epilogue(), out_dev=A, workspace_dev=A, workspace_bytes_=ws_bytes, stream=0)
    E = hl.Epilogue
    cases = [("unknown activation", dict(epilogue=E(activation=5)), "INVALID_ARG"),
             ("unknown type", dict(epilogue=E(out_type=2)), "INVALID_ARG"),
             ("no out", dict(out_dev=None), "INVALID_ARG"),
             ("fp32 out off 4 bytes", dict(out_dev=A + 2), "INVALID_ARG"),
             ("16-bit out off 2 bytes", dict(out_dev=A + 1, epilogue=E(out_type=hl.ELEM_16)), "INVALID_ARG"),
             ("residual off its type", dict(epilogue=E(residual=A + 2)), "INVALID_ARG"),
             ("bias off its type", dict(epilogue=E(bias=A + 1)), "INVALID_ARG"),
             ("short out stride", dict(epilogue=E(out_stride=desc.rows - 1)), "INVALID_ARG"),
             ("short residual stride", dict(epilogue=E(residual=A, residual_stride=1)), "INVALID_ARG"),
             ("in place with another stride", dict(epilogue=E(residual=A, residual_stride=desc.rows, out_stride=desc.rows + 8)), "INVALID_ARG"),
             ("gates of another blob", dict(epilogue=E(gated_rows=desc.rows // 2 + 1)), "INVALID_ARG"),
             ("too few gates", dict(epilogue=E(gated_rows=desc.rows // 2 - 8)), "INVALID_ARG"),
             ("gates without end", dict(epilogue=E(gated_rows=(1 << 64) - 1)), "INVALID_ARG"),
             ("gated with residual", dict(epilogue=E(gated_rows=desc.rows // 2, residual=A)), "UNSUPPORTED"),
             ("no vectors", dict(batch=0), "INVALID_ARG"),
             ("too many vectors", dict(batch=65), "INVALID_ARG"),
             ("small workspace", dict(workspace_bytes_=ws_bytes - 1), "BUFFER_TOO_SMALL"),
             ("x off 16 bytes", dict(x_dev=A + 8), "INVALID_ARG")]
    return [(what, {**good, **change}, want) for what, change, want in cases]


def test_epilogues_are_refused_before_anything_is_launched(hl):
    w = wl.gaussian_weights(64, 96, 0.02, 1)
    b = Blob(hl, None, w, "bf16")
    ws_bytes = hl.workspace_bytes(b.desc, 2)
    for what, args, want in refusals(hl, b.desc, ws_bytes):
        blob, rest = args.pop("blob_dev"), args
        assert status(lambda: hl.decode_gemm_epilogue(b.desc, blob, **rest)) == want, what
        multi = dict(blobs_dev=[blob] * 2, xs_dev=[rest["x_dev"]] * 2, batch=rest["batch"], epilogues=[hl.Epilogue(), rest["epilogue"]],
                     outs_dev=[1 << 20, rest["out_dev"]], workspaces_dev=[1 << 20, 1 << 21], workspace_bytes_each=rest["workspace_bytes_"], stream=0)
        assert status(lambda: hl.decode_gemm_multi_epilogue([b.desc, b.desc], **multi)) == want, what
    assert hl.lib().huffllm_decode_gemm_epilogue(b.desc, 256, 256, 1, None, 256, 256, ws_bytes, None, None) == 1
    odd = Blob(hl, None, wl.gaussian_weights(32, 40, 0.02, 1), "bf16")
    assert status(lambda: hl.decode_gemm_epilogue(odd.desc, 256, 256, 1, hl.Epilogue(), 256, 256, 1 << 20, stream=0)) == "UNSUPPORTED"


def test_norms_are_refused(hl):
    A = 1 << 20
    good = dict(dtype=0, vectors=2, cols=64, x=A, x_type=hl.ELEM_F32, gain=A, eps=1e-5, out=A)
    for change, want in [(dict(dtype=2), "INVALID_ARG"), (dict(x_type=2), "INVALID_ARG"), (dict(delta_type=2), "INVALID_ARG"), (dict(x=None), "INVALID_ARG"),
                         (dict(out=None), "INVALID_ARG"), (dict(vectors=0), "INVALID_ARG"), (dict(cols=0), "INVALID_ARG"), (dict(eps=-1.0), "INVALID_ARG"),
                         (dict(eps=float("nan")), "INVALID_ARG"), (dict(vectors=1 << 31), "UNSUPPORTED"), (dict(cols=(1 << 31) + 1), "UNSUPPORTED"),
                         (dict(x=A + 2), "INVALID_ARG"), (dict(sum=A + 2), "INVALID_ARG"), (dict(delta=A + 1, delta_type=1), "INVALID_ARG"),
                         (dict(gain=A + 1), "INVALID_ARG"), (dict(out=A + 1), "INVALID_ARG"), (dict(x_stride=63), "INVALID_ARG"),
                         (dict(out_stride=1), "INVALID_ARG"), (dict(sum=A, sum_stride=64, x_stride=128), "INVALID_ARG"),
                         (dict(delta=A + 4096, sum=A + 4096, delta_type=1), "INVALID_ARG"),
                         (dict(delta=A + 4096, sum=A + 4096, delta_stride=72), "INVALID_ARG")]:
        assert status(lambda: hl.add_rms_norm(hl.Norm(**{**good, **change}), stream=0)) == want, change
    assert hl.lib().huffllm_add_rms_norm(None, None) == 1


def test_feed_forward_calls_are_refused(hl):
    n, hidden = 64, 96
    gate_up = Blob(hl, None, wl.gaussian_weights(hl.stacked_rows(n), hidden, 0.02, 1), "bf16")
    down = Blob(hl, None, wl.gaussian_weights(hidden, n, 0.02, 2), "bf16")
    fp16 = Blob(hl, None, wl.gaussian_weights(hidden, n, 0.02, 2, "fp16"), "fp16")
    A = 1 << 20

    def call(gu=gate_up, dn=down, rows=n, act=hl.ACT_SILU, h=A, batch=2, out=A, h_type=0, ws=A, ws_bytes=None, h_stride=0, out_stride=0, gu_blob=A):
        f = hl.Ffn(gu.desc, gu_blob, dn.desc, A, rows, None, 1e-5, act)
        size = hl.ffn_workspace_bytes(f, 2) if ws_bytes is None else ws_bytes
        hl.decode_ffn(f, h, batch, out, h_type, ws, size, None, h_stride, out_stride, stream=0)

    for change, want in [(dict(rows=n - 8), "INVALID_ARG"), (dict(rows=0), "INVALID_ARG"), (dict(gu=down), "INVALID_ARG"), (dict(dn=gate_up), "INVALID_ARG"),
                         (dict(dn=fp16), "UNSUPPORTED"), (dict(act=9), "INVALID_ARG"), (dict(h=None), "INVALID_ARG"), (dict(out=None), "INVALID_ARG"),
                         (dict(h=A + 2), "INVALID_ARG"), (dict(h_type=2), "INVALID_ARG"), (dict(batch=0), "INVALID_ARG"), (dict(batch=65), "INVALID_ARG"),
                         (dict(ws=A + 16), "INVALID_ARG"), (dict(ws=None), "INVALID_ARG"), (dict(ws_bytes=0), "BUFFER_TOO_SMALL"),
                         (dict(ws_bytes=8192), "BUFFER_TOO_SMALL"), (dict(h_stride=hidden - 1), "INVALID_ARG"), (dict(out_stride=1), "INVALID_ARG"),
                         (dict(h_stride=hidden + 8), "INVALID_ARG")]:
        assert status(lambda: call(**change)) == want, change


# ------------------------------------------------------------------------------------------------ products with epilogues (GPU)

def run_product(hl, torch, w, dtype, batch, act, bias, residual, out16, chunk=1024, limit=0, stride=0, in_place=False, seed=0):
    rows, cols = w.shape
    blob = Blob(hl, torch, w, dtype, chunk, limit)
    x = x_of(batch, cols, seed + 1, dtype)
    rng = np.random.default_rng(seed + 2)
    b = f_to_bits(rng.standard_normal(rows), dtype) if bias else None
    ld = rows + stride
    out_t = half(torch, dtype) if out16 else torch.float32
    out = torch.full((batch * ld + 8,), 77.0, dtype=out_t, device="cuda")
    r = None
    if residual:
        host = 3 * rng.standard_normal((batch, ld)).astype(np.float32)
        r = torch.from_numpy(host).cuda().to(out_t)
        r64 = values(r)[:, :rows]
        if in_place:
            out[:batch * ld] = r.reshape(-1)
            r = out
    n, (ws,) = workspace(hl, torch, [blob], batch)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    bd = up(torch, b, dtype) if bias else None
    ep = hl.Epilogue(getattr(hl, "ACT_" + act.upper()), hl.ELEM_16 if out16 else hl.ELEM_F32, bd, r, ld if residual else 0, ld)
    xd = up(torch, x, dtype)
    before = out.clone()
    hl.decode_gemm_epilogue(blob.desc, blob.dev, xd, batch, ep, out, ws, n, err)
    torch.cuda.synchronize()
    assert_clean(hl, blob, ws, err)
    s = Sums(bits_to_f64(w, dtype), bits_to_f64(x, dtype)).plus(bits_to_f64(b, dtype) if bias else None)
    want, tol = s.through(act)
    if residual:
        want = want + r64
        tol = tol + F32 * (np.abs(want) + tol)
    got = out[:batch * ld].view(batch, ld)
    check(values(got)[:, :rows], want, tol, dtype if out16 else "f32")
    # what lies behind the rows and behind the last vector is left as it was
    keep = before[:batch * ld].view(batch, ld)[:, rows:]
    assert torch.equal(got[:, rows:], keep) and torch.equal(out[batch * ld:], before[batch * ld:])


PRODUCTS = [
    # rows, cols, dtype, chunk, limit
    (16, 32, "bf16", 512, 0),             # one block
    (1, 96, "bf16", 1024, 0),             # one row
    (100, 1056, "bf16", 1024, 0),         # ragged rows and last chunk
    (2049, 2048, "bf16", 4096, 0),        # row groups shared by warps and CTAs; as wide as tall but for a row
    (2048, 4096, "bf16", 4096, 0),        # tensor-core shapes
    (333, 1024, "bf16", 2048, 9),         # the other table size
    (77, 640, "bf16", 1024, 12),          # two-level lookups
    (300, 1056, "bf16", 2048, 10),
    (90, 672, "fp16", 1024, 12),
    (96, 1024, "fp16", 8192, 0),          # records too large for the tensor-core kernel's slots: passes of 8 vectors
    (130, 1056, "fp16", 1024, 0),
    (515, 512, "fp16", 1024, 7),          # tables of 128 entries
    (64, 8192, "bf16", 16384, 0),         # single slots
    (2000, 1024, "bf16", 16384, 0),       # single slots on the tensor-core path too
    (1500, 1056, "fp16", 4096, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,dtype,chunk,limit", PRODUCTS)
@pytest.mark.parametrize("batch", [1, 2, 7, 8, 9, 16, 17, 33, 64])
def test_products_with_epilogues(hl, torch, rows, cols, dtype, chunk, limit, batch):
    """Every path that a product can take; the epilogue's parts take turns over the batches."""
    w = wl.gaussian_weights(rows, cols, 0.05, rows + cols, dtype)
    i = [1, 2, 7, 8, 9, 16, 17, 33, 64].index(batch) + PRODUCTS.index((rows, cols, dtype, chunk, limit))
    run_product(hl, torch, w, dtype, batch, ACTS[i % 5], i % 2 == 0, i % 3 == 0, i % 4 < 2, chunk, limit, stride=(0, 1, 24)[i % 3], seed=i)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype,out16", [("bf16", True), ("bf16", False), ("fp16", True)])
@pytest.mark.parametrize("batch", [1, 5, 12, 40])
def test_every_activation_on_every_path(hl, torch, act, dtype, out16, batch):
    w = wl.gaussian_weights(300, 512, 0.15, 7, dtype)                 # sums of up to some twenty: both ends of the activations
    run_product(hl, torch, w, dtype, batch, act, True, True, out16, seed=batch)
    run_product(hl, torch, w, dtype, batch, act, False, False, out16, stride=5, seed=batch + 50)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 4, 16, 64])
@pytest.mark.parametrize("out16", [False, True])
@pytest.mark.parametrize("dtype,chunk,limit", [("bf16", 1024, 0), ("bf16", 1024, 12), ("fp16", 8192, 0)])
def test_the_residual_stream_is_updated_in_place(hl, torch, batch, out16, dtype, chunk, limit):
    w = wl.gaussian_weights(528, 1024, 0.05, 9, dtype)
    run_product(hl, torch, w, dtype, batch, "none", True, True, out16, chunk, limit, stride=16, in_place=True, seed=batch)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,batch", [(1000, 1), (1000, 8), (2048, 9), (2048, 16), (1000, 32)])
def test_without_an_epilogue_the_sums_are_those_of_the_plain_product(hl, torch, rows, batch):
    """Where both calls take the same kernel it adds in the same order: bit for bit the plain call's sums, and their rounding.  (At 9..16
    vectors the plain call does only where the matrix is as wide as tall and has 2048 rows.)"""
    w = wl.gaussian_weights(rows, 2048, 0.05, 11)
    blob = Blob(hl, torch, w, "bf16", 4096)
    x = up(torch, x_of(batch, 2048, 3, "bf16"), "bf16")
    n, (ws,) = workspace(hl, torch, [blob], batch)
    y = torch.empty((batch, rows), dtype=torch.float32, device="cuda")
    out32, out16 = torch.empty_like(y), torch.empty((batch, rows), dtype=torch.bfloat16, device="cuda")
    hl.decode_gemm(blob.desc, blob.dev, x, batch, y, ws, n)
    hl.decode_gemm_epilogue(blob.desc, blob.dev, x, batch, hl.Epilogue(), out32, ws, n)
    hl.decode_gemm_epilogue(blob.desc, blob.dev, x, batch, hl.Epilogue(out_type=hl.ELEM_16), out16, ws, n)
    torch.cuda.synchronize()
    assert torch.equal(y, out32) and torch.equal(y.to(torch.bfloat16), out16)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,limit", [("bf16", 9), ("bf16", 10), ("bf16", 12), ("fp16", 7), ("fp16", 9), ("fp16", 12)])
@pytest.mark.parametrize("batch", [3, 9, 32, 64])
def test_codewords_of_every_length_on_every_path(hl, torch, dtype, limit, batch):
    """Weights whose fields have codewords up to the limit: exponents that fall off by halves."""
    w = wl.skewed_exponent_weights(200, 1056, 17, dtype=dtype)
    run_product(hl, torch, w, dtype, batch, "relu", False, False, False, 1024, limit, seed=batch)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 6, 13, 30])
def test_infinities_and_nans_of_bias_and_residual_stay_in_their_places(hl, torch, batch):
    rows, cols = 96, 256
    w = wl.gaussian_weights(rows, cols, 0.05, 13)
    blob = Blob(hl, torch, w, "bf16")
    x = x_of(batch, cols, 5, "bf16")
    b = np.zeros(rows, np.float32)
    b[3], b[4], b[5], b[20] = np.inf, -np.inf, np.nan, 3e38
    bias, xd = up(torch, f_to_bits(b, "bf16"), "bf16"), up(torch, x, "bf16")
    res = torch.zeros((batch, rows), dtype=torch.bfloat16, device="cuda")
    res[:, 7], res[batch - 1, 9], res[0, 11] = float("nan"), float("inf"), float("-inf")
    n, (ws,) = workspace(hl, torch, [blob], batch)
    v = bits_to_f64(x, "bf16") @ bits_to_f64(w, "bf16").T + b.astype(np.float64)
    for act in ("none", "relu"):
        out = torch.empty((batch, rows), dtype=torch.bfloat16, device="cuda")
        hl.decode_gemm_epilogue(blob.desc, blob.dev, xd, batch, hl.Epilogue(getattr(hl, "ACT_" + act.upper()), hl.ELEM_16, bias, res), out, ws, n)
        torch.cuda.synchronize()
        want = act64(v, act) + values(res)
        got = values(out)
        fine = np.isfinite(want)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isfinite(got), fine)
        assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
        assert np.all(np.abs(got[fine] - want[fine]) <= 0.01 * np.abs(want[fine]) + 0.01)      # (the places matter here: values are another test's)


@pytest.mark.gpu
def test_fp16_results_beyond_the_range_become_infinite_and_small_ones_denormal(hl, torch):
    w = np.full((32, 32), np.float16(1.0).view(np.uint16), np.uint16)
    blob = Blob(hl, torch, w, "fp16")
    x = torch.zeros((2, 32), dtype=torch.float16, device="cuda")
    x[0, 0], x[1, 0], x[1, 1] = 2.0 ** -24, 65504.0, 65504.0
    n, (ws,) = workspace(hl, torch, [blob], 2)
    out = torch.empty((2, 32), dtype=torch.float16, device="cuda")
    hl.decode_gemm_epilogue(blob.desc, blob.dev, x, 2, hl.Epilogue(out_type=hl.ELEM_16), out, ws, n)
    torch.cuda.synchronize()
    assert torch.all(out[0] == 2.0 ** -24) and torch.all(torch.isinf(out[1]))


# ------------------------------------------------------------------------------------------------ gated products (GPU)

def gated_case(hl, torch, n, cols, dtype, batch, act, bias, out16, chunk, limit, stride=0, seed=0):
    gate, up_ = wl.gaussian_weights(n, cols, 0.05, seed + 1, dtype), wl.gaussian_weights(n, cols, 0.05, seed + 2, dtype)
    blob = Blob(hl, torch, hl.stack_gate_up(gate, up_), dtype, chunk, limit)
    x = x_of(batch, cols, seed + 3, dtype)
    rng = np.random.default_rng(seed)
    gb, ub = (f_to_bits(rng.standard_normal(n), dtype) for _ in range(2))
    bd = up(torch, hl.stack_gate_up(gb, ub), dtype) if bias else None
    ld = n + stride
    out = torch.full((batch * ld + 8,), 77.0, dtype=half(torch, dtype) if out16 else torch.float32, device="cuda")
    ws_n, (ws,) = workspace(hl, torch, [blob], batch)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ep = hl.Epilogue(getattr(hl, "ACT_" + act.upper()), hl.ELEM_16 if out16 else hl.ELEM_F32, bd, out_stride=ld if stride else 0, gated_rows=n)
    xd = up(torch, x, dtype)
    hl.decode_gemm_epilogue(blob.desc, blob.dev, xd, batch, ep, out, ws, ws_n, err)
    torch.cuda.synchronize()
    assert_clean(hl, blob, ws, err)
    x64 = bits_to_f64(x, dtype)
    g, gt = Sums(bits_to_f64(gate, dtype), x64).plus(bits_to_f64(gb, dtype) if bias else None).through(act)
    s = Sums(bits_to_f64(up_, dtype), x64).plus(bits_to_f64(ub, dtype) if bias else None)
    want = g * s.v
    tol = np.abs(g) * s.tol + np.abs(s.v) * gt + gt * s.tol
    tol = tol + F32 * (np.abs(want) + tol)
    got = out[:batch * ld].view(batch, ld)
    check(values(got)[:, :n], want, tol, dtype if out16 else "f32")
    assert torch.all(got[:, n:] == 77.0) and torch.all(out[batch * ld:] == 77.0)


@pytest.mark.gpu
@pytest.mark.parametrize("n,cols,dtype,chunk,limit", [(1, 32, "bf16", 512, 0), (7, 96, "bf16", 1024, 0), (8, 512, "bf16", 1024, 0), (201, 1056, "bf16", 1024, 0),
                                                      (1030, 2048, "bf16", 4096, 0), (333, 1024, "bf16", 2048, 9), (45, 640, "bf16", 1024, 12),
                                                      (131, 1056, "fp16", 1024, 0), (60, 512, "fp16", 1024, 7), (1024, 4096, "bf16", 4096, 0), (70, 512, "fp16", 8192, 0)])
@pytest.mark.parametrize("batch", [1, 2, 8, 9, 16, 17, 48, 64])
def test_gated_products(hl, torch, n, cols, dtype, chunk, limit, batch):
    i = n + batch
    gated_case(hl, torch, n, cols, dtype, batch, ACTS[1 + i % 4], i % 2 == 0, i % 3 != 0, chunk, limit, stride=(0, 3)[i % 2], seed=i)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("batch", [1, 3, 15, 31])
def test_gated_products_with_every_activation(hl, torch, act, batch):
    gated_case(hl, torch, 90, 256, "bf16", batch, act, True, True, 1024, 0, seed=batch)


@pytest.mark.gpu
@pytest.mark.parametrize("n,cols", [(1, 1), (5, 64), (8, 33), (203, 96)])
def test_stacking_on_the_device(hl, torch, n, cols):
    rng = np.random.default_rng(n)
    gate, up_ = (rng.integers(0, 65536, (n, cols), dtype=np.uint16) for _ in range(2))
    gd, ud = (torch.from_numpy(a.view(np.int16)).cuda() for a in (gate, up_))
    rows = hl.stacked_rows(n)
    out = torch.full((rows * cols + 8,), 0x5A5A, dtype=torch.int16, device="cuda")
    hl.stack_gate_up_device(gd, ud, n, cols, out)
    torch.cuda.synchronize()
    got = out.cpu().numpy().view(np.uint16)
    assert np.array_equal(got[:rows * cols].reshape(rows, cols), hl.stack_gate_up(gate, up_)) and np.all(got[rows * cols:] == 0x5A5A)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [12, 20, 64])
@pytest.mark.parametrize("rows,cols,chunk", [(90000, 128, 512), (40000, 1024, 512)])
def test_more_work_items_than_ctas(hl, torch, rows, cols, chunk, batch):
    """CTAs that fetch items from the counter in the workspace; three calls in a row on one workspace, whose counters must be zero behind each."""
    w = wl.gaussian_weights(rows, cols, 0.05, rows)
    blob = Blob(hl, torch, w, "bf16", chunk)
    n, (ws,) = workspace(hl, torch, [blob], batch)
    x = x_of(batch, cols, 3, "bf16")
    bias = f_to_bits(np.random.default_rng(4).standard_normal(rows), "bf16")
    bd, xd = up(torch, bias, "bf16"), up(torch, x, "bf16")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    want, tol = Sums(bits_to_f64(w, "bf16"), bits_to_f64(x, "bf16")).plus(bits_to_f64(bias, "bf16")).through("silu")
    first = None
    for _ in range(3):
        out = torch.empty((batch, rows), dtype=torch.float32, device="cuda")
        hl.decode_gemm_epilogue(blob.desc, blob.dev, xd, batch, hl.Epilogue(hl.ACT_SILU, hl.ELEM_F32, bd), out, ws, n, err)
        torch.cuda.synchronize()
        assert_clean(hl, blob, ws, err)
        first = out if first is None else first
        assert torch.equal(out, first)
    check(values(out), want, tol, "f32")
    assert hl.gemm_launch_plan([blob.desc], batch, n)["work_items"][0] > torch.cuda.get_device_properties(0).multi_processor_count


# ------------------------------------------------------------------------------------------------ several matrices in a launch (GPU)

@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 5, 12, 20, 64])
@pytest.mark.parametrize("dtype,chunk,limit", [("bf16", 1024, 0), ("bf16", 8192, 0), ("fp16", 1024, 0), ("fp16", 2048, 7), ("bf16", 2048, 11), ("fp16", 1024, 10), ("fp16", 8192, 0)])
def test_several_matrices_with_an_epilogue_each(hl, torch, batch, dtype, chunk, limit):
    """A gated product, one with bias and one with residual in one launch; one fp32 output among 16-bit ones."""
    cols, n = 512, 100
    gate, up_ = wl.gaussian_weights(n, cols, 0.05, 1, dtype), wl.gaussian_weights(n, cols, 0.05, 2, dtype)
    mats = [hl.stack_gate_up(gate, up_), wl.gaussian_weights(300, cols, 0.05, 3, dtype), wl.gaussian_weights(77, cols, 0.05, 4, dtype)]
    blobs = [Blob(hl, torch, m, dtype, chunk, limit) for m in mats]
    x = x_of(batch, cols, 5, dtype)
    rng = np.random.default_rng(6)
    bias = f_to_bits(rng.standard_normal(300), dtype)
    res = torch.from_numpy(rng.standard_normal((batch, 77)).astype(np.float32)).cuda()
    outs = [torch.empty((batch, n), dtype=half(torch, dtype), device="cuda"), torch.empty((batch, 300), dtype=half(torch, dtype), device="cuda"),
            torch.empty((batch, 77), dtype=torch.float32, device="cuda")]
    bd = up(torch, bias, dtype)
    eps = [hl.Epilogue(hl.ACT_SILU, hl.ELEM_16, gated_rows=n), hl.Epilogue(hl.ACT_GELU, hl.ELEM_16, bd), hl.Epilogue(residual=res)]
    ws_n, wss = workspace(hl, torch, blobs, batch)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    xd = up(torch, x, dtype)
    hl.decode_gemm_multi_epilogue([b.desc for b in blobs], [b.dev for b in blobs], [xd] * 3, batch, eps, outs, wss, ws_n, err)
    torch.cuda.synchronize()
    for b, ws in zip(blobs, wss):
        assert_clean(hl, b, ws, err)
    x64 = bits_to_f64(x, dtype)
    g, gt = Sums(bits_to_f64(gate, dtype), x64).through("silu")
    s = Sums(bits_to_f64(up_, dtype), x64)
    tol = np.abs(g) * s.tol + np.abs(s.v) * gt + gt * s.tol
    check(values(outs[0]), g * s.v, tol + F32 * (np.abs(g * s.v) + tol), dtype)
    check(values(outs[1]), *Sums(bits_to_f64(mats[1], dtype), x64).plus(bits_to_f64(bias, dtype)).through("gelu"), dtype)
    s = Sums(bits_to_f64(mats[2], dtype), x64)
    check(values(outs[2]), s.v + values(res), s.tol + F32 * (np.abs(s.v + values(res)) + s.tol), "f32")


# ------------------------------------------------------------------------------------------------ residual addition and norm (GPU)

def norm64(h, gain, eps):
    return h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps) * gain


def norm_case(hl, torch, vectors, cols, dtype, x16, delta, want_sum, gain, pad=0, off=0, eps=1e-5, seed=0):
    """pad: values between vectors; off: values in front of every buffer (alignment); delta: None, "f32" or "16"."""
    rng = np.random.default_rng(seed)
    ht = half(torch, dtype)
    ld = cols + pad

    def make(t, factor=1.0):
        buf = torch.full((vectors * ld + 16,), 55.0, dtype=t, device="cuda")
        view = buf[off:off + vectors * ld].view(vectors, ld)
        view[:, :cols] = torch.from_numpy((factor * rng.standard_normal((vectors, cols))).astype(np.float32)).cuda().to(t)
        return buf, view
    xt = ht if x16 else torch.float32
    xb, x = make(xt, 3.0)
    db, d = make(torch.float32 if delta == "f32" else ht) if delta else (None, None)
    sb, s = make(xt) if want_sum else (None, None)
    ob, o = make(ht)
    gt = (1 + 0.2 * torch.from_numpy(rng.standard_normal(cols + off).astype(np.float32)).cuda()).to(ht)[off:] if gain else None
    sb0, ob0 = sb.clone() if want_sum else None, ob.clone()
    a = hl.Norm(hl.BF16 if dtype == "bf16" else hl.FP16, vectors, cols, x, hl.ELEM_16 if x16 else hl.ELEM_F32, gt, eps, o, d,
                hl.ELEM_16 if delta == "16" else hl.ELEM_F32, s, ld, ld, ld, ld)
    hl.add_rms_norm(a)
    torch.cuda.synchronize()
    h = values(x)[:, :cols] + (values(d)[:, :cols] if delta else 0.0)
    want = norm64(h, values(gt) if gain else 1.0, eps)
    # h rounds once (2^-24); the squares' sum of cols terms is off by at most (cols + 8) 2^-24 of itself, its root by half of that; the root's
    # reciprocal, the quotient and the two products by 2^-22 at most together
    add = F32 * (np.abs(h) + (np.abs(values(d)[:, :cols]) if delta else 0.0))
    rms = np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    g = np.abs(values(gt)) if gain else 1.0
    tol = add / rms * g + np.abs(want) * ((cols + 8) * F32 / 2 + 2 * F32 + 2.0 ** -22)
    check(values(o)[:, :cols], want, tol, dtype)
    if want_sum:
        check(values(s)[:, :cols], h, add, dtype if x16 else "f32")
    for buf, was in ((ob, ob0), (sb, sb0)):                              # gaps, front and tail as they were
        if buf is not None:
            mask = torch.ones_like(buf, dtype=torch.bool)
            mask[off:off + vectors * ld].view(vectors, ld)[:, :cols] = False
            assert torch.equal(buf[mask], was[mask])


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [1, 7, 8, 33, 250, 4096, 8191, 8200, 16384, 16392, 40001])
@pytest.mark.parametrize("vectors", [1, 3, 64])
def test_residual_addition_and_norm(hl, torch, vectors, cols):
    i = cols + vectors
    for k in range(4):
        norm_case(hl, torch, vectors, cols, ("bf16", "fp16")[(i + k) % 2], k % 2 == 0, (None, "f32", "16")[(i + k) % 3], (i + k) % 4 != 0, k != 3,
                  pad=(0, 8, 3)[(i + k) % 3], off=(0, 8, 1)[k % 3], seed=i + k)


@pytest.mark.gpu
@pytest.mark.parametrize("vectors,cols", [(2000, 512), (300, 8192), (5000, 33), (400, 20000)])
def test_norm_of_many_vectors(hl, torch, vectors, cols):
    norm_case(hl, torch, vectors, cols, "bf16", True, "16", True, True, seed=cols)
    norm_case(hl, torch, vectors, cols, "fp16", False, "f32", True, True, pad=4, seed=cols)


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [96, 4096, 4099, 20000])
@pytest.mark.parametrize("over", ["x", "delta"])
def test_the_sum_may_lie_over_x_or_delta(hl, torch, cols, over):
    g = torch.Generator(device="cuda").manual_seed(cols)
    for t, elem in ((torch.bfloat16, hl.ELEM_16), (torch.float32, hl.ELEM_F32)):
        x, d = (torch.randn((5, cols), generator=g, device="cuda").to(t) for _ in range(2))
        outs = []
        for place in (None, over):
            a, b = x.clone(), d.clone()
            s = torch.empty_like(a) if place is None else a if place == "x" else b
            o = torch.empty((5, cols), dtype=torch.bfloat16, device="cuda")
            hl.add_rms_norm(hl.Norm(hl.BF16, 5, cols, a, elem, None, 1e-6, o, b, elem, s))
            torch.cuda.synchronize()
            outs.append((s.clone(), o))
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.gpu
def test_norm_of_zeros_tiny_and_special_values(hl, torch):
    cols = 264
    x = torch.randn((6, cols), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    x[0] = 0
    x[1] *= 1e-20
    x[2, 5] = float("nan")
    x[3, 7] = float("inf")
    x[4] *= 1e15
    o, s = torch.empty((6, cols), dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    hl.add_rms_norm(hl.Norm(hl.BF16, 6, cols, x, hl.ELEM_F32, None, 1e-5, o, sum=s))
    torch.cuda.synchronize()
    assert torch.equal(s.nan_to_num(9.0), x.nan_to_num(9.0))
    got = values(o)
    assert np.all(got[0] == 0) and np.all(np.abs(got[1]) < 1e-16) and np.all(np.isnan(got[2]))
    assert np.isnan(got[3, 7]) and np.all(got[3][np.arange(cols) != 7] == 0)
    want = norm64(values(x)[4:], 1.0, 1e-5)
    assert np.all(np.abs(got[4:] - want) <= (2.0 ** -8 + 1e-4) * np.abs(want))
    # no eps: a vector of zeros is 0 * inf
    hl.add_rms_norm(hl.Norm(hl.BF16, 1, cols, x, hl.ELEM_F32, None, 0.0, o))
    torch.cuda.synchronize()
    assert torch.all(torch.isnan(o[0]))


# ------------------------------------------------------------------------------------------------ the feed-forward sub-layer (GPU)

class FfnCase:
    def __init__(self, hl, torch, hidden, n, dtype, bias=True, seed=0, chunk=1024, limit=0):
        self.w = [wl.gaussian_weights(n, hidden, 0.03, seed + 1, dtype), wl.gaussian_weights(n, hidden, 0.03, seed + 2, dtype),
                  wl.gaussian_weights(hidden, n, 0.03, seed + 3, dtype)]
        self.gate_up = Blob(hl, torch, hl.stack_gate_up(self.w[0], self.w[1]), dtype, chunk, limit)
        self.down = Blob(hl, torch, self.w[2], dtype, chunk, limit)
        rng = np.random.default_rng(seed)
        self.gain = f_to_bits(1 + 0.2 * rng.standard_normal(hidden), dtype)
        self.b = [f_to_bits(0.5 * rng.standard_normal(k), dtype) for k in (n, n, hidden)] if bias else None
        self.dev = [up(torch, self.gain, dtype)] + ([up(torch, hl.stack_gate_up(self.b[0], self.b[1]), dtype), up(torch, self.b[2], dtype)] if bias else [None, None])
        self.n, self.hidden, self.dtype = n, hidden, dtype
        self.ffn = hl.Ffn(self.gate_up.desc, self.gate_up.dev, self.down.desc, self.down.dev, n, self.dev[0], 1e-5, hl.ACT_SILU, self.dev[1], self.dev[2])


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 4, 11, 24, 64])
@pytest.mark.parametrize("dtype,h16,hidden,n", [("bf16", True, 512, 1376), ("bf16", False, 1024, 96), ("fp16", True, 96, 2080), ("fp16", False, 288, 800)])
def test_the_feed_forward_sub_layer(hl, torch, batch, dtype, h16, hidden, n):
    """Against 64 bits, with the roundings of the norm's and the gated product's outputs carried through, and bit for bit what its three
    steps give one by one; in place too."""
    c = FfnCase(hl, torch, hidden, n, dtype, seed=batch)
    ht = half(torch, dtype)
    ld = hidden + 8
    h = torch.full((batch, ld), 9.0, dtype=ht if h16 else torch.float32, device="cuda")
    h[:, :hidden] = torch.from_numpy(2 * np.random.default_rng(batch).standard_normal((batch, hidden)).astype(np.float32)).cuda().to(h.dtype)
    elem = hl.ELEM_16 if h16 else hl.ELEM_F32
    size = hl.ffn_workspace_bytes(c.ffn, batch)
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((batch, hidden), 9.0, dtype=h.dtype, device="cuda")
    hl.decode_ffn(c.ffn, h, batch, out, elem, ws, size, err, h_stride=ld)
    torch.cuda.synchronize()
    assert int(err.item()) == 0

    # its steps one by one
    nrm, mid, out2 = torch.empty((batch, hidden), dtype=ht, device="cuda"), torch.empty((batch, n), dtype=ht, device="cuda"), torch.empty_like(out)
    hl.add_rms_norm(hl.Norm(hl.BF16 if dtype == "bf16" else hl.FP16, batch, hidden, h, elem, c.dev[0], 1e-5, nrm, x_stride=ld))
    w0, (ws0,) = workspace(hl, torch, [c.gate_up], batch)
    hl.decode_gemm_epilogue(c.gate_up.desc, c.gate_up.dev, nrm, batch, hl.Epilogue(hl.ACT_SILU, hl.ELEM_16, c.dev[1], gated_rows=n), mid, ws0, w0, err)
    w1, (ws1,) = workspace(hl, torch, [c.down], batch)
    hl.decode_gemm_epilogue(c.down.desc, c.down.dev, mid, batch, hl.Epilogue(out_type=elem, bias=c.dev[2], residual=h, residual_stride=ld), out2, ws1, w1, err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0 and torch.equal(out, out2)

    # in place, again with the same workspace
    h64 = values(h)[:, :hidden]
    hl.decode_ffn(c.ffn, h, batch, h, elem, ws, size, err, h_stride=ld, out_stride=ld)
    torch.cuda.synchronize()
    assert int(err.item()) == 0 and torch.equal(h[:, :hidden], out) and torch.all(h[:, hidden:] == 9.0)

    # 64 bits
    f = lambda b: bits_to_f64(b, dtype)
    n64 = norm64(h64, f(c.gain), 1e-5)
    ntol = np.abs(n64) * ((hidden + 16) * F32 + 2.0 ** -22)
    ntol = ntol + rounding(np.abs(n64) + ntol, dtype)
    def spread(w, x, xtol, b):                                          # W x + b where x is off by xtol
        s = Sums(w, x)
        s.tol = s.tol * 1.02 + xtol @ np.abs(w).T
        return s.plus(b)
    g, gt = spread(f(c.w[0]), n64, ntol, f(c.b[0])).through("silu")
    u = spread(f(c.w[1]), n64, ntol, f(c.b[1]))
    m64 = g * u.v
    mtol = np.abs(g) * u.tol + np.abs(u.v) * gt + gt * u.tol + F32 * np.abs(m64)
    mtol = mtol + rounding(np.abs(m64) + mtol, dtype)
    d = spread(f(c.w[2]), m64, mtol, f(c.b[2]))
    want = h64 + d.v
    check(values(out), want, d.tol + F32 * np.abs(want), dtype if h16 else "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 20])
def test_a_decoders_sub_layers_on_one_stream_and_as_a_captured_graph(hl, torch, batch):
    """Residual stream, attention's output projection added to it, norm, feed-forward: twice in a row on a stream of its own, then
    captured and replayed on other inputs; the workspaces are shared by the calls of the stream."""
    hidden, n = 512, 640
    c = FfnCase(hl, torch, hidden, n, "bf16", seed=3)
    wo = wl.gaussian_weights(hidden, hidden, 0.03, 40)
    o = Blob(hl, torch, wo, "bf16")
    size = hl.ffn_workspace_bytes(c.ffn, batch)
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    w0, (ws0,) = workspace(hl, torch, [o], batch)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    attn = torch.empty((batch, hidden), dtype=torch.bfloat16, device="cuda")
    h, mid, total = (torch.empty((batch, hidden), dtype=torch.float32, device="cuda") for _ in range(3))
    nrm = torch.empty((batch, hidden), dtype=torch.bfloat16, device="cuda")
    stream = torch.cuda.Stream()

    def steps(s):
        hl.decode_gemm_epilogue(o.desc, o.dev, attn, batch, hl.Epilogue(residual=h), mid, ws0, w0, err, s)
        for _ in range(2):
            hl.decode_ffn(c.ffn, mid, batch, mid, hl.ELEM_F32, ws, size, err, stream=s)
        hl.add_rms_norm(hl.Norm(hl.BF16, batch, hidden, mid, hl.ELEM_F32, c.dev[0], 1e-5, nrm, h, hl.ELEM_F32, total), s)

    def inputs(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        attn.copy_(torch.randn((batch, hidden), generator=g, device="cuda"))
        h.copy_(torch.randn((batch, hidden), generator=g, device="cuda"))

    results = {}
    for seed in (1, 2):
        inputs(seed)
        torch.cuda.synchronize()
        steps(stream)
        stream.synchronize()
        results[seed] = (mid.clone(), total.clone(), nrm.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        steps(stream)
    for seed in (2, 1, 2):
        inputs(seed)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results[seed], (mid, total, nrm)))
    assert int(err.item()) == 0


# ------------------------------------------------------------------------------------------------ calls that nothing above makes (GPU)

@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,chunk,batch", [(64, 1024, 1024, 1), (64, 1024, 1024, 4), (64, 1024, 1024, 12), (64, 1024, 1024, 32),
                                                   (6000, 5120, 8192, 12), (6000, 5120, 8192, 32)])
def test_bad_records_add_nothing_and_are_reported(hl, torch, rows, cols, chunk, batch):
    """A record offset that points outside the payload: the two chunks that it bounds add nothing, the epilogue runs over what is left, the flag
    is set; the workspace, cleared, serves the next call.  (The large matrix: records behind each other in single slots.)"""
    w = wl.gaussian_weights(rows, cols, 0.05, 31)
    blob = Blob(hl, torch, w, "bf16", chunk)
    d = blob.desc
    host = blob.host.copy()
    idx = host[d.off_index:d.off_index + 4 * (d.n_chunks + 1)].view(np.uint32)
    victim = int(d.n_chunks) // 2
    idx[victim + 1] = 0x7FFFFFFF
    bad = torch.from_numpy(host).cuda()
    kept = np.ones((rows, cols), bool)
    for v in (victim, victim + 1):
        rg, kc = divmod(v, d.col_chunks)
        kept[rg * 16:(rg + 1) * 16, kc * d.chunk_cols:(kc + 1) * d.chunk_cols] = False
    x = x_of(batch, cols, 3, "bf16")
    xd = up(torch, x, "bf16")
    n, (ws,) = workspace(hl, torch, [blob], batch)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    res = torch.randn((batch, rows), device="cuda")
    for dev, weights, codes in ((bad, np.where(kept, w, np.uint16(0)), (victim + 1, victim + 2)), (blob.dev, w, (0,))):
        out = torch.full((batch, rows), float("nan"), device="cuda")
        err.zero_()
        hl.decode_gemm_epilogue(d, dev, xd, batch, hl.Epilogue(residual=res), out, ws, n, err)
        torch.cuda.synchronize()
        assert int(err.item()) in codes
        s = Sums(bits_to_f64(weights, "bf16"), bits_to_f64(x, "bf16"))
        check(values(out), s.v + values(res), s.tol + F32 * (np.abs(s.v + values(res)) + s.tol), "f32")
        ws[:hl.workspace_control_bytes(d)].zero_()


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 20])
def test_two_calls_at_once_and_results_straight_to_pinned_host_memory(hl, torch, batch):
    rows, cols = 512, 1024
    blob = Blob(hl, torch, wl.gaussian_weights(rows, cols, 0.05, 1), "bf16")
    n, wss = workspace(hl, torch, [blob] * 2, batch)
    wss.append(torch.zeros_like(wss[0]))
    xs = [up(torch, x_of(batch, cols, i, "bf16"), "bf16") for i in range(2)]
    alone = [torch.empty((batch, rows), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ep = hl.Epilogue(hl.ACT_GELU, hl.ELEM_16)
    for x, out in zip(xs, alone):
        hl.decode_gemm_epilogue(blob.desc, blob.dev, x, batch, ep, out, wss[0], n)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty((batch, rows), dtype=torch.bfloat16, device="cuda"), torch.empty((batch, rows), dtype=torch.bfloat16).pin_memory()]
    for _ in range(20):
        for s, x, out, ws in zip(streams, xs, outs, wss):
            hl.decode_gemm_epilogue(blob.desc, blob.dev, x, batch, ep, out, ws, n, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], alone[0]) and torch.equal(outs[1], alone[1].cpu())


@pytest.mark.gpu
def test_offsets_past_32_bits(hl, torch):
    """Vectors 2^31 values apart: a product's out and residual, a norm's input and output; and 9 vectors (tensor cores) 2^29 values apart."""
    rows, cols, far = 32, 64, (1 << 31) + 8
    w = wl.gaussian_weights(rows, cols, 0.05, 1)
    blob = Blob(hl, torch, w, "bf16")
    big = torch.empty(2 * far + 64, dtype=torch.bfloat16, device="cuda")
    at = lambda b: big[b * far:b * far + rows]
    batch = 3
    n, (ws,) = workspace(hl, torch, [blob], batch)
    x = x_of(batch, cols, 2, "bf16")
    r = torch.randn((batch, rows), device="cuda").to(torch.bfloat16)
    for b in range(batch):
        at(b).copy_(r[b])
    xd = up(torch, x, "bf16")
    hl.decode_gemm_epilogue(blob.desc, blob.dev, xd, batch, hl.Epilogue(0, hl.ELEM_16, None, big, far, far), big, ws, n)
    torch.cuda.synchronize()
    s = Sums(bits_to_f64(w, "bf16"), bits_to_f64(x, "bf16"))
    want = s.v + values(r)
    check(np.stack([values(at(b)) for b in range(batch)]), want, s.tol + F32 * np.abs(want), "bf16")
    o = torch.empty((3, rows), dtype=torch.bfloat16, device="cuda")
    h = np.stack([values(at(b)) for b in range(3)])
    hl.add_rms_norm(hl.Norm(hl.BF16, 3, rows, big, hl.ELEM_16, None, 1e-5, o, x_stride=far))
    hl.add_rms_norm(hl.Norm(hl.BF16, 3, rows, o, hl.ELEM_16, None, 1e-5, big, out_stride=far))
    torch.cuda.synchronize()
    check(values(o), norm64(h, 1.0, 1e-5), np.abs(norm64(h, 1.0, 1e-5)) * 2.0 ** -20, "bf16")
    check(np.stack([values(at(b)) for b in range(3)]), norm64(values(o), 1.0, 1e-5), np.abs(norm64(values(o), 1.0, 1e-5)) * 2.0 ** -20, "bf16")
    near = 1 << 29
    n, (ws,) = workspace(hl, torch, [blob], 9)
    x = x_of(9, cols, 4, "bf16")
    xd = up(torch, x, "bf16")
    big = torch.empty(8 * near + 64, dtype=torch.bfloat16, device="cuda")
    hl.decode_gemm_epilogue(blob.desc, blob.dev, xd, 9, hl.Epilogue(hl.ACT_RELU, hl.ELEM_16, None, None, 0, near), big, ws, n)
    torch.cuda.synchronize()
    got = np.stack([values(big[b * near:b * near + rows]) for b in range(9)])
    check(got, *Sums(bits_to_f64(w, "bf16"), bits_to_f64(x, "bf16")).through("relu"), "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [65, 1000, 9001])
@pytest.mark.parametrize("strides", [(0, 0, 0, 0), (8, 16, 24, 40), (3, 11, 19, 35), (1, 2, 3, 4), (4, 8, 4, 8)])
@pytest.mark.parametrize("vectors", [5, 700])
def test_norms_whose_buffers_have_strides_of_their_own(hl, torch, cols, strides, vectors):
    """x, delta, sum and out each with their own distance between vectors: alike modulo eight values, multiples of 16 bytes, neither."""
    g = torch.Generator(device="cuda").manual_seed(cols + vectors)
    lds = [cols + k for k in strides]
    x = torch.randn(vectors * lds[0], generator=g, device="cuda")
    d = torch.randn(vectors * lds[1], generator=g, device="cuda").to(torch.float16)
    s = torch.full((vectors * lds[2],), 55.0, device="cuda")
    o = torch.full((vectors * lds[3],), 55.0, dtype=torch.float16, device="cuda")
    gain = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(torch.float16)
    hl.add_rms_norm(hl.Norm(hl.FP16, vectors, cols, x, hl.ELEM_F32, gain, 1e-5, o, d, hl.ELEM_16, s, *lds))
    torch.cuda.synchronize()
    of = lambda t, ld: values(t.view(vectors, ld)[:, :cols])
    h = of(x, lds[0]) + of(d, lds[1])
    add = F32 * (np.abs(of(x, lds[0])) + np.abs(of(d, lds[1])))
    want = norm64(h, values(gain), 1e-5)
    rms = np.sqrt(np.mean(h * h, axis=1, keepdims=True) + 1e-5)
    check(of(s, lds[2]), h, add, "f32")
    check(of(o, lds[3]), want, add / rms * np.abs(values(gain)) + np.abs(want) * ((cols + 8) * F32 / 2 + 2 * F32 + 2.0 ** -22), "fp16")
    assert torch.all(s.view(vectors, lds[2])[:, cols:] == 55.0) and torch.all(o.view(vectors, lds[3])[:, cols:] == 55.0)


@pytest.mark.gpu
def test_one_workspace_for_every_batch_and_kind_of_call(hl, torch):
    """A feed-forward workspace larger than asked for, at changing batches; a product's workspace under plain calls and calls with epilogues in
    turn, on the register path and on the tensor cores: what a call leaves behind does not reach the next one."""
    c = FfnCase(hl, torch, 512, 640, "bf16", seed=5)
    size = hl.ffn_workspace_bytes(c.ffn, 64) + 1000
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    hs = {b: torch.randn((b, 512), device="cuda") for b in (1, 6, 12, 64)}
    def sub_layer(b, w):
        out = torch.empty_like(hs[b])
        hl.decode_ffn(c.ffn, hs[b], b, out, hl.ELEM_F32, w, w.numel(), err)
        return out
    want = {b: sub_layer(b, torch.zeros(size, dtype=torch.uint8, device="cuda")) for b in hs}
    for b in (64, 1, 12, 6, 64, 12, 1):
        assert torch.equal(sub_layer(b, ws), want[b]), b

    rows, cols = 40000, 1024                                    # more work items than CTAs in chunks of 512
    blob = Blob(hl, torch, wl.gaussian_weights(rows, cols, 0.05, 6), "bf16", 512)
    n, (ws,) = workspace(hl, torch, [blob], 64)
    xs = {b: up(torch, x_of(b, cols, b, "bf16"), "bf16") for b in (1, 12, 40)}
    def product(b, kind, w):
        out = torch.empty((b, rows), device="cuda")
        if kind:
            hl.decode_gemm_epilogue(blob.desc, blob.dev, xs[b], b, hl.Epilogue(hl.ACT_RELU), out, w, n, err)
        else:
            hl.decode_gemm(blob.desc, blob.dev, xs[b], b, out, w, n, err)
        return out
    want = {(b, k): product(b, k, torch.zeros_like(ws)) for b in xs for k in (0, 1)}
    for b, k in ((40, 1), (40, 0), (1, 1), (40, 1), (12, 1), (12, 0), (1, 0), (40, 1), (12, 1)):
        assert torch.equal(product(b, k, ws), want[b, k]), (b, k)
    torch.cuda.synchronize()
    assert_clean(hl, blob, ws, err)
