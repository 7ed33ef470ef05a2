"""Layer operators over weights that were trained in fewer mantissa bits and are stored as FP16: BF16-trained ones, of whose mantissa halves the upper
one alone is flat, and ones of three mantissa bits, where neither is.  They run through kernels of their own (one flat half: two tables; none: three);
the checks are those of the other types."""
import numpy as np
import pytest

import test_layer_operators as ops
import workloads as wl
from test_layer_operators import hl, torch  # noqa: F401  (fixtures)

gaussian = wl.gaussian_weights


def trained(kind, rows, cols, std, seed):
    if kind == "from_bf16":
        return gaussian(rows, cols, std, seed, "fp16_from_bf16")
    w = gaussian(rows, cols, std, seed, "fp16")
    return ((w + 0x40) & np.uint16(0xFF80)).astype(np.uint16)            # (the carry goes into the exponent: values far below the largest)


@pytest.fixture(params=["from_bf16", "three_bits"])
def kind(request, monkeypatch):
    """All FP16 weights of a test are of this kind."""
    monkeypatch.setattr(wl, "gaussian_weights",
                        lambda r, c, std, seed, dtype="bf16": trained(request.param, r, c, std, seed) if dtype == "fp16" else gaussian(r, c, std, seed, dtype))
    return request.param


@pytest.mark.parametrize("kind_,flat", [("from_bf16", 2), ("three_bits", 0)])
def test_which_mantissa_halves_are_flat(hl, kind_, flat):  # noqa: F811
    for rows, cols, chunk in ((300, 1056, 1024), (96, 512, 2048)):
        d = ops.Blob(hl, None, trained(kind_, rows, cols, 0.05, rows), "fp16", chunk).desc
        assert d.lut_bits == 8 and d.flat_fields & 6 == flat


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,chunk", [(16, 32, 512), (130, 1056, 1024), (1500, 1056, 4096), (2049, 2048, 2048), (515, 512, 1024)])
@pytest.mark.parametrize("batch", [1, 2, 7, 8, 9, 16, 17, 33, 64])
def test_products(hl, torch, kind, rows, cols, chunk, batch):  # noqa: F811
    i = rows + batch
    w = wl.gaussian_weights(rows, cols, 0.05, rows + cols, "fp16")
    ops.run_product(hl, torch, w, "fp16", batch, ops.ACTS[i % 5], i % 2 == 0, i % 3 == 0, i % 4 < 2, chunk, 0, stride=(0, 1, 24)[i % 3], in_place=i % 6 == 0, seed=i)


@pytest.mark.gpu
@pytest.mark.parametrize("n,cols,chunk", [(7, 96, 1024), (201, 1056, 1024), (600, 512, 2048)])
@pytest.mark.parametrize("batch", [1, 3, 9, 24, 64])
def test_gated(hl, torch, kind, n, cols, chunk, batch):  # noqa: F811
    ops.gated_case(hl, torch, n, cols, "fp16", batch, ops.ACTS[1 + (n + batch) % 4], batch % 2 == 0, True, chunk, 0, stride=3, seed=n + batch)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 5, 12, 20, 64])
@pytest.mark.parametrize("chunk", [1024, 2048])
def test_several_matrices(hl, torch, kind, batch, chunk):  # noqa: F811
    ops.test_several_matrices_with_an_epilogue_each(hl, torch, batch, "fp16", chunk, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 4, 11, 24, 64])
@pytest.mark.parametrize("h16,hidden,n", [(True, 96, 2080), (False, 288, 800)])
def test_the_sub_layer(hl, torch, kind, batch, h16, hidden, n):  # noqa: F811
    ops.test_the_feed_forward_sub_layer(hl, torch, batch, "fp16", h16, hidden, n)


@pytest.mark.gpu
@pytest.mark.parametrize("limit", [7, 9, 12])
@pytest.mark.parametrize("batch", [1, 6, 16, 24, 64])
def test_other_table_sizes(hl, torch, kind, limit, batch):  # noqa: F811
    w = wl.gaussian_weights(300, 1056, 0.05, limit, "fp16")
    ops.run_product(hl, torch, w, "fp16", batch, "silu", True, True, True, 1024, limit, seed=batch)
