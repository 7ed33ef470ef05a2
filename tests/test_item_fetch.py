"""Work items that a CTA of the tensor-core kernel with epilogues fetches from the counter in the workspace: how the CTA's warps learn the next
item's number (a model, every interleaving) and launches whose items have a single step, in every shape of a CTA (GPU)."""
import numpy as np
import pytest

import workloads as wl
from test_layer_operators import Blob, Sums, assert_clean, bits_to_f64, check, up, values, workspace


@pytest.fixture(scope="module")
def hl():
    import paper_2502_00922_b200 as m
    m.lib()
    return m


@pytest.fixture(scope="module")
def torch():
    import torch as t
    return t


RING = 3


def programs(steps, items, meeting):
    """What the issuer and two decoders do, item by item, in steps of one stage.  `meeting`: a barrier of all warps at an item's end; else an mbarrier on
    which the issuer arrives when it has fetched, which it does in front of the item's last step."""
    issuer, decoder = [], []
    for t in range(items):
        for j in range(steps):
            if j + 1 == steps:
                issuer.append(("write", t))
                if not meeting:
                    issuer.append(("arrive", t))
            issuer += [("full", t * steps + j), ("commit", 0)]
            decoder += [("empty", t * steps + j), ("stage", 0)]
        for p in (issuer, decoder):
            p += [("meet" if meeting else "phase", t), ("read", t)]
    return [issuer, decoder, list(decoder)]


def explore(steps, meeting, items=4):
    """(states in which a warp waits for good, reads of a place that holds another item's number)"""
    prog = programs(steps, items, meeting)
    seen, todo, stuck, stale = set(), [((0, 0, 0), (0, 0), 0, 0, (None, None))], 0, 0
    while todo:
        state = todo.pop()
        if state in seen:
            continue
        seen.add(state)
        at, staged, commits, phases, places = state
        moved = False
        for w in range(3):
            if at[w] == len(prog[w]):
                continue
            what, n = prog[w][at[w]]
            free = (min(staged) > n if what == "full" else
                    commits > n - RING if what == "empty" else
                    phases % 2 != n % 2 if what == "phase" else                  # (try_wait.parity: the phase of this parity is not the current one)
                    all(at[v] >= prog[v].index(("meet", n)) for v in range(3)) if what == "meet" else True)
            if not free:
                continue
            moved = True
            s, pl = list(staged), list(places)
            if what == "stage":
                s[w - 1] += 1
            elif what == "write":
                pl[n % 2] = n
            elif what == "read":
                stale += pl[n % 2] != n
            now = tuple(a + (v == w) for v, a in enumerate(at))
            todo.append((now, tuple(s), commits + (what == "commit"), phases + (what == "arrive"), tuple(pl)))
        stuck += not moved and any(at[w] < len(prog[w]) for w in range(3))
    return stuck, stale


@pytest.mark.parametrize("steps", [1, 2, 3])
def test_a_meeting_at_each_items_end_hands_on_its_successor(steps):
    assert explore(steps, True) == (0, 0)


def test_an_arrival_of_the_issuer_alone_can_overtake_a_warp_where_items_have_one_step():
    """Why the warps meet."""
    assert explore(1, False)[0] > 0
    assert explore(2, False) == (0, 0) and explore(3, False) == (0, 0)


ONE_STEP = [
    # rows, cols, dtype, chunk
    (20000, 32, "bf16", 16384),      # tiles of 8 row groups, one block an item
    (40000, 32, "bf16", 8192),       # two tiles
    (57344, 256, "fp16", 4096),      # fewer than four tiles: the issuer has no part in the epilogue
    (20000, 1024, "fp16", 4096),     # row groups that fill no tile; ranges of one chunk
    (57344, 64, "fp16", 2048),       # three tiles
    (75000, 32, "bf16", 512),        # four tiles
    (40000, 1024, "bf16", 4096),     # several ranges
    (75000, 512, "bf16", 4096),      # two slices: a chunk each
]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,dtype,chunk", ONE_STEP)
def test_items_of_one_step(hl, torch, rows, cols, dtype, chunk):
    w = wl.gaussian_weights(rows, cols, 0.05, rows + cols, dtype)
    blob = Blob(hl, torch, w, dtype, chunk)
    w64 = bits_to_f64(w, dtype)
    for batch in (12, 24, 64):
        n, (ws,) = workspace(hl, torch, [blob], batch)
        x = wl.activations(batch, cols, 3, dtype)
        xd = up(torch, x, dtype)
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        res = torch.randn((batch, rows), device="cuda", generator=torch.Generator(device="cuda").manual_seed(batch))
        first = None
        for _ in range(4):
            out = torch.empty((batch, rows), dtype=torch.float32, device="cuda")
            hl.decode_gemm_epilogue(blob.desc, blob.dev, xd, batch, hl.Epilogue(residual=res), out, ws, n, err)
            torch.cuda.synchronize()
            assert_clean(hl, blob, ws, err)
            first = out if first is None else first
            assert torch.equal(out, first)
        s = Sums(w64, bits_to_f64(x, dtype))
        want = s.v + values(res)
        check(values(first), want, s.tol + 2.0 ** -24 * (np.abs(want) + s.tol), "f32")
