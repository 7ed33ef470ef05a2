"""Launch plans of the products with epilogues on the tensor cores (no GPU needed)."""
import pytest

from test_host_codec import planned_desc
from test_layer_operators import status


@pytest.fixture(scope="module")
def hl():
    import paper_2502_00922_b200 as m
    m.lib()
    return m


BF16, FP16 = 0, 1


@pytest.mark.parametrize("rows,cols", [(1024, 4096), (4096, 11008), (11008, 4096), (57344, 8192), (333, 1024)])
@pytest.mark.parametrize("batch", [9, 16, 17, 32, 64])
def test_with_room_for_every_warp_the_plan_is_the_plain_calls(hl, rows, cols, batch):
    d = planned_desc(rows, cols, 4096)
    assert hl.gemm_epilogue_launch_plan([d], batch) == {"slots_per_warp": 2, **hl.gemm_launch_plan([d], batch)}


@pytest.mark.parametrize("dtype,limit", [(BF16, 10), (BF16, 12), (FP16, 7), (FP16, 9), (FP16, 12)])
@pytest.mark.parametrize("batch", [9, 17, 64])
def test_long_codes_have_a_plan_with_epilogues_alone(hl, dtype, limit, batch):
    d = planned_desc(2000, 2048, 1024, limit, dtype)
    assert status(lambda: hl.gemm_launch_plan([d], batch)) == "UNSUPPORTED"
    plan = hl.gemm_epilogue_launch_plan([d], batch)
    assert plan["slots_per_warp"] in (1, 2) and plan["work_items"][0] == -(-d.row_groups // plan["row_groups"]) * plan["ranges"][0]


def test_several_matrices_say_which_path_they_take(hl):
    plan = lambda batch, *ds: hl.gemm_epilogue_launch_plan(list(ds), batch)["slots_per_warp"]
    short, long, nine = planned_desc(4096, 4096, 4096), planned_desc(1024, 4096, 8192), planned_desc(1024, 4096, 8192, 9)
    assert plan(12, short, short) == 2 and plan(17, short, long) > 0 and plan(12, nine, nine) > 0
    assert hl.gemm_epilogue_launch_plan([short, long], 12) == {"slots_per_warp": 0}       # the register path
    assert plan(12, long) > 0                                                              # (one matrix: the tensor cores)


def test_plans_are_refused(hl):
    d = planned_desc(512, 1024, 8192, 0, FP16)            # records for which eight warps find no room
    assert status(lambda: hl.gemm_epilogue_launch_plan([d], 32)) == "UNSUPPORTED"
    good = planned_desc(512, 1024, 1024)
    for batch in (0, 8, 65):
        assert status(lambda: hl.gemm_epilogue_launch_plan([good], batch)) == "INVALID_ARG"
    assert status(lambda: hl.gemm_epilogue_launch_plan([good, d], 32)) == "UNSUPPORTED"    # types differ
    assert status(lambda: hl.gemm_epilogue_launch_plan([good] * 9, 32)) == "INVALID_ARG"
    assert hl.lib().huffllm_gemm_epilogue_launch_plan(1, None, 32, 0, None, None, None, None, None, None) == 1


# Records so large that two slots a warp leave few warps a place: (rows, cols, dtype, chunk, limit).
LARGE_RECORDS = [(22016, 4096, FP16, 2048, 0), (11008, 4096, FP16, 4096, 0), (10000, 4096, FP16, 2048, 0), (28672, 1024, FP16, 4096, 0), (10086, 4576, FP16, 4096, 0),
                 (54663, 14080, FP16, 4096, 0), (30673, 1184, FP16, 4096, 0), (17996, 22208, FP16, 4096, 0), (8999, 4544, FP16, 4096, 0), (11008, 4096, BF16, 8192, 0),
                 (33485, 13536, BF16, 8192, 0), (20000, 2048, BF16, 8192, 9), (11008, 4096, BF16, 16384, 0), (7528, 8832, BF16, 16384, 0), (2000, 4096, FP16, 2048, 7)]


@pytest.mark.parametrize("rows,cols,dtype,chunk,limit", LARGE_RECORDS)
@pytest.mark.parametrize("batch", [9, 12, 16, 17, 24, 32, 33, 45, 56, 64])
def test_single_slots_make_no_sum_longer(hl, rows, cols, dtype, chunk, limit, batch):
    """Rounding is not traded for time: no accumulator adds up more columns than with two slots a warp, as in the call without an epilogue."""
    d = planned_desc(rows, cols, chunk, limit, dtype)
    plan = hl.gemm_epilogue_launch_plan([d], batch)
    if limit != 7:
        assert plan["chunks_per_sum"][0] <= hl.gemm_launch_plan([d], batch)["chunks_per_sum"][0]


def test_single_slots_are_taken(hl):
    taken = {(rows, chunk, batch) for rows, cols, dtype, chunk, limit in LARGE_RECORDS for batch in (12, 32, 64)
             if hl.gemm_epilogue_launch_plan([planned_desc(rows, cols, chunk, limit, dtype)], batch)["slots_per_warp"] == 1}
    assert {(22016, 2048, 32), (11008, 4096, 32), (28672, 4096, 12), (11008, 16384, 32)} <= taken


def test_single_slots_make_no_sum_longer_whatever_the_shape(hl):
    import random
    rng = random.Random(11)
    single = 0
    for _ in range(300):
        dtype = rng.choice([BF16, FP16])
        chunk = rng.choice([4096, 8192, 16384] if dtype == BF16 else [2048, 4096])
        d = planned_desc(int(200 * 280 ** rng.random()), 32 * int(10 * 90 ** rng.random()), chunk, rng.choice([0, 9]) if dtype == BF16 else 0, dtype)
        batch = rng.randrange(9, 65)
        if status(lambda: hl.gemm_launch_plan([d], batch)) == "UNSUPPORTED":
            continue                                       # (records that the kernel has no room for)
        plan = hl.gemm_epilogue_launch_plan([d], batch)
        single += plan["slots_per_warp"] == 1
        assert plan["chunks_per_sum"][0] <= hl.gemm_launch_plan([d], batch)["chunks_per_sum"][0], (d.rows, d.cols, dtype, chunk, batch)
    assert single > 100


@pytest.mark.parametrize("rows,cols,dtype,chunk,limit", LARGE_RECORDS)
def test_the_plan_is_the_same_in_the_workspace_asked_for_and_in_any(hl, rows, cols, dtype, chunk, limit):
    """A buffer's size decides neither about rounding nor about time, also when it was sized for more vectors."""
    d = planned_desc(rows, cols, chunk, limit, dtype)
    for batch in (9, 12, 16, 17, 24, 32, 33, 45, 56, 64):
        free = hl.gemm_epilogue_launch_plan([d], batch)
        for sized_for in sorted({batch, 16, 32, 64}):
            if sized_for >= batch:
                assert hl.gemm_epilogue_launch_plan([d], batch, hl.workspace_bytes(d, sized_for)) == free, (batch, sized_for)


def test_the_plan_is_the_same_in_the_workspace_asked_for_whatever_the_shape(hl):
    import random
    rng = random.Random(12)
    for _ in range(300):
        dtype = rng.choice([BF16, FP16])
        chunk = rng.choice([1024, 4096, 8192, 16384] if dtype == BF16 else [1024, 2048, 4096])
        limit = rng.choice([0, 0, 9, 12]) if dtype == BF16 else rng.choice([0, 0, 7, 9, 12])
        d = planned_desc(int(200 * 280 ** rng.random()), 32 * int(10 * 90 ** rng.random()), chunk, limit, dtype)
        batch = rng.randrange(9, 65)
        if status(lambda: hl.gemm_epilogue_launch_plan([d], batch)) == "UNSUPPORTED":
            continue                                       # (records that the kernel has no room for)
        assert hl.gemm_epilogue_launch_plan([d], batch, hl.workspace_bytes(d, batch)) == hl.gemm_epilogue_launch_plan([d], batch), (d.rows, d.cols, dtype, chunk, limit, batch)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,dtype,chunk,limit,batch", [(28672, 1024, "fp16", 4096, 0, 12), (28672, 1024, "fp16", 4096, 0, 56), (11008, 4096, "fp16", 4096, 0, 32),
                                                               (20000, 2048, "bf16", 8192, 9, 17), (22016, 1024, "bf16", 16384, 0, 40), (11008, 4096, "fp16", 4096, 7, 24)])
def test_single_slots_in_the_workspace_asked_for(hl, rows, cols, dtype, chunk, limit, batch):
    """The plans above at work: one slot a warp, some with more work items than CTAs; against 64 bits on sampled rows, twice the same bits,
    and no further from 64 bits than the bound of an accumulator of that many columns."""
    import numpy as np
    import torch

    import workloads as wl
    from test_layer_operators import Blob, Sums, assert_clean, bits_to_f64, check, up, values, workspace
    w = wl.gaussian_weights(rows, cols, 0.05, rows + cols, dtype)
    blob = Blob(hl, torch, w, dtype, chunk, limit)
    n, (ws,) = workspace(hl, torch, [blob], batch)
    plan = hl.gemm_epilogue_launch_plan([blob.desc], batch, n)
    assert plan["slots_per_warp"] == 1 and plan == hl.gemm_epilogue_launch_plan([blob.desc], batch)
    x = wl.activations(batch, cols, 3, dtype)
    xd = up(torch, x, dtype)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    outs = []
    for _ in range(2):
        outs.append(torch.empty((batch, rows), dtype=torch.float32, device="cuda"))
        hl.decode_gemm_epilogue(blob.desc, blob.dev, xd, batch, hl.Epilogue(hl.ACT_RELU), outs[-1], ws, n, err)
        torch.cuda.synchronize()
        assert_clean(hl, blob, ws, err)
    assert torch.equal(*outs)
    pick = np.unique(np.concatenate([np.arange(0, rows, 37), np.arange(rows - 40, rows)]))
    check(values(outs[0])[:, pick], *Sums(bits_to_f64(w[pick], dtype), bits_to_f64(x, dtype)).through("relu"), "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [12, 24, 64])
@pytest.mark.parametrize("dtype,chunk", [("bf16", 512), ("fp16", 4096)])
def test_several_matrices_with_more_items_than_ctas_each(hl, dtype, chunk, batch):
    """Every matrix of a launch has a counter of its own in its own workspace."""
    import torch

    import workloads as wl
    from test_layer_operators import Blob, Sums, assert_clean, bits_to_f64, check, up, values, workspace
    shapes = [(60000, 256), (20000, 512), (60000, 128)]
    ws_ = [wl.gaussian_weights(r, c, 0.05, r + c, dtype) for r, c in shapes]
    blobs = [Blob(hl, torch, w, dtype, chunk) for w in ws_]
    n, wss = workspace(hl, torch, blobs, batch)
    xs = [wl.activations(batch, c, c, dtype) for _, c in shapes]
    xd = [up(torch, x, dtype) for x in xs]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    for act in ("relu", "silu"):
        outs = [torch.empty((batch, r), dtype=torch.float32, device="cuda") for r, _ in shapes]
        eps = [hl.Epilogue(getattr(hl, "ACT_" + act.upper()))] * 3
        hl.decode_gemm_multi_epilogue([b.desc for b in blobs], [b.dev for b in blobs], xd, batch, eps, outs, wss, n, err)
        torch.cuda.synchronize()
        for b, w, x, ws, out in zip(blobs, ws_, xs, wss, outs):
            assert_clean(hl, b, ws, err)
            check(values(out), *Sums(bits_to_f64(w, dtype), bits_to_f64(x, dtype)).through(act), "f32")


def test_remembered_plans_are_those_worked_out_anew(hl):
    """Questions with and without epilogues in several orders against threads that have kept nothing."""
    import random
    import threading
    descs = [planned_desc(rows, cols, chunk, limit, dtype) for rows, cols, dtype, chunk, limit in LARGE_RECORDS if limit != 7]
    questions = [(epi, d, b, w) for d in descs for b in (12, 33) for w in (0, hl.workspace_bytes(d, b), hl.workspace_bytes(d, 9)) for epi in (False, True)]

    def ask(q):
        epi, d, batch, ws = q
        return (hl.gemm_epilogue_launch_plan if epi else hl.gemm_launch_plan)([d], batch, ws)
    anew = []
    for q in questions:
        t = threading.Thread(target=lambda: anew.append(ask(q)))
        t.start()
        t.join()
    assert len(anew) == len(questions)
    order = list(range(len(questions)))
    for seed in range(3):
        random.Random(seed).shuffle(order)
        for i in order + order[::-1]:
            assert ask(questions[i]) == anew[i]
