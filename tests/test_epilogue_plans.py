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
