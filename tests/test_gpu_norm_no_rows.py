"""What is summed over tokens when there are none: zeros, also where the sums' factors are no numbers."""
import pytest
import torch

import row_ops as ro

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan"), 1.0])
@pytest.mark.parametrize("dtype", ro.DTYPES, ids=str)
@pytest.mark.parametrize("H", [8, 1001, 4096])
def test_sums_over_no_rows(H, dtype, value):
    import paper_2502_19811_amd as moe
    none, factor = torch.empty((0, H), dtype=dtype, device="cuda"), torch.full((H,), value, dtype=dtype, device="cuda")
    ws = torch.full((moe.moe_norm_workspace_bytes(0, H),), 0xff, dtype=torch.uint8, device="cuda")
    for norm in (moe.MOE_NORM_RMS, moe.MOE_NORM_LAYER):
        sums = [torch.full((H,), 7.0, device="cuda") for _ in range(3)]
        moe.moe_norm_after_backward(none, factor, factor, factor, moe.MOE_GATE_CHANNEL, 1.0, none, norm, 1e-5, none, *sums, ws)
        assert all(bool((s == 0).all()) for s in sums)
        sums = [torch.full((H,), 7.0, device="cuda") for _ in range(2)]
        moe.moe_norm_before_backward(none, factor, none, None, 1.0, norm, 1e-5, none, None, *sums, ws)
        assert all(bool((s == 0).all()) for s in sums)
