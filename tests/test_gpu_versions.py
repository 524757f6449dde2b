"""Gradients of torch's that need what a call has overwritten: an error instead of a wrong gradient."""
import pytest
import torch

import row_ops as ro

pytestmark = pytest.mark.gpu

T, H, E, k = 24, 256, 4, 2


def _plan(moe):
    return moe.moe_plan_create(T, H, 256, E, k, 1, moe.MOE_ACT_SWIGLU, [0, T])


def _calls(moe):
    f32, bf, i32 = torch.float32, torch.bfloat16, torch.int32
    new = lambda *shape, dt=f32: torch.zeros(shape, dtype=dt, device="cuda")  # noqa: E731
    logits, ids, w = ro.dev((T, E), f32, 1), new(T, k, dt=i32), new(T, k)
    x, out = ro.dev((T, H), bf, 2, 0.1), new(T, H, dt=bf)
    W1, W2 = ro.dev((E, 2 * 256, H), bf, 3, 0.05), ro.dev((E, H, 256), bf, 4, 0.05)
    rows, offsets, perm, inv, gamma = new(T * k, H, dt=bf), new(E + 1, dt=i32), new(T * k, dt=i32), new(T, k, dt=i32), ro.dev((H,), bf, 5)

    def forward():
        plan = _plan(moe)
        ws = torch.empty(moe.moe_plan_workspace_bytes(plan) + 256, dtype=torch.uint8, device="cuda")
        ws = ws[-ws.data_ptr() % 256:]
        moe.moe_layer_forward(plan, x, ids, w, W1, W2, moe.MOE_ACT_SWIGLU, out, ws)
        torch.cuda.synchronize()
        moe.moe_plan_destroy(plan)
    return [
        ("norm", x, lambda: moe.moe_norm_before(x, None, 1.0, gamma, None, moe.MOE_NORM_RMS, 1e-5, None, x)),
        ("gate", w, lambda: moe.moe_route_topk(logits, k, ids, w)),
        ("gate's ids", ids, lambda: moe.moe_route_topk(logits, k, ids, w)),
        ("sort", inv, lambda: moe.moe_sort_tokens(ids, E, offsets, perm, inv, new(moe.moe_sort_workspace_bytes(T, E, k), dt=torch.uint8))),
        ("dispatch", rows, lambda: moe.moe_dispatch(x, inv, rows)),
        ("combine", out, lambda: moe.moe_combine(rows, inv, w, out)),
        ("layer", out, forward),
    ]


def test_saved_tensors_that_a_call_overwrites():
    import paper_2502_19811_amd as moe
    for name, target, call in _calls(moe):
        print(name, flush=True)
        if target.dtype == torch.int32:              # saved as an index
            factor = torch.ones(16, 128, device="cuda", requires_grad=True)
            loss = torch.gather(factor, 1, torch.zeros((1, 1), dtype=torch.int64, device="cuda")).sum() + factor.sum()
            version = target._version
            call()
            assert target._version == version + 1
            loss.backward()                          # what was not overwritten does not mind
            continue
        factor = torch.ones(target.shape[1], device="cuda", dtype=target.dtype, requires_grad=True)
        loss = (target * factor).sum()
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
