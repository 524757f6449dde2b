"""The operators around the experts on streams of the caller's: every result holds something else before each run, and whatever the streams
need of each other is waited for."""
import pytest
import torch

import row_ops as ro
import test_gpu_train_block as tb

pytestmark = pytest.mark.gpu


def _spoil(b):
    for v in tb._results(b):
        v.fill_(77)


def _spoil_and_check(b, eager, run):
    _spoil(b)
    torch.cuda.synchronize()
    run()
    torch.cuda.synchronize()
    for i, (a, c) in enumerate(zip(tb._results(b), eager)):
        assert torch.equal(a, c), i


def _block(T, H, E, k, seed, layer):
    """A block whose forward has run, and the results of its operators in order, on the current stream."""
    b = tb.Block(T, H, E, k, torch.bfloat16, seed, layer)
    b.forward()
    tb._without_products(b)
    torch.cuda.synchronize()
    eager = [v.clone() for v in tb._results(b)]
    torch.cuda.synchronize()
    return b, eager


def test_the_current_stream():
    b, eager = _block(900, 264, 8, 2, 80, True)
    side = torch.cuda.Stream()
    for _ in range(3):
        def run():
            with torch.cuda.stream(side):
                tb._without_products(b)
        _spoil_and_check(b, eager, run)


def test_a_stream_by_name():
    """Each call's input is there late, and on its own stream only: a call that goes elsewhere reads what was there before."""
    b, eager = _block(900, 264, 8, 2, 81, True)
    m, side, busy = b.moe, torch.cuda.Stream(), ro.dev((4096, 4096), torch.float32, 1)
    torch.cuda.synchronize()
    beta = b.b2
    rows = eager[5]
    calls = [      # (input, call, outputs, what they are)
        (b.h, lambda: m.moe_norm_before(b.h, b.u, tb.SCALE, b.g1, b.b1, b.norm, tb.EPS, b.s, b.x, stream=side), (b.s, b.x)),
        (b.ids, lambda: m.moe_sort_tokens(b.ids, b.E, b.offsets, b.perm, b.inv, b.sort_ws, stream=side), (b.offsets, b.perm, b.inv)),
        (b.x, lambda: m.moe_dispatch(b.x, b.inv, b.rows, stream=side), (b.rows,)),
        (b.rows, lambda: m.moe_combine(b.rows, b.inv, b.w, b.y, stream=side), (b.y,)),
        (b.y, lambda: m.moe_norm_after(b.s, b.y, b.g2, beta, b.gate, m.MOE_GATE_CHANNEL, tb.SCALE, b.norm, tb.EPS, b.out, stream=side), (b.out,)),
        (b.grad_out, lambda: m.moe_norm_after_backward(b.y, b.g2, beta, b.gate, m.MOE_GATE_CHANNEL, tb.SCALE, b.grad_out, b.norm, tb.EPS, b.gy,
                                                       b.gg2, None, b.ggate, b.norm_ws, stream=side), (b.gy, b.gg2, b.ggate)),
        (b.gy, lambda: m.moe_combine_backward(b.gy, b.rows, b.inv, b.w, b.g_expert_out, b.gw, stream=side), (b.g_expert_out, b.gw)),
        (b.gw, lambda: m.moe_route_topk_backward(b.ids, b.w, b.gw, b.glogits, stream=side), (b.glogits,)),
        (b.g_expert_out, lambda: m.moe_dispatch_backward(b.g_expert_out, b.inv, b.gx, stream=side), (b.gx,)),
        (b.gx, lambda: m.moe_norm_before_backward(b.s, b.g1, b.gx, b.grad_out, tb.SCALE, b.norm, tb.EPS, b.gr, b.gu, b.gg1, None, b.norm_ws,
                                                  stream=side), (b.gr, b.gu, b.gg1)),
    ]
    assert torch.equal(rows, b.rows)
    for i, (late, call, outputs) in enumerate(calls):
        print(f"call {i}", flush=True)
        want, value = [o.clone() for o in outputs], late.clone()
        late.zero_()
        for o in outputs:
            o.fill_(77)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(6):
                busy @ busy                     # some milliseconds
            late.copy_(value)
        call()                                  # the current stream is the default one, and idle
        side.synchronize()
        for o, w in zip(outputs, want):
            assert torch.equal(o, w)


def test_two_streams_with_workspaces_of_their_own():
    blocks = [_block(2500, 520, 16, 4, 90 + i, bool(i)) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in blocks]
    for rep in range(5):
        for b, _ in blocks:
            _spoil(b)
        torch.cuda.synchronize()
        for (b, _), s in zip(blocks, streams):
            with torch.cuda.stream(s):
                tb._without_products(b)
        torch.cuda.synchronize()
        for b, eager in blocks:
            for i, (a, c) in enumerate(zip(tb._results(b), eager)):
                assert torch.equal(a, c), (rep, i)
