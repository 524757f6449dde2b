"""Row order, dispatch, combine, their gradients and the gate's against definitions in 64 bits: sizes on both sides of every variant
(one workgroup / many, pairs counted by every workgroup / by a launch of its own, the counts summed by the scatter / beforehand, 8 / 32 / 64 lanes a token, numbers of slots with and without a
kernel of their own, rows of odd lengths), slots without an expert, and what lies where nothing may be read or written."""
import numpy as np
import pytest
import torch

import row_ops as ro

pytestmark = pytest.mark.gpu


def _sort(moe, ids, E):
    T, k = ids.shape
    ws = torch.empty(moe.moe_sort_workspace_bytes(T, E, k), dtype=torch.uint8, device="cuda")
    offsets, perm, inv = (torch.full(n, -7, dtype=torch.int32, device="cuda") for n in ((E + 1,), (T * k,), (T, k)))
    moe.moe_sort_tokens(ids, E, offsets, perm, inv, ws)
    return offsets, perm, inv


@pytest.mark.parametrize("T,E,k,dropped", [
    (1, 1, 1, 0.0), (1, 256, 64, 0.0), (3, 4, 2, 0.5), (16, 8, 2, 0.0), (31, 200, 33, 0.1), (13, 8, 5, 0.1), (128, 8, 2, 0.0), (43, 8, 6, 0.1), (512, 8, 2, 0.0), (513, 8, 2, 0.2), (2048, 64, 2, 0.0),
    (2049, 64, 2, 0.3), (1000, 63, 8, 0.0), (1000, 64, 8, 0.1), (1000, 127, 8, 0.1), (1000, 128, 8, 0.0), (4096, 16, 8, 0.1), (4097, 16, 8, 0.1), (8000, 100, 8, 0.1),
    (5000, 256, 8, 0.1),
    (65536, 8, 8, 0.05), (70001, 8, 8, 0.05), (262144 + 77, 256, 8, 0.01)])
def test_row_order(T, E, k, dropped):
    import paper_2502_19811_amd as moe
    print(f"row order T {T} E {E} k {k} dropped {dropped}", flush=True)
    ids = ro.slots(T, E, k, T + E + k, dropped)
    got = [v.cpu().numpy() for v in _sort(moe, ids.cuda(), E)]
    for name, a, b in zip(("offsets", "perm", "inv_perm"), got, ro.sort(ids, E)):
        np.testing.assert_array_equal(a, b, err_msg=name)


@pytest.mark.parametrize("T,k,what", [(0, 2, "none"), (100, 2, "dropped"), (40000, 2, "dropped"), (100, 4, "one"), (40000, 4, "one"), (40000, 1, "twice"), (300, 3, "twice")])
def test_row_order_of_one_sided_batches(T, k, what):
    """No tokens, no slot with an expert, every slot with the same one, the same expert several times in a token."""
    import paper_2502_19811_amd as moe
    E = 16
    ids = {"none": torch.zeros((T, k)), "dropped": torch.full((T, k), -3), "one": torch.full((T, k), 11),
           "twice": torch.arange(T)[:, None].expand(T, k) * 7 % E}[what].to(torch.int32).contiguous()
    print(f"row order T {T} k {k} {what}", flush=True)
    got = [v.cpu().numpy() for v in _sort(moe, ids.cuda(), E)]
    for a, b in zip(got, ro.sort(ids, E)):
        np.testing.assert_array_equal(a, b)


def test_row_order_is_the_layers():
    import paper_2502_19811_amd as moe
    import gpu_harness as H
    import workloads as wl
    from oracle import moe_oracle as orc
    cfg = wl.CONFIGS["tiny"]
    inp = wl.make_inputs(cfg, threads=2)
    ids, w = orc.route_topk(inp.logits, cfg.k)
    layer = H.GpuLayer(cfg, inp, ids, w)
    layer.forward()
    run = layer.results()
    layer.close()
    offsets, perm, inv = (v.cpu().numpy() for v in _sort(moe, torch.from_numpy(ids).cuda(), cfg.E))
    np.testing.assert_array_equal(offsets, run.offsets)
    np.testing.assert_array_equal(perm, run.perm)
    np.testing.assert_array_equal(inv.reshape(-1), run.inv_perm)


# rows of 16 bytes and a little more, of 8, 32 and 64 lanes, of one span and several, odd ones
WIDTHS = [8, 9, 33, 64, 65, 100, 256, 257, 1000, 1001, 2048, 4096, 4097, 8200]


def _pairs(T, E, k, seed, dropped):
    ids = ro.slots(T, E, k, seed, dropped)
    inv = torch.from_numpy(ro.sort(ids, E)[2]).cuda()
    g = torch.Generator()
    g.manual_seed(seed + 1)
    w = torch.softmax(torch.randn((T, k), generator=g), dim=1).contiguous().cuda()
    return ids.cuda(), inv, w


@pytest.mark.parametrize("dtype", ro.DTYPES, ids=str)
@pytest.mark.parametrize("H", WIDTHS)
def test_dispatch(H, dtype):
    import paper_2502_19811_amd as moe
    for T, E, k, dropped in ((1, 8, 1, 0.0), (37, 8, 3, 0.3), (130, 16, 9, 0.1)):
        print(f"dispatch T {T} H {H} k {k} {dtype}", flush=True)
        _, inv, _ = _pairs(T, E, k, H + T, dropped)
        x = ro.dev((T, H), dtype, 3)
        x[0, H // 2], x[T // 2, 0] = float("nan"), float("inf")       # moved, not computed with
        rows, check = ro.guarded((T * k, H), dtype, 7.0)
        moe.moe_dispatch(x, inv, rows)
        ref = torch.full((T * k, H), 7.0, dtype=dtype, device="cuda")   # rows that no pair has stay
        kept = inv >= 0
        ref[inv[kept].long()] = x[torch.nonzero(kept)[:, 0]]
        assert torch.equal(rows.view(torch.uint8), ref.view(torch.uint8))
        check()


@pytest.mark.parametrize("dtype", ro.DTYPES, ids=str)
@pytest.mark.parametrize("H", WIDTHS)
def test_combine_and_gradient_of_dispatch(H, dtype):
    import paper_2502_19811_amd as moe
    for T, E, k, dropped in ((1, 8, 1, 0.0), (37, 8, 2, 0.3), (40, 8, 3, 0.2), (41, 8, 4, 0.0), (42, 16, 7, 0.1), (43, 16, 8, 0.1), (30, 32, 17, 0.1)):
        print(f"combine T {T} H {H} k {k} {dtype}", flush=True)
        _, inv, w = _pairs(T, E, k, H + T, dropped)
        rows = ro.dev((T * k, H), dtype, 4)
        n = int((inv >= 0).sum())
        rows[n:] = float("nan")                                        # rows of no pair do not matter
        for weights in (w, None):
            out, check = ro.guarded((T, H), dtype, 7.0)
            if weights is None:
                moe.moe_dispatch_backward(rows, inv, out)
            else:
                moe.moe_combine(rows, inv, weights, out)
            ref, size = ro.combine(rows, inv, weights)
            ro.close(out, ref, (k + 1) * ro.STEP32 * size, "combine")
            assert bool((out[(inv < 0).all(dim=1)] == 0).all())
            check()
        plain = torch.empty_like(out)
        moe.moe_combine(rows, inv, None, plain)
        assert torch.equal(plain, out)


@pytest.mark.parametrize("dtype", ro.DTYPES, ids=str)
@pytest.mark.parametrize("H", WIDTHS)
def test_gradient_of_combine(H, dtype):
    import paper_2502_19811_amd as moe
    for T, E, k, dropped in ((1, 8, 1, 0.0), (37, 8, 2, 0.3), (40, 8, 3, 0.2), (42, 16, 7, 0.1), (43, 16, 8, 0.1), (30, 32, 17, 0.1), (4099, 8, 2, 0.1), (4100, 16, 5, 0.0),
                             (4098, 16, 9, 0.0)):
        if T > 4096 and H not in (1001, 4096):
            continue
        print(f"combine gradient T {T} H {H} k {k} {dtype}", flush=True)
        _, inv, w = _pairs(T, E, k, H + T, dropped)
        rows, g = ro.dev((T * k, H), dtype, 5), ro.dev((T, H), dtype, 6)
        kept = inv >= 0
        rows[int(kept.sum()):] = float("nan")
        at, tok = inv[kept].long(), torch.nonzero(kept)[:, 0]
        products = g[tok].double() * rows[at].double()
        for weights in (w, None):
            grad_rows, check = ro.guarded((T * k, H), dtype, 7.0)
            grad_w, check_w = ro.guarded((T, k), torch.float32, 7.0)
            moe.moe_combine_backward(g, rows, inv, weights, grad_rows, grad_w)
            ref = torch.full((T * k, H), 7.0, dtype=torch.float64, device="cuda")
            ref[at] = g[tok].double() * (1.0 if weights is None else weights[kept].double()[:, None])
            ro.close(grad_rows, ref, ro.STEP32 * ref.abs(), "grad_rows")
            ref = torch.zeros((T, k), dtype=torch.float64, device="cuda")
            size = torch.zeros_like(ref)
            ref[kept], size[kept] = products.sum(dim=1), products.abs().sum(dim=1)
            ro.close(grad_w, ref, (H / 8 + 24) * ro.STEP32 * size, "grad_weights")     # at most H/8 products of a lane in a row
            assert bool((grad_w[~kept] == 0).all())
            check()
            check_w()
        only, check = ro.guarded((T * k, H), dtype, 7.0)
        moe.moe_combine_backward(g, None, inv, None, only, None)
        assert torch.equal(only, grad_rows)
        check()


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (5, 2, 2), (203, 8, 2), (100, 63, 8), (64, 64, 64), (333, 65, 17), (70, 256, 5), (9000, 64, 8)])
def test_gradient_of_the_gate(T, E, k):
    import paper_2502_19811_amd as moe
    print(f"gate gradient T {T} E {E} k {k}", flush=True)
    g = torch.Generator()
    g.manual_seed(T + E)
    logits = torch.randn((T, E), generator=g).cuda()
    ids = torch.zeros((T, k), dtype=torch.int32, device="cuda")
    w = torch.zeros((T, k), device="cuda")
    if E > k:
        logits[1::3, 0] = float("-inf")          # a masked expert
    moe.moe_route_topk(logits, k, ids, w)
    gw = torch.randn((T, k), generator=g).cuda()
    out, check = ro.guarded((T, E), torch.float32, 7.0)
    moe.moe_route_topk_backward(ids, w, gw, out)
    W, G = w.double(), gw.double()
    d = W * (G - (W * G).sum(dim=1, keepdim=True))
    size = W * (G.abs() + (W * G).abs().sum(dim=1, keepdim=True))
    ref, extra = torch.zeros((T, E), dtype=torch.float64, device="cuda"), torch.zeros((T, E), dtype=torch.float64, device="cuda")
    ref.scatter_(1, ids.long(), d)
    extra.scatter_(1, ids.long(), (k + 4) * ro.STEP32 * size)
    ro.close(out, ref, extra, "grad_logits")
    check()
    # against differences: the loss sum(w * gw) of softmax over the kept logits, in 64 bits
    rows = torch.arange(min(T, 50), device="cuda")
    kept = torch.gather(logits.double(), 1, ids.long())[rows]
    for j in range(min(k, 3)):
        step = torch.zeros_like(kept)
        step[:, j] = 1e-6
        diff = ((torch.softmax(kept + step, 1) - torch.softmax(kept - step, 1)) * G[rows]).sum(dim=1) / 2e-6
        got = torch.gather(out[rows].double(), 1, ids[rows].long())[:, j]
        # W is off by fp32 steps (1e-6 of it), the difference by 1e-16 / 1e-6 and 1e-12
        assert bool(((got - diff).abs() <= 2e-5 * (G[rows].abs().sum(dim=1) + 1e-3)).all())


def test_gate_gradient_of_dropped_and_repeated_slots():
    import paper_2502_19811_amd as moe
    ids = torch.tensor([[0, 0, 2], [-1, 1, 5], [4, -1, 4]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[0.5, 0.25, 0.25]] * 3, device="cuda")
    gw = torch.tensor([[1.0, 2.0, 4.0], [0.0, 3.0, 0.0], [1.0, 0.0, -1.0]], device="cuda")
    out = torch.full((3, 5), 7.0, device="cuda")
    moe.moe_route_topk_backward(ids, w, gw, out)
    # sums: 2, 0.75, 0.25 -- all values are exact
    assert out.tolist() == [[-0.5, 0.0, 0.5, 0.0, 0.0], [0.0, 0.5625, 0.0, 0.0, 0.0], [0.0, 0.0, 0.0, 0.0, 0.0625]]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_indices_outside_are_no_row(dtype):
    """inv_perm with values behind the last row and before the first: nothing outside is touched."""
    import paper_2502_19811_amd as moe
    T, H, k = 50, 264, 2
    inv = torch.arange(T * k, dtype=torch.int32).reshape(T, k)
    inv[::3, 0], inv[1::3, 1], inv[2::3, 0] = T * k, -2 ** 31, 2 ** 31 - 1
    inv = inv.cuda()
    clean = torch.where((inv >= 0) & (inv < T * k), inv, -1)
    x, rows = ro.dev((T, H), dtype, 8), ro.dev((T * k, H), dtype, 9)
    a, check = ro.guarded((T * k, H), dtype, 7.0)
    b = torch.full((T * k, H), 7.0, dtype=dtype, device="cuda")
    moe.moe_dispatch(x, inv, a)
    moe.moe_dispatch(x, clean, b)
    assert torch.equal(a, b)
    check()
    a, b = torch.empty_like(x), torch.empty_like(x)
    moe.moe_combine(rows, inv, None, a)
    moe.moe_combine(rows, clean, None, b)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
@pytest.mark.parametrize("H", [30001, 65536])
def test_the_widest_rows(H, dtype):
    import paper_2502_19811_amd as moe
    T, k = 7, 3
    print(f"widest rows H {H} {dtype}", flush=True)
    _, inv, w = _pairs(T, 8, k, H, 0.2)
    x, g = ro.dev((T, H), dtype, 11), ro.dev((T, H), dtype, 12)
    rows, check = ro.guarded((T * k, H), dtype, 7.0)
    moe.moe_dispatch(x, inv, rows)
    kept = inv >= 0
    at, tok = inv[kept].long(), torch.nonzero(kept)[:, 0]
    assert torch.equal(rows[at], x[tok])
    check()
    out = torch.empty_like(x)
    moe.moe_combine(rows, inv, w, out)
    ref, size = ro.combine(rows, inv, w)
    ro.close(out, ref, (k + 1) * ro.STEP32 * size, "combine")
    grad_rows, check = ro.guarded((T * k, H), dtype, 7.0)
    grad_w = torch.empty((T, k), device="cuda")
    moe.moe_combine_backward(g, rows, inv, w, grad_rows, grad_w)
    ref = g[tok].double() * w[kept].double()[:, None]
    ro.close(grad_rows[at], ref, ro.STEP32 * ref.abs(), "grad_rows")
    products = g[tok].double() * rows[at].double()
    ro.close(grad_w[kept], products.sum(dim=1), (H / 8 + 24) * ro.STEP32 * products.abs().sum(dim=1), "grad_weights")
    check()


@pytest.mark.parametrize("dtype", ro.DTYPES, ids=str)
def test_no_tokens(dtype):
    import paper_2502_19811_amd as moe
    x, rows, inv = (torch.empty(s, dtype=d, device="cuda") for s, d in (((0, 64), dtype), ((0, 64), dtype), ((0, 2), torch.int32)))
    w, logits = torch.empty((0, 2), device="cuda"), torch.empty((0, 4), device="cuda")
    moe.moe_dispatch(x, inv, rows)
    moe.moe_dispatch_backward(rows, inv, x)
    moe.moe_combine(rows, inv, w, x)
    moe.moe_combine_backward(x, rows, inv, w, rows, w)
    moe.moe_route_topk_backward(inv, w, w, logits)
    torch.cuda.synchronize()


def test_rows_beyond_4_gib():
    import paper_2502_19811_amd as moe
    T, H, k = 140000, 8192, 2                                   # rows of 4.6 GB
    print(f"T {T} H {H} k {k}: {T * k * H * 2 / 2 ** 30:.1f} GiB of rows", flush=True)
    ids = (torch.arange(T * k, dtype=torch.int32) * 5 % 8).reshape(T, k).contiguous().cuda()
    offsets, perm, inv = _sort(moe, ids, 8)
    x = torch.empty((T, H), dtype=torch.bfloat16, device="cuda").normal_()
    rows = torch.empty((T * k, H), dtype=torch.bfloat16, device="cuda")
    moe.moe_dispatch(x, inv, rows)
    at = torch.randint(0, T * k, (3000,), device="cuda")
    at[:2] = torch.tensor([0, T * k - 1])
    assert torch.equal(rows[at], x[(perm[at] // k).long()])
    back = torch.empty_like(x)
    moe.moe_combine(rows, inv, torch.full((T, k), 0.5, device="cuda"), back)
    assert torch.equal(back, x)                                 # halves of the same value: exact
    grad_rows, grad_w = torch.empty_like(rows), torch.empty((T, k), device="cuda")
    moe.moe_combine_backward(x, rows, inv, None, grad_rows, grad_w)
    assert torch.equal(grad_rows[at], rows[at])
    t = torch.randint(0, T, (500,), device="cuda")
    ref = x[t].double().square().sum(dim=1)
    ro.close(grad_w[t, 1], ref, (H / 8 + 24) * ro.STEP32 * ref, "grad_weights")
