"""The norms on either side of the block and their gradients against definitions in 64 bits: every number of wavefronts a row may
have, rows of odd lengths and rows that do not fill their lanes, more rows than groups of rows, every gate, outputs in the place of inputs."""
import itertools

import pytest
import torch

import row_ops as ro

pytestmark = pytest.mark.gpu

EPS = 1e-5
# bf16 pieces of 16 bytes: 1, 2, 5, 64, 65, 126, 138, 250, 256, 321 (the last piece alone in its wavefront), 448, 512, 513, 577, 1025, 2048
WIDTHS = [8, 9, 33, 512, 513, 1003, 1100, 2000, 2048, 2561, 3584, 4096, 4097, 4609, 8200, 16384]
CASES = [(1, False), (5, True), (300, False), (301, True)]
GATES = ["none", "channel", "token", "full"]


def _kind(moe, gate):
    return [moe.MOE_GATE_NONE, moe.MOE_GATE_CHANNEL, moe.MOE_GATE_TOKEN, moe.MOE_GATE_FULL][GATES.index(gate)]


def _gate(gate, T, H, dtype, seed):
    return {"none": lambda: None, "channel": lambda: ro.dev((H,), dtype, seed, 0.5, 0.5), "token": lambda: ro.dev((T,), torch.float32, seed, 0.5, 0.5),
            "full": lambda: ro.dev((T, H), dtype, seed, 0.5, 0.5)}[gate]()


def _wide(gate, v):
    """A gate, or what goes with it, as something that multiplies rows, in 64 bits."""
    return 1.0 if v is None else v.double()[:, None] if gate == "token" else v.double()


def _rows(T, H, dtype, seed):
    v = ro.dev((T, H), dtype, seed, 2.0, 0.7)
    v[:, H // 3] *= 20.0                       # a large channel
    return v


@pytest.mark.parametrize("dtype", ro.DTYPES, ids=str)
@pytest.mark.parametrize("H", WIDTHS)
def test_before(H, dtype):
    import paper_2502_19811_amd as moe
    for T, layer in CASES:
        print(f"before T {T} H {H} layer {layer} {dtype}", flush=True)
        res, upd = _rows(T, H, dtype, 1), ro.dev((T, H), dtype, 2)
        gamma, beta = ro.dev((H,), dtype, 3, 0.2, 1.0), ro.dev((H,), dtype, 4) if layer else None
        norm = moe.MOE_NORM_LAYER if layer else moe.MOE_NORM_RMS
        for update, scale in ((upd, 0.37), (None, 1.0)):
            s, check_s = ro.guarded((T, H), dtype, 7.0)
            x, check_x = ro.guarded((T, H), dtype, 7.0)
            moe.moe_norm_before(res, update, scale, gamma, beta, norm, EPS, s, x)
            v = res.double() + (0.0 if update is None else torch.tensor(scale, dtype=torch.float32).double().item() * update.double())
            ro.close(s, v, ro.STEP32 * v.abs(), "sum")
            d = ro.Norm(v, layer, EPS)
            G, B = gamma.double(), 0.0 if beta is None else beta.double()
            size = d.size * G.abs() * (1.0 if not layer else d.size.square().mean(dim=1, keepdim=True).clamp(min=1.0)) + (0.0 if beta is None else B.abs())
            ro.close(x, d.n * G + B, ro.CHAIN * ro.STEP32 * size, "x")
            check_s()
            check_x()
            # without the sum, and in place of either input: the same bits
            again = torch.empty_like(x)
            moe.moe_norm_before(res, update, scale, gamma, beta, norm, EPS, None, again)
            assert torch.equal(again, x)
            a = res.clone()
            moe.moe_norm_before(a, update, scale, gamma, beta, norm, EPS, a, again)
            assert torch.equal(a, s) and torch.equal(again, x)
            if update is not None:
                a, b = res.clone(), upd.clone()
                moe.moe_norm_before(a, b, scale, gamma, beta, norm, EPS, a, b)
                assert torch.equal(a, s) and torch.equal(b, x)


@pytest.mark.parametrize("dtype", ro.DTYPES, ids=str)
@pytest.mark.parametrize("H", WIDTHS)
def test_gradient_of_before(H, dtype):
    import paper_2502_19811_amd as moe
    for T, layer in CASES + [(4, True), (31, False), (2500, H % 2 == 0), (4099, H % 2 == 1)]:      # 4099: groups of narrow rows that do not fill a workgroup
        if T > 2000 and H > (4097 if T == 2500 else 1100):
            continue
        print(f"before gradient T {T} H {H} layer {layer} {dtype}", flush=True)
        v, gx, gs = _rows(T, H, dtype, 1), ro.dev((T, H), dtype, 2), ro.dev((T, H), dtype, 3)
        gamma = ro.dev((H,), dtype, 4, 0.2, 1.0)
        norm = moe.MOE_NORM_LAYER if layer else moe.MOE_NORM_RMS
        ws = torch.full((moe.moe_norm_workspace_bytes(T, H),), 0xff, dtype=torch.uint8, device="cuda")
        scale = 0.37
        d = ro.Norm(v, layer, EPS)
        GX = gx.double()
        ref, size = d.backward(GX * gamma.double())
        for more, want_beta in ((gs, layer), (None, not layer)):
            out = [ro.guarded((T, H), dtype, 7.0), ro.guarded((T, H), dtype, 7.0), ro.guarded((H,), torch.float32, 7.0), ro.guarded((H,), torch.float32, 7.0)]
            grad_res, grad_upd, grad_gamma, grad_beta = (o[0] for o in out)
            moe.moe_norm_before_backward(v, gamma, gx, more, scale, norm, EPS, grad_res, grad_upd, grad_gamma, grad_beta if want_beta else None, ws)
            total = ref + (0.0 if more is None else more.double())
            extra = ro.CHAIN * ro.STEP32 * size + 2 * ro.STEP32 * total.abs()
            ro.close(grad_res, total, extra, "grad_residual")
            s32 = torch.tensor(scale, dtype=torch.float32).double().item()
            ro.close(grad_upd, s32 * total, s32 * extra + ro.STEP32 * total.abs(), "grad_update")
            # rows of a group one after the other (256 groups and more, or one row each), then 8 or so sums and 32 more
            chain = ro.STEP32 * (ro.CHAIN + T / 256 + 64 + 32)
            deviation = d.size.square().mean(dim=1, keepdim=True).clamp(min=1.0) if layer else 1.0
            ro.close(grad_gamma, (GX * d.n).sum(dim=0), chain * (GX.abs() * d.size * deviation).sum(dim=0), "grad_gamma")
            if want_beta:
                ro.close(grad_beta, GX.sum(dim=0), chain * GX.abs().sum(dim=0), "grad_beta")
            for _, check in out:
                check()
            # in place, and without what is not wanted: the same bits
            a, b = (gs.clone() if more is not None else v.clone()), gx.clone()
            moe.moe_norm_before_backward(v if more is not None else a, gamma, b, a if more is not None else None, scale, norm, EPS, a, b, None, None, None)
            assert torch.equal(a, grad_res) and torch.equal(b, grad_upd)
            a = torch.empty_like(gx)
            again = torch.full((H,), 7.0, device="cuda")
            moe.moe_norm_before_backward(v, gamma, gx, more, scale, norm, EPS, a, None, again, None, ws)
            assert torch.equal(a, grad_res) and torch.equal(again, grad_gamma)


@pytest.mark.parametrize("dtype", ro.DTYPES, ids=str)
@pytest.mark.parametrize("H", WIDTHS)
def test_after(H, dtype):
    import paper_2502_19811_amd as moe
    for (T, layer), gate in itertools.product(CASES, GATES):
        if T > 100 and gate == "none":
            continue
        print(f"after T {T} H {H} layer {layer} gate {gate} {dtype}", flush=True)
        res, y = _rows(T, H, dtype, 1), _rows(T, H, dtype, 2)
        gamma, beta = ro.dev((H,), dtype, 3, 0.2, 1.0), ro.dev((H,), dtype, 4) if layer else None
        h, kind, norm, scale = _gate(gate, T, H, dtype, 5), _kind(moe, gate), moe.MOE_NORM_LAYER if layer else moe.MOE_NORM_RMS, -0.6
        out, check = ro.guarded((T, H), dtype, 7.0)
        moe.moe_norm_after(res, y, gamma, beta, h, kind, scale, norm, EPS, out)
        d = ro.Norm(y, layer, EPS)
        G, B, m = gamma.double(), 0.0 if beta is None else beta.double(), torch.tensor(scale, dtype=torch.float32).double().item() * _wide(gate, h)
        size = d.size * G.abs() * (1.0 if not layer else d.size.square().mean(dim=1, keepdim=True).clamp(min=1.0)) + (0.0 if beta is None else B.abs())
        m_abs = m.abs() if isinstance(m, torch.Tensor) else abs(m)
        extra = ro.CHAIN * ro.STEP32 * size * m_abs
        branch = m * (d.n * G + B)
        ro.close(out, res.double() + branch, extra + ro.STEP32 * (res.double() + branch).abs(), "out")
        check()
        alone = torch.empty_like(out)
        moe.moe_norm_after(None, y, gamma, beta, h, kind, scale, norm, EPS, alone)
        ro.close(alone, branch + torch.zeros_like(y.double()), extra, "out without a residual stream")
        for place in ("residual", "y") + (("gate",) if gate == "full" else ()):
            a, b, c = res.clone(), y.clone(), h.clone() if h is not None else None
            o = {"residual": a, "y": b, "gate": c}[place]
            moe.moe_norm_after(a, b, gamma, beta, c, kind, scale, norm, EPS, o)
            assert torch.equal(o, out), place


@pytest.mark.parametrize("dtype", ro.DTYPES, ids=str)
@pytest.mark.parametrize("H", WIDTHS)
def test_gradient_of_after(H, dtype):
    import paper_2502_19811_amd as moe
    for (T, layer), gate in itertools.product(CASES + [(4, False), (31, True), (2500, H % 2 == 1), (4099, H % 2 == 0)], GATES):
        if (T > 2000 and (H > (4097 if T == 2500 else 1100) or gate == "none")) or (T == 1 and gate == "none"):
            continue
        print(f"after gradient T {T} H {H} layer {layer} gate {gate} {dtype}", flush=True)
        y, g = _rows(T, H, dtype, 1), ro.dev((T, H), dtype, 2)
        gamma, beta = ro.dev((H,), dtype, 3, 0.2, 1.0), ro.dev((H,), dtype, 4) if layer else None
        h, kind, norm, scale = _gate(gate, T, H, dtype, 5), _kind(moe, gate), moe.MOE_NORM_LAYER if layer else moe.MOE_NORM_RMS, 0.6
        ws = torch.full((moe.moe_norm_workspace_bytes(T, H),), 0xff, dtype=torch.uint8, device="cuda")
        gate_type = dtype if gate == "full" else torch.float32
        out = [ro.guarded((T, H), dtype, 7.0), ro.guarded((H,), torch.float32, 7.0), ro.guarded((H,), torch.float32, 7.0)]
        if h is not None:
            out.append(ro.guarded(tuple(h.shape), gate_type, 7.0))
        grad_y, grad_gamma, grad_beta = (o[0] for o in out[:3])
        grad_gate = out[3][0] if h is not None else None
        moe.moe_norm_after_backward(y, gamma, beta, h, kind, scale, g, norm, EPS, grad_y, grad_gamma, grad_beta if layer else None, grad_gate, ws)
        d = ro.Norm(y, layer, EPS)
        deviation = d.size.square().mean(dim=1, keepdim=True).clamp(min=1.0) if layer else torch.ones((), device="cuda", dtype=torch.float64)
        G, B = gamma.double(), torch.zeros(H, device="cuda", dtype=torch.float64) if beta is None else beta.double()
        GS = torch.tensor(scale, dtype=torch.float32).double().item() * g.double()
        F = GS * _wide(gate, h)
        ref, size = d.backward(F * G)
        if gate == "token":    # its mean is taken before the token's gate is multiplied in: one rounding more
            size = size * 2
        ro.close(grad_y, ref, ro.CHAIN * ro.STEP32 * size, "grad_y")
        chain = ro.STEP32 * (ro.CHAIN + T / 256 + 64 + 32)
        n_size = d.size * deviation
        ro.close(grad_gamma, (F * d.n).sum(dim=0), chain * (F.abs() * n_size).sum(dim=0), "grad_gamma")
        if layer:
            ro.close(grad_beta, F.sum(dim=0), chain * F.abs().sum(dim=0), "grad_beta")
        if gate != "none":
            full, full_size = GS * (d.n * G + B), GS.abs() * (n_size * G.abs() + B.abs())
            if gate == "channel":
                ro.close(grad_gate, full.sum(dim=0), chain * full_size.sum(dim=0), "grad_gate")
            elif gate == "token":
                ro.close(grad_gate, full.sum(dim=1), ro.CHAIN * ro.STEP32 * full_size.sum(dim=1), "grad_gate")
            else:
                ro.close(grad_gate, full, ro.CHAIN * ro.STEP32 * full_size, "grad_gate")
        for _, check in out:
            check()
        # in place, and without what is not wanted: the same bits
        a, b, c = y.clone(), g.clone(), h.clone() if h is not None else None
        moe.moe_norm_after_backward(a, gamma, beta, c, kind, scale, b, norm, EPS, b, None, None, c if gate == "full" else None, None)
        assert torch.equal(b, grad_y) and (gate != "full" or torch.equal(c, grad_gate))
        if gate in ("token", "full"):       # the gate's gradient not wanted
            again, other = torch.full((H,), 7.0, device="cuda"), torch.empty_like(y)
            moe.moe_norm_after_backward(y, gamma, beta, h, kind, scale, g, norm, EPS, other, again, None, None, ws)
            assert torch.equal(again, grad_gamma) and torch.equal(other, grad_y)
        if gate == "channel":
            again = torch.full((H,), 7.0, device="cuda")
            moe.moe_norm_after_backward(y, gamma, beta, h, kind, scale, g, norm, EPS, a, None, None, again, ws)
            assert torch.equal(again, grad_gate) and torch.equal(a, grad_y)


@pytest.mark.parametrize("layer", [False, True])
def test_rows_of_zeros_and_of_one_value(layer):
    """Deviation 0: eps alone holds the quotient; with eps 0 a row of zeros has no norm (NaN) and the others are as ever."""
    import paper_2502_19811_amd as moe
    T, H = 6, 1000
    norm = moe.MOE_NORM_LAYER if layer else moe.MOE_NORM_RMS
    gamma = ro.dev((H,), torch.float32, 1)
    v = ro.dev((T, H), torch.float32, 2)
    v[1], v[4] = 0.0, 2.0
    x, x0 = torch.empty_like(v), torch.empty_like(v)
    moe.moe_norm_before(v, None, 1.0, gamma, None, norm, EPS, None, x)
    assert bool(torch.isfinite(x).all()) and bool((x[1] == 0).all())
    if layer:
        assert bool((x[4] == 0).all())
    moe.moe_norm_before(v, None, 1.0, gamma, None, norm, 0.0, None, x0)
    assert bool(torch.isnan(x0[1]).all())
    rest = [0, 2, 3, 5]
    assert bool(torch.isfinite(x0[rest]).all())
    gx, ws = ro.dev((T, H), torch.float32, 3), torch.empty(moe.moe_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    gr, gg = torch.empty_like(v), torch.empty(H, device="cuda")
    moe.moe_norm_before_backward(v, gamma, gx, None, 1.0, norm, EPS, gr, None, gg, None, ws)
    ref, size = ro.Norm(v, layer, EPS).backward(gx.double() * gamma.double())
    ro.close(gr[[0, 1, 2, 3, 5]], ref[[0, 1, 2, 3, 5]], ro.CHAIN * ro.STEP32 * size[[0, 1, 2, 3, 5]], "grad_residual")
    assert bool(torch.isfinite(gr).all()) and bool(torch.isfinite(gg).all())


@pytest.mark.parametrize("H", [2000, 4097, 8192])
def test_a_broken_row_stays_alone(H):
    """Rows with a NaN, an infinity, or the type's largest values leave the other rows' bits as they are."""
    import paper_2502_19811_amd as moe
    T, dtype = 700, torch.bfloat16
    gamma = ro.dev((H,), dtype, 1)
    good, g = ro.dev((T, H), dtype, 2), ro.dev((T, H), dtype, 3)
    bad = good.clone()
    bad[3, 5], bad[600, H - 1], bad[77] = float("nan"), float("-inf"), torch.finfo(dtype).max
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[[3, 600, 77]] = False
    outs = []
    for v in (good, bad):
        x, gr, y = torch.empty_like(v), torch.empty_like(v), torch.empty_like(v)
        moe.moe_norm_before(v, g, 0.5, gamma, None, moe.MOE_NORM_RMS, EPS, None, x)
        moe.moe_norm_before_backward(v, gamma, g, None, 1.0, moe.MOE_NORM_RMS, EPS, gr, None, None, None, None)
        moe.moe_norm_after(g, v, gamma, None, None, moe.MOE_GATE_NONE, 1.0, moe.MOE_NORM_LAYER, EPS, y)
        outs.append((x, gr, y))
    for a, b in zip(*outs):
        assert torch.equal(a[rest], b[rest])
        assert bool(torch.isnan(b[3]).all()) and bool(torch.isnan(b[600]).any())


def test_no_tokens_give_zero_sums():
    import paper_2502_19811_amd as moe
    for H in (8, 4096, 16384):
        none, gamma = torch.empty((0, H), dtype=torch.bfloat16, device="cuda"), ro.dev((H,), torch.bfloat16, 1)
        ws = torch.full((moe.moe_norm_workspace_bytes(0, H),), 0xff, dtype=torch.uint8, device="cuda")
        a, b, c = (torch.full((H,), 7.0, device="cuda") for _ in range(3))
        moe.moe_norm_before_backward(none, gamma, none, None, 1.0, 0, EPS, none, None, a, b, ws)
        assert bool((a == 0).all()) and bool((b == 0).all())
        a.fill_(7.0), b.fill_(7.0)
        moe.moe_norm_after_backward(none, gamma, gamma, gamma, moe.MOE_GATE_CHANNEL, 1.0, none, 0, EPS, none, a, b, c, ws)
        assert bool((a == 0).all()) and bool((b == 0).all()) and bool((c == 0).all())
        moe.moe_norm_before(none, None, 1.0, gamma, None, 0, EPS, None, none)
        moe.moe_norm_after(none, none, gamma, None, None, 0, 1.0, 0, EPS, none)


def test_streams_beyond_4_gib():
    import paper_2502_19811_amd as moe
    T, H = 150000, 16384
    print(f"T {T} H {H}: {T * H * 2 / 2 ** 30:.1f} GiB", flush=True)
    v = torch.empty((T, H), dtype=torch.bfloat16, device="cuda").normal_()
    gamma = ro.dev((H,), torch.bfloat16, 1)
    x = torch.empty_like(v)
    moe.moe_norm_before(v, None, 1.0, gamma, None, moe.MOE_NORM_RMS, EPS, None, x)
    at = torch.tensor([0, 1, 65535, 131071, 131072, T - 2, T - 1], device="cuda")
    d = ro.Norm(v[at], False, EPS)
    ro.close(x[at], d.n * gamma.double(), ro.CHAIN * ro.STEP32 * d.size * gamma.double().abs(), "x")
    ws = torch.empty(moe.moe_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    gr, gg = torch.empty_like(v), torch.empty(H, device="cuda")
    moe.moe_norm_before_backward(v, gamma, x, None, 1.0, moe.MOE_NORM_RMS, EPS, gr, None, gg, None, ws)
    ref, size = d.backward(x[at].double() * gamma.double())
    ro.close(gr[at], ref, ro.CHAIN * ro.STEP32 * size, "grad_residual")
    cols = [0, 1, 8191, H - 1]
    total, absolute = torch.zeros(4, dtype=torch.float64, device="cuda"), torch.zeros(4, dtype=torch.float64, device="cuda")
    for p in torch.arange(T, device="cuda").split(10000):
        n = ro.Norm(v[p], False, EPS).n[:, cols]
        total += (x[p][:, cols].double() * n).sum(dim=0)
        absolute += (x[p][:, cols].double() * n).abs().sum(dim=0)
    ro.close(gg[cols], total, ro.STEP32 * (ro.CHAIN + T / 256 + 96) * absolute, "grad_gamma")
