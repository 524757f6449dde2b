"""The operators around the experts together: a block's forward and backward as a program runs them, against automatic
differentiation in 64 bits and against differences; captured in a graph; on another stream; what the binding refuses.

Streams share a few hardware queues in the order in which they come into use.  The tests of ready flags need one that
runs beside the default stream, so this file, which uses several, comes after theirs."""
import pytest
import torch

import row_ops as ro

pytestmark = pytest.mark.gpu

EPS, SCALE = 1e-5, 0.7


class Block:
    """h -> s = h + SCALE * u, x = norm(s), gate, experts (one matrix each), combine, out = s + SCALE * gate * norm(y)."""

    def __init__(self, T, H, E, k, dtype, seed, layer):
        import paper_2502_19811_amd as moe
        self.moe, self.T, self.H, self.E, self.k, self.dtype = moe, T, H, E, k, dtype
        self.norm = moe.MOE_NORM_LAYER if layer else moe.MOE_NORM_RMS
        self.layer = layer
        self.h, self.u = ro.dev((T, H), dtype, seed), ro.dev((T, H), dtype, seed + 1)
        self.router = ro.dev((H, E), torch.float32, seed + 2, H ** -0.5)
        self.experts = ro.dev((E, H, H), torch.float32, seed + 3, H ** -0.5)
        self.g1, self.g2 = ro.dev((H,), dtype, seed + 4, 0.2, 1.0), ro.dev((H,), dtype, seed + 5, 0.2, 1.0)
        self.b1, self.b2 = (ro.dev((H,), dtype, seed + 6, 0.1), ro.dev((H,), dtype, seed + 7, 0.1)) if layer else (None, None)
        self.gate = ro.dev((H,), dtype, seed + 8, 0.3, 0.5)
        self.grad_out = ro.dev((T, H), dtype, seed + 9)
        new = lambda *shape, dt=dtype: torch.zeros(shape, dtype=dt, device="cuda")  # noqa: E731
        f32, i32 = torch.float32, torch.int32
        R = T * k
        self.s, self.x, self.y, self.out = new(T, H), new(T, H), new(T, H), new(T, H)
        self.ids, self.w = new(T, k, dt=i32), new(T, k, dt=f32)
        self.offsets, self.perm, self.inv = new(E + 1, dt=i32), new(R, dt=i32), new(T, k, dt=i32)
        self.rows, self.expert_out = new(R, H), new(R, H)
        self.sort_ws = torch.zeros(moe.moe_sort_workspace_bytes(T, E, k), dtype=torch.uint8, device="cuda")
        self.norm_ws = torch.zeros(moe.moe_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
        self.gy, self.gx, self.gx_rows, self.gr, self.gu = (new(T, H) for _ in range(5))
        self.g_expert_out, self.g_rows = new(R, H), new(R, H)
        self.gw, self.glogits = new(T, k, dt=f32), new(T, E, dt=f32)
        self.gg1, self.gg2, self.gb1, self.gb2, self.ggate = (new(H, dt=f32) for _ in range(5))

    def products(self, rows, transposed):
        """The caller's experts, here one product in fp32 for each."""
        out = torch.zeros_like(rows)
        bounds = self.offsets.tolist()
        for e in range(self.E):
            a, b = bounds[e], bounds[e + 1]
            W = self.experts[e].T.contiguous() if transposed else self.experts[e]
            out[a:b] = (rows[a:b].float() @ W).to(self.dtype)
        return out

    def forward(self):
        m = self.moe
        m.moe_norm_before(self.h, self.u, SCALE, self.g1, self.b1, self.norm, EPS, self.s, self.x)
        logits = self.x.float() @ self.router
        m.moe_route_topk(logits, self.k, self.ids, self.w)
        m.moe_sort_tokens(self.ids, self.E, self.offsets, self.perm, self.inv, self.sort_ws)
        m.moe_dispatch(self.x, self.inv, self.rows)
        self.expert_out = self.products(self.rows, False)
        m.moe_combine(self.expert_out, self.inv, self.w, self.y)
        m.moe_norm_after(self.s, self.y, self.g2, self.b2, self.gate, m.MOE_GATE_CHANNEL, SCALE, self.norm, EPS, self.out)

    def backward(self):
        m = self.moe
        beta = self.b2 is not None
        m.moe_norm_after_backward(self.y, self.g2, self.b2, self.gate, m.MOE_GATE_CHANNEL, SCALE, self.grad_out, self.norm, EPS, self.gy,
                                  self.gg2, self.gb2 if beta else None, self.ggate, self.norm_ws)
        m.moe_combine_backward(self.gy, self.expert_out, self.inv, self.w, self.g_expert_out, self.gw)
        m.moe_route_topk_backward(self.ids, self.w, self.gw, self.glogits)
        self.g_rows = self.products(self.g_expert_out, True)
        m.moe_dispatch_backward(self.g_rows, self.inv, self.gx_rows)
        self.gx.copy_((self.gx_rows.float() + self.glogits @ self.router.T.contiguous()).to(self.dtype))
        m.moe_norm_before_backward(self.s, self.g1, self.gx, self.grad_out, SCALE, self.norm, EPS, self.gr, self.gu, self.gg1,
                                   self.gb1 if beta else None, self.norm_ws)

    def definition(self, params):
        """The block in 64 bits on the CPU for the experts that were picked."""
        h, u, g1, b1, g2, b2, gate = params
        scale = torch.tensor(SCALE, dtype=torch.float32).double().item()

        def norm(v, gamma, beta):
            if self.layer:
                v = v - v.mean(dim=1, keepdim=True)
            n = v * (v.square().mean(dim=1, keepdim=True) + EPS).rsqrt() * gamma
            return n if beta is None else n + beta
        s = h + scale * u
        x = norm(s, g1, b1)
        ids = self.ids.cpu().long()
        w = torch.softmax(torch.gather(x @ self.router.cpu().double(), 1, ids), dim=1)
        y = torch.zeros_like(x)
        W = self.experts.cpu().double()
        for e in range(self.E):
            part = ((ids == e) * w).sum(dim=1, keepdim=True)
            y = y + part * (x @ W[e])
        return s + scale * gate * norm(y, g2, b2)

    def params(self):
        return [None if p is None else p.cpu().double().requires_grad_() for p in (self.h, self.u, self.g1, self.b1, self.g2, self.b2, self.gate)]

    def gradients(self):
        return [self.gr, self.gu, self.gg1, self.gb1, self.gg2, self.gb2, self.ggate]


@pytest.mark.parametrize("layer", [False, True], ids=["rms", "layer"])
def test_block_forward_and_backward(layer):
    """fp32 rows: every operator is off by at most a hundred or so fp32 steps (6e-6), the products of 96 terms by less, and a chain of
    ten of them, none of which magnifies by more than a few times, by 2e-4 in the 2-norm."""
    b = Block(150, 96, 8, 2, torch.float32, 50, layer)
    b.forward()
    b.backward()
    params = b.params()
    out = b.definition(params)
    norm = lambda v: float(v.norm())  # noqa: E731
    assert norm(b.out.cpu().double() - out.detach()) <= 2e-4 * norm(out.detach())
    loss = (out * b.grad_out.cpu().double()).sum()
    grads = torch.autograd.grad(loss, [p for p in params if p is not None])
    got = [g.cpu().double() for p, g in zip(params, b.gradients()) if p is not None]
    for i, (a, r) in enumerate(zip(got, grads)):
        assert norm(a - r) <= 2e-4 * norm(r), i
    # and against differences of the definition, in a direction for each
    with torch.no_grad():
        for i, p in enumerate(params):
            if p is None:
                continue
            d = torch.randn(p.shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64)
            values = []
            for sign in (1e-6, -1e-6):
                moved = [q if j != i else p + sign * d for j, q in enumerate(params)]
                values.append(float((b.definition(moved) * b.grad_out.cpu().double()).sum()))
            diff, g = (values[0] - values[1]) / 2e-6, b.gradients()[i].cpu().double()
            assert abs(diff - float((g * d).sum())) <= 3e-4 * norm(g) * norm(d)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_the_same_call_gives_the_same_bits(dtype):
    runs = []
    for _ in range(3):
        b = Block(700, 264, 16, 4, dtype, 60, False)
        b.forward()
        b.backward()
        runs.append([v.clone() for v in (b.out, b.gr, b.gu, b.gg1, b.gg2, b.ggate, b.gw, b.glogits, b.perm)])
    for r in runs[1:]:
        for a, c in zip(r, runs[0]):
            assert torch.equal(a, c)


@pytest.mark.parametrize("H", [264, 1001, 3584, 4097])
def test_a_row_does_not_depend_on_the_batch_around_it(H):
    """The first rows of a batch against a batch of them alone: every result that belongs to a row."""
    import paper_2502_19811_amd as moe
    bf, T, k = torch.bfloat16, 5000, 2
    norm, kind = moe.MOE_NORM_LAYER, moe.MOE_GATE_TOKEN
    h, u, g, y = (ro.dev((T, H), bf, 100 + i) for i in range(4))
    gamma, beta, gate = ro.dev((H,), bf, 104), ro.dev((H,), bf, 105), ro.dev((T,), torch.float32, 106)
    inv = torch.arange(T * k, dtype=torch.int32, device="cuda").reshape(T, k)
    rows, w = ro.dev((T * k, H), bf, 107), ro.dev((T, k), torch.float32, 108)
    results = []
    for n in (T, 3, 33):
        H1, U, G, Y, GATE, INV, ROWS, W = h[:n], u[:n], g[:n], y[:n], gate[:n].contiguous(), inv[:n], rows[:n * k], w[:n].contiguous()
        new = lambda: torch.empty((n, H), dtype=bf, device="cuda")  # noqa: E731
        s, x, out, gr, gu, gy, c = (new() for _ in range(7))
        grad_rows, grad_w, grad_gate = torch.empty_like(ROWS), torch.empty_like(W), torch.empty_like(GATE)
        sums, ws = torch.empty(H, device="cuda"), torch.empty(moe.moe_norm_workspace_bytes(n, H), dtype=torch.uint8, device="cuda")
        moe.moe_norm_before(H1, U, SCALE, gamma, beta, norm, EPS, s, x)
        moe.moe_norm_before_backward(H1, gamma, G, U, SCALE, norm, EPS, gr, gu, sums, None, ws)
        moe.moe_norm_after(H1, Y, gamma, beta, GATE, kind, SCALE, norm, EPS, out)
        moe.moe_norm_after_backward(Y, gamma, beta, GATE, kind, SCALE, G, norm, EPS, gy, sums, None, grad_gate, ws)
        moe.moe_combine(ROWS, INV, W, c)
        moe.moe_combine_backward(G, ROWS, INV, W, grad_rows, grad_w)
        results.append((s, x, gr, gu, out, gy, grad_gate, c, grad_rows, grad_w))
    for few in results[1:]:
        for a, b in zip(few, results[0]):
            assert torch.equal(a, b[:a.shape[0]])


def _without_products(b):
    """The operators alone, for a graph and another stream: the experts' results are what they were."""
    m = b.moe
    m.moe_norm_before(b.h, b.u, SCALE, b.g1, b.b1, b.norm, EPS, b.s, b.x)
    m.moe_sort_tokens(b.ids, b.E, b.offsets, b.perm, b.inv, b.sort_ws)
    m.moe_dispatch(b.x, b.inv, b.rows)
    m.moe_combine(b.rows, b.inv, b.w, b.y)
    m.moe_norm_after(b.s, b.y, b.g2, b.b2, b.gate, m.MOE_GATE_CHANNEL, SCALE, b.norm, EPS, b.out)
    m.moe_norm_after_backward(b.y, b.g2, b.b2, b.gate, m.MOE_GATE_CHANNEL, SCALE, b.grad_out, b.norm, EPS, b.gy, b.gg2, None, b.ggate, b.norm_ws)
    m.moe_combine_backward(b.gy, b.rows, b.inv, b.w, b.g_expert_out, b.gw)
    m.moe_route_topk_backward(b.ids, b.w, b.gw, b.glogits)
    m.moe_dispatch_backward(b.g_expert_out, b.inv, b.gx)
    m.moe_norm_before_backward(b.s, b.g1, b.gx, b.grad_out, SCALE, b.norm, EPS, b.gr, b.gu, b.gg1, None, b.norm_ws)


def _results(b):
    return (b.s, b.x, b.offsets, b.perm, b.inv, b.rows, b.y, b.out, b.gy, b.gg2, b.ggate, b.g_expert_out, b.gw, b.glogits, b.gx, b.gr, b.gu, b.gg1)


@pytest.mark.parametrize("T", [100, 3000])
def test_captured_in_a_graph(T):
    b = Block(T, 520, 16, 4, torch.bfloat16, 70, False)
    b.forward()                                # picks experts
    _without_products(b)
    torch.cuda.synchronize()
    eager = [v.clone() for v in _results(b)]
    print(f"capturing T {T}", flush=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _without_products(b)
    ids = b.ids.clone()
    for rep in range(4):
        for v in _results(b):
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(_results(b), eager):
            assert torch.equal(a, c)
        if rep == 1:                           # the program's own work in between: another routing, eagerly, then the first one again
            b.ids.copy_(ids.flip(0))
            _without_products(b)
            torch.cuda.synchronize()
            assert not torch.equal(b.perm, eager[3])
            b.ids.copy_(ids)
        print(f"  replay {rep} ok", flush=True)


def test_two_graphs_with_the_same_workspaces():
    """Scratch holds nothing between calls: graphs that share it may be replayed in any order, one after the other."""
    a, b = Block(1500, 264, 16, 4, torch.bfloat16, 71, False), Block(900, 264, 16, 4, torch.bfloat16, 72, True)
    b.sort_ws, b.norm_ws = a.sort_ws, a.norm_ws            # those of the larger batch
    graphs, eager = [], []
    for blk in (a, b):
        blk.forward()
        _without_products(blk)
        torch.cuda.synchronize()
        eager.append([v.clone() for v in _results(blk)])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _without_products(blk)
        graphs.append(g)
    for i in (0, 1, 1, 0, 1):
        blk = (a, b)[i]
        for v in _results(blk):
            v.zero_()
        a.sort_ws.fill_(0xff)
        a.norm_ws.fill_(0xff)
        graphs[i].replay()
        torch.cuda.synchronize()
        for x, y in zip(_results(blk), eager[i]):
            assert torch.equal(x, y)


def test_on_another_stream():
    b = Block(900, 264, 8, 2, torch.bfloat16, 80, True)
    b.forward()
    _without_products(b)
    torch.cuda.synchronize()
    eager = [v.clone() for v in _results(b)]
    for v in _results(b):
        v.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):              # the current stream
        _without_products(b)
    side.synchronize()
    for a, c in zip(_results(b), eager):
        assert torch.equal(a, c)
    b.x.zero_()
    b.moe.moe_norm_before(b.h, b.u, SCALE, b.g1, b.b1, b.norm, EPS, b.s, b.x, stream=side)     # a stream by name
    side.synchronize()
    assert torch.equal(b.x, eager[1])


def test_two_streams_at_once():
    """Calls that overlap in time, each with workspaces of its own."""
    blocks = [Block(2500, 520, 16, 4, torch.bfloat16, 90 + i, False) for i in range(2)]
    eager = []
    for b in blocks:
        b.forward()
        _without_products(b)
        torch.cuda.synchronize()
        eager.append([v.clone() for v in _results(b)])
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(5):
        for b, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                _without_products(b)
    torch.cuda.synchronize()
    for b, e in zip(blocks, eager):
        for a, c in zip(_results(b), e):
            assert torch.equal(a, c)


def test_the_binding_refuses():
    """Wrong types, shapes, strides and devices, before any launch."""
    import paper_2502_19811_amd as moe
    T, H, E, k = 20, 64, 4, 2
    bf = torch.bfloat16
    x, rows, inv = ro.dev((T, H), bf, 1), ro.dev((T * k, H), bf, 2), torch.zeros((T, k), dtype=torch.int32, device="cuda")
    w, gamma = torch.ones((T, k), device="cuda"), ro.dev((H,), bf, 3)
    ids, offsets, perm = inv.clone(), torch.zeros(E + 1, dtype=torch.int32, device="cuda"), torch.zeros(T * k, dtype=torch.int32, device="cuda")
    ws = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    wide = torch.zeros((T, 2 * H), dtype=bf, device="cuda")[:, :H]
    out = torch.empty_like(x)
    bad = [
        lambda: moe.moe_dispatch(x.cpu(), inv, rows),
        lambda: moe.moe_dispatch(x, inv.cpu(), rows),
        lambda: moe.moe_dispatch(x, inv.long(), rows),
        lambda: moe.moe_dispatch(x.half(), inv, rows),
        lambda: moe.moe_dispatch(x.double(), inv, rows),
        lambda: moe.moe_dispatch(wide, inv, rows),
        lambda: moe.moe_dispatch(x, inv, rows[:-1]),
        lambda: moe.moe_dispatch(x, inv[:-1], rows),
        lambda: moe.moe_dispatch(x[0], inv, rows),
        lambda: moe.moe_dispatch(x, inv.reshape(-1), rows),
        lambda: moe.moe_dispatch(x, inv.t().contiguous().t(), rows),
        lambda: moe.moe_combine(rows, inv, w.to(bf), out),
        lambda: moe.moe_combine(rows, inv, w[:, :1], out),
        lambda: moe.moe_combine(rows, inv, w, out.t()),
        lambda: moe.moe_combine_backward(x, None, inv, w, rows, torch.empty_like(w)),
        lambda: moe.moe_combine_backward(x, rows, inv, w, torch.empty_like(rows), torch.empty_like(w).to(bf)),
        lambda: moe.moe_sort_tokens(ids, E, offsets[:-1], perm, inv, ws),
        lambda: moe.moe_sort_tokens(ids, E, offsets, perm[:-1], inv, ws),
        lambda: moe.moe_sort_tokens(ids, E, offsets, perm, inv, ws.to(torch.int32)),
        lambda: moe.moe_sort_tokens(ids, E, offsets, perm, inv, ws[:16]),
        lambda: moe.moe_route_topk_backward(ids, w, w.to(bf), torch.zeros((T, E), device="cuda")),
        lambda: moe.moe_route_topk_backward(ids, w, w, torch.zeros((T - 1, E), device="cuda")),
        lambda: moe.moe_norm_before(x, None, 1.0, gamma.float(), None, 0, EPS, None, out),
        lambda: moe.moe_norm_before(x, None, 1.0, gamma[:-1], None, 0, EPS, None, out),
        lambda: moe.moe_norm_before(x, None, float("nan"), gamma, None, 0, EPS, None, out),
        lambda: moe.moe_norm_before(x, wide, 1.0, gamma, None, 0, EPS, None, out),
        lambda: moe.moe_norm_before(x, None, 1.0, gamma, None, 2, EPS, None, out),
        lambda: moe.moe_norm_before_backward(x, gamma, x, None, 1.0, 0, EPS, out, None, torch.zeros(H, dtype=bf, device="cuda"), None, ws),
        lambda: moe.moe_norm_before_backward(x, gamma, x, None, 1.0, 0, EPS, out, None, torch.zeros(H, device="cuda"), None, None),
        lambda: moe.moe_norm_after(None, x, gamma, None, gamma, moe.MOE_GATE_NONE, 1.0, 0, EPS, out),
        lambda: moe.moe_norm_after(None, x, gamma, None, None, moe.MOE_GATE_TOKEN, 1.0, 0, EPS, out),
        lambda: moe.moe_norm_after(None, x, gamma, None, gamma, moe.MOE_GATE_TOKEN, 1.0, 0, EPS, out),
        lambda: moe.moe_norm_after(None, x, gamma, None, w[:, 0], moe.MOE_GATE_TOKEN, 1.0, 0, EPS, out),
        lambda: moe.moe_norm_after(None, x, gamma, None, gamma, 4, 1.0, 0, EPS, out),
        lambda: moe.moe_norm_after_backward(x, gamma, None, gamma, moe.MOE_GATE_CHANNEL, 1.0, x, 0, EPS, out, None, None, gamma.clone(), ws),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(moe.MoEError):
            call()
            pytest.fail(f"call {i} was not refused")
