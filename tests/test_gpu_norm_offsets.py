"""Layer norms of rows whose mean is large against their deviation, down to rows of one value, and their gradients, against definitions in
64 bits.

Bounds, with u = 2^-24 and C = CHAIN roundings in a row behind a sum: the first mean is off by D <= C u mean|v|; with x = v - mean the
differences d from it are right to u |d|, |d| <= |x| + D, and so is what is taken off them to C u (mean|x| + D); the sum of squares is
right to 3 C u (x^2 + D^2) an element, which moves r by (1 + q) 3/2 C u of itself, q = (D r)^2.  No term has the size of the mean but in D,
which is squared or multiplied by u again."""
import pytest
import torch

import row_ops as ro

pytestmark = pytest.mark.gpu

U, C = ro.STEP32, ro.CHAIN
WIDTHS = [33, 1000, 3584, 4097, 16384]        # one wavefront; three of one piece; even; ragged; eight or sixteen of two and four


class Layer:
    """n of the rows in 64 bits and what it may be off by, in units of C u; the same of gradients."""

    def __init__(self, v, eps):
        v = v.double()
        self.x = v - v.mean(dim=1, keepdim=True)
        self.r = (self.x.square().mean(dim=1, keepdim=True) + eps).rsqrt()
        self.n = self.x * self.r
        D = C * U * v.abs().mean(dim=1, keepdim=True)
        self.Dr, self.q = D * self.r, (D * self.r).square()
        self.mean_n = self.n.abs().mean(dim=1, keepdim=True)
        self.size = self.n.abs() + self.mean_n + 2 * self.Dr + 2 * self.n.abs() * (1 + self.q)

    def sums(self, e):
        """(mean of e n, what it may be off by)."""
        en = (e * self.n).mean(dim=1, keepdim=True)
        size = (e.abs() * (self.n.abs() + self.Dr)).mean(dim=1, keepdim=True) + e.abs().mean(dim=1, keepdim=True) * (self.mean_n + self.Dr)
        return en, 4 * (1 + self.q) * size

    def backward(self, e):
        en, en_size = self.sums(e)
        me = e.mean(dim=1, keepdim=True)
        g = self.r * (e - me - self.n * en)
        parts = e.abs() + me.abs() + (self.n * en).abs()
        return g, self.r * (e.abs() + e.abs().mean(dim=1, keepdim=True) + self.size * en.abs() + self.n.abs() * en_size + 2 * (1 + self.q) * parts)


def _new(*shape, dtype):
    return torch.full(shape, 7.0, dtype=dtype, device="cuda")


def _all(v, g, gamma, beta, gate, eps):
    """(x, grad_v, grad_gamma, grad_beta) in front of the block; (out, grad_y, grad_gamma, grad_beta, grad_gate) behind it."""
    import paper_2502_19811_amd as moe
    T, H = v.shape
    ws = torch.empty(moe.moe_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    x, gv, out, gy = (_new(T, H, dtype=v.dtype) for _ in range(4))
    gg, gb, gg2, gb2 = (_new(H, dtype=torch.float32) for _ in range(4))
    ggate = _new(T, dtype=torch.float32)
    moe.moe_norm_before(v, None, 1.0, gamma, beta, moe.MOE_NORM_LAYER, eps, None, x)
    moe.moe_norm_before_backward(v, gamma, g, None, 1.0, moe.MOE_NORM_LAYER, eps, gv, None, gg, gb, ws)
    moe.moe_norm_after(None, v, gamma, beta, gate, moe.MOE_GATE_TOKEN, 1.0, moe.MOE_NORM_LAYER, eps, out)
    moe.moe_norm_after_backward(v, gamma, beta, gate, moe.MOE_GATE_TOKEN, 1.0, g, moe.MOE_NORM_LAYER, eps, gy, gg2, gb2, ggate, ws)
    return (x, gv, gg, gb), (out, gy, gg2, gb2, ggate)


def _check(v, g, gamma, beta, gate, eps):
    T = v.shape[0]
    (x, gv, gg, gb), (out, gy, gg2, gb2, ggate) = _all(v, g, gamma, beta, gate, eps)
    ref, G, ga, be, w = Layer(v, eps), g.double(), gamma.double(), beta.double(), gate.double()[:, None]
    y, size = ref.n * ga + be, U * (C * ref.size * ga.abs() + 4 * ((ref.n * ga).abs() + be.abs()))
    ro.close(x, y, size, "x")
    ro.close(out, w * y, w.abs() * (size + 2 * U * y.abs()), "out")
    dv, dv_size = ref.backward(G * ga)
    ro.close(gv, dv, C * U * dv_size, "grad before")
    ro.close(gy, w * dv, w.abs() * C * U * dv_size, "grad behind")
    for got, f, what in ((gg, G, "before"), (gg2, G * w, "behind")):
        ro.close(got, (f * ref.n).sum(dim=0), U * (f.abs() * (C * ref.size + (T + 8) * ref.n.abs())).sum(dim=0), f"grad gamma {what}")
    for got, f, what in ((gb, G, "before"), (gb2, G * w, "behind")):
        ro.close(got, f.sum(dim=0), U * (T + 8) * f.abs().sum(dim=0), f"grad beta {what}")
    ro.close(ggate, (G * y).sum(dim=1), U * C * (G.abs() * (ref.size * ga.abs() + 2 * (ref.n * ga).abs() + 2 * be.abs())).sum(dim=1), "grad gate")
    return (x, gv, gg, gb), (out, gy, gg2, gb2, ggate)


@pytest.mark.parametrize("dtype,offset", [(torch.float32, 1e3), (torch.float32, -1e5), (torch.float16, 100.0), (torch.bfloat16, -30.0)], ids=str)
@pytest.mark.parametrize("H", WIDTHS)
def test_rows_far_from_zero(H, dtype, offset):
    for T in (1, 37):
        print(f"T {T} H {H} {dtype} offset {offset}", flush=True)
        _check(ro.dev((T, H), dtype, 1, 1.0, offset), ro.dev((T, H), dtype, 2), ro.dev((H,), dtype, 3, 0.2, 1.0), ro.dev((H,), dtype, 4, 0.3),
               ro.dev((T,), torch.float32, 5, 0.5, 1.0), 1e-5)


@pytest.mark.parametrize("dtype", ro.DTYPES, ids=str)
@pytest.mark.parametrize("H", WIDTHS)
def test_rows_of_one_whole_number(H, dtype):
    """Their sums are exact, so is the mean, and n is 0 whatever r is: x = beta, no gradient of gamma, r (e - mean(e)) for the row's."""
    values = [1.0, 3.0, 100.0, 300.0 if dtype is not torch.bfloat16 else 304.0, -7.0, 0.0] * 2
    v = torch.tensor(values, device="cuda")[:, None].expand(-1, H).to(dtype).contiguous()
    T = v.shape[0]
    g, gamma, beta = ro.dev((T, H), dtype, 2), ro.dev((H,), dtype, 3, 0.2, 1.0), ro.dev((H,), dtype, 4, 0.3)
    gate = torch.full((T,), 2.0, device="cuda")
    for eps in (1e-5, 1e-12):
        print(f"H {H} {dtype} eps {eps}", flush=True)
        held = dtype is not torch.float16 or eps > 1e-8    # r (e - mean(e)) lies beyond 65504 otherwise
        (x, gv, gg, gb), (out, gy, gg2, gb2, ggate) = _check(v, g, gamma, beta, gate, eps) if held else _all(v, g, gamma, beta, gate, eps)
        assert torch.equal(x, beta.expand(T, H)) and torch.equal(out, 2 * beta.expand(T, H))
        assert bool((gg == 0).all()) and bool((gg2 == 0).all())
        one = torch.full_like(g, 3.0)                       # e of one whole number: no gradient at all
        (_, gv, _, _), (_, gy, _, _, _) = _all(v, one, torch.full_like(gamma, 2.0), beta, gate, eps)
        assert bool((gv == 0).all()) and bool((gy == 0).all())


@pytest.mark.parametrize("H", WIDTHS)
def test_rows_of_one_value(H):
    """fp32 values whose sums are rounded: D is not 0, and what is left of it is squared or multiplied by u."""
    v = torch.tensor([0.1, 1.7, -100.1, 1 / 3, 1e-3], device="cuda")[:, None].expand(-1, H).contiguous()
    T = v.shape[0]
    f32 = torch.float32
    _check(v, ro.dev((T, H), f32, 2), ro.dev((H,), f32, 3, 0.2, 1.0), ro.dev((H,), f32, 4, 0.3), ro.dev((T,), f32, 5, 0.5, 1.0), 1e-5)
