"""Sums over rows of small whole numbers: fp32 holds every one of them, in whatever order they are added, so results are compared for being
equal, and an element that is left out or counted twice shows wherever it is."""
import pytest
import torch

import row_ops as ro

pytestmark = pytest.mark.gpu

# rows that end inside a piece, inside a wavefront's pieces, that their wavefronts take in one turn and in several, and even ones
WIDTHS = [8, 9, 63, 64, 65, 255, 257, 300, 513, 1001, 2049, 2339, 4096, 4097, 4099, 8191, 8200, 16385, 30001, 65529, 65536]


def _whole(shape, dtype, seed, most=3):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g).to(dtype).cuda()


@pytest.mark.parametrize("dtype", ro.DTYPES, ids=str)
@pytest.mark.parametrize("H", WIDTHS)
def test_combine_and_its_gradient(H, dtype):
    """Products are at most 9, sums of 65536 of them below 2^24; a token's sum over 10 slots is below 256, which 8 bits hold."""
    import paper_2502_19811_amd as moe
    for T, k in ((1, 1), (7, 2), (5, 3), (4, 8), (3, 10), (2, 17)):
        print(f"T {T} H {H} k {k} {dtype}", flush=True)
        R = T * k
        rows, g = _whole((R, H), dtype, 1), _whole((T, H), dtype, 2)
        inv = torch.randperm(R, generator=torch.Generator().manual_seed(3)).to(torch.int32).reshape(T, k).cuda()
        inv[T - 1, k - 1] = -1                                       # a slot without a row
        w = _whole((T, k), torch.float32, 4, 2)
        kept, at = (inv >= 0).cpu(), inv.clamp(min=0).long().cpu()
        r64, g64, w64 = rows.cpu().double(), g.cpu().double(), w.cpu().double()
        picked = torch.where(kept[:, :, None], r64[at], 0.0)         # [T, k, H]

        out, grad_x = torch.full((T, H), 77, dtype=dtype, device="cuda"), torch.full((T, H), 77, dtype=dtype, device="cuda")
        moe.moe_combine(rows, inv, w, out)
        moe.moe_dispatch_backward(rows, inv, grad_x)
        assert torch.equal(out.cpu().double(), (w64[:, :, None] * picked).sum(dim=1))
        assert torch.equal(grad_x.cpu().double(), picked.sum(dim=1))

        for weights in (w, None):
            grad_rows, grad_w = torch.full((R, H), 77, dtype=dtype, device="cuda"), torch.full((T, k), 77.0, device="cuda")
            moe.moe_combine_backward(g, rows, inv, weights, grad_rows, grad_w)
            assert torch.equal(grad_w.cpu().double(), (g64[:, None, :] * picked).sum(dim=2))
            want = torch.full((R, H), 77, dtype=torch.float64)
            factor = w64 if weights is not None else torch.ones_like(w64)
            want[at[kept]] = (factor[:, :, None] * g64[:, None, :])[kept]
            assert torch.equal(grad_rows.cpu().double(), want)


@pytest.mark.parametrize("dtype", ro.DTYPES, ids=str)
@pytest.mark.parametrize("H", [h for h in WIDTHS if h <= 16384])
def test_sums_over_tokens(H, dtype):
    """The gradients of a bias: sums over 33 and more rows, of whole numbers; the gate 2 and the scale 0.5 cancel."""
    import paper_2502_19811_amd as moe
    for T in (1, 4, 33, 700):
        print(f"T {T} H {H} {dtype}", flush=True)
        v, g, gamma = ro.dev((T, H), dtype, 1), _whole((T, H), dtype, 2), ro.dev((H,), dtype, 3)
        gate, ws = torch.full((T,), 2.0, device="cuda"), torch.empty(moe.moe_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
        want, rows = g.double().sum(dim=0), torch.empty_like(v)
        for norm in (moe.MOE_NORM_RMS, moe.MOE_NORM_LAYER):
            sums = [torch.full((H,), 77.0, device="cuda") for _ in range(2)]
            moe.moe_norm_before_backward(v, gamma, g, None, 1.0, norm, 1e-5, rows, None, None, sums[0], ws)
            moe.moe_norm_after_backward(v, gamma, None, gate, moe.MOE_GATE_TOKEN, 0.5, g, norm, 1e-5, rows, None, sums[1], None, ws)
            assert torch.equal(sums[0].double(), want) and torch.equal(sums[1].double(), want)
