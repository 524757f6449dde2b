"""Definitions of the operators around the experts in 64 bits, with the error that each result may have, and helpers of their tests.

A result may be off by half a step of its type for its one rounding, and by what fp32 arithmetic adds: STEP32 times the number of
roundings in a row times the sum of the absolute values that went into it."""
import numpy as np
import torch

STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}      # half a step, relative
SUBNORMAL = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}   # half a step of the smallest values
STEP32 = 2.0 ** -24
# fp32 roundings in a row behind a sum over a row: at most 32 elements of a lane, 6 steps over lanes, 16 wavefronts, and the ten or so
# operations before and after; twice that for a sum of squares of differences from a mean that is such a sum
CHAIN = 128
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


def dev(shape, dtype, seed, scale=1.0, mean=0.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + mean).to(dtype).cuda()


def guarded(shape, dtype, fill):
    """A tensor inside a larger buffer that holds `fill` all around it; returns (tensor, check)."""
    n, pad = int(np.prod(shape)), 256
    buf = torch.full((n + 2 * pad,), fill, dtype=dtype, device="cuda")
    view = buf[pad:pad + n].view(shape)

    def check():
        assert bool((buf[:pad] == fill).all()) and bool((buf[pad + n:] == fill).all()), "something was written beside the output"
    return view, check


def close(got, ref, extra, what):
    """got: tensor of its type; ref, extra: fp64."""
    dt = got.dtype
    err = (got.double() - ref).abs()
    tol = STEP[dt] * (ref.abs() + extra) + extra + SUBNORMAL[dt]
    bad = ~(err <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, by {float((err / tol)[bad].max()):.2f} of what they may be"


def sort(ids, E):
    """(offsets, perm, inv_perm) on the CPU, int32."""
    flat = ids.cpu().reshape(-1).numpy().astype(np.int64)
    kept = (flat >= 0) & (flat < E)
    order = np.argsort(np.where(kept, flat, E), kind="stable")
    n = int(kept.sum())
    perm = np.where(np.arange(flat.size) < n, order, -1).astype(np.int32)
    inv = np.full(flat.size, -1, dtype=np.int32)
    inv[order[:n]] = np.arange(n)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[kept], minlength=E))]).astype(np.int32)
    return offsets, perm, inv.reshape(tuple(ids.shape))


def slots(T, E, k, seed, dropped=0.0):
    """Distinct experts of each token, a share of the slots without one (some tokens lose all of them)."""
    g = torch.Generator()
    g.manual_seed(seed)
    ids = torch.argsort(torch.rand((T, E), generator=g), dim=1)[:, :k].to(torch.int32)
    if dropped > 0:
        out = torch.rand((T, k), generator=g) < dropped
        out[torch.rand(T, generator=g) < dropped / 2] = True
        ids = torch.where(out, torch.where(torch.rand((T, k), generator=g) < 0.5, -1, E), ids).to(torch.int32)
    return ids.contiguous()


def combine(rows, inv, w):
    """(result, sum of absolute values)."""
    kept = inv >= 0
    v = torch.where(kept[:, :, None], rows[inv.clamp(min=0).long()].double(), 0.0)
    if w is not None:
        v = v * w.double()[:, :, None]
    return v.sum(dim=1), v.abs().sum(dim=1)


class Norm:
    """norm(v) of rows in 64 bits, what it may be off by in fp32 (in units of STEP32 * CHAIN), and its gradient."""

    def __init__(self, v, layer, eps):
        v = v.double()
        mean = v.mean(dim=1, keepdim=True) if layer else torch.zeros_like(v[:, :1])
        self.layer = layer
        self.r = ((v - mean).square().mean(dim=1, keepdim=True) + eps).rsqrt()
        self.n = (v - mean) * self.r
        # each element carries the rounding of v and of the mean
        self.size = self.r * (v.abs() + (v.abs().mean(dim=1, keepdim=True) if layer else 0.0))

    def backward(self, e):
        """(gradient of v for the gradient e of n, sum of the absolute values that go into it)."""
        mean_e = e.mean(dim=1, keepdim=True) if self.layer else 0.0
        g = self.r * (e - mean_e - self.n * (e * self.n).mean(dim=1, keepdim=True))
        abs_e = e.abs().mean(dim=1, keepdim=True) if self.layer else 0.0
        size = self.r * (e.abs() + abs_e + 3 * self.size * (e.abs() * self.size).mean(dim=1, keepdim=True))
        if self.layer:   # the deviation's error is that of the differences, relative to the deviation
            size = size * self.size.square().mean(dim=1, keepdim=True).clamp(min=1.0)
        return g, size
