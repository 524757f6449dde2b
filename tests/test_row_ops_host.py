"""What the operators around the experts refuse, at the C entry points and without a GPU: every refusal comes before any launch, so the
addresses here are arithmetic only."""
import ctypes as C

import pytest

import paper_2502_19811_amd as moe

INVALID, TOO_SMALL, UNSUPPORTED = -1, -3, -4
A = 1 << 40             # aligned addresses, far apart
B, D, E_, F, G = (A + i * (1 << 38) for i in range(1, 6))
BIG = 1 << 36           # bytes of workspace


def _args(**kw):
    return dict(kw)


CALLS = {
    "moe_sort_tokens": _args(ids=A, T=100, E=8, k=2, offsets=B, perm=D, inv=E_, ws=F, ws_bytes=BIG),
    "moe_dispatch": _args(x=A, inv=B, T=100, H=256, k=2, dtype=0, rows=D),
    "moe_dispatch_backward": _args(grad_rows=A, inv=B, T=100, H=256, k=2, dtype=0, grad_x=D),
    "moe_combine": _args(rows=A, inv=B, w=D, T=100, H=256, k=2, dtype=0, out=E_),
    "moe_combine_backward": _args(grad_out=A, rows=B, inv=D, w=E_, T=100, H=256, k=2, dtype=0, grad_rows=F, grad_weights=G),
    "moe_route_topk_backward": _args(ids=A, w=B, grad_weights=D, T=100, E=8, k=2, grad_logits=E_),
    "moe_norm_before": _args(residual=A, update=B, scale=1.0, gamma=D, beta=None, norm=0, eps=1e-5, T=100, H=256, dtype=0, sum=E_, x=F),
    "moe_norm_before_backward": _args(sum=A, gamma=B, grad_x=D, grad_sum=None, scale=1.0, norm=0, eps=1e-5, T=100, H=256, dtype=0,
                                      grad_residual=E_, grad_update=None, grad_gamma=F, grad_beta=None, ws=G, ws_bytes=BIG),
    "moe_norm_after": _args(residual=A, y=B, gamma=D, beta=None, gate=None, gate_kind=0, scale=1.0, norm=0, eps=1e-5, T=100, H=256,
                            dtype=0, out=E_),
    "moe_norm_after_backward": _args(y=A, gamma=B, beta=None, gate=None, gate_kind=0, scale=1.0, grad_out=D, norm=0, eps=1e-5, T=100,
                                     H=256, dtype=0, grad_y=E_, grad_gamma=F, grad_beta=None, grad_gate=None, ws=G, ws_bytes=BIG),
}
ROWS = ("moe_dispatch", "moe_dispatch_backward", "moe_combine", "moe_combine_backward")
NORMS = ("moe_norm_before", "moe_norm_before_backward", "moe_norm_after", "moe_norm_after_backward")

REFUSED = []
for name, base in CALLS.items():
    REFUSED.append((name, dict(T=-1), INVALID))
    for key, value in base.items():
        if value in (A, B, D, E_, F, G):
            REFUSED.append((name, {key: value + 2}, INVALID))                # misaligned
            if (name, key) not in {("moe_combine", "w"), ("moe_combine_backward", "w"), ("moe_combine_backward", "grad_weights"),
                                   ("moe_norm_before", "update"), ("moe_norm_before", "sum"), ("moe_norm_after", "residual"),
                                   ("moe_norm_before_backward", "grad_gamma"), ("moe_norm_after_backward", "grad_gamma")}:
                REFUSED.append((name, {key: None}, INVALID))                 # missing
for name in ROWS:
    REFUSED += [(name, dict(H=0), INVALID), (name, dict(k=0), INVALID), (name, dict(dtype=3), INVALID), (name, dict(dtype=-1), INVALID),
                (name, dict(H=7), UNSUPPORTED), (name, dict(H=65537), UNSUPPORTED), (name, dict(k=65), UNSUPPORTED),
                (name, dict(T=1 << 23, k=2), UNSUPPORTED), (name, dict(T=1 << 20, k=1, H=16384, dtype=0), UNSUPPORTED)]
for name in NORMS:
    REFUSED += [(name, dict(H=0), INVALID), (name, dict(dtype=3), INVALID), (name, dict(norm=2), INVALID), (name, dict(norm=-1), INVALID),
                (name, dict(eps=-1e-9), INVALID), (name, dict(eps=float("nan")), INVALID), (name, dict(eps=float("inf")), INVALID),
                (name, dict(scale=float("nan")), INVALID), (name, dict(scale=float("inf")), INVALID),
                (name, dict(H=7), UNSUPPORTED), (name, dict(H=16385), UNSUPPORTED), (name, dict(T=1 << 24), UNSUPPORTED),
                (name, dict(T=1 << 20, H=16384, dtype=0), UNSUPPORTED), (name, dict(T=1 << 20, H=8192, dtype=2), UNSUPPORTED)]
for name in ("moe_sort_tokens", "moe_route_topk_backward"):
    REFUSED += [(name, dict(E=0), INVALID), (name, dict(k=0), INVALID), (name, dict(E=257), UNSUPPORTED),
                (name, dict(T=1 << 23), UNSUPPORTED)]
REFUSED += [
    ("moe_sort_tokens", dict(k=65), UNSUPPORTED),
    ("moe_sort_tokens", dict(ws_bytes=moe.moe_sort_workspace_bytes(100, 8, 2) - 1), TOO_SMALL),
    ("moe_route_topk_backward", dict(k=9), INVALID),
    # buffers that lie across each other
    ("moe_dispatch", dict(rows=A), INVALID),
    ("moe_dispatch", dict(rows=A + 100 * 512 - 16), INVALID),
    ("moe_dispatch", dict(rows=A - 200 * 512 + 16), INVALID),
    ("moe_combine", dict(out=A + 16), INVALID),
    ("moe_combine_backward", dict(grad_rows=A), INVALID),
    ("moe_combine_backward", dict(grad_rows=B), INVALID),
    ("moe_combine_backward", dict(rows=None), INVALID),
    ("moe_norm_before", dict(x=A + 512), INVALID),
    ("moe_norm_before", dict(sum=B + 16), INVALID),
    ("moe_norm_before", dict(x=E_), INVALID),
    ("moe_norm_before_backward", dict(grad_residual=A + 16), INVALID),
    ("moe_norm_before_backward", dict(grad_update=E_), INVALID),
    ("moe_norm_before_backward", dict(ws_bytes=moe.moe_norm_workspace_bytes(100, 256) - 1), TOO_SMALL),
    ("moe_norm_after", dict(out=B + 16), INVALID),
    ("moe_norm_after", dict(gate=F, gate_kind=3, out=F + 16), INVALID),
    ("moe_norm_after_backward", dict(grad_y=D + 512), INVALID),
    ("moe_norm_after_backward", dict(gate=F + (1 << 37), gate_kind=3, grad_gate=E_), INVALID),
    ("moe_norm_after_backward", dict(ws_bytes=moe.moe_norm_workspace_bytes(100, 256) - 1), TOO_SMALL),
    ("moe_sort_tokens", dict(inv=A), INVALID),
    ("moe_sort_tokens", dict(perm=E_ + 400), INVALID),
    ("moe_sort_tokens", dict(ws=B), INVALID),
    ("moe_dispatch", dict(rows=B), INVALID),
    ("moe_combine", dict(out=D), INVALID),
    ("moe_combine_backward", dict(grad_weights=E_), INVALID),
    ("moe_combine_backward", dict(grad_weights=F + 512), INVALID),
    ("moe_route_topk_backward", dict(grad_logits=B), INVALID),
    ("moe_norm_before", dict(x=D), INVALID),
    ("moe_norm_before", dict(sum=D), INVALID),
    ("moe_norm_before_backward", dict(grad_gamma=B), INVALID),
    ("moe_norm_before_backward", dict(grad_gamma=D), INVALID),
    ("moe_norm_before_backward", dict(grad_beta=F), INVALID),
    ("moe_norm_before_backward", dict(ws=A), INVALID),
    ("moe_norm_after", dict(gate=F, gate_kind=1, out=F), INVALID),
    ("moe_norm_after", dict(out=D), INVALID),
    ("moe_norm_after_backward", dict(grad_gamma=E_ + 512), INVALID),
    ("moe_norm_after_backward", dict(gate=A + (1 << 37), gate_kind=2, grad_gate=A + (1 << 37)), INVALID),
    ("moe_norm_after_backward", dict(gate=A + (1 << 37), gate_kind=1, grad_gate=F), INVALID),
    # gates that do not fit their kind
    ("moe_norm_after", dict(gate_kind=4), INVALID),
    ("moe_norm_after", dict(gate_kind=-1), INVALID),
    ("moe_norm_after", dict(gate=F, gate_kind=0), INVALID),
    ("moe_norm_after", dict(gate_kind=1), INVALID),
    ("moe_norm_after", dict(gate_kind=2), INVALID),
    ("moe_norm_after", dict(gate=F + 4, gate_kind=2), INVALID),
    ("moe_norm_after_backward", dict(gate_kind=3), INVALID),
    ("moe_norm_after_backward", dict(gate_kind=0, grad_gate=A + (1 << 37)), INVALID),
    ("moe_norm_after_backward", dict(gate=A + (1 << 37), gate_kind=1, grad_gamma=None, grad_gate=A + (3 << 36), ws=None), INVALID),
]


@pytest.mark.parametrize("name,change,status", REFUSED, ids=[f"{n}-{'-'.join(c)}-{i}" for i, (n, c, _) in enumerate(REFUSED)])
def test_refused_before_any_launch(name, change, status):
    assert getattr(moe.load_library(), name)(*{**CALLS[name], **change}.values(), None) == status


def test_the_tables_follow_the_header():
    """Every call of the tables has as many arguments as its binding says (the last one is the stream)."""
    lib = moe.load_library()
    for name, base in CALLS.items():
        assert len(base) + 1 == len(getattr(lib, name).argtypes), name
        assert getattr(lib, name).restype is C.c_int


def test_nothing_to_do_is_no_error():
    """Without tokens, what writes nothing needs no pointers and launches nothing."""
    lib = moe.load_library()
    for name in ROWS + ("moe_route_topk_backward", "moe_norm_before", "moe_norm_after"):
        args = {key: (None if value in (A, B, D, E_, F, G) else value) for key, value in CALLS[name].items()}
        assert getattr(lib, name)(*{**args, "T": 0}.values(), None) == 0, name
    for name in ("moe_norm_before_backward", "moe_norm_after_backward"):
        args = {key: (None if value in (A, B, D, E_, F, G) and key != "gamma" else value) for key, value in CALLS[name].items()}
        assert getattr(lib, name)(*{**args, "T": 0}.values(), None) == 0, name


def test_workspace_sizes():
    assert moe.moe_sort_workspace_bytes(0, 8, 2) > 0
    assert moe.moe_sort_workspace_bytes(1 << 20, 8, 2) >= (1 << 11) * 9 * 4           # counts of 9 buckets for 2048 chunks
    for bad in ((-1, 8, 2), (1, 0, 2), (1, 257, 2), (1, 8, 0), (1, 8, 65), (1 << 23, 8, 2)):
        assert moe.moe_sort_workspace_bytes(*bad) == 0
    assert moe.moe_norm_workspace_bytes(0, 8) > 0
    sizes = [moe.moe_norm_workspace_bytes(T, 4096) for T in (1, 10, 100, 1000, 100000)]
    assert sizes == sorted(sizes) and sizes[0] == 2 * 4096 * 4
    assert sizes[-1] <= 2 * 2048 * 4096 * 4                                           # bounded, however many tokens
    for bad in ((-1, 256), (1, 0), (1, 7), (1, 16385), (1 << 24, 256)):
        assert moe.moe_norm_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("H", [8, 300, 1000, 2049, 3584, 4096, 4104, 8192, 16384])
def test_a_workspace_of_a_batch_does_for_smaller_ones(H):
    sizes = [moe.moe_norm_workspace_bytes(T, H) for T in [*range(1300), *range(1300, 9000, 37)]]
    assert sizes == sorted(sizes)
    sizes = [moe.moe_sort_workspace_bytes(T, 64, 4) for T in range(0, 9000, 37)]
    assert sizes == sorted(sizes)
