"""What the binding does before any launch, without a GPU: tensors without memory stand in for those on the device."""
import sys

import pytest
import torch

import paper_2502_19811_amd as moe
from paper_2502_19811_amd import binding

INVALID, UNSUPPORTED = -1, -4
HUGE = [1 << 31, 1 << 32, (1 << 32) + 8, 1 << 40]      # 32 bits make a negative number, none, 8, none out of them


@pytest.fixture
def no_device(monkeypatch):
    """Calls go through the binding with tensors that are on no device (their device is -1)."""
    binding._first_call()
    monkeypatch.setattr(binding, "_current_device", lambda: -1)
    monkeypatch.setattr(binding, "_raw_stream", lambda device: None)
    monkeypatch.setattr(binding, "_stream", lambda stream: None)


def _t(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


def _i(*shape):
    return _t(*shape, dtype=torch.int32)


def _f(*shape):
    return _t(*shape, dtype=torch.float32)


def _calls(T=0, H=64, E=8, k=2, norm=0, kind=0):
    """Every call with these sizes; without tokens nothing is launched and no pointer is needed but a gradient's gamma."""
    ws = _t(1 << 20, dtype=torch.uint8)
    rows, all_rows, pairs = _t(T, H), _t(T * k, H), (T, k)
    gate = None
    return {
        "moe_route_topk": lambda: moe.moe_route_topk(_f(T, E), k, _i(*pairs), _f(*pairs)),
        "moe_sort_tokens": lambda: moe.moe_sort_tokens(_i(*pairs), E, _i(E + 1), _i(T * k), _i(*pairs), ws),
        "moe_dispatch": lambda: moe.moe_dispatch(rows, _i(*pairs), all_rows),
        "moe_dispatch_backward": lambda: moe.moe_dispatch_backward(all_rows, _i(*pairs), rows),
        "moe_combine": lambda: moe.moe_combine(all_rows, _i(*pairs), _f(*pairs), rows),
        "moe_combine_backward": lambda: moe.moe_combine_backward(rows, all_rows, _i(*pairs), _f(*pairs), all_rows, _f(*pairs)),
        "moe_route_topk_backward": lambda: moe.moe_route_topk_backward(_i(*pairs), _f(*pairs), _f(*pairs), _f(T, E)),
        "moe_norm_before": lambda: moe.moe_norm_before(rows, None, 1.0, _t(H), None, norm, 1e-5, None, rows),
        "moe_norm_before_backward": lambda: moe.moe_norm_before_backward(rows, _t(H), rows, None, 1.0, norm, 1e-5, rows, None, None, None, None),
        "moe_norm_after": lambda: moe.moe_norm_after(None, rows, _t(H), None, gate, kind, 1.0, norm, 1e-5, rows),
        "moe_norm_after_backward": lambda: moe.moe_norm_after_backward(rows, _t(H), None, gate, kind, 1.0, rows, norm, 1e-5, rows, None, None,
                                                                       None, None),
    }


ROWS = ["moe_dispatch", "moe_dispatch_backward", "moe_combine", "moe_combine_backward"]
NORMS = ["moe_norm_before", "moe_norm_before_backward", "moe_norm_after", "moe_norm_after_backward"]
SIZES = [(name, "T") for name in _calls()] + [(name, "H") for name in ROWS + NORMS] + \
        [(name, "k") for name in ROWS + ["moe_route_topk", "moe_sort_tokens", "moe_route_topk_backward"]] + \
        [(name, "E") for name in ("moe_route_topk", "moe_sort_tokens", "moe_route_topk_backward")]


@pytest.mark.parametrize("value", HUGE)
@pytest.mark.parametrize("name,size", SIZES)
def test_sizes_beyond_32_bits_are_refused(no_device, name, size, value):
    with pytest.raises(moe.MoEError) as error:
        _calls(**{size: value})[name]()
    assert error.value.status == UNSUPPORTED


@pytest.mark.parametrize("value", [*HUGE, 2, -1, -(1 << 32)])
@pytest.mark.parametrize("name", NORMS)
def test_norms_that_there_are_not(no_device, name, value):
    with pytest.raises(moe.MoEError) as error:
        _calls(norm=value)[name]()
    assert error.value.status == INVALID


@pytest.mark.parametrize("value", [*HUGE, 4, -1, -(1 << 32)])
@pytest.mark.parametrize("name", NORMS[2:])
def test_gates_that_there_are_not(no_device, name, value):
    with pytest.raises(moe.MoEError) as error:
        _calls(kind=value)[name]()
    assert error.value.status == INVALID


def test_negative_numbers_of_experts(no_device):
    for E in (-1, -(1 << 32)):
        with pytest.raises(moe.MoEError) as error:
            moe.moe_sort_tokens(_i(4, 2), E, _i(8), _i(8), _i(4, 2), None)
        assert error.value.status == INVALID


def test_plans_take_offsets_that_are_read_once():
    for offsets in (iter([0, 40, 64]), (v for v in (0, 40, 64)), torch.tensor([0, 40, 64]), range(0, 65, 32)):
        moe.moe_plan_destroy(moe.moe_plan_create(64, 256, 256, 8, 2, 2, moe.MOE_ACT_SWIGLU, offsets))


@pytest.mark.parametrize("value", [*HUGE, -(1 << 32)])
def test_workspaces_and_plans_of_sizes_beyond_32_bits(value):
    for at in range(3):
        sizes = [8, 8, 2]
        sizes[at] = value
        assert moe.moe_sort_workspace_bytes(*sizes) == 0
    assert moe.moe_norm_workspace_bytes(value, 256) == 0 and moe.moe_norm_workspace_bytes(1, value) == 0
    good = dict(T=64, H=256, F=256, E=8, k=2, S=1, act=moe.MOE_ACT_SWIGLU, seg_offsets=[0, 64])
    moe.moe_plan_destroy(moe.moe_plan_create(**good))
    for name in ("T", "H", "F", "E", "k", "act"):
        with pytest.raises(moe.MoEError) as error:
            moe.moe_plan_create(**{**good, name: value})
        assert error.value.status == UNSUPPORTED
    with pytest.raises(moe.MoEError):
        moe.moe_plan_create(**{**good, "seg_offsets": [0, (1 << 32) + 64]})


def test_the_first_call_of_two_threads(monkeypatch):
    """Whenever another thread could look, between any two lines of the first call: what it takes for done is done."""
    names = ["_INT32", "_FLOAT32", "_UINT8", "_current_device", "_raw_stream", "_increment_version"]
    for name in names:
        monkeypatch.setattr(binding, name, None)
    monkeypatch.setattr(binding, "_DTYPES", {})
    looks = []

    def look(frame, event, arg):
        if frame.f_code is binding._first_call.__code__:
            if binding._INT32 is not None:       # what _Call looks at
                looks.append(len(binding._DTYPES) == 3 and all(getattr(binding, name) is not None for name in names))
            return look
        return None

    before = sys.gettrace()
    sys.settrace(look)
    try:
        binding._first_call()
    finally:
        sys.settrace(before)
    assert looks and all(looks)
    assert binding._INT32 is torch.int32


def _all_arguments(T=0, H=64, E=8, k=2):
    """(call, arguments by name, names of what it writes), every result wanted; the names are those of the call."""
    ws = _t(1 << 20, dtype=torch.uint8)

    def rows():
        return _t(T, H)

    def all_rows():
        return _t(T * k, H)
    pairs, gate = (T, k), moe.MOE_GATE_FULL
    return [
        (moe.moe_dispatch, dict(x=rows(), inv_perm=_i(*pairs), rows=all_rows()), "rows"),
        (moe.moe_dispatch_backward, dict(grad_rows=all_rows(), inv_perm=_i(*pairs), grad_x=rows()), "grad_x"),
        (moe.moe_combine, dict(rows=all_rows(), inv_perm=_i(*pairs), topk_weights=_f(*pairs), out=rows()), "out"),
        (moe.moe_combine_backward, dict(grad_out=rows(), rows=all_rows(), inv_perm=_i(*pairs), topk_weights=_f(*pairs), grad_rows=all_rows(),
                                        grad_weights=_f(*pairs)), "grad_rows grad_weights"),
        (moe.moe_route_topk_backward, dict(topk_ids=_i(*pairs), topk_weights=_f(*pairs), grad_weights=_f(*pairs), grad_logits=_f(T, E)),
         "grad_logits"),
        (moe.moe_norm_before, dict(residual=rows(), update=rows(), residual_scale=1.0, gamma=_t(H), beta=_t(H), norm=0, eps=1e-5, sum=rows(),
                                   x=rows()), "sum x"),
        (moe.moe_norm_after, dict(residual=rows(), y=rows(), gamma=_t(H), beta=_t(H), gate=rows(), gate_kind=gate, residual_scale=1.0, norm=0,
                                  eps=1e-5, out=rows()), "out"),
        # without tokens these two would still clear sums on the device: none are wanted
        (moe.moe_norm_before_backward, dict(sum=rows(), gamma=torch.empty(H, dtype=torch.bfloat16), grad_x=rows(), grad_sum=rows(), residual_scale=1.0,
                                            norm=0, eps=1e-5, grad_residual=rows(), grad_update=rows(), grad_gamma=None, grad_beta=None,
                                            workspace=ws), "grad_residual grad_update"),
        (moe.moe_norm_after_backward, dict(y=rows(), gamma=torch.empty(H, dtype=torch.bfloat16), beta=_t(H), gate=rows(), gate_kind=gate,
                                           residual_scale=1.0, grad_out=rows(), norm=0, eps=1e-5, grad_y=rows(), grad_gamma=None, grad_beta=None,
                                           grad_gate=rows(), workspace=ws), "grad_y grad_gate"),
    ]


@pytest.mark.parametrize("case", _all_arguments(), ids=lambda case: case[0].__name__)
def test_what_is_written_has_another_version(no_device, case):
    call, args, outputs = case
    tensors = {name: t for name, t in args.items() if isinstance(t, torch.Tensor)}
    before = {name: t._version for name, t in tensors.items()}
    call(**args)
    changed = {name for name, t in tensors.items() if t._version != before[name]}
    assert changed == set(outputs.split())
    with pytest.raises(moe.MoEError):          # a refused call has written nothing
        call(**args, stream=type("Stream", (), {"device_index": 0, "cuda_stream": None})())     # of another device
    assert changed == {name for name, t in tensors.items() if t._version != before[name]} and all(
        t._version == before[name] + 1 for name, t in tensors.items() if name in changed)
    with torch.inference_mode():               # tensors without a version
        call(**{name: torch.empty_like(t) if name in outputs.split() else t for name, t in args.items()})


def test_a_gradient_that_needs_overwritten_rows(no_device):
    """The stream is saved for the gradient of what follows, then a call in place takes it: no wrong gradient, but an error."""
    h, w = _t(0, 64, dtype=torch.float32), torch.ones(64, device="meta", requires_grad=True)
    loss = (h * w).sum()
    moe.moe_norm_before(h, None, 1.0, _f(64), None, moe.MOE_NORM_RMS, 1e-5, h, _f(0, 64))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
