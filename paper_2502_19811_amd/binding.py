"""ctypes binding with the same names as the C entry points of include/moe_gfx950.h.

Tensor arguments are torch tensors on the GPU (or None where the C call accepts NULL); only their
data pointers are passed on.  `stream` is a torch.cuda.Stream or None for the current stream.

No call becomes a node of torch's graph of gradients, whatever its tensors require: a program that wants that wraps a call and
its backward call in a torch.autograd.Function.  What the gate, the layer and the operators around the experts write counts as written
there, as after an operation in place: a gradient that needs the former values raises an error (replays of a graph do not count).
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

MOE_ERR_INVALID_ARG, MOE_ERR_UNSUPPORTED = -1, -4
MOE_ACT_GELU = 0
MOE_ACT_SWIGLU = 1
MOE_BF16, MOE_FP16, MOE_FP32 = 0, 1, 2
MOE_NORM_RMS, MOE_NORM_LAYER = 0, 1
MOE_GATE_NONE, MOE_GATE_CHANNEL, MOE_GATE_TOKEN, MOE_GATE_FULL = 0, 1, 2, 3

_LIB_NAME = "libmoe_gfx950.so"
_lib = None

EXPORTS = [
    "moe_plan_create", "moe_plan_destroy", "moe_plan_set_option", "moe_plan_get_option",
    "moe_plan_workspace_bytes", "moe_plan_max_tiles", "moe_receive_buffer_bytes", "moe_route_topk",
    "moe_layer_forward", "moe_get_index_outputs", "moe_get_tile_table", "moe_last_device_status",
    "moe_status_string", "moe_plan_phase_times", "moe_plan_forward_times", "moe_play_arrival",
    "moe_probe_mfma", "moe_probe_copy", "moe_pack_weights", "moe_layer_forward_static", "moe_get_schedule",
    "moe_plan_schedule_capacity", "moe_probe_mix",
    "moe_sort_workspace_bytes", "moe_sort_tokens", "moe_dispatch", "moe_dispatch_backward", "moe_combine", "moe_combine_backward",
    "moe_route_topk_backward", "moe_norm_workspace_bytes", "moe_norm_before", "moe_norm_before_backward", "moe_norm_after",
    "moe_norm_after_backward",
]


class MoEError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {moe_status_string(status)} ({status})")


class MoEShape(C.Structure):
    _fields_ = [("T", C.c_int32), ("H", C.c_int32), ("F", C.c_int32), ("E", C.c_int32), ("k", C.c_int32),
                ("S", C.c_int32), ("act", C.c_int32)]


def lib_path() -> str:
    """The in-tree library; MOE_GFX950_LIB names another build of the same sources (the measurement tools use it for
    builds with extra instrumentation)."""
    return os.environ.get("MOE_GFX950_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)), _LIB_NAME)


def load_library():
    """Loads the built library.  Raises if it is missing: there is no other implementation to fall back to."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is not built; run `python -m paper_2502_19811_amd.build` "
                                f"(or __graft_entry__.build()) first")
    lib = C.CDLL(path)
    vp, i32p, f32p, u32p = C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p
    lib.moe_plan_create.argtypes = [C.POINTER(C.c_void_p), C.POINTER(MoEShape), C.POINTER(C.c_int32)]
    lib.moe_plan_create.restype = C.c_int
    lib.moe_plan_destroy.argtypes = [C.c_void_p]
    lib.moe_plan_destroy.restype = C.c_int
    lib.moe_plan_set_option.argtypes = [C.c_void_p, C.c_char_p, C.c_int64]
    lib.moe_plan_set_option.restype = C.c_int
    lib.moe_plan_get_option.argtypes = [C.c_void_p, C.c_char_p, C.POINTER(C.c_int64)]
    lib.moe_plan_get_option.restype = C.c_int
    lib.moe_plan_workspace_bytes.argtypes = [C.c_void_p]
    lib.moe_plan_workspace_bytes.restype = C.c_size_t
    lib.moe_plan_max_tiles.argtypes = [C.c_void_p]
    lib.moe_plan_max_tiles.restype = C.c_int32
    lib.moe_receive_buffer_bytes.argtypes = [C.c_int64, C.c_int64]
    lib.moe_receive_buffer_bytes.restype = C.c_size_t
    lib.moe_route_topk.argtypes = [f32p, C.c_int32, C.c_int32, C.c_int32, i32p, f32p, vp]
    lib.moe_route_topk.restype = C.c_int
    lib.moe_layer_forward.argtypes = [C.c_void_p, vp, i32p, f32p, vp, vp, C.c_int32, vp, vp, C.c_size_t, u32p,
                                      C.c_uint32, vp]
    lib.moe_layer_forward.restype = C.c_int
    lib.moe_layer_forward_static.argtypes = [C.c_void_p, vp, i32p, f32p, vp, vp, C.c_int32, vp, u32p, C.c_uint32, vp]
    lib.moe_layer_forward_static.restype = C.c_int
    lib.moe_get_index_outputs.argtypes = [C.c_void_p, vp, i32p, i32p, i32p, i32p, vp]
    lib.moe_get_index_outputs.restype = C.c_int
    lib.moe_get_schedule.argtypes = [C.c_void_p, vp, C.c_int32, i32p, C.POINTER(C.c_int32), vp]
    lib.moe_get_schedule.restype = C.c_int
    lib.moe_plan_schedule_capacity.argtypes = [C.c_void_p, C.c_int32]
    lib.moe_plan_schedule_capacity.restype = C.c_int64
    lib.moe_get_tile_table.argtypes = [C.c_void_p, vp, i32p, i32p, i32p, i32p, i32p, i32p, vp]
    lib.moe_get_tile_table.restype = C.c_int
    lib.moe_last_device_status.argtypes = [C.c_void_p, vp, vp]
    lib.moe_last_device_status.restype = C.c_int
    lib.moe_plan_phase_times.argtypes = [C.c_void_p, C.POINTER(C.c_float), C.POINTER(C.c_int32)]
    lib.moe_plan_phase_times.restype = C.c_int
    lib.moe_plan_forward_times.argtypes = [C.c_void_p, C.POINTER(C.c_float), C.c_int32, C.POINTER(C.c_int32)]
    lib.moe_plan_forward_times.restype = C.c_int
    lib.moe_probe_mfma.argtypes = [C.c_int32, C.c_int32, vp, C.c_size_t, C.POINTER(C.c_float), vp]
    lib.moe_probe_mfma.restype = C.c_int
    lib.moe_probe_mix.argtypes = [C.c_int32, C.c_int32, vp, C.c_size_t, C.POINTER(C.c_float), C.POINTER(C.c_float), vp]
    lib.moe_probe_mix.restype = C.c_int
    lib.moe_probe_copy.argtypes = [vp, vp, C.c_size_t, C.POINTER(C.c_float), vp]
    lib.moe_probe_copy.restype = C.c_int
    lib.moe_play_arrival.argtypes = [C.c_void_p, vp, vp, u32p, u32p, C.c_uint32, C.c_double, C.c_int32, vp]
    lib.moe_play_arrival.restype = C.c_int
    lib.moe_pack_weights.argtypes = [C.c_void_p, vp, vp, vp, vp, vp]
    lib.moe_pack_weights.restype = C.c_int
    i32, f32, size = C.c_int32, C.c_float, C.c_size_t
    lib.moe_sort_workspace_bytes.argtypes = [i32, i32, i32]
    lib.moe_sort_workspace_bytes.restype = size
    lib.moe_sort_tokens.argtypes = [i32p, i32, i32, i32, i32p, i32p, i32p, vp, size, vp]
    lib.moe_dispatch.argtypes = [vp, i32p, i32, i32, i32, i32, vp, vp]
    lib.moe_dispatch_backward.argtypes = [vp, i32p, i32, i32, i32, i32, vp, vp]
    lib.moe_combine.argtypes = [vp, i32p, f32p, i32, i32, i32, i32, vp, vp]
    lib.moe_combine_backward.argtypes = [vp, vp, i32p, f32p, i32, i32, i32, i32, vp, f32p, vp]
    lib.moe_route_topk_backward.argtypes = [i32p, f32p, f32p, i32, i32, i32, f32p, vp]
    lib.moe_norm_workspace_bytes.argtypes = [i32, i32]
    lib.moe_norm_workspace_bytes.restype = size
    lib.moe_norm_before.argtypes = [vp, vp, f32, vp, vp, i32, f32, i32, i32, i32, vp, vp, vp]
    lib.moe_norm_before_backward.argtypes = [vp, vp, vp, vp, f32, i32, f32, i32, i32, i32, vp, vp, f32p, f32p, vp, size, vp]
    lib.moe_norm_after.argtypes = [vp, vp, vp, vp, vp, i32, f32, i32, f32, i32, i32, i32, vp, vp]
    lib.moe_norm_after_backward.argtypes = [vp, vp, vp, vp, i32, f32, vp, i32, f32, i32, i32, i32, vp, f32p, f32p, vp, vp, size, vp]
    for name in ("moe_sort_tokens", "moe_dispatch", "moe_dispatch_backward", "moe_combine", "moe_combine_backward",
                 "moe_route_topk_backward", "moe_norm_before", "moe_norm_before_backward", "moe_norm_after", "moe_norm_after_backward"):
        getattr(lib, name).restype = C.c_int
    lib.moe_status_string.argtypes = [C.c_int]
    lib.moe_status_string.restype = C.c_char_p
    _lib = lib
    return lib


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream


def _check(status: int, where: str) -> None:
    if status != 0:
        raise MoEError(status, where)


def _written(tensors) -> None:
    """A call has written these: whoever saved them for a gradient is told by their version (0.1 to 0.2 us)."""
    if _increment_version is None:
        _first_call()
    _increment_version(tensors)


# The C calls take sizes as 32-bit integers, and ctypes cuts what is longer without a word: 2**32 rows would be none.  So sizes are
# tested first, where calls are short those of a call together: (a | b | ...) >> 31 is 0 if all of them fit and none is negative.
def _check_int32(where: str, *values: int) -> None:
    if any(not -1 << 31 <= v < 1 << 31 for v in values):
        raise MoEError(MOE_ERR_UNSUPPORTED, where)


def moe_status_string(status: int) -> str:
    return load_library().moe_status_string(status).decode()


def moe_plan_create(T: int, H: int, F: int, E: int, k: int, S: int, act: int, seg_offsets: Sequence[int]) -> int:
    """Returns the plan handle.  seg_offsets: S+1 host integers."""
    lib = load_library()
    offsets = [int(v) for v in seg_offsets]
    _check_int32("moe_plan_create", T, H, F, E, k, S, act, *offsets)
    shape = MoEShape(T, H, F, E, k, S, act)
    seg = (C.c_int32 * (S + 1))(*offsets)
    handle = C.c_void_p()
    _check(lib.moe_plan_create(C.byref(handle), C.byref(shape), seg), "moe_plan_create")
    return handle.value


def moe_plan_destroy(plan: int) -> None:
    _check(load_library().moe_plan_destroy(plan), "moe_plan_destroy")


def moe_plan_set_option(plan: int, key: str, value: int) -> None:
    _check(load_library().moe_plan_set_option(plan, key.encode(), int(value)), f"moe_plan_set_option({key})")


def moe_plan_get_option(plan: int, key: str) -> int:
    v = C.c_int64()
    _check(load_library().moe_plan_get_option(plan, key.encode(), C.byref(v)), f"moe_plan_get_option({key})")
    return v.value


def moe_plan_workspace_bytes(plan: int) -> int:
    return load_library().moe_plan_workspace_bytes(plan)


def moe_plan_max_tiles(plan: int) -> int:
    return load_library().moe_plan_max_tiles(plan)


def moe_receive_buffer_bytes(M: int, N: int) -> int:
    return load_library().moe_receive_buffer_bytes(M, N)


def moe_route_topk(logits, k: int, topk_ids, topk_weights, stream=None) -> None:
    T, E = logits.shape
    if (T | E | k) >> 31:
        _check_int32("moe_route_topk", T, E, k)
    _check(load_library().moe_route_topk(_ptr(logits), T, E, k, _ptr(topk_ids), _ptr(topk_weights), _stream(stream)),
           "moe_route_topk")
    _written((topk_ids, topk_weights))


def moe_layer_forward(plan: int, x, topk_ids, topk_weights, W1, W2, act: int, out, workspace, seg_ready=None,
                      ready_epoch: int = 0, stream=None) -> None:
    _check(load_library().moe_layer_forward(plan, _ptr(x), _ptr(topk_ids), _ptr(topk_weights), _ptr(W1), _ptr(W2), act,
                                            _ptr(out), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                            _ptr(seg_ready), ready_epoch, _stream(stream)), "moe_layer_forward")
    _written((out,))


def moe_layer_forward_static(plan: int, x, topk_ids, topk_weights, W1, W2, act: int, out, seg_ready=None,
                             ready_epoch: int = 0, stream=None) -> None:
    """moe_layer_forward on the library's own fixed workspace (no allocation; plans up to 32 MiB of workspace)."""
    _check(load_library().moe_layer_forward_static(plan, _ptr(x), _ptr(topk_ids), _ptr(topk_weights), _ptr(W1), _ptr(W2),
                                                   act, _ptr(out), _ptr(seg_ready), ready_epoch, _stream(stream)),
           "moe_layer_forward_static")
    _written((out,))


def moe_pack_weights(plan: int, W1, W2, W1_packed, W2_packed, stream=None) -> None:
    _check(load_library().moe_pack_weights(plan, _ptr(W1), _ptr(W2), _ptr(W1_packed), _ptr(W2_packed), _stream(stream)),
           "moe_pack_weights")


def moe_get_index_outputs(plan: int, workspace, expert_counts=None, expert_offsets=None, perm=None, inv_perm=None,
                          stream=None) -> None:
    _check(load_library().moe_get_index_outputs(plan, _ptr(workspace), _ptr(expert_counts), _ptr(expert_offsets),
                                                _ptr(perm), _ptr(inv_perm), _stream(stream)), "moe_get_index_outputs")


def moe_get_tile_table(plan: int, workspace, n_tiles, tile_expert, tile_row0, tile_rows, tile_ready_seg,
                       tile_height=None, stream=None) -> None:
    _check(load_library().moe_get_tile_table(plan, _ptr(workspace), _ptr(n_tiles), _ptr(tile_expert), _ptr(tile_row0),
                                             _ptr(tile_rows), _ptr(tile_ready_seg), _ptr(tile_height),
                                             _stream(stream)),
           "moe_get_tile_table")


def moe_plan_schedule_capacity(plan: int, layer: int) -> int:
    return load_library().moe_plan_schedule_capacity(plan, layer)


def moe_get_schedule(plan: int, workspace, layer: int, items=None, stream=None):
    """Queues of the last forward's tile schedule: (first position, items, stride) per XCD; items (a device int32
    tensor [capacity, 8]) receives the item records."""
    q = (C.c_int32 * 24)()
    _check(load_library().moe_get_schedule(plan, _ptr(workspace), layer, _ptr(items), q, _stream(stream)),
           "moe_get_schedule")
    return [(q[x], q[8 + x], q[16 + x]) for x in range(8)]


def moe_last_device_status(plan: int, workspace, stream=None) -> int:
    return load_library().moe_last_device_status(plan, _ptr(workspace), _stream(stream))


def moe_plan_phase_times(plan: int):
    """(ms per phase [index build, layer0, layer1 (+fused combine), stand-alone combine], forwards averaged)."""
    ms = (C.c_float * 4)()
    n = C.c_int32()
    _check(load_library().moe_plan_phase_times(plan, ms, C.byref(n)), "moe_plan_phase_times")
    return [float(v) for v in ms], n.value


def moe_play_arrival(plan: int, staging, x, seg_ready, seg_counters, ready_epoch: int, gbytes_per_s: float,
                     n_workgroups: int = 1, stream=None) -> None:
    _check(load_library().moe_play_arrival(plan, _ptr(staging), _ptr(x), _ptr(seg_ready), _ptr(seg_counters),
                                           ready_epoch, float(gbytes_per_s), n_workgroups, _stream(stream)),
           "moe_play_arrival")


def moe_plan_forward_times(plan: int, capacity: int = 256):
    """ms of each forward recorded since the last moe_plan_phase_times call (needs the "profile" option)."""
    ms = (C.c_float * capacity)()
    n = C.c_int32()
    _check(load_library().moe_plan_forward_times(plan, ms, capacity, C.byref(n)), "moe_plan_forward_times")
    return [float(ms[i]) for i in range(n.value)]


def moe_probe_mfma(random_data, iters: int, scratch, stream=None) -> float:
    """TFLOP/s of the library's register-only bf16 MFMA loop on this device (scratch: a device tensor of >= 1 MiB).
    random_data: False zeros, True random operands, 2 random operands with the 16x16x32 instruction."""
    out = C.c_float()
    _check(load_library().moe_probe_mfma(int(random_data), iters, _ptr(scratch), scratch.numel() * scratch.element_size(),
                                         C.byref(out), _stream(stream)), "moe_probe_mfma")
    return float(out.value)


def moe_probe_mix(mode: int, iters: int, scratch, stream=None, with_clock: bool = False):
    """TFLOP/s of the MFMA loop with GroupGEMM-like data movement around it (mode bits: 1 LDS reads, 2 global->LDS
    loads, 4 barrier, 8 a quarter of the loads from HBM, 16 the 16x16x32 instruction); iters K steps; scratch: a device tensor, see the header for its size.
    with_clock: returns (TFLOP/s, core clock in GHz inside the loop)."""
    out, ghz = C.c_float(), C.c_float()
    _check(load_library().moe_probe_mix(mode, iters, _ptr(scratch), scratch.numel() * scratch.element_size(),
                                        C.byref(out), C.byref(ghz) if with_clock else None, _stream(stream)),
           "moe_probe_mix")
    return (float(out.value), float(ghz.value)) if with_clock else float(out.value)


def moe_probe_copy(dst, src, stream=None) -> float:
    """GB/s (read + written) of a plain device copy of src into dst."""
    out = C.c_float()
    nbytes = src.numel() * src.element_size()
    _check(load_library().moe_probe_copy(_ptr(dst), _ptr(src), nbytes, C.byref(out), _stream(stream)), "moe_probe_copy")
    return float(out.value)


# ---- operators around the experts ----
# The C calls see addresses only, so what they cannot check is checked here: every tensor has the type and shape its call
# says, is contiguous, and lies on the current device, as the stream does.  These calls are often a few microseconds of work:
# checking a tensor takes 0.3 us, and the current stream is asked for by its address (0.1 us; as an object 1.1).  With the test of the
# sizes and the versions of what is written a call takes 0.2 to 0.35 us more than without.

_DTYPES = {}            # torch's row types -> their numbers, filled at the first call
_INT32 = _FLOAT32 = _UINT8 = _current_device = _raw_stream = _increment_version = None


def _first_call() -> None:
    global _INT32, _FLOAT32, _UINT8, _current_device, _raw_stream, _increment_version
    import torch
    _FLOAT32, _UINT8 = torch.float32, torch.uint8
    _current_device = torch.cuda.current_device
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
    _increment_version = getattr(torch._C, "_increment_version", None) or torch.autograd.graph.increment_version
    _DTYPES.update({torch.bfloat16: MOE_BF16, torch.float16: MOE_FP16, torch.float32: MOE_FP32})
    _INT32 = torch.int32    # last: another thread goes on once this is there


class _Call:
    """The tensors of one call: arg() checks one and gives its address."""

    __slots__ = ("where", "device", "stream")

    def __init__(self, where: str, stream):
        if _INT32 is None:
            _first_call()
        self.where = where
        self.device = _current_device()
        if stream is None:
            self.stream = _raw_stream(self.device)
        elif stream.device_index == self.device:
            self.stream = stream.cuda_stream
        else:
            self.refuse()

    def refuse(self, status: int = MOE_ERR_INVALID_ARG):
        raise MoEError(status, self.where)

    def arg(self, t, dtype, shape) -> int:
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self.device or not t.is_contiguous():
            self.refuse()
        return t.data_ptr()

    def opt(self, t, dtype, shape) -> Optional[int]:
        return None if t is None else self.arg(t, dtype, shape)

    def rows(self, t):
        """(shape, type, its number) of a tensor of rows."""
        if t.dim() != 2 or t.dtype not in _DTYPES:
            self.refuse()
        T, H = shape = t.shape
        if (T | H) >> 31:
            self.refuse(MOE_ERR_UNSUPPORTED)
        return shape, t.dtype, _DTYPES[t.dtype]

    def pairs(self, t):
        """(T, k) of a tensor of pairs."""
        if t.dim() != 2:
            self.refuse()
        T, k = shape = t.shape
        if (T | k) >> 31:
            self.refuse(MOE_ERR_UNSUPPORTED)
        return shape

    def workspace(self, t):
        if t is None:
            return None, 0
        return self.arg(t, _UINT8, (t.numel(),)), t.numel()

    def done(self, status: int, *written) -> None:
        if status != 0:
            raise MoEError(status, self.where)
        _increment_version(written)


def _given(*tensors):
    return [t for t in tensors if t is not None]


def moe_sort_workspace_bytes(T: int, E: int, k: int) -> int:
    if (T | E | k) >> 31:      # (negative ones, too: no such shape)
        return 0
    return load_library().moe_sort_workspace_bytes(T, E, k)


def moe_sort_tokens(topk_ids, E: int, expert_offsets, perm, inv_perm, workspace, stream=None) -> None:
    """topk_ids int32 [T,k] -> expert_offsets int32 [E+1], perm int32 [T*k], inv_perm int32 [T,k]; workspace uint8."""
    c = _Call("moe_sort_tokens", stream)
    T, k = pairs = c.pairs(topk_ids)
    if E >> 31:
        c.refuse(MOE_ERR_INVALID_ARG if E < 0 else MOE_ERR_UNSUPPORTED)
    c.done(load_library().moe_sort_tokens(
        c.arg(topk_ids, _INT32, pairs), T, E, k, c.arg(expert_offsets, _INT32, (E + 1,)), c.arg(perm, _INT32, (T * k,)),
        c.arg(inv_perm, _INT32, pairs), *c.workspace(workspace), c.stream), expert_offsets, perm, inv_perm)


def moe_dispatch(x, inv_perm, rows, stream=None) -> None:
    """x [T,H], inv_perm int32 [T,k] -> rows [T*k,H]."""
    c = _Call("moe_dispatch", stream)
    (T, H), t, dtype = c.rows(x)
    k = c.pairs(inv_perm)[1]
    c.done(load_library().moe_dispatch(c.arg(x, t, (T, H)), c.arg(inv_perm, _INT32, (T, k)), T, H, k, dtype, c.arg(rows, t, (T * k, H)), c.stream),
           rows)


def moe_dispatch_backward(grad_rows, inv_perm, grad_x, stream=None) -> None:
    """grad_rows [T*k,H], inv_perm int32 [T,k] -> grad_x [T,H]."""
    c = _Call("moe_dispatch_backward", stream)
    (T, H), t, dtype = c.rows(grad_x)
    k = c.pairs(inv_perm)[1]
    c.done(load_library().moe_dispatch_backward(c.arg(grad_rows, t, (T * k, H)), c.arg(inv_perm, _INT32, (T, k)), T, H, k, dtype,
                                                c.arg(grad_x, t, (T, H)), c.stream), grad_x)


def moe_combine(rows, inv_perm, topk_weights, out, stream=None) -> None:
    """rows [T*k,H], inv_perm int32 [T,k], topk_weights fp32 [T,k] or None -> out [T,H]."""
    c = _Call("moe_combine", stream)
    (T, H), t, dtype = c.rows(out)
    k = c.pairs(inv_perm)[1]
    c.done(load_library().moe_combine(c.arg(rows, t, (T * k, H)), c.arg(inv_perm, _INT32, (T, k)), c.opt(topk_weights, _FLOAT32, (T, k)),
                                      T, H, k, dtype, c.arg(out, t, (T, H)), c.stream), out)


def moe_combine_backward(grad_out, rows, inv_perm, topk_weights, grad_rows, grad_weights, stream=None) -> None:
    """grad_out [T,H], rows [T*k,H] -> grad_rows [T*k,H], grad_weights fp32 [T,k] (None: not wanted, rows may be None)."""
    c = _Call("moe_combine_backward", stream)
    (T, H), t, dtype = c.rows(grad_out)
    k = c.pairs(inv_perm)[1]
    pairs, all_rows = (T, k), (T * k, H)
    c.done(load_library().moe_combine_backward(
        c.arg(grad_out, t, (T, H)), c.opt(rows, t, all_rows), c.arg(inv_perm, _INT32, pairs), c.opt(topk_weights, _FLOAT32, pairs),
        T, H, k, dtype, c.arg(grad_rows, t, all_rows), c.opt(grad_weights, _FLOAT32, pairs), c.stream),
        *((grad_rows,) if grad_weights is None else (grad_rows, grad_weights)))


def moe_route_topk_backward(topk_ids, topk_weights, grad_weights, grad_logits, stream=None) -> None:
    """topk_ids int32 [T,k], topk_weights and grad_weights fp32 [T,k] -> grad_logits fp32 [T,E]."""
    c = _Call("moe_route_topk_backward", stream)
    T, k = pairs = c.pairs(topk_ids)
    E = c.pairs(grad_logits)[1]
    c.done(load_library().moe_route_topk_backward(
        c.arg(topk_ids, _INT32, pairs), c.arg(topk_weights, _FLOAT32, pairs), c.arg(grad_weights, _FLOAT32, pairs), T, E, k,
        c.arg(grad_logits, _FLOAT32, (T, E)), c.stream), grad_logits)


def moe_norm_workspace_bytes(T: int, H: int) -> int:
    if (T | H) >> 31:
        return 0
    return load_library().moe_norm_workspace_bytes(T, H)


def moe_norm_before(residual, update, residual_scale: float, gamma, beta, norm: int, eps: float, sum, x, stream=None) -> None:
    """sum = residual + residual_scale * update, x = norm of it; update, beta and sum may be None."""
    c = _Call("moe_norm_before", stream)
    s, t, dtype = c.rows(residual)
    T, H = s
    if norm >> 31:
        c.refuse()
    c.done(load_library().moe_norm_before(
        c.arg(residual, t, s), c.opt(update, t, s), residual_scale, c.arg(gamma, t, (H,)), c.opt(beta, t, (H,)), norm, eps, T, H, dtype,
        c.opt(sum, t, s), c.arg(x, t, s), c.stream), *((x,) if sum is None else (sum, x)))


def moe_norm_before_backward(sum, gamma, grad_x, grad_sum, residual_scale: float, norm: int, eps: float, grad_residual, grad_update,
                             grad_gamma, grad_beta, workspace, stream=None) -> None:
    """grad_sum, grad_update, grad_gamma and grad_beta may be None; without the last two workspace may be, too."""
    c = _Call("moe_norm_before_backward", stream)
    s, t, dtype = c.rows(sum)
    T, H = s
    if norm >> 31:
        c.refuse()
    c.done(load_library().moe_norm_before_backward(
        c.arg(sum, t, s), c.arg(gamma, t, (H,)), c.arg(grad_x, t, s), c.opt(grad_sum, t, s), residual_scale, norm, eps, T, H, dtype,
        c.arg(grad_residual, t, s), c.opt(grad_update, t, s), c.opt(grad_gamma, _FLOAT32, (H,)), c.opt(grad_beta, _FLOAT32, (H,)),
        *c.workspace(workspace), c.stream), *_given(grad_residual, grad_update, grad_gamma, grad_beta))


def _gate(c: _Call, gate, kind: int, shape, t) -> Optional[int]:
    """A gate of this kind; shape: of the rows; t: type of a channel or full one."""
    if gate is None:
        return None
    if kind == MOE_GATE_TOKEN:
        return c.arg(gate, _FLOAT32, shape[:1])
    return c.arg(gate, t, shape[1:] if kind == MOE_GATE_CHANNEL else shape)


def moe_norm_after(residual, y, gamma, beta, gate, gate_kind: int, residual_scale: float, norm: int, eps: float, out,
                   stream=None) -> None:
    """out = residual + residual_scale * gate * norm of y; residual and beta may be None, gate is with MOE_GATE_NONE."""
    c = _Call("moe_norm_after", stream)
    s, t, dtype = c.rows(y)
    T, H = s
    if (norm | gate_kind) >> 31:
        c.refuse()
    c.done(load_library().moe_norm_after(
        c.opt(residual, t, s), c.arg(y, t, s), c.arg(gamma, t, (H,)), c.opt(beta, t, (H,)), _gate(c, gate, gate_kind, s, t), gate_kind,
        residual_scale, norm, eps, T, H, dtype, c.arg(out, t, s), c.stream), out)


def moe_norm_after_backward(y, gamma, beta, gate, gate_kind: int, residual_scale: float, grad_out, norm: int, eps: float, grad_y,
                            grad_gamma, grad_beta, grad_gate, workspace, stream=None) -> None:
    """grad_gamma, grad_beta and grad_gate may be None; workspace too if nothing is summed over tokens."""
    c = _Call("moe_norm_after_backward", stream)
    s, t, dtype = c.rows(y)
    T, H = s
    if (norm | gate_kind) >> 31:
        c.refuse()
    c.done(load_library().moe_norm_after_backward(
        c.arg(y, t, s), c.arg(gamma, t, (H,)), c.opt(beta, t, (H,)), _gate(c, gate, gate_kind, s, t), gate_kind, residual_scale,
        c.arg(grad_out, t, s), norm, eps, T, H, dtype, c.arg(grad_y, t, s), c.opt(grad_gamma, _FLOAT32, (H,)), c.opt(grad_beta, _FLOAT32, (H,)),
        _gate(c, grad_gate, gate_kind, s, _FLOAT32 if gate_kind == MOE_GATE_CHANNEL else t), *c.workspace(workspace), c.stream),
        *_given(grad_y, grad_gamma, grad_beta, grad_gate))
