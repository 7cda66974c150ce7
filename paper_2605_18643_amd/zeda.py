"""Thin Python binding of libzeda's C ABI (include/zeda.h): argument marshalling only.

Tensors are PyTorch-ROCm device tensors used as plain device buffers; every step of the layer runs
inside the HIP library.  There is no fallback: if the library is missing, importing the entry points
raises, and nothing here computes on the CPU.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from typing import Optional, Tuple

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "libzeda.so")

ZEDA_OK, ZEDA_EINVAL, ZEDA_EUNSUPPORTED, ZEDA_EWORKSPACE, ZEDA_EHIP = 0, -1, -2, -3, -4
ZEDA_F32, ZEDA_BF16 = 0, 1
GATE_SOFTMAX, GATE_TOPK_NORM, GATE_REAL_RENORM = 0, 1, 2
WEIGHTS_ROW_MAJOR, WEIGHTS_TILED = 0, 1
EXPERT_ZERO, EXPERT_COPY = 0, 1
STAGES = ("route", "dispatch", "gateup", "down", "combine")

EXPORTS = ("zeda_status_string", "zeda_workspace_bytes", "zeda_route_workspace_bytes", "zeda_dispatch_workspace_bytes",
           "zeda_expert_ffn_workspace_bytes", "zeda_workspace_layout", "zeda_route", "zeda_dispatch",
           "zeda_dispatch_noalloc", "zeda_dispatch_noalloc_max_slots",
           "zeda_expert_ffn", "zeda_combine", "zeda_moe_forward", "zeda_moe_forward_events", "zeda_moe_block_forward",
           "zeda_rmsnorm",
           "zeda_residual_add", "zeda_pack_expert_weights", "zeda_routing_stats_workspace_bytes", "zeda_routing_stats",
           "zeda_init_zero_expert_rows", "zeda_stream_read_probe", "zeda_mfma_probe", "zeda_token_zero_slots", "zeda_overlap_probe",
           "zeda_quantize_rows_fp8", "zeda_quantize_weights_fp8", "zeda_fp8_expert_bytes", "zeda_pack_expert_weights_fp8",
           "zeda_expert_ffn_workspace_bytes_fp8", "zeda_workspace_bytes_fp8", "zeda_workspace_layout_fp8", "zeda_expert_ffn_fp8",
           "zeda_moe_forward_fp8", "zeda_moe_block_forward_fp8",
           "zeda_route_train_workspace_bytes", "zeda_route_train", "zeda_route_backward_workspace_bytes", "zeda_route_backward",
           "zeda_combine_backward")


class LayerDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "H", "I", "N", "Z", "K", "dtype", "gate_norm", "weight_layout",
                                                 "free_expert")]


class WsLayout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in ("topk_ids", "topk_gates", "expert_offsets", "sorted_slot",
                                               "slot_to_row", "num_real", "dispatch_ws", "act", "y_slot", "route_ws",
                                               "total")]


class Fp8Experts(ctypes.Structure):
    """Packed 8-bit expert weights (zeda_fp8_experts): the C struct, and the device buffers that it points to in `buffers`.
    desc: the layer that they were packed for (only its N, H and I count), which calls with another one are then refused by; without
    it they are taken for any layer whose packed sizes they have."""

    _fields_ = [(n, ctypes.c_void_p) for n in ("w_gateup", "w_down", "s_gateup", "s_down")]

    def __init__(self, buffers, desc: Optional[LayerDesc] = None):
        super().__init__(*[b.data_ptr() for b in buffers])
        self.buffers = tuple(buffers)
        self.shape = None
        if desc is not None:
            self.check(desc, "Fp8Experts")
            self.shape = (desc.N, desc.H, desc.I)

    def check(self, desc: LayerDesc, where: str) -> None:
        if self.shape is not None:
            _need(self.shape == (desc.N, desc.H, desc.I), where)
            return
        sizes = fp8_expert_bytes(desc)
        _need(len(self.buffers) == 4 and all(b.numel() * b.element_size() >= n and b.is_contiguous() for b, n in zip(self.buffers, sizes)), where)


class ZedaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2605_18643_amd.build`")
        L = ctypes.CDLL(_LIB_PATH)
        vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
        dp = ctypes.POINTER(LayerDesc)
        L.zeda_status_string.restype = ctypes.c_char_p
        L.zeda_status_string.argtypes = [i32]
        for name in ("zeda_workspace_bytes", "zeda_route_workspace_bytes", "zeda_dispatch_workspace_bytes",
                     "zeda_expert_ffn_workspace_bytes", "zeda_routing_stats_workspace_bytes"):
            getattr(L, name).restype = sz
            getattr(L, name).argtypes = [dp]
        L.zeda_workspace_layout.restype = i32
        L.zeda_workspace_layout.argtypes = [dp, ctypes.POINTER(WsLayout)]
        L.zeda_route.restype = i32
        L.zeda_route.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.zeda_dispatch.restype = i32
        L.zeda_dispatch.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.zeda_dispatch_noalloc.restype = i32
        L.zeda_dispatch_noalloc.argtypes = [dp, vp, vp, vp, vp, vp, vp]
        L.zeda_dispatch_noalloc_max_slots.restype = i32
        L.zeda_dispatch_noalloc_max_slots.argtypes = []
        L.zeda_expert_ffn.restype = i32
        L.zeda_expert_ffn.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.zeda_combine.restype = i32
        L.zeda_combine.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp]
        L.zeda_moe_forward.restype = i32
        L.zeda_moe_forward.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.zeda_moe_forward_events.restype = i32
        L.zeda_moe_forward_events.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, ctypes.POINTER(vp)]
        L.zeda_moe_block_forward.restype = i32
        L.zeda_moe_block_forward.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, sz, vp]
        L.zeda_rmsnorm.restype = i32
        L.zeda_rmsnorm.argtypes = [i32, i32, i32, vp, vp, ctypes.c_float, vp, vp]
        L.zeda_residual_add.restype = i32
        L.zeda_residual_add.argtypes = [i32, i32, i32, vp, vp, vp]
        L.zeda_routing_stats.restype = i32
        L.zeda_routing_stats.argtypes = [dp, vp, vp, vp, ctypes.c_float, ctypes.c_float, vp, vp, vp, vp, sz, vp]
        L.zeda_init_zero_expert_rows.restype = i32
        L.zeda_init_zero_expert_rows.argtypes = [dp, vp, vp, vp, vp]
        L.zeda_token_zero_slots.restype = i32
        L.zeda_token_zero_slots.argtypes = [dp, vp, vp, i32, vp]
        L.zeda_overlap_probe.restype = i32
        L.zeda_overlap_probe.argtypes = [vp, sz, i32, i32, vp, vp]
        L.zeda_mfma_probe.restype = i32
        L.zeda_mfma_probe.argtypes = [i32, i32, vp, vp]
        L.zeda_stream_read_probe.restype = i32
        L.zeda_stream_read_probe.argtypes = [vp, sz, vp, vp]
        L.zeda_pack_expert_weights.restype = i32
        L.zeda_pack_expert_weights.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp]
        L.zeda_quantize_rows_fp8.restype = i32
        L.zeda_quantize_rows_fp8.argtypes = [i32, i32, i32, vp, vp, vp, vp]
        L.zeda_quantize_weights_fp8.restype = i32
        L.zeda_quantize_weights_fp8.argtypes = [i32, i32, i32, i32, vp, vp, vp, vp]
        ep = ctypes.POINTER(Fp8Experts)
        L.zeda_fp8_expert_bytes.restype = i32
        L.zeda_fp8_expert_bytes.argtypes = [dp, ctypes.POINTER(sz)]
        L.zeda_pack_expert_weights_fp8.restype = i32
        L.zeda_pack_expert_weights_fp8.argtypes = [dp, vp, vp, vp, vp, vp, vp, ep, vp]
        for name in ("zeda_expert_ffn_workspace_bytes_fp8", "zeda_workspace_bytes_fp8", "zeda_route_train_workspace_bytes",
                     "zeda_route_backward_workspace_bytes"):
            getattr(L, name).restype = sz
            getattr(L, name).argtypes = [dp]
        L.zeda_workspace_layout_fp8.restype = i32
        L.zeda_workspace_layout_fp8.argtypes = [dp, ctypes.POINTER(WsLayout)]
        L.zeda_expert_ffn_fp8.restype = i32
        L.zeda_expert_ffn_fp8.argtypes = [dp, vp, ep, vp, vp, vp, vp, vp, sz, vp]
        L.zeda_moe_forward_fp8.restype = i32
        L.zeda_moe_forward_fp8.argtypes = [dp, vp, vp, vp, ep, vp, vp, vp, sz, vp]
        L.zeda_moe_block_forward_fp8.restype = i32
        L.zeda_moe_block_forward_fp8.argtypes = [dp, vp, vp, vp, vp, ep, vp, ctypes.c_float, vp, vp, vp, sz, vp]
        fl = ctypes.c_float
        L.zeda_route_train.restype = i32
        L.zeda_route_train.argtypes = [dp, vp, vp, vp, vp, fl, fl, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.zeda_route_backward.restype = i32
        L.zeda_route_backward.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, fl, fl, vp, vp, vp, vp, vp, vp, sz, vp]
        L.zeda_combine_backward.restype = i32
        L.zeda_combine_backward.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().zeda_status_string(int(status)).decode()


def make_desc(T, H, I, N, Z, K, dtype, gate_norm=GATE_TOPK_NORM, weight_layout=0, free_expert=0) -> LayerDesc:
    if isinstance(dtype, torch.dtype):
        dtype = ZEDA_BF16 if dtype == torch.bfloat16 else ZEDA_F32
    elif isinstance(dtype, str):
        dtype = ZEDA_BF16 if dtype == "bf16" else ZEDA_F32
    return LayerDesc(T, H, I, N, Z, K, int(dtype), int(gate_norm), int(weight_layout), int(free_expert))


# Arguments go to ctypes as plain integers (the functions' argtypes say what they are), and the current stream is asked for
# by its handle, where this torch has the (private) function for it: ten c_void_p objects and a Stream object a call were 4 us
# of a small layer's 18 us on the host.
def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return torch.cuda.current_stream().cuda_stream if raw is None else raw(torch.cuda.current_device())


def _on(stream):
    """Context for allocations that a call on `stream` fills: they come from that stream's blocks.  One of the current stream's may have been
    freed with work on it still queued there, which the call on `stream` would not wait for."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _check(rc: int, where: str) -> None:
    if rc != ZEDA_OK:
        raise ZedaError(rc, where)


def workspace_bytes(desc: LayerDesc) -> int:
    return int(lib().zeda_workspace_bytes(ctypes.byref(desc)))


def dispatch_workspace_bytes(desc: LayerDesc) -> int:
    return int(lib().zeda_dispatch_workspace_bytes(ctypes.byref(desc)))


def expert_ffn_workspace_bytes(desc: LayerDesc) -> int:
    return int(lib().zeda_expert_ffn_workspace_bytes(ctypes.byref(desc)))


def workspace_layout(desc: LayerDesc) -> WsLayout:
    out = WsLayout()
    _check(lib().zeda_workspace_layout(ctypes.byref(desc), ctypes.byref(out)), "zeda_workspace_layout")
    return out


def route_workspace_bytes(desc: LayerDesc) -> int:
    return int(lib().zeda_route_workspace_bytes(ctypes.byref(desc)))


def zeda_route(desc, x, w_router, router_bias, topk_ids, topk_gates, ws=None, stream=None) -> None:
    """ws: uint8 scratch of route_workspace_bytes(desc) or None (see include/zeda.h)."""
    _check(lib().zeda_route(ctypes.byref(desc), _ptr(x), _ptr(w_router), _ptr(router_bias), _ptr(topk_ids),
                            _ptr(topk_gates), _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)), "zeda_route")


def zeda_dispatch(desc, topk_ids, expert_offsets, sorted_slot, slot_to_row, num_real, ws, stream=None) -> None:
    _check(lib().zeda_dispatch(ctypes.byref(desc), _ptr(topk_ids), _ptr(expert_offsets), _ptr(sorted_slot),
                               _ptr(slot_to_row), _ptr(num_real), _ptr(ws), ws.numel() * ws.element_size(),
                               _stream(stream)), "zeda_dispatch")


def zeda_dispatch_noalloc(desc, topk_ids, expert_offsets, sorted_slot, slot_to_row, num_real, stream=None) -> None:
    """zeda_dispatch on the library's own static scratch (no workspace argument, nothing allocated)."""
    _check(lib().zeda_dispatch_noalloc(ctypes.byref(desc), _ptr(topk_ids), _ptr(expert_offsets), _ptr(sorted_slot),
                                       _ptr(slot_to_row), _ptr(num_real), _stream(stream)), "zeda_dispatch_noalloc")


def dispatch_noalloc_max_slots() -> int:
    return int(lib().zeda_dispatch_noalloc_max_slots())


def zeda_expert_ffn(desc, x, w_gate, w_up, w_down, expert_offsets, sorted_slot, num_real, y_slot, ws,
                    stream=None) -> None:
    _check(lib().zeda_expert_ffn(ctypes.byref(desc), _ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(w_down),
                                 _ptr(expert_offsets), _ptr(sorted_slot), _ptr(num_real), _ptr(y_slot), _ptr(ws),
                                 ws.numel() * ws.element_size(), _stream(stream)), "zeda_expert_ffn")


def zeda_combine(desc, y_slot, topk_ids, topk_gates, slot_to_row, out, x=None, stream=None) -> None:
    """x (the layer input) is only needed with desc.free_expert == EXPERT_COPY."""
    _check(lib().zeda_combine(ctypes.byref(desc), _ptr(y_slot), _ptr(topk_ids), _ptr(topk_gates), _ptr(slot_to_row),
                              _ptr(x), _ptr(out), _stream(stream)), "zeda_combine")


def zeda_moe_forward(desc, x, w_router, router_bias, w_gate, w_up, w_down, out, num_real_out, ws,
                     stream=None) -> None:
    _check(lib().zeda_moe_forward(ctypes.byref(desc), _ptr(x), _ptr(w_router), _ptr(router_bias), _ptr(w_gate),
                                  _ptr(w_up), _ptr(w_down), _ptr(out), _ptr(num_real_out), _ptr(ws),
                                  ws.numel() * ws.element_size(), _stream(stream)), "zeda_moe_forward")


def zeda_moe_forward_events(desc, x, w_router, router_bias, w_gate, w_up, w_down, out, num_real_out, ws, events,
                            stream=None) -> None:
    """`events`: len(STAGES)+1 recorded-once torch.cuda.Event(enable_timing=True) objects."""
    arr = (ctypes.c_void_p * len(events))(*[ctypes.c_void_p(e.cuda_event) for e in events])
    _check(lib().zeda_moe_forward_events(ctypes.byref(desc), _ptr(x), _ptr(w_router), _ptr(router_bias),
                                         _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(out), _ptr(num_real_out),
                                         _ptr(ws), ws.numel() * ws.element_size(), _stream(stream), arr),
           "zeda_moe_forward_events")


def zeda_moe_block_forward(desc, xn, x_res, w_router, router_bias, w_gate, w_up, w_down, gamma_next, eps: float,
                           xn_next, num_real_out, ws, stream=None) -> None:
    """x_res += layer(xn) in place; xn_next (None to skip, may be xn itself) = RMSNorm(x_res) * gamma_next."""
    _check(lib().zeda_moe_block_forward(ctypes.byref(desc), _ptr(xn), _ptr(x_res), _ptr(w_router), _ptr(router_bias),
                                        _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(gamma_next), float(eps),
                                        _ptr(xn_next), _ptr(num_real_out), _ptr(ws), ws.numel() * ws.element_size(),
                                        _stream(stream)), "zeda_moe_block_forward")


def _dtype_of(desc: LayerDesc) -> torch.dtype:
    return torch.bfloat16 if desc.dtype == ZEDA_BF16 else torch.float32


def _dtype_code(t: torch.Tensor) -> int:
    return ZEDA_BF16 if t.dtype == torch.bfloat16 else ZEDA_F32


def zeda_rmsnorm(x, gamma, eps: float, out, stream=None) -> None:
    T, H = x.shape
    _check(lib().zeda_rmsnorm(T, H, _dtype_code(x), _ptr(x), _ptr(gamma), float(eps), _ptr(out), _stream(stream)),
           "zeda_rmsnorm")


def zeda_stream_read_probe(buf: torch.Tensor, sink: torch.Tensor, stream=None) -> None:
    """Measurement aid: one plain streaming read of all bytes of `buf` (contiguous, a multiple of 16 bytes)."""
    _check(lib().zeda_stream_read_probe(_ptr(buf), buf.numel() * buf.element_size(), _ptr(sink), _stream(stream)),
           "zeda_stream_read_probe")


def zeda_token_zero_slots(desc, topk_ids, zero_slots, accumulate: bool = False, stream=None) -> None:
    """zero_slots[t] (int32[T], device) = or += the number of token t's K slots on zero experts (Section 4.1)."""
    _check(lib().zeda_token_zero_slots(ctypes.byref(desc), _ptr(topk_ids), _ptr(zero_slots), int(bool(accumulate)),
                                       _stream(stream)), "zeda_token_zero_slots")


PROBE_READ, PROBE_MFMA, PROBE_SPLIT_SIMD = 1, 2, 4


def zeda_overlap_probe(buf: torch.Tensor, mfmas_per_wave: int, mode: int, sink: torch.Tensor, stream=None) -> None:
    """Measurement aid: streaming read of buf (a multiple of 1 MiB) and / or register-only MFMAs in one kernel.
    sink: fp32, at least (MiB of buf) * 512 + 8 elements; the last six of these hold two int64 (shader-clock cycles
    and 100 MHz ticks of one mid-launch wave)."""
    nbytes = buf.numel() * buf.element_size()
    assert sink.dtype == torch.float32 and sink.numel() >= (nbytes >> 20) * 512 + 8
    _check(lib().zeda_overlap_probe(_ptr(buf), nbytes, int(mfmas_per_wave), int(mode), _ptr(sink), _stream(stream)),
           "zeda_overlap_probe")


def zeda_mfma_probe(workgroups: int, iters: int, sink: torch.Tensor, stream=None) -> float:
    """Measurement aid: launches the register-only MFMA loop; returns the FLOPs of the launch.  sink: fp32, at least
    workgroups * 256 elements."""
    assert sink.dtype == torch.float32 and sink.numel() >= workgroups * 256
    _check(lib().zeda_mfma_probe(int(workgroups), int(iters), _ptr(sink), _stream(stream)), "zeda_mfma_probe")
    return 2.0 * 32 * 32 * 16 * 8 * iters * 4 * workgroups


def zeda_residual_add(x, y, stream=None) -> None:
    T, H = x.shape
    _check(lib().zeda_residual_add(T, H, _dtype_code(x), _ptr(x), _ptr(y), _stream(stream)), "zeda_residual_add")


def zeda_routing_stats(desc, x, w_router, router_bias, alpha=1.0, w=1.0, stream=None):
    """Section 2.2 statistics over the batch of all tokens; allocates the outputs and the scratch.
    Returns device tensors (f[N+Z], P[N+Z], summary[7] = f_E, P_E, f_Z, P_Z, r_ZE, L_A, L_GA)."""
    NE = desc.N + desc.Z
    nbytes = int(lib().zeda_routing_stats_workspace_bytes(ctypes.byref(desc)))
    with _on(stream):
        f = torch.empty(NE, dtype=torch.float32, device=x.device)
        P = torch.empty(NE, dtype=torch.float32, device=x.device)
        summary = torch.empty(7, dtype=torch.float32, device=x.device)
        ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=x.device)
    _check(lib().zeda_routing_stats(ctypes.byref(desc), _ptr(x), _ptr(w_router), _ptr(router_bias), float(alpha), float(w),
                                    _ptr(f), _ptr(P), _ptr(summary), _ptr(ws), ws.numel(), _stream(stream)),
           "zeda_routing_stats")
    return f, P, summary


def zeda_init_zero_expert_rows(desc, w_router, normals, stream=None):
    """Fills rows N.. of w_router in place (see include/zeda.h); returns the device tensor {mean, variance}."""
    with _on(stream):
        stats = torch.empty(2, dtype=torch.float32, device=w_router.device)
    _check(lib().zeda_init_zero_expert_rows(ctypes.byref(desc), _ptr(w_router), _ptr(normals), _ptr(stats), _stream(stream)),
           "zeda_init_zero_expert_rows")
    return stats


def zeda_pack_expert_weights(desc, w_gate, w_up, w_down, stream=None):
    """Tiled copies of the three expert tensors (any of them may be None); allocates the outputs."""
    with _on(stream):
        outs = [None if w is None else torch.empty_like(w) for w in (w_gate, w_up, w_down)]
    _check(lib().zeda_pack_expert_weights(ctypes.byref(desc), _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(outs[0]),
                                          _ptr(outs[1]), _ptr(outs[2]), _stream(stream)), "zeda_pack_expert_weights")
    return tuple(outs)


def _need(ok: bool, where: str) -> None:
    """What the C side cannot see of a tensor (type, shape, strides)."""
    if not ok:
        raise ZedaError(ZEDA_EINVAL, where)


def _typed(where: str, *args) -> None:
    """(tensor or None, type, elements): types and sizes that the C side cannot see of a pointer."""
    for t, dtype, n in args:
        _need(t is None or (t.dtype == dtype and t.numel() >= n and t.is_contiguous()), where)


def _is_float_buffer(t, dim: int) -> bool:
    return t.dim() == dim and t.dtype in (torch.bfloat16, torch.float32) and t.is_contiguous()


def zeda_quantize_rows_fp8(x, stream=None):
    """x [rows, cols] (bf16 or fp32, contiguous) -> (q float8_e4m3fn [rows, cols], scales uint8 [rows, ceil(cols / 128)]):
    x is nearly q * 2^(scale - 127)."""
    _need(_is_float_buffer(x, 2), "zeda_quantize_rows_fp8")
    rows, cols = x.shape
    with _on(stream):
        q = torch.empty((rows, cols), dtype=torch.float8_e4m3fn, device=x.device)
        scales = torch.empty((rows, -(-cols // 128)), dtype=torch.uint8, device=x.device)
    _check(lib().zeda_quantize_rows_fp8(rows, cols, _dtype_code(x), _ptr(x), _ptr(q), _ptr(scales), _stream(stream)), "zeda_quantize_rows_fp8")
    return q, scales


def zeda_quantize_weights_fp8(w, stream=None):
    """w [count, rows, cols] (bf16 or fp32, contiguous) -> (q float8_e4m3fn like w, scales uint8 [count, ceil(rows / 128), ceil(cols / 128)])."""
    _need(_is_float_buffer(w, 3), "zeda_quantize_weights_fp8")
    count, rows, cols = w.shape
    with _on(stream):
        q = torch.empty((count, rows, cols), dtype=torch.float8_e4m3fn, device=w.device)
        scales = torch.empty((count, -(-rows // 128), -(-cols // 128)), dtype=torch.uint8, device=w.device)
    _check(lib().zeda_quantize_weights_fp8(count, rows, cols, _dtype_code(w), _ptr(w), _ptr(q), _ptr(scales), _stream(stream)),
           "zeda_quantize_weights_fp8")
    return q, scales


def fp8_expert_bytes(desc: LayerDesc) -> Tuple[int, ...]:
    """Sizes of the four buffers of packed 8-bit expert weights, in the order of Fp8Experts' fields."""
    sizes = (ctypes.c_size_t * 4)()
    _check(lib().zeda_fp8_expert_bytes(ctypes.byref(desc), sizes), "zeda_fp8_expert_bytes")
    return tuple(sizes)


def zeda_pack_expert_weights_fp8(desc, q_gate, s_gate, q_up, s_up, q_down, s_down, stream=None) -> Fp8Experts:
    """The experts' 8-bit weights in the layout of the kernels (allocates the buffers); row-major inputs as
    zeda_quantize_weights_fp8 gives them: q_gate, q_up [N, I, H], q_down [N, H, I]."""
    N, H, I, Ib = desc.N, desc.H, desc.I, -(-desc.I // 128)
    for t, shape in ((q_gate, (N, I, H)), (s_gate, (N, Ib, H // 128)), (q_up, (N, I, H)), (s_up, (N, Ib, H // 128)), (q_down, (N, H, I)),
                     (s_down, (N, H // 128, Ib))):
        _need(tuple(t.shape) == shape and t.element_size() == 1 and t.is_contiguous(), "zeda_pack_expert_weights_fp8")
    with _on(stream):
        e = Fp8Experts([torch.empty(n, dtype=torch.uint8, device=q_gate.device) for n in fp8_expert_bytes(desc)], desc)
    _check(lib().zeda_pack_expert_weights_fp8(ctypes.byref(desc), _ptr(q_gate), _ptr(s_gate), _ptr(q_up), _ptr(s_up), _ptr(q_down), _ptr(s_down),
                                              ctypes.byref(e), _stream(stream)), "zeda_pack_expert_weights_fp8")
    return e


def workspace_bytes_fp8(desc: LayerDesc) -> int:
    return int(lib().zeda_workspace_bytes_fp8(ctypes.byref(desc)))


def expert_ffn_workspace_bytes_fp8(desc: LayerDesc) -> int:
    return int(lib().zeda_expert_ffn_workspace_bytes_fp8(ctypes.byref(desc)))


def workspace_layout_fp8(desc: LayerDesc) -> WsLayout:
    out = WsLayout()
    _check(lib().zeda_workspace_layout_fp8(ctypes.byref(desc), ctypes.byref(out)), "zeda_workspace_layout_fp8")
    return out


def zeda_expert_ffn_fp8(desc, x, experts: Fp8Experts, expert_offsets, sorted_slot, num_real, y_slot, ws, stream=None) -> None:
    S, dt, i32 = desc.T * desc.K, _dtype_of(desc), torch.int32
    _typed("zeda_expert_ffn_fp8", (x, dt, desc.T * desc.H), (expert_offsets, i32, desc.N + 1), (sorted_slot, i32, S), (num_real, i32, 1), (y_slot, dt, S * desc.H))
    experts.check(desc, "zeda_expert_ffn_fp8")
    _check(lib().zeda_expert_ffn_fp8(ctypes.byref(desc), _ptr(x), ctypes.byref(experts), _ptr(expert_offsets), _ptr(sorted_slot), _ptr(num_real),
                                     _ptr(y_slot), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)), "zeda_expert_ffn_fp8")


def zeda_moe_forward_fp8(desc, x, w_router, router_bias, experts: Fp8Experts, out, num_real_out, ws, stream=None) -> None:
    n, NE, dt = desc.T * desc.H, desc.N + desc.Z, _dtype_of(desc)
    _typed("zeda_moe_forward_fp8", (x, dt, n), (w_router, dt, NE * desc.H), (router_bias, torch.float32, NE), (out, dt, n), (num_real_out, torch.int32, 1))
    experts.check(desc, "zeda_moe_forward_fp8")
    _check(lib().zeda_moe_forward_fp8(ctypes.byref(desc), _ptr(x), _ptr(w_router), _ptr(router_bias), ctypes.byref(experts), _ptr(out),
                                      _ptr(num_real_out), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)), "zeda_moe_forward_fp8")


def zeda_moe_block_forward_fp8(desc, xn, x_res, w_router, router_bias, experts: Fp8Experts, gamma_next, eps: float, xn_next, num_real_out, ws,
                               stream=None) -> None:
    """zeda_moe_block_forward with 8-bit experts."""
    n, NE, dt = desc.T * desc.H, desc.N + desc.Z, _dtype_of(desc)
    _typed("zeda_moe_block_forward_fp8", (xn, dt, n), (x_res, dt, n), (w_router, dt, NE * desc.H), (router_bias, torch.float32, NE), (gamma_next, dt, desc.H),
           (xn_next, dt, n), (num_real_out, torch.int32, 1))
    experts.check(desc, "zeda_moe_block_forward_fp8")
    _check(lib().zeda_moe_block_forward_fp8(ctypes.byref(desc), _ptr(xn), _ptr(x_res), _ptr(w_router), _ptr(router_bias), ctypes.byref(experts),
                                            _ptr(gamma_next), float(eps), _ptr(xn_next), _ptr(num_real_out), _ptr(ws),
                                            ws.numel() * ws.element_size(), _stream(stream)), "zeda_moe_block_forward_fp8")


def route_train_workspace_bytes(desc: LayerDesc) -> int:
    return int(lib().zeda_route_train_workspace_bytes(ctypes.byref(desc)))


def route_backward_workspace_bytes(desc: LayerDesc) -> int:
    return int(lib().zeda_route_backward_workspace_bytes(ctypes.byref(desc)))


def _token_mask(mask, T: int, where: str) -> None:
    _need(mask is None or (mask.dtype in (torch.uint8, torch.bool) and mask.numel() == T and mask.is_contiguous()), where)


def zeda_route_train(desc, x, w_router, router_bias, token_mask, alpha: float, w: float, topk_ids, topk_gates, probs, counts, mean_probs, summary,
                     ws, stream=None) -> None:
    """zeda_route that also leaves probs[T, N+Z], and over the tokens with token_mask (uint8[T] or None) != 0 counts[N+Z], mean_probs[N+Z] and
    summary[7] (as zeda_routing_stats: the balance losses are summary[5] and summary[6])."""
    S, NE, f = desc.T * desc.K, desc.N + desc.Z, torch.float32
    _token_mask(token_mask, desc.T, "zeda_route_train")
    _typed("zeda_route_train", (x, _dtype_of(desc), desc.T * desc.H), (w_router, _dtype_of(desc), NE * desc.H), (router_bias, f, NE), (topk_ids, torch.int32, S),
           (topk_gates, f, S), (probs, f, desc.T * NE), (counts, torch.int32, NE), (mean_probs, f, NE), (summary, f, 7))
    _check(lib().zeda_route_train(ctypes.byref(desc), _ptr(x), _ptr(w_router), _ptr(router_bias), _ptr(token_mask), float(alpha), float(w),
                                  _ptr(topk_ids), _ptr(topk_gates), _ptr(probs), _ptr(counts), _ptr(mean_probs), _ptr(summary), _ptr(ws),
                                  ws.numel() * ws.element_size(), _stream(stream)), "zeda_route_train")


def zeda_route_backward(desc, x, w_router, probs, topk_ids, topk_gates, token_mask, counts, alpha: float, w: float, d_loss, d_gates, dx, dw_router,
                        dbias, ws, stream=None) -> None:
    """Gradients of d_loss[0] L_A + d_loss[1] L_GA + <d_gates, topk_gates>: dx (type of x), dw_router and dbias (fp32); each may be None."""
    S, NE, f, dt = desc.T * desc.K, desc.N + desc.Z, torch.float32, _dtype_of(desc)
    _token_mask(token_mask, desc.T, "zeda_route_backward")
    _typed("zeda_route_backward", (x, dt, desc.T * desc.H), (w_router, dt, NE * desc.H), (probs, f, desc.T * NE), (topk_ids, torch.int32, S), (topk_gates, f, S),
           (counts, torch.int32, NE), (d_loss, f, 2), (d_gates, f, S), (dx, dt, desc.T * desc.H), (dw_router, f, NE * desc.H), (dbias, f, NE))
    _check(lib().zeda_route_backward(ctypes.byref(desc), _ptr(x), _ptr(w_router), _ptr(probs), _ptr(topk_ids), _ptr(topk_gates), _ptr(token_mask),
                                     _ptr(counts), float(alpha), float(w), _ptr(d_loss), _ptr(d_gates), _ptr(dx), _ptr(dw_router), _ptr(dbias),
                                     _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)), "zeda_route_backward")


def zeda_combine_backward(desc, d_out, y_slot, topk_ids, topk_gates, slot_to_row, x, d_gates, d_y_slot, dx, stream=None) -> None:
    """Backward of zeda_combine.  d_y_slot may be None; x and dx belong to EXPERT_COPY (None otherwise, dx None if not wanted)."""
    S, f, dt = desc.T * desc.K, torch.float32, _dtype_of(desc)
    _typed("zeda_combine_backward", (d_out, dt, desc.T * desc.H), (y_slot, dt, S * desc.H), (topk_ids, torch.int32, S), (topk_gates, f, S), (slot_to_row, torch.int32, S),
           (x, dt, desc.T * desc.H), (d_gates, f, S), (d_y_slot, dt, S * desc.H), (dx, dt, desc.T * desc.H))
    _check(lib().zeda_combine_backward(ctypes.byref(desc), _ptr(d_out), _ptr(y_slot), _ptr(topk_ids), _ptr(topk_gates), _ptr(slot_to_row), _ptr(x),
                                       _ptr(d_gates), _ptr(d_y_slot), _ptr(dx), _stream(stream)), "zeda_combine_backward")


def ws_views(desc: LayerDesc, ws: torch.Tensor, fp8: bool = False):
    """Typed views of the intermediate results zeda_moe_forward leaves in its workspace (fp8: zeda_moe_forward_fp8, whose
    activations and expert outputs are in forms of the kernels' own: only the routing)."""
    L = workspace_layout_fp8(desc) if fp8 else workspace_layout(desc)
    S = desc.T * desc.K
    dt = torch.bfloat16 if desc.dtype == ZEDA_BF16 else torch.float32
    es = 2 if desc.dtype == ZEDA_BF16 else 4
    b = ws.view(torch.uint8)

    def view(off, n, dtype, size):
        return b[off: off + n * size].view(dtype)

    views = {
        "topk_ids": view(L.topk_ids, S, torch.int32, 4).view(desc.T, desc.K),
        "topk_gates": view(L.topk_gates, S, torch.float32, 4).view(desc.T, desc.K),
        "expert_offsets": view(L.expert_offsets, desc.N + 1, torch.int32, 4),
        "sorted_slot": view(L.sorted_slot, S, torch.int32, 4),
        "slot_to_row": view(L.slot_to_row, S, torch.int32, 4),
        "num_real": view(L.num_real, 1, torch.int32, 4),
    }
    if not fp8:
        views["act"] = view(L.act, S * desc.I, dt, es).view(S, desc.I)
        views["y_slot"] = view(L.y_slot, S * desc.H, dt, es).view(S, desc.H)
    return views
