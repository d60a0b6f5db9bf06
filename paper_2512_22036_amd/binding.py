"""Python binding of libfusco.so (ctypes; the shuffle's calls through _fastcall): same names as the C boundary, argument
marshalling only.

Every step of the shuffle runs in the library's HIP kernels.  This module checks tensor shapes
against the layout (the C side sees bare pointers), passes pointers and the current HIP stream,
and turns negative return codes into FuscoError.  It never computes on the data and has no
fallback path: a missing library is an error.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from types import SimpleNamespace
from typing import Optional

import torch

BF16, F32, E4M3 = 0, 1, 2
DISPATCH_EXPERT, DISPATCH_WIRE, DISPATCH_TWO_HOP, DISPATCH_STREAMING = 1, 2, 4, 8
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
GATE_NONE, GATE_CHANNEL, GATE_TOKEN = 0, 1, 2

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libfusco.so")

EXPORTS = ("fusco_version", "fusco_status_string", "fusco_layout_bytes", "fusco_scratch_bytes",
           "fusco_layout_bind", "fusco_plan", "fusco_plan_static", "fusco_dispatch", "fusco_dispatch_in_transfer_order", "fusco_combine", "fusco_plan_dispatch", "fusco_probe_copy", "fusco_probe_rows", "fusco_probe_pieces", "fusco_probe_consume_slices", "fusco_probe_time_next_call", "fusco_probe_source_chunk_bytes", "fusco_probe_dispatch_kernel", "fusco_probe_dispatch_occupancy", "fusco_probe_dispatch_pull", "fusco_probe_dispatch_walk", "fusco_probe_dispatch_route", "fusco_probe_plan_through", "fusco_probe_plan_dispatch_through", "fusco_probe_segments_wide", "fusco_probe_experts_tile_rows", "fusco_probe_experts_tile_outputs",
           "fusco_combine_two_hop", "fusco_balance_groups", "fusco_cross_node_load", "fusco_segments_scan", "fusco_segments_copy",
           "fusco_disaggregated_plan", "fusco_disaggregated_dispatch", "fusco_disaggregated_combine",
           "fusco_combine_backward", "fusco_route", "fusco_route_backward", "fusco_norm_before", "fusco_norm_after", "fusco_norm_scratch_bytes",
           "fusco_norm_before_backward", "fusco_norm_after_backward",
           "fusco_experts_gated", "fusco_experts_linear", "fusco_experts_input_grad", "fusco_experts_weight_grad",
           "fusco_to_fp8", "fusco_from_fp8", "fusco_experts_gated_fp8", "fusco_experts_linear_fp8",
           "fusco_experts_input_grad_fp8", "fusco_experts_weight_grad_fp8", "fusco_moe_few_scratch_bytes", "fusco_moe_few")


class FuscoError(RuntimeError):
    pass


class _CLayout(ctypes.Structure):
    """Mirror of struct fusco_layout."""
    _fields_ = [("N", ctypes.c_int32), ("k", ctypes.c_int32), ("E", ctypes.c_int32), ("D", ctypes.c_int32),
                ("P", ctypes.c_int32), ("send_cap", ctypes.c_int32),
                ("exp_count", ctypes.c_void_p), ("exp_off", ctypes.c_void_p),
                ("send_count", ctypes.c_void_p), ("send_off", ctypes.c_void_p),
                ("pair_slot", ctypes.c_void_p), ("slot_pair", ctypes.c_void_p),
                ("slot_token", ctypes.c_void_p), ("send_src", ctypes.c_void_p),
                ("pair_send_row", ctypes.c_void_p), ("slot_send_row", ctypes.c_void_p),
                ("pair_first", ctypes.c_void_p), ("status", ctypes.c_void_p),
                ("tile_slots", ctypes.c_void_p), ("tile_tokens", ctypes.c_int32), ("tile_count", ctypes.c_int32)]


class _CRouter(ctypes.Structure):
    """Mirror of struct fusco_router."""
    _fields_ = [(n, ctypes.c_int32) for n in ("N", "E", "k", "score", "groups", "keep_groups", "group_best", "renorm", "logits_dtype")] + [
        ("scale", ctypes.c_float), ("logits_stride", ctypes.c_int64)]


class _CNorm(ctypes.Structure):
    """Mirror of struct fusco_norm."""
    _fields_ = [(n, ctypes.c_int32) for n in ("N", "H", "stream_dtype", "block_dtype", "gain_dtype", "gate_kind")] + [
        ("scale", ctypes.c_float), ("eps", ctypes.c_float)]


class _CFp8(ctypes.Structure):
    """Mirror of struct fusco_fp8."""
    _fields_ = [("rows", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("columns", "dtype", "matrix_rows", "scale_stride")]


class _CFew(ctypes.Structure):
    """Mirror of struct fusco_few."""
    _fields_ = [(n, ctypes.c_int32) for n in ("N", "E", "k", "H", "I", "weight_dtype", "out_dtype")]


_lib = None
_fast = None   # csrc/fastcall.cpp, bound to _lib


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load libfusco.so (built by paper_2512_22036_amd.build / __graft_entry__.build)."""
    global _lib, _fast
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FuscoError("libfusco.so is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                         "(there is no fallback path)")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, sz, u32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_uint32
    lib.fusco_version.restype = ctypes.c_int
    lib.fusco_version.argtypes = []
    lib.fusco_status_string.restype = ctypes.c_char_p
    lib.fusco_status_string.argtypes = [ctypes.c_int]
    lib.fusco_layout_bytes.restype = sz
    lib.fusco_layout_bytes.argtypes = [i32, i32, i32, i32]
    lib.fusco_scratch_bytes.restype = sz
    lib.fusco_scratch_bytes.argtypes = [i32, i32, i32, i32]
    lib.fusco_layout_bind.restype = ctypes.c_int
    lib.fusco_layout_bind.argtypes = [ctypes.POINTER(_CLayout), i32, i32, i32, i32, vp, sz]
    lib.fusco_plan.restype = ctypes.c_int
    lib.fusco_plan.argtypes = [ctypes.POINTER(_CLayout), vp, vp, sz, vp]
    lib.fusco_plan_static.restype = ctypes.c_int
    lib.fusco_plan_static.argtypes = [ctypes.POINTER(_CLayout), vp, vp]
    lib.fusco_dispatch.restype = ctypes.c_int
    lib.fusco_dispatch.argtypes = [ctypes.POINTER(_CLayout), vp, sz, vp, sz, vp, vp, vp, vp, u32, vp]
    lib.fusco_dispatch_in_transfer_order.restype = ctypes.c_int
    lib.fusco_dispatch_in_transfer_order.argtypes = [ctypes.POINTER(_CLayout), sz, sz, u32]
    lib.fusco_plan_dispatch.restype = ctypes.c_int
    lib.fusco_plan_dispatch.argtypes = [ctypes.POINTER(_CLayout), vp, vp, sz, vp, sz, vp, vp, vp]
    lib.fusco_combine.restype = ctypes.c_int
    lib.fusco_combine.argtypes = [ctypes.POINTER(_CLayout), vp, ctypes.c_int, vp, vp, ctypes.c_int, i32, u32, vp]
    lib.fusco_probe_copy.restype = ctypes.c_int
    lib.fusco_probe_copy.argtypes = [vp, vp, sz, vp]
    lib.fusco_probe_dispatch_kernel.restype = ctypes.c_int
    lib.fusco_probe_dispatch_kernel.argtypes = [ctypes.c_int]
    lib.fusco_probe_dispatch_occupancy.restype = ctypes.c_int
    lib.fusco_probe_dispatch_occupancy.argtypes = [ctypes.c_int]
    lib.fusco_probe_dispatch_walk.restype = ctypes.c_int
    lib.fusco_probe_dispatch_walk.argtypes = [ctypes.c_int]
    lib.fusco_probe_dispatch_pull.restype = ctypes.c_int
    lib.fusco_probe_dispatch_pull.argtypes = [ctypes.c_int]
    lib.fusco_probe_segments_wide.restype = ctypes.c_int
    lib.fusco_probe_segments_wide.argtypes = [ctypes.c_uint64, ctypes.c_uint64]
    lib.fusco_probe_experts_tile_rows.restype = ctypes.c_int
    lib.fusco_probe_experts_tile_rows.argtypes = [ctypes.POINTER(_CLayout), ctypes.c_int, i32, i32]
    lib.fusco_probe_experts_tile_outputs.restype = ctypes.c_int
    lib.fusco_probe_experts_tile_outputs.argtypes = [ctypes.POINTER(_CLayout), ctypes.c_int, i32, i32]
    lib.fusco_probe_plan_dispatch_through.restype = ctypes.c_int
    lib.fusco_probe_plan_dispatch_through.argtypes = [ctypes.POINTER(_CLayout), sz, sz, vp]
    lib.fusco_probe_plan_through.restype = ctypes.c_int
    lib.fusco_probe_plan_through.argtypes = [ctypes.POINTER(_CLayout)]
    lib.fusco_probe_dispatch_route.restype = ctypes.c_int
    lib.fusco_probe_dispatch_route.argtypes = [ctypes.POINTER(_CLayout), sz, sz, vp, vp, vp, vp, u32]
    lib.fusco_probe_source_chunk_bytes.restype = ctypes.c_size_t
    lib.fusco_probe_source_chunk_bytes.argtypes = [sz]
    lib.fusco_probe_time_next_call.restype = ctypes.c_int
    lib.fusco_probe_time_next_call.argtypes = [vp, vp]
    lib.fusco_probe_rows.restype = ctypes.c_int
    lib.fusco_probe_rows.argtypes = [vp, u32, vp, u32, sz, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                     vp, vp]
    lib.fusco_probe_pieces.restype = ctypes.c_int
    lib.fusco_probe_pieces.argtypes = [vp, sz, ctypes.c_int, u32, ctypes.c_int, vp, vp]
    lib.fusco_probe_consume_slices.restype = ctypes.c_int
    lib.fusco_probe_consume_slices.argtypes = [vp, ctypes.c_uint64, ctypes.c_uint64, vp, u32, vp, vp]
    lp = ctypes.POINTER(_CLayout)
    u64, i64 = ctypes.c_uint64, ctypes.c_int64
    lib.fusco_segments_scan.restype = ctypes.c_int
    lib.fusco_segments_scan.argtypes = [vp, i64, vp, vp, vp]
    lib.fusco_segments_copy.restype = ctypes.c_int
    lib.fusco_segments_copy.argtypes = [vp, u64, vp, vp, u64, vp, vp, i64, u64, u64, vp, vp, vp]
    lib.fusco_cross_node_load.restype = ctypes.c_int
    lib.fusco_cross_node_load.argtypes = [ctypes.POINTER(_CLayout), i32, i32, sz, vp, vp]
    lib.fusco_balance_groups.restype = ctypes.c_int
    lib.fusco_balance_groups.argtypes = [vp, i32, i32, vp]
    lib.fusco_combine_two_hop.restype = ctypes.c_int
    lib.fusco_combine_two_hop.argtypes = [lp, vp, ctypes.c_int, vp, vp, vp, ctypes.c_int, i32, vp]
    lib.fusco_disaggregated_plan.restype = ctypes.c_int
    lib.fusco_disaggregated_plan.argtypes = [lp, lp, vp, vp, vp, sz, vp]
    lib.fusco_disaggregated_dispatch.restype = ctypes.c_int
    lib.fusco_disaggregated_dispatch.argtypes = [lp, lp, vp, sz, vp, vp, vp, vp]
    lib.fusco_disaggregated_combine.restype = ctypes.c_int
    lib.fusco_disaggregated_combine.argtypes = [lp, lp, vp, ctypes.c_int, vp, vp, vp, vp, ctypes.c_int, i32, vp]
    rp, np_ = ctypes.POINTER(_CRouter), ctypes.POINTER(_CNorm)
    lib.fusco_combine_backward.restype = ctypes.c_int
    lib.fusco_combine_backward.argtypes = [lp, vp, ctypes.c_int, vp, vp, ctypes.c_int, vp, vp, i32, vp]
    lib.fusco_route.restype = ctypes.c_int
    lib.fusco_route.argtypes = [rp, vp, vp, vp, vp, vp]
    lib.fusco_route_backward.restype = ctypes.c_int
    lib.fusco_route_backward.argtypes = [rp, vp, vp, vp, vp, vp]
    lib.fusco_norm_scratch_bytes.restype = sz
    lib.fusco_norm_scratch_bytes.argtypes = [i32, i32]
    lib.fusco_norm_before.restype = ctypes.c_int
    lib.fusco_norm_before.argtypes = [np_, vp, vp, vp, vp]
    lib.fusco_norm_after.restype = ctypes.c_int
    lib.fusco_norm_after.argtypes = [np_, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.fusco_norm_before_backward.restype = ctypes.c_int
    lib.fusco_norm_before_backward.argtypes = [np_, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.fusco_norm_after_backward.restype = ctypes.c_int
    lib.fusco_norm_after_backward.argtypes = [np_] + [vp] * 13 + [sz, vp]
    lib.fusco_experts_gated.restype = ctypes.c_int
    lib.fusco_experts_gated.argtypes = [lp, vp, vp, vp, vp, i32, i32, vp]
    lib.fusco_experts_linear.restype = ctypes.c_int
    lib.fusco_experts_linear.argtypes = [lp, vp, vp, vp, i32, i32, vp]
    lib.fusco_experts_input_grad.restype = ctypes.c_int
    lib.fusco_experts_input_grad.argtypes = [lp, vp, vp, vp, vp, i32, i32, vp]
    lib.fusco_experts_weight_grad.restype = ctypes.c_int
    lib.fusco_experts_weight_grad.argtypes = [lp, vp, vp, vp, ctypes.c_int, i32, i32, vp]
    fp = ctypes.POINTER(_CFp8)
    lib.fusco_to_fp8.restype = ctypes.c_int
    lib.fusco_to_fp8.argtypes = [fp, vp, vp, vp, vp]
    lib.fusco_from_fp8.restype = ctypes.c_int
    lib.fusco_from_fp8.argtypes = [fp, vp, vp, vp, vp]
    lib.fusco_experts_gated_fp8.restype = ctypes.c_int
    lib.fusco_experts_gated_fp8.argtypes = [lp, vp, vp, i32, vp, vp, vp, vp, i32, i32, vp]
    lib.fusco_experts_linear_fp8.restype = ctypes.c_int
    lib.fusco_experts_linear_fp8.argtypes = [lp, vp, vp, i32, vp, vp, vp, i32, i32, vp]
    lib.fusco_experts_input_grad_fp8.restype = ctypes.c_int
    lib.fusco_experts_input_grad_fp8.argtypes = [lp, vp, vp, vp, vp, vp, i32, i32, i32, vp]
    lib.fusco_experts_weight_grad_fp8.restype = ctypes.c_int
    lib.fusco_experts_weight_grad_fp8.argtypes = [lp, vp, vp, vp, i32, vp, ctypes.c_int, i32, i32, vp]
    lib.fusco_moe_few_scratch_bytes.restype = sz
    lib.fusco_moe_few_scratch_bytes.argtypes = [i32, i32, i32]
    lib.fusco_moe_few.restype = ctypes.c_int
    lib.fusco_moe_few.argtypes = [ctypes.POINTER(_CFew)] + [vp] * 9 + [sz, vp]
    _lib = lib
    _fast = _bind_fastcall(lib)
    return lib


def _bind_fastcall(lib):
    """The module that makes the common calls without ctypes in between (csrc/fastcall.cpp), bound to the library's
    entry points; None where it was not built or this torch cannot load it, and every call goes through ctypes."""
    if not os.path.exists(os.path.join(_HERE, "_fastcall.so")):
        return None
    try:
        from . import _fastcall
    except ImportError:
        return None
    _fastcall.bind(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value
                     for name in ("fusco_plan", "fusco_dispatch", "fusco_plan_dispatch", "fusco_combine", "fusco_combine_two_hop")))
    _fastcall.bind_block(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value
                           for name in ("fusco_route", "fusco_norm_before", "fusco_norm_after", "fusco_experts_gated", "fusco_experts_linear")))
    _fastcall.bind_fp8(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in ("fusco_to_fp8", "fusco_from_fp8", "fusco_moe_few")))
    return _fastcall


def _check(rc: int, what: str) -> None:
    if rc != 0:
        raise FuscoError("%s failed: %s (%d)" % (what, load_library().fusco_status_string(rc).decode(), rc))


# handle of a device's current stream without the torch.cuda.Stream object around it (2.5 us a call, as long as a
# launch takes); absent from builds of torch without a GPU runtime, where no call gets this far
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _rows(t: torch.Tensor, name: str, min_rows: int, row_bytes: Optional[int] = None) -> int:
    if not t.is_cuda or t.dim() != 2 or not t.is_contiguous():
        raise FuscoError("%s must be a contiguous 2-D device tensor" % name)
    if t.shape[0] < min_rows:
        raise FuscoError("%s has %d rows, needs %d" % (name, t.shape[0], min_rows))
    rb = t.shape[1] * t.element_size()
    if row_bytes is not None and rb != row_bytes:
        raise FuscoError("%s rows are %d bytes, expected %d" % (name, rb, row_bytes))
    return rb


def fusco_version() -> int:
    return load_library().fusco_version()


_I32_FIELDS = {"exp_count": "E", "exp_off": "E+1", "send_count": "D", "send_off": "D+1", "pair_slot": "P",
               "slot_pair": "P", "slot_token": "P", "send_src": "send_cap", "pair_send_row": "P",
               "slot_send_row": "P", "status": "1", "tile_slots": "tiles"}


class Layout:
    """Device-resident layout descriptor: owns the device block the C struct points into and the
    planner scratch.  Arrays are exposed as torch views of that block (no copies)."""

    def __init__(self, N: int, k: int, E: int, D: int, device="cuda"):
        lib = load_library()
        nbytes = lib.fusco_layout_bytes(N, k, E, D)
        if nbytes == 0:
            raise FuscoError("invalid layout sizes N=%d k=%d E=%d D=%d" % (N, k, E, D))
        self.mem = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.scratch = torch.empty(lib.fusco_scratch_bytes(N, k, E, D), dtype=torch.uint8, device=device)
        self.c = _CLayout()
        _check(lib.fusco_layout_bind(ctypes.byref(self.c), N, k, E, D, self.mem.data_ptr(), nbytes),
               "fusco_layout_bind")
        self.N, self.k, self.E, self.D = N, k, E, D
        self.P, self.send_cap = int(self.c.P), int(self.c.send_cap)
        self.tile_tokens, self.tile_count = int(self.c.tile_tokens), int(self.c.tile_count)

    def array(self, name: str) -> torch.Tensor:
        """Torch view of one descriptor array (int32, or uint8 for pair_first)."""
        sizes = {"E": self.E, "E+1": self.E + 1, "D": self.D, "D+1": self.D + 1, "P": self.P,
                 "send_cap": self.send_cap, "1": 1, "tiles": self.tile_count * self.tile_tokens * self.k}
        off = getattr(self.c, name) - self.mem.data_ptr()
        if name == "pair_first":
            return self.mem[off:off + self.P]
        n = sizes[_I32_FIELDS[name]]
        return self.mem[off:off + 4 * n].view(torch.int32)

    def to_host(self) -> SimpleNamespace:
        """Synchronising copy of every array to numpy (send_src cut to its U valid rows)."""
        out = {n: self.array(n).cpu().numpy() for n in list(_I32_FIELDS) + ["pair_first"]}
        U = int(out["send_off"][self.D])
        out["send_src"] = out["send_src"][:max(0, min(U, self.send_cap))]
        return SimpleNamespace(N=self.N, k=self.k, E=self.E, D=self.D, P=self.P, U=U, **out)


def fusco_plan(layout: Layout, topk_idx: torch.Tensor, stream=None) -> None:
    if stream is None and _fast is not None:
        rc = _fast.plan(layout, topk_idx)
        if rc is not None:
            return _check(rc, "fusco_plan")
    if (not topk_idx.is_cuda or topk_idx.dtype != torch.int32 or not topk_idx.is_contiguous()
            or tuple(topk_idx.shape) != (layout.N, layout.k)):
        raise FuscoError("topk_idx must be a contiguous int32 device tensor of shape [N, k]")
    _check(load_library().fusco_plan(ctypes.byref(layout.c), topk_idx.data_ptr(), layout.scratch.data_ptr(),
                                     layout.scratch.numel(), _stream(stream)), "fusco_plan")


def fusco_plan_static(layout: Layout, topk_idx: torch.Tensor, stream=None) -> None:
    """fusco_plan on the library's own static scratch array: nothing is allocated or passed in."""
    if (not topk_idx.is_cuda or topk_idx.dtype != torch.int32 or not topk_idx.is_contiguous()
            or tuple(topk_idx.shape) != (layout.N, layout.k)):
        raise FuscoError("topk_idx must be a contiguous int32 device tensor of shape [N, k]")
    _check(load_library().fusco_plan_static(ctypes.byref(layout.c), topk_idx.data_ptr(), _stream(stream)),
           "fusco_plan_static")


def fusco_dispatch(layout: Layout, x: torch.Tensor, expert_buf: Optional[torch.Tensor] = None,
                   x_aux: Optional[torch.Tensor] = None, expert_aux: Optional[torch.Tensor] = None,
                   send_buf: Optional[torch.Tensor] = None, send_aux: Optional[torch.Tensor] = None,
                   flags: int = 0, stream=None) -> None:
    if stream is None and _fast is not None:
        rc = _fast.dispatch(layout, x, expert_buf, x_aux, expert_aux, send_buf, send_aux, flags)
        if rc is not None:
            return _check(rc, "fusco_dispatch")
    rb = _rows(x, "x", layout.N)
    ab = _rows(x_aux, "x_aux", layout.N) if x_aux is not None else 0
    eff = (flags & ~DISPATCH_STREAMING) or DISPATCH_EXPERT
    if eff & DISPATCH_TWO_HOP:
        eff |= DISPATCH_EXPERT | DISPATCH_WIRE
    if eff & DISPATCH_EXPERT:
        if expert_buf is None:
            raise FuscoError("expert_buf is required")
        _rows(expert_buf, "expert_buf", layout.P, rb)
        if ab:
            if expert_aux is None:
                raise FuscoError("expert_aux is required")
            _rows(expert_aux, "expert_aux", layout.P, ab)
    if eff & DISPATCH_WIRE:
        if send_buf is None:
            raise FuscoError("send_buf is required")
        _rows(send_buf, "send_buf", layout.send_cap, rb)
        if ab:
            if send_aux is None:
                raise FuscoError("send_aux is required")
            _rows(send_aux, "send_aux", layout.send_cap, ab)
    _check(load_library().fusco_dispatch(ctypes.byref(layout.c), x.data_ptr(), rb, _ptr(x_aux), ab,
                                         _ptr(expert_buf), _ptr(expert_aux), _ptr(send_buf), _ptr(send_aux),
                                         flags, _stream(stream)), "fusco_dispatch")


def fusco_dispatch_in_transfer_order(layout: Layout, row_bytes: int, aux_row_bytes: int = 0, flags: int = 0) -> bool:
    rc = load_library().fusco_dispatch_in_transfer_order(ctypes.byref(layout.c), row_bytes, aux_row_bytes, flags)
    if rc < 0:
        _check(rc, "fusco_dispatch_in_transfer_order")
    return bool(rc)


def fusco_plan_dispatch(layout: Layout, topk_idx: torch.Tensor, x: torch.Tensor, expert_buf: torch.Tensor,
                        x_aux: Optional[torch.Tensor] = None, expert_aux: Optional[torch.Tensor] = None,
                        stream=None) -> None:
    """fusco_plan and fusco_dispatch (expert tensor only) in one launch; inputs of one planner tile only
    (N <= 2048 // k), FuscoError otherwise."""
    if stream is None and _fast is not None:
        rc = _fast.plan_dispatch(layout, topk_idx, x, expert_buf, x_aux, expert_aux)
        if rc is not None:
            return _check(rc, "fusco_plan_dispatch")
    if (not topk_idx.is_cuda or topk_idx.dtype != torch.int32 or not topk_idx.is_contiguous()
            or tuple(topk_idx.shape) != (layout.N, layout.k)):
        raise FuscoError("topk_idx must be a contiguous int32 device tensor of shape [N, k]")
    rb = _rows(x, "x", layout.N)
    ab = _rows(x_aux, "x_aux", layout.N) if x_aux is not None else 0
    _rows(expert_buf, "expert_buf", layout.P, rb)
    if ab:
        if expert_aux is None:
            raise FuscoError("expert_aux is required")
        _rows(expert_aux, "expert_aux", layout.P, ab)
    _check(load_library().fusco_plan_dispatch(ctypes.byref(layout.c), topk_idx.data_ptr(), x.data_ptr(), rb,
                                              _ptr(x_aux), ab, expert_buf.data_ptr(), _ptr(expert_aux),
                                              _stream(stream)), "fusco_plan_dispatch")


def _dtype_code(t: torch.Tensor, name: str) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise FuscoError("%s must be bfloat16 or float32" % name)


def fusco_combine(layout: Layout, y: torch.Tensor, w: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    if stream is None and _fast is not None:
        rc = _fast.combine(layout, y, w, out)
        if rc is not None:
            return _check(rc, "fusco_combine")
    _rows(y, "y", layout.P)
    H = y.shape[1]
    _rows(out, "out", layout.N)
    if out.shape[1] != H:
        raise FuscoError("out must have %d columns" % H)
    if (not w.is_cuda or w.dtype != torch.float32 or not w.is_contiguous()
            or tuple(w.shape) != (layout.N, layout.k)):
        raise FuscoError("w must be a contiguous float32 device tensor of shape [N, k]")
    _check(load_library().fusco_combine(ctypes.byref(layout.c), y.data_ptr(), _dtype_code(y, "y"), w.data_ptr(),
                                        out.data_ptr(), _dtype_code(out, "out"), H, 0, _stream(stream)),
           "fusco_combine")


def fusco_combine_backward(layout: Layout, y: torch.Tensor, w: torch.Tensor, dout: torch.Tensor, dy: torch.Tensor,
                           dw: torch.Tensor, stream=None) -> None:
    """Gradients of fusco_combine: dout [N, H] in, dy [P, H] (of y's type) and dw [N, k] float32 out."""
    _rows(y, "y", layout.P)
    _rows(dy, "dy", layout.P)
    _rows(dout, "dout", layout.N)
    H = y.shape[1]
    if dy.dtype != y.dtype or dy.shape[1] != H or dout.shape[1] != H:
        raise FuscoError("dy must be of y's type, dy and dout must have %d columns" % H)
    for t, name in ((w, "w"), (dw, "dw")):
        _fp32(t, name, (layout.N, layout.k))
    _check(load_library().fusco_combine_backward(ctypes.byref(layout.c), y.data_ptr(), _dtype_code(y, "y"), w.data_ptr(),
                                                 dout.data_ptr(), _dtype_code(dout, "dout"), dy.data_ptr(), dw.data_ptr(), H,
                                                 _stream(stream)), "fusco_combine_backward")


def _fp32(t: torch.Tensor, name: str, shape) -> torch.Tensor:
    if not t.is_cuda or t.dtype != torch.float32 or not t.is_contiguous() or tuple(t.shape) != tuple(shape):
        raise FuscoError("%s must be a contiguous float32 device tensor of shape %s" % (name, list(shape)))
    return t


def _router(logits: torch.Tensor, topk_idx: torch.Tensor, score: int, groups: int, keep_groups: int, group_best: int,
            renorm: bool, scale: float) -> _CRouter:
    if not logits.is_cuda or logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise FuscoError("logits must be a 2-D device tensor whose rows are contiguous")
    N, E = logits.shape
    if (not topk_idx.is_cuda or topk_idx.dtype != torch.int32 or not topk_idx.is_contiguous() or topk_idx.dim() != 2
            or topk_idx.shape[0] != N):
        raise FuscoError("topk_idx must be a contiguous int32 device tensor of shape [N, k]")
    stride = logits.stride(0) if N > 1 else max(E, 1)
    return _CRouter(N, E, topk_idx.shape[1], score, groups, keep_groups, group_best, int(bool(renorm)), _dtype_code(logits, "logits"),
                    scale, stride)


def fusco_route(logits: torch.Tensor, topk_idx: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None,
                score: int = SCORE_SOFTMAX, groups: int = 1, keep_groups: int = 1, group_best: int = 1, renorm: bool = True,
                scale: float = 1.0, stream=None) -> None:
    """Routing: logits [N, E] (bfloat16 or float32, rows may lie apart) to topk_idx [N, k] int32 and w [N, k] float32, as
    fusco_plan and fusco_combine take them.  bias: float32 [E], added to the scores for the choice alone."""
    if stream is None and _fast is not None:
        rc = _fast.route(logits, topk_idx, w, bias, score, groups, keep_groups, group_best, renorm, scale)
        if rc is not None:
            return _check(rc, "fusco_route")
    R = _router(logits, topk_idx, score, groups, keep_groups, group_best, renorm, scale)
    _fp32(w, "w", topk_idx.shape)
    if bias is not None:
        _fp32(bias, "bias", (R.E,))
    _check(load_library().fusco_route(ctypes.byref(R), logits.data_ptr(), _ptr(bias), topk_idx.data_ptr(), w.data_ptr(),
                                      _stream(stream)), "fusco_route")


def fusco_route_backward(logits: torch.Tensor, topk_idx: torch.Tensor, dw: torch.Tensor, dlogits: torch.Tensor,
                         score: int = SCORE_SOFTMAX, renorm: bool = True, scale: float = 1.0, stream=None) -> None:
    """Gradient of fusco_route's weights: dw [N, k] float32 to dlogits [N, E], contiguous and of logits' type."""
    R = _router(logits, topk_idx, score, 1, 1, 1, renorm, scale)
    _fp32(dw, "dw", topk_idx.shape)
    if not dlogits.is_cuda or dlogits.dtype != logits.dtype or dlogits.shape != logits.shape or not dlogits.is_contiguous():
        raise FuscoError("dlogits must be a contiguous device tensor of logits' shape and type")
    _check(load_library().fusco_route_backward(ctypes.byref(R), logits.data_ptr(), topk_idx.data_ptr(), dw.data_ptr(),
                                               dlogits.data_ptr(), _stream(stream)), "fusco_route_backward")


def _norm(stream: torch.Tensor, block_dtype: torch.dtype, params, gate: Optional[torch.Tensor], gate_kind: Optional[int],
          scale: float, eps: float) -> _CNorm:
    """The struct for rows like `stream` [N, H]; params: (name, tensor or None) of [H] each, of one type with the gate."""
    if not stream.is_cuda or stream.dim() != 2 or not stream.is_contiguous():
        raise FuscoError("the stream must be a contiguous 2-D device tensor")
    N, H = stream.shape
    given = [(n, t) for n, t in params if t is not None]
    kind = GATE_NONE
    if gate is not None:
        kind = gate_kind
        if kind is None:
            if N == H:
                raise FuscoError("gate [%d] may be per channel or per token: give gate_kind" % N)
            kind = GATE_TOKEN if gate.dim() == 1 and gate.shape[0] == N else GATE_CHANNEL
        if kind not in (GATE_CHANNEL, GATE_TOKEN):
            raise FuscoError("gate_kind must be GATE_CHANNEL or GATE_TOKEN")
    for name, t in given + ([("gate", gate)] if gate is not None else []):
        want = N if name == "gate" and kind == GATE_TOKEN else H
        if not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != (want,) or t.dtype != given[0][1].dtype:
            raise FuscoError("%s must be a contiguous device tensor of shape [%d], gains and gate of one type" % (name, want))
    code = {torch.bfloat16: BF16, torch.float32: F32}
    if stream.dtype not in code or block_dtype not in code or given[0][1].dtype not in code:
        raise FuscoError("tensors must be bfloat16 or float32")
    return _CNorm(N, H, code[stream.dtype], code[block_dtype], code[given[0][1].dtype], kind, scale, eps)


def _like(n: _CNorm, dtype: torch.dtype, **tensors) -> None:
    for name, t in tensors.items():
        if t is not None and (not t.is_cuda or t.dtype != dtype or not t.is_contiguous() or tuple(t.shape) != (n.N, n.H)):
            raise FuscoError("%s must be a contiguous %s device tensor of shape [%d, %d]" % (name, dtype, n.N, n.H))


def fusco_norm_before(x: torch.Tensor, gain: torch.Tensor, out: torch.Tensor, eps: float = 1e-6, stream=None) -> None:
    """out = x / sqrt(mean(x^2) + eps) * gain, row by row: the norm before a block; x is the residual stream."""
    if stream is None and _fast is not None:
        rc = _fast.norm_before(x, gain, out, eps)
        if rc is not None:
            return _check(rc, "fusco_norm_before")
    n = _norm(x, out.dtype, [("gain", gain)], None, None, 1.0, eps)
    _like(n, out.dtype, out=out)
    _check(load_library().fusco_norm_before(ctypes.byref(n), x.data_ptr(), gain.data_ptr(), out.data_ptr(), _stream(stream)),
           "fusco_norm_before")


def fusco_norm_after(r: torch.Tensor, y: torch.Tensor, gain: torch.Tensor, out: torch.Tensor, gate: Optional[torch.Tensor] = None,
                     scale: float = 1.0, next_gain: Optional[torch.Tensor] = None, next_out: Optional[torch.Tensor] = None,
                     eps: float = 1e-6, gate_kind: Optional[int] = None, stream=None) -> None:
    """out = r + scale * gate * norm(y) * gain: the norm after a block, its gate and the sum with the residual stream r; with
    next_out also the norm before the next block, norm(out) * next_gain.  gate: [H] (per channel) or [N] (per token);
    gate_kind says which where N == H."""
    if stream is None and _fast is not None:
        rc = _fast.norm_after(r, y, gain, out, gate, scale, next_gain, next_out, eps, gate_kind)
        if rc is not None:
            return _check(rc, "fusco_norm_after")
    if (next_gain is None) != (next_out is None):
        raise FuscoError("next_gain and next_out go together")
    n = _norm(r, y.dtype, [("gain", gain), ("next_gain", next_gain)], gate, gate_kind, scale, eps)
    _like(n, r.dtype, out=out)
    _like(n, y.dtype, y=y, next_out=next_out)
    _check(load_library().fusco_norm_after(ctypes.byref(n), r.data_ptr(), y.data_ptr(), gain.data_ptr(), _ptr(gate), out.data_ptr(),
                                           _ptr(next_gain), _ptr(next_out), _stream(stream)), "fusco_norm_after")


def fusco_norm_scratch_bytes(N: int, H: int) -> int:
    return load_library().fusco_norm_scratch_bytes(N, H)


def _norm_scratch(n: _CNorm, scratch: Optional[torch.Tensor], device, stream) -> torch.Tensor:
    return _scratch(fusco_norm_scratch_bytes(n.N, n.H), scratch, device, stream)


def _scratch(nbytes: int, scratch: Optional[torch.Tensor], device, stream) -> torch.Tensor:
    """The caller's scratch, or one for this call alone.  That one is given up when the call returns, with its kernels still to
    run: it is made on their stream, whose later work is all that may get the block again."""
    if scratch is None:
        own = contextlib.nullcontext()
        if stream is not None:
            own = torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(_stream(stream), device=device))
        with own:
            return torch.empty(nbytes, dtype=torch.uint8, device=device)
    if not scratch.is_cuda or not scratch.is_contiguous():
        raise FuscoError("scratch must be a contiguous device tensor")
    return scratch


def fusco_norm_before_backward(dout: torch.Tensor, x: torch.Tensor, gain: torch.Tensor, dx: torch.Tensor, dgain: torch.Tensor,
                               dres: Optional[torch.Tensor] = None, eps: float = 1e-6, scratch: Optional[torch.Tensor] = None,
                               stream=None) -> None:
    """Gradients of fusco_norm_before: dx = dres + what comes through the norm, dgain float32 [H].  dres: the gradient that
    reaches x past the block.  scratch: fusco_norm_scratch_bytes(N, H) bytes, made here on the call's stream if not given."""
    n = _norm(x, dout.dtype, [("gain", gain)], None, None, 1.0, eps)
    _like(n, dout.dtype, dout=dout)
    _like(n, x.dtype, dx=dx, dres=dres)
    _fp32(dgain, "dgain", (n.H,))
    scratch = _norm_scratch(n, scratch, x.device, stream)
    _check(load_library().fusco_norm_before_backward(ctypes.byref(n), dout.data_ptr(), x.data_ptr(), gain.data_ptr(), _ptr(dres),
                                                     dx.data_ptr(), dgain.data_ptr(), scratch.data_ptr(),
                                                     scratch.numel() * scratch.element_size(), _stream(stream)),
           "fusco_norm_before_backward")


def fusco_norm_after_backward(dout: Optional[torch.Tensor], y: torch.Tensor, gain: torch.Tensor, dr: torch.Tensor, dy: torch.Tensor,
                              dgain: torch.Tensor, gate: Optional[torch.Tensor] = None, dgate: Optional[torch.Tensor] = None,
                              scale: float = 1.0, dnext: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                              next_gain: Optional[torch.Tensor] = None, dnext_gain: Optional[torch.Tensor] = None,
                              eps: float = 1e-6, gate_kind: Optional[int] = None, scratch: Optional[torch.Tensor] = None,
                              stream=None) -> None:
    """Gradients of fusco_norm_after: dr and dy [N, H], dgain, dgate and dnext_gain float32.  dnext, out (as fusco_norm_after
    wrote it), next_gain and dnext_gain go together; dout may be None beside them."""
    asked = [t is not None for t in (dnext, out, next_gain, dnext_gain)]
    if any(asked) != all(asked) or (dout is None and dnext is None):
        raise FuscoError("dnext, out, next_gain and dnext_gain go together, and dout or dnext must be given")
    if (gate is None) != (dgate is None):
        raise FuscoError("gate and dgate go together")
    n = _norm(dr, y.dtype, [("gain", gain), ("next_gain", next_gain)], gate, gate_kind, scale, eps)
    _like(n, dr.dtype, dout=dout, out=out)
    _like(n, y.dtype, y=y, dy=dy, dnext=dnext)
    _fp32(dgain, "dgain", (n.H,))
    if dnext is not None:
        _fp32(dnext_gain, "dnext_gain", (n.H,))
    if gate is not None:
        _fp32(dgate, "dgate", gate.shape)
    scratch = _norm_scratch(n, scratch, dr.device, stream)
    _check(load_library().fusco_norm_after_backward(ctypes.byref(n), _ptr(dout), _ptr(dnext), y.data_ptr(), _ptr(out), gain.data_ptr(),
                                                    _ptr(gate), _ptr(next_gain), dr.data_ptr(), dy.data_ptr(), dgain.data_ptr(),
                                                    _ptr(dgate), _ptr(dnext_gain), scratch.data_ptr(),
                                                    scratch.numel() * scratch.element_size(), _stream(stream)),
           "fusco_norm_after_backward")


def _bf16(t: torch.Tensor, name: str, shape) -> torch.Tensor:
    if not t.is_cuda or t.dtype != torch.bfloat16 or not t.is_contiguous() or tuple(t.shape) != tuple(shape):
        raise FuscoError("%s must be a contiguous bfloat16 device tensor of shape %s" % (name, list(shape)))
    return t


def _weights(layout: Layout, w: torch.Tensor, name: str):
    if w.dim() != 3 or w.shape[0] != layout.E:
        raise FuscoError("%s must have three dimensions, the first of them the %d experts" % (name, layout.E))
    return _bf16(w, name, w.shape)


def fusco_experts_gated(layout: Layout, x: torch.Tensor, w: torch.Tensor, h: torch.Tensor, pre: Optional[torch.Tensor] = None,
                        stream=None) -> None:
    """h = silu(x Wg^T) * (x Wu^T), expert by expert: x [P, H] as fusco_dispatch wrote it, w [E, 2 I, H] with the gate rows
    first, h [P, I], all bfloat16.  pre [P, 2 I]: also keep both factors before the activation, for the gradient."""
    if stream is None and _fast is not None:
        rc = _fast.experts_gated(layout, x, w, h, pre)
        if rc is not None:
            return _check(rc, "fusco_experts_gated")
    _weights(layout, w, "w")
    I, H = w.shape[1] // 2, w.shape[2]
    if w.shape[1] % 2:
        raise FuscoError("w must have an even number of rows per expert")
    _bf16(x, "x", (layout.P, H))
    _bf16(h, "h", (layout.P, I))
    if pre is not None:
        _bf16(pre, "pre", (layout.P, 2 * I))
    _check(load_library().fusco_experts_gated(ctypes.byref(layout.c), x.data_ptr(), w.data_ptr(), h.data_ptr(), _ptr(pre), H, I,
                                              _stream(stream)), "fusco_experts_gated")


def fusco_experts_linear(layout: Layout, x: torch.Tensor, w: torch.Tensor, y: torch.Tensor, stream=None) -> None:
    """y = x W^T, expert by expert: x [P, C], w [E, M, C], y [P, M], all bfloat16."""
    if stream is None and _fast is not None:
        rc = _fast.experts_linear(layout, x, w, y)
        if rc is not None:
            return _check(rc, "fusco_experts_linear")
    _weights(layout, w, "w")
    M, C = w.shape[1], w.shape[2]
    _bf16(x, "x", (layout.P, C))
    _bf16(y, "y", (layout.P, M))
    _check(load_library().fusco_experts_linear(ctypes.byref(layout.c), x.data_ptr(), w.data_ptr(), y.data_ptr(), C, M,
                                               _stream(stream)), "fusco_experts_linear")


def fusco_experts_input_grad(layout: Layout, dy: torch.Tensor, w: torch.Tensor, dx: torch.Tensor,
                             pre: Optional[torch.Tensor] = None, stream=None, *, pre_scale: Optional[torch.Tensor] = None) -> None:
    """dx = dy W, expert by expert: dy [P, M], w [E, M, C], dx [P, C], all bfloat16.  With pre [P, 2 C] (from
    fusco_experts_gated) dx is the gradient of pre, [P, 2 C].  pre may have been kept as float8_e4m3fn: then pre_scale, float32
    [P, S], has its scales (fusco_to_fp8)."""
    _weights(layout, w, "w")
    M, C = w.shape[1], w.shape[2]
    _bf16(dy, "dy", (layout.P, M))
    _bf16(dx, "dx", (layout.P, C if pre is None else 2 * C))
    if pre_scale is not None:
        if pre is None:
            raise FuscoError("pre_scale goes with pre")
        _fp8(pre, "pre", (layout.P, 2 * C))
        stride = _row_scale(pre_scale, "pre_scale", layout.P, 2 * C)
        return _check(load_library().fusco_experts_input_grad_fp8(ctypes.byref(layout.c), dy.data_ptr(), w.data_ptr(), dx.data_ptr(), pre.data_ptr(), pre_scale.data_ptr(), stride, M, C,
                                                                  _stream(stream)), "fusco_experts_input_grad_fp8")
    if pre is not None:
        _bf16(pre, "pre", (layout.P, 2 * C))
    _check(load_library().fusco_experts_input_grad(ctypes.byref(layout.c), dy.data_ptr(), w.data_ptr(), dx.data_ptr(), _ptr(pre),
                                                   M, C, _stream(stream)), "fusco_experts_input_grad")


def fusco_experts_weight_grad(layout: Layout, dy: torch.Tensor, x: torch.Tensor, dw: torch.Tensor,
                              stream=None, *, x_scale: Optional[torch.Tensor] = None) -> None:
    """dw = dy^T x, expert by expert: dy [P, M], x [P, C] bfloat16, dw [E, M, C] bfloat16 or float32.  x may have been kept as
    float8_e4m3fn: then x_scale, float32 [P, S], has its scales (fusco_to_fp8)."""
    if not dw.is_cuda or dw.dim() != 3 or dw.shape[0] != layout.E or not dw.is_contiguous():
        raise FuscoError("dw must be a contiguous device tensor of three dimensions, the first of them the %d experts" % layout.E)
    M, C = dw.shape[1], dw.shape[2]
    _bf16(dy, "dy", (layout.P, M))
    if x_scale is not None:
        _fp8(x, "x", (layout.P, C))
        stride = _row_scale(x_scale, "x_scale", layout.P, C)
        return _check(load_library().fusco_experts_weight_grad_fp8(ctypes.byref(layout.c), dy.data_ptr(), x.data_ptr(), x_scale.data_ptr(), stride, dw.data_ptr(), _dtype_code(dw, "dw"), M, C,
                                                                   _stream(stream)), "fusco_experts_weight_grad_fp8")
    _bf16(x, "x", (layout.P, C))
    _check(load_library().fusco_experts_weight_grad(ctypes.byref(layout.c), dy.data_ptr(), x.data_ptr(), dw.data_ptr(),
                                                    _dtype_code(dw, "dw"), M, C, _stream(stream)), "fusco_experts_weight_grad")


FP8 = torch.float8_e4m3fn
_BLOCK = 128


def _blocks(n: int) -> int:
    return -(-n // _BLOCK)


def _fp8(t: torch.Tensor, name: str, shape) -> torch.Tensor:
    if not t.is_cuda or t.dtype != FP8 or not t.is_contiguous() or tuple(t.shape) != tuple(shape):
        raise FuscoError("%s must be a contiguous float8_e4m3fn device tensor of shape %s" % (name, list(shape)))
    return t


def _row_scale(t: torch.Tensor, name: str, rows: int, columns: int) -> int:
    """Scales of rows, a value per 128 columns; rows of scales may be longer than that.  Their length."""
    if not t.is_cuda or t.dtype != torch.float32 or not t.is_contiguous() or t.dim() != 2 or t.shape[0] != rows or t.shape[1] < _blocks(columns):
        raise FuscoError("%s must be a contiguous float32 device tensor of %d rows with at least %d columns" % (name, rows, _blocks(columns)))
    return t.shape[1]


def _scaled(x: torch.Tensor, q: torch.Tensor, scale: torch.Tensor) -> _CFp8:
    if not x.is_cuda or x.dim() not in (2, 3) or not x.is_contiguous():
        raise FuscoError("x must be a contiguous device tensor of rows or of matrices")
    if max(x.shape) >= 2 ** 31 or scale.numel() and max(scale.shape) >= 2 ** 31:
        raise FuscoError("x and scale must have fewer than 2^31 rows and columns")
    _fp8(q, "q", x.shape)
    if x.dim() == 2:
        return _CFp8(x.shape[0], x.shape[1], _dtype_code(x, "x"), 0, _row_scale(scale, "scale", *x.shape))
    E, M, C = x.shape
    _fp32(scale, "scale", (E, _blocks(M), _blocks(C)))
    return _CFp8(E * M, C, _dtype_code(x, "x"), M, _blocks(C))


def fusco_to_fp8(x: torch.Tensor, q: torch.Tensor, scale: torch.Tensor, stream=None) -> None:
    """x, bfloat16 or float32, as q (float8_e4m3fn, of x's shape) with scales that are powers of two: per 128 columns of each
    row for x [R, C] (scale float32 [R, S], S at least ceil(C / 128)), per 128 x 128 for matrices [E, M, C] (scale
    [E, ceil(M / 128), ceil(C / 128)])."""
    if stream is None and _fast is not None:
        rc = _fast.to_fp8(x, q, scale)
        if rc is not None:
            return _check(rc, "fusco_to_fp8")
    f = _scaled(x, q, scale)
    _check(load_library().fusco_to_fp8(ctypes.byref(f), x.data_ptr(), q.data_ptr(), scale.data_ptr(), _stream(stream)), "fusco_to_fp8")


def fusco_from_fp8(q: torch.Tensor, scale: torch.Tensor, x: torch.Tensor, stream=None) -> None:
    """x = q * scale, tensors as in fusco_to_fp8, scales any numbers."""
    if stream is None and _fast is not None:
        rc = _fast.from_fp8(q, scale, x)
        if rc is not None:
            return _check(rc, "fusco_from_fp8")
    f = _scaled(x, q, scale)
    _check(load_library().fusco_from_fp8(ctypes.byref(f), q.data_ptr(), scale.data_ptr(), x.data_ptr(), _stream(stream)), "fusco_from_fp8")


def _fp8_weights(layout: Layout, w: torch.Tensor, w_scale: torch.Tensor, matrices: int) -> None:
    if w.dim() != 3 or w.shape[0] != layout.E:
        raise FuscoError("w must have three dimensions, the first of them the %d experts" % layout.E)
    _fp8(w, "w", w.shape)
    _fp32(w_scale, "w_scale", (layout.E, matrices * _blocks(w.shape[1] // matrices), _blocks(w.shape[2])))


def fusco_experts_gated_fp8(layout: Layout, x: torch.Tensor, x_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor,
                            h: torch.Tensor, pre: Optional[torch.Tensor] = None, stream=None) -> None:
    """fusco_experts_gated on float8_e4m3fn: x [P, H] with x_scale float32 [P, S] as fusco_dispatch moves both, w [E, 2 I, H] with
    w_scale [E, 2 ceil(I / 128), ceil(H / 128)] (gate and up rows are matrices of their own); h [P, I] and pre [P, 2 I] bfloat16.
    Scales: any numbers whose products x_scale * w_scale float32 holds."""
    if w.dim() == 3 and w.shape[1] % 2:
        raise FuscoError("w must have an even number of rows per expert")
    _fp8_weights(layout, w, w_scale, 2)
    I, H = w.shape[1] // 2, w.shape[2]
    _fp8(x, "x", (layout.P, H))
    stride = _row_scale(x_scale, "x_scale", layout.P, H)
    _bf16(h, "h", (layout.P, I))
    if pre is not None:
        _bf16(pre, "pre", (layout.P, 2 * I))
    _check(load_library().fusco_experts_gated_fp8(ctypes.byref(layout.c), x.data_ptr(), x_scale.data_ptr(), stride, w.data_ptr(), w_scale.data_ptr(), h.data_ptr(), _ptr(pre),
                                                  H, I, _stream(stream)), "fusco_experts_gated_fp8")


def fusco_experts_linear_fp8(layout: Layout, x: torch.Tensor, x_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor,
                             y: torch.Tensor, stream=None) -> None:
    """fusco_experts_linear on float8_e4m3fn: x [P, C] with x_scale float32 [P, S], w [E, M, C] with w_scale
    [E, ceil(M / 128), ceil(C / 128)], y [P, M] bfloat16."""
    _fp8_weights(layout, w, w_scale, 1)
    M, C = w.shape[1], w.shape[2]
    _fp8(x, "x", (layout.P, C))
    stride = _row_scale(x_scale, "x_scale", layout.P, C)
    _bf16(y, "y", (layout.P, M))
    _check(load_library().fusco_experts_linear_fp8(ctypes.byref(layout.c), x.data_ptr(), x_scale.data_ptr(), stride, w.data_ptr(), w_scale.data_ptr(), y.data_ptr(), C, M,
                                                   _stream(stream)), "fusco_experts_linear_fp8")


def fusco_moe_few_scratch_bytes(N: int, k: int, I: int) -> int:
    return load_library().fusco_moe_few_scratch_bytes(N, k, I)


def fusco_moe_few(x: torch.Tensor, topk_idx: torch.Tensor, w: torch.Tensor, w_in: torch.Tensor, w_out: torch.Tensor, out: torch.Tensor,
                  w_in_scale: Optional[torch.Tensor] = None, w_out_scale: Optional[torch.Tensor] = None, scratch: Optional[torch.Tensor] = None,
                  stream=None) -> None:
    """The experts of a layer for a few tokens, N of 1 to 64: x [N, H] bfloat16, topk_idx [N, k] int32, w [N, k] float32 as
    fusco_route writes them, out [N, H] bfloat16 or float32.  Weights w_in [E, 2 I, H] and w_out [E, H, I] are bfloat16, or
    float8_e4m3fn with the scales that fusco_experts_gated_fp8 and fusco_experts_linear_fp8 take.  scratch:
    fusco_moe_few_scratch_bytes(N, k, I) bytes, made here on the call's stream if not given.  Up to some 8 tokens this is faster than
    the calls one by one, from 16 on they are in most sizes."""
    if stream is None and scratch is not None and _fast is not None:
        rc = _fast.moe_few(x, topk_idx, w, w_in, w_out, out, w_in_scale, w_out_scale, scratch)
        if rc is not None:
            return _check(rc, "fusco_moe_few")
    if not x.is_cuda or x.dim() != 2 or w_in.dim() != 3 or w_in.shape[1] % 2:
        raise FuscoError("x must be a 2-D device tensor, w_in have three dimensions and an even number of rows per expert")
    (N, H), E, I = x.shape, w_in.shape[0], w_in.shape[1] // 2
    if not topk_idx.is_cuda or topk_idx.dtype != torch.int32 or not topk_idx.is_contiguous() or topk_idx.dim() != 2 or topk_idx.shape[0] != N:
        raise FuscoError("topk_idx must be a contiguous int32 device tensor of shape [N, k]")
    _bf16(x, "x", (N, H))
    _fp32(w, "w", topk_idx.shape)
    if (w_in_scale is None) != (w_out_scale is None):
        raise FuscoError("w_in_scale and w_out_scale go together")
    weights = _bf16 if w_in_scale is None else _fp8
    weights(w_in, "w_in", (E, 2 * I, H))
    weights(w_out, "w_out", (E, H, I))
    if w_in_scale is not None:
        _fp32(w_in_scale, "w_in_scale", (E, 2 * _blocks(I), _blocks(H)))
        _fp32(w_out_scale, "w_out_scale", (E, _blocks(H), _blocks(I)))
    if not out.is_cuda or not out.is_contiguous() or tuple(out.shape) != (N, H):
        raise FuscoError("out must be a contiguous device tensor of shape [%d, %d]" % (N, H))
    if max(N, E, topk_idx.shape[1], H, I) >= 2 ** 31:
        raise FuscoError("sizes must be below 2^31")
    f = _CFew(N, E, topk_idx.shape[1], H, I, BF16 if w_in_scale is None else E4M3, _dtype_code(out, "out"))
    scratch = _scratch(fusco_moe_few_scratch_bytes(N, f.k, I), scratch, x.device, stream)
    _check(load_library().fusco_moe_few(ctypes.byref(f), x.data_ptr(), topk_idx.data_ptr(), w.data_ptr(), w_in.data_ptr(), _ptr(w_in_scale), w_out.data_ptr(),
                                        _ptr(w_out_scale), out.data_ptr(), scratch.data_ptr(), scratch.numel() * scratch.element_size(), _stream(stream)),
           "fusco_moe_few")


def fusco_combine_two_hop(layout: Layout, y: torch.Tensor, w: torch.Tensor, partial: torch.Tensor,
                          out: torch.Tensor, stream=None) -> None:
    if stream is None and _fast is not None:
        rc = _fast.combine_two_hop(layout, y, w, partial, out)
        if rc is not None:
            return _check(rc, "fusco_combine_two_hop")
    _rows(y, "y", layout.P)
    H = y.shape[1]
    _rows(out, "out", layout.N)
    _rows(partial, "partial", layout.send_cap, 4 * H)
    if partial.dtype != torch.float32:
        raise FuscoError("partial must be float32")
    if out.shape[1] != H or H % 4 != 0:
        raise FuscoError("out must have %d columns and H must be a multiple of 4" % H)
    if (not w.is_cuda or w.dtype != torch.float32 or not w.is_contiguous()
            or tuple(w.shape) != (layout.N, layout.k)):
        raise FuscoError("w must be a contiguous float32 device tensor of shape [N, k]")
    _check(load_library().fusco_combine_two_hop(ctypes.byref(layout.c), y.data_ptr(), _dtype_code(y, "y"),
                                                w.data_ptr(), partial.data_ptr(), out.data_ptr(),
                                                _dtype_code(out, "out"), H, _stream(stream)),
           "fusco_combine_two_hop")


def fusco_cross_node_load(layout: Layout, devices_per_node: int, home_node: int, row_bytes: int,
                          load: torch.Tensor, stream=None) -> None:
    """load: one-element int64 device tensor (e.g. a cell of the [nodes, gpus] load matrix)."""
    if not load.is_cuda or load.dtype != torch.int64 or load.numel() != 1:
        raise FuscoError("load must be a one-element int64 device tensor")
    _check(load_library().fusco_cross_node_load(ctypes.byref(layout.c), devices_per_node, home_node, row_bytes,
                                                load.data_ptr(), _stream(stream)), "fusco_cross_node_load")


def fusco_balance_groups(load) -> "numpy.ndarray":
    """Algorithm 1 on a host [nodes, gpus] int64 load matrix; returns group_gpu [gpus, nodes] int32."""
    import numpy as np
    load = np.ascontiguousarray(load, dtype=np.int64)
    if load.ndim != 2:
        raise FuscoError("load must be a [nodes, gpus] matrix")
    nodes, gpus = load.shape
    out = np.empty((gpus, nodes), dtype=np.int32)
    _check(load_library().fusco_balance_groups(load.ctypes.data, nodes, gpus, out.ctypes.data), "fusco_balance_groups")
    return out


def _desc_ok(desc: Optional[torch.Tensor], n: int, name: str) -> None:
    if desc is None:
        return
    if not desc.is_cuda or desc.dtype != torch.int64 or not desc.is_contiguous() or tuple(desc.shape) != (n, 2):
        raise FuscoError("%s must be a contiguous int64 device tensor of shape [n, 2] (offset, size)" % name)


def fusco_segments_scan(desc: torch.Tensor, cum: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    """desc: int64 [n, 2] (offset, size) on the device; cum: int64 [n + 1]; status: int32 [1]."""
    n = desc.shape[0]
    _desc_ok(desc, n, "desc")
    if not cum.is_cuda or cum.dtype != torch.int64 or not cum.is_contiguous() or cum.numel() != n + 1:
        raise FuscoError("cum must be a contiguous int64 device tensor with n + 1 entries")
    if not status.is_cuda or status.dtype != torch.int32 or status.numel() != 1:
        raise FuscoError("status must be an int32 device tensor with one entry")
    _check(load_library().fusco_segments_scan(desc.data_ptr(), n, cum.data_ptr(), status.data_ptr(), _stream(stream)),
           "fusco_segments_scan")


def fusco_segments_copy(src: torch.Tensor, src_desc: Optional[torch.Tensor], dst: torch.Tensor,
                        dst_desc: Optional[torch.Tensor], cum: torch.Tensor, stream_capacity: int,
                        status: torch.Tensor, slice_bytes: int = 0, slice_fill: Optional[torch.Tensor] = None,
                        stream=None) -> None:
    """src / dst: contiguous device tensors viewed as bytes; a None descriptor list means that side is the
    contiguous stream.  slice_fill: int32 [ceil(stream_capacity / slice_bytes)] or None."""
    n = cum.numel() - 1
    _desc_ok(src_desc, n, "src_desc")
    _desc_ok(dst_desc, n, "dst_desc")
    if not (src.is_cuda and dst.is_cuda and src.is_contiguous() and dst.is_contiguous()):
        raise FuscoError("src and dst must be contiguous device tensors")
    if not cum.is_cuda or cum.dtype != torch.int64 or not cum.is_contiguous() or n < 0:
        raise FuscoError("cum must be a contiguous int64 device tensor with n + 1 entries")
    if not status.is_cuda or status.dtype != torch.int32 or status.numel() != 1:
        raise FuscoError("status must be an int32 device tensor with one entry")
    src_bytes, dst_bytes = src.numel() * src.element_size(), dst.numel() * dst.element_size()
    if src_desc is None and src_bytes < stream_capacity or dst_desc is None and dst_bytes < stream_capacity:
        raise FuscoError("the contiguous side is smaller than stream_capacity")
    if slice_fill is not None:
        if slice_bytes <= 0:
            raise FuscoError("slice_bytes must be positive with slice_fill")
        need = (stream_capacity + slice_bytes - 1) // slice_bytes
        if (not slice_fill.is_cuda or slice_fill.dtype != torch.int32 or not slice_fill.is_contiguous()
                or slice_fill.numel() < need):
            raise FuscoError("slice_fill must be a contiguous int32 device tensor with %d entries" % need)
    _check(load_library().fusco_segments_copy(src.data_ptr(), src_bytes, _ptr(src_desc), dst.data_ptr(), dst_bytes,
                                              _ptr(dst_desc), cum.data_ptr(), n, stream_capacity, slice_bytes,
                                              _ptr(slice_fill), status.data_ptr(), _stream(stream)),
           "fusco_segments_copy")


def fusco_probe_copy(dst: torch.Tensor, src: torch.Tensor, stream=None) -> None:
    nbytes = src.numel() * src.element_size()
    if not (dst.is_cuda and src.is_cuda and dst.is_contiguous() and src.is_contiguous()):
        raise FuscoError("probe copy needs contiguous device tensors")
    if dst.numel() * dst.element_size() < nbytes:
        raise FuscoError("dst is smaller than src")
    _check(load_library().fusco_probe_copy(dst.data_ptr(), src.data_ptr(), nbytes, _stream(stream)),
           "fusco_probe_copy")


def fusco_probe_dispatch_kernel(which: int = -1) -> int:
    """Which kernel fusco_dispatch uses where it has a choice: 0 automatic, 1 token walk, 2 transfer order wherever
    its shape allows; < 0 reads the setting.  Returns the previous setting."""
    rc = int(load_library().fusco_probe_dispatch_kernel(int(which)))
    if rc < 0:
        _check(rc, "fusco_probe_dispatch_kernel")
    return rc


def fusco_probe_dispatch_occupancy(wgs: int = -1) -> int:
    """Workgroups of the tiled dispatch per compute unit: 0 automatic, 3 ... 15 that many, 16 no cap; < 0 reads the
    setting.  Returns the previous setting."""
    rc = int(load_library().fusco_probe_dispatch_occupancy(int(wgs)))
    if rc < 0:
        _check(rc, "fusco_probe_dispatch_occupancy")
    return rc


def fusco_probe_dispatch_walk(which: int = -1) -> int:
    """Loads and stores of the token walk: 0 automatic, 1 non-temporal loads + plain stores, 2 cached loads + plain
    stores, 3 non-temporal loads and stores, 4 cached loads + non-temporal stores; < 0 reads the setting.  Returns the
    previous setting."""
    rc = int(load_library().fusco_probe_dispatch_walk(int(which)))
    if rc < 0:
        _check(rc, "fusco_probe_dispatch_walk")
    return rc


def fusco_probe_dispatch_pull(which: int = -1) -> int:
    """Whether the tiled dispatch pulls a tile's source rows towards the L2 at the start of the tile: 0 automatic,
    1 off, 2 on; < 0 reads the setting.  Returns the previous setting."""
    rc = int(load_library().fusco_probe_dispatch_pull(int(which)))
    if rc < 0:
        _check(rc, "fusco_probe_dispatch_pull")
    return rc


ROUTE_TOKENS, ROUTE_TILES, ROUTE_BOTH_BY_TILES, ROUTE_TILES_THEN_TOKENS = 0, 1, 2, 3
WALK_PLAIN, WALK_STREAMING, WALK_THROUGH = 0, 16, 32


def fusco_probe_dispatch_route(layout: Layout, row_bytes: int, aux_row_bytes: int = 0, expert_buf=None, expert_aux=None, send_buf=None, send_aux=None,
                               flags: int = DISPATCH_EXPERT) -> int:
    """How fusco_dispatch moves the rows of a call with these sizes and tensors: one of ROUTE_*, for the two that walk tokens together with
    one of WALK_* for the walk's stores (fusco_probe.h).  Host-only; the tensors are not read."""
    rc = int(load_library().fusco_probe_dispatch_route(ctypes.byref(layout.c), row_bytes, aux_row_bytes, _ptr(expert_buf), _ptr(expert_aux),
                                                       _ptr(send_buf), _ptr(send_aux), flags))
    if rc < 0:
        _check(rc, "fusco_probe_dispatch_route")
    return rc


def fusco_probe_plan_through(layout: Layout) -> bool:
    """Whether fusco_plan writes the layout's arrays that are indexed by pair through the L2s (fusco_probe.h).  Host-only."""
    rc = int(load_library().fusco_probe_plan_through(ctypes.byref(layout.c)))
    if rc < 0:
        _check(rc, "fusco_probe_plan_through")
    return bool(rc)


def fusco_probe_plan_dispatch_through(layout: Layout, row_bytes: int, aux_row_bytes: int = 0, expert_buf=None) -> bool:
    """Whether fusco_plan_dispatch writes the rows of such a call through the L2s (fusco_probe.h).  Host-only; the tensor is not read."""
    rc = int(load_library().fusco_probe_plan_dispatch_through(ctypes.byref(layout.c), row_bytes, aux_row_bytes, _ptr(expert_buf)))
    if rc < 0:
        _check(rc, "fusco_probe_plan_dispatch_through")
    return bool(rc)


def fusco_probe_segments_wide(stream_capacity: int, slice_bytes: int) -> bool:
    """Whether fusco_segments_copy packs into such slices with workgroups of twice the usual width (fusco_probe.h).  Host-only."""
    rc = int(load_library().fusco_probe_segments_wide(stream_capacity, slice_bytes))
    if rc < 0:
        _check(rc, "fusco_probe_segments_wide")
    return bool(rc)


PRODUCT_GATED, PRODUCT_LINEAR, PRODUCT_INPUT_GRAD, PRODUCT_INPUT_GRAD_ACTIVATION = 0, 1, 2, 3


def fusco_probe_experts_tile_rows(layout: Layout, which: int, outputs: int, sum: int) -> int:
    """Rows per tile of an expert product (one of PRODUCT_*) with `outputs` values per row, each the sum of `sum` products
    (fusco_probe.h).  Host-only."""
    rc = int(load_library().fusco_probe_experts_tile_rows(ctypes.byref(layout.c), which, outputs, sum))
    if rc < 0:
        _check(rc, "fusco_probe_experts_tile_rows")
    return rc


def fusco_probe_experts_tile_outputs(layout: Layout, which: int, outputs: int, sum: int) -> int:
    """Outputs per tile of the same products (PRODUCT_GATED: units) (fusco_probe.h).  Host-only."""
    rc = int(load_library().fusco_probe_experts_tile_outputs(ctypes.byref(layout.c), which, outputs, sum))
    if rc < 0:
        _check(rc, "fusco_probe_experts_tile_outputs")
    return rc


def fusco_probe_source_chunk_bytes(nbytes: int = 0) -> int:
    """Largest source tensor the tiled dispatch takes in one piece; a non-zero value replaces it (returns the
    previous one)."""
    return int(load_library().fusco_probe_source_chunk_bytes(int(nbytes)))


def fusco_probe_time_next_call(start: torch.cuda.Event, stop: torch.cuda.Event) -> None:
    """The next plan / dispatch / combine call of this thread records its own device time into the two events
    (created with enable_timing=True and recorded once before, so that their HIP handles exist)."""
    h0, h1 = int(start.cuda_event or 0), int(stop.cuda_event or 0)
    if not h0 or not h1:
        raise FuscoError("events must have been recorded once (torch creates the HIP event on first use)")
    _check(load_library().fusco_probe_time_next_call(h0, h1), "fusco_probe_time_next_call")


def fusco_probe_rows(src, dst, reads: int, writes: int, scatter: bool, write_through: bool = False,
                     sink: torch.Tensor | None = None, stream=None) -> None:
    """src / dst: 2-D contiguous device tensors of rows with the same row size in bytes (either may be None
    when its side is unused); sink: one int32 on the device, needed for the read-only shape."""
    rows, row_bytes = [0, 0], 0
    for i, t in enumerate((src, dst)):
        if t is None:
            continue
        if not t.is_cuda or t.dim() != 2 or not t.is_contiguous():
            raise FuscoError("probe rows needs 2-D contiguous device tensors")
        rb = t.shape[1] * t.element_size()
        if row_bytes and rb != row_bytes:
            raise FuscoError("src and dst rows differ in size")
        rows[i], row_bytes = t.shape[0], rb
    if sink is not None and (not sink.is_cuda or sink.numel() < 1 or sink.element_size() != 4):
        raise FuscoError("sink must be one 32-bit word on the device")
    _check(load_library().fusco_probe_rows(_ptr(src), rows[0], _ptr(dst), rows[1], row_bytes, int(reads), int(writes),
                                           int(bool(scatter)), int(bool(write_through)), _ptr(sink), _stream(stream)),
           "fusco_probe_rows")


def fusco_probe_pieces(buf: torch.Tensor, write: bool, run_pieces: int = 1, scatter: bool = False,
                       sink: torch.Tensor | None = None, stream=None) -> None:
    """buf: contiguous device tensor whose size is a multiple of 4096 bytes; see fusco_probe.h."""
    if not buf.is_cuda or not buf.is_contiguous():
        raise FuscoError("probe pieces needs a contiguous device tensor")
    if sink is not None and (not sink.is_cuda or sink.numel() < 1 or sink.element_size() != 4):
        raise FuscoError("sink must be one 32-bit word on the device")
    _check(load_library().fusco_probe_pieces(buf.data_ptr(), buf.numel() * buf.element_size(), int(bool(write)),
                                             int(run_pieces), int(bool(scatter)), _ptr(sink), _stream(stream)),
           "fusco_probe_pieces")


def fusco_probe_consume_slices(packed: torch.Tensor, total_bytes: int, slice_bytes: int, slice_fill: torch.Tensor,
                               max_polls: int, report: torch.Tensor, stream=None) -> None:
    """report: int32 [slices, 4] on the device (ready, polls, checksum low, checksum high per slice)."""
    slices = (total_bytes + slice_bytes - 1) // slice_bytes if slice_bytes > 0 else 0
    if not packed.is_cuda or not packed.is_contiguous() or packed.numel() * packed.element_size() < total_bytes:
        raise FuscoError("packed must be a contiguous device tensor of at least total_bytes")
    if not slice_fill.is_cuda or slice_fill.dtype != torch.int32 or slice_fill.numel() < slices:
        raise FuscoError("slice_fill must be an int32 device tensor with one entry per slice")
    if not report.is_cuda or report.dtype != torch.int32 or not report.is_contiguous() or report.numel() < 4 * slices:
        raise FuscoError("report must be a contiguous int32 device tensor of shape [slices, 4]")
    _check(load_library().fusco_probe_consume_slices(packed.data_ptr(), total_bytes, slice_bytes, slice_fill.data_ptr(),
                                                     max_polls, report.data_ptr(), _stream(stream)),
           "fusco_probe_consume_slices")


def fusco_disaggregated_plan(rank_layout: Layout, layout: Layout, topk_idx: torch.Tensor, topk_dev: torch.Tensor,
                             stream=None) -> None:
    """rank_layout must be Layout(N, k, D, D); topk_dev is an int32 [N, k] scratch tensor."""
    for t, name in ((topk_idx, "topk_idx"), (topk_dev, "topk_dev")):
        if (not t.is_cuda or t.dtype != torch.int32 or not t.is_contiguous()
                or tuple(t.shape) != (layout.N, layout.k)):
            raise FuscoError("%s must be a contiguous int32 device tensor of shape [N, k]" % name)
    _check(load_library().fusco_disaggregated_plan(ctypes.byref(rank_layout.c), ctypes.byref(layout.c),
                                                   topk_idx.data_ptr(), topk_dev.data_ptr(),
                                                   rank_layout.scratch.data_ptr(), rank_layout.scratch.numel(),
                                                   _stream(stream)), "fusco_disaggregated_plan")


def fusco_disaggregated_dispatch(layout: Layout, rank_layout: Layout, x: torch.Tensor, stage_a: torch.Tensor,
                                 stage_b: torch.Tensor, expert_buf: torch.Tensor, stream=None) -> None:
    rb = _rows(x, "x", layout.N)
    for t, name in ((stage_a, "stage_a"), (stage_b, "stage_b"), (expert_buf, "expert_buf")):
        _rows(t, name, layout.P, rb)
    _check(load_library().fusco_disaggregated_dispatch(ctypes.byref(layout.c), ctypes.byref(rank_layout.c),
                                                       x.data_ptr(), rb, stage_a.data_ptr(), stage_b.data_ptr(),
                                                       expert_buf.data_ptr(), _stream(stream)),
           "fusco_disaggregated_dispatch")


def fusco_disaggregated_combine(layout: Layout, rank_layout: Layout, y: torch.Tensor, w: torch.Tensor,
                                stage_a: torch.Tensor, stage_b: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    rb = _rows(y, "y", layout.P)
    H = y.shape[1]
    for t, name in ((stage_a, "stage_a"), (stage_b, "stage_b")):
        _rows(t, name, layout.P, rb)
    _rows(out, "out", layout.N)
    if out.shape[1] != H:
        raise FuscoError("out must have %d columns" % H)
    if (not w.is_cuda or w.dtype != torch.float32 or not w.is_contiguous()
            or tuple(w.shape) != (layout.N, layout.k)):
        raise FuscoError("w must be a contiguous float32 device tensor of shape [N, k]")
    _check(load_library().fusco_disaggregated_combine(ctypes.byref(layout.c), ctypes.byref(rank_layout.c),
                                                      y.data_ptr(), _dtype_code(y, "y"), w.data_ptr(),
                                                      stage_a.data_ptr(), stage_b.data_ptr(), out.data_ptr(),
                                                      _dtype_code(out, "out"), H, _stream(stream)),
           "fusco_disaggregated_combine")
