"""Python binding of libodb, the MI355X Online Dynamic Batching window pipeline.

The functions named ``odb_*`` mirror the C ABI in ``include/odb.h`` one to one: they
convert torch device tensors and host arrays into the pointers and structs the library
takes, call it, and turn its status into an exception.  All computation happens in the
HIP kernels of ``libodb.so``; there is no fallback path -- if the library is missing or
fails to load, every call raises.

:class:`Pipeline` owns the device buffers of one window and runs the three stages
(grouping, alignment, collation) in order on one stream, and on request the loss-scaling
weights of the aligned plan, a policy loss, a preference loss and a distillation loss over its
tiles.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libodb.so")

ODB_OK = 0
ODB_E_INVALID_ARG = 1
ODB_E_INVALID_DATA = 2
ODB_E_WORKSPACE = 3
ODB_E_CAPACITY = 4
ODB_E_HIP = 5
ODB_E_COVERAGE = 6
ODB_E_INTERNAL = 7

ODB_MODE_JOIN = 0
ODB_MODE_NONJOIN_QUOTA = 1
ODB_STOP_DRAINED, ODB_STOP_QUOTA, ODB_STOP_RANK_FINISHED = 0, 1, 2
ODB_WEIGHT_SAMPLE, ODB_WEIGHT_TOKEN_APPROX, ODB_WEIGHT_TOKEN_EXACT = 0, 1, 2
ODB_LABEL_IGNORE = -100
ODB_LIST_MAX = 128
ODB_FLOAT32, ODB_BFLOAT16, ODB_FLOAT16 = 0, 1, 2
ODB_KL_NONE, ODB_KL_LINEAR, ODB_KL_SQUARE, ODB_KL_EXP = 0, 1, 2, 3
ODB_REDUCE_TOKEN_MEAN, ODB_REDUCE_ROW_MEAN, ODB_REDUCE_SUM = 0, 1, 2
ODB_DISTILL_FORWARD, ODB_DISTILL_REVERSE, ODB_DISTILL_MIXTURE = 0, 1, 2
ODB_SUPPORT_LISTED, ODB_SUPPORT_RENORMALIZED, ODB_SUPPORT_REST = 0, 1, 2
ODB_PREFERENCE_SIGMOID, ODB_PREFERENCE_HINGE, ODB_PREFERENCE_SQUARE = 0, 1, 2

EXPORTED = [
    "odb_status_string", "odb_last_error_message", "odb_workspace_size", "odb_form_groups",
    "odb_align_groups", "odb_collate", "odb_collate_status", "odb_check_coverage", "odb_loss_weights",
    "odb_length_sketch", "odb_stream_workspace_size", "odb_stream_plan", "odb_collate_static",
    "odb_token_logprobs", "odb_token_logprobs_backward", "odb_loss_workspace_size", "odb_policy_loss",
    "odb_preference_loss", "odb_token_list_logprobs", "odb_token_list_logprobs_backward",
    "odb_token_top_workspace_size", "odb_token_top_logprobs", "odb_distill_workspace_size", "odb_distill_loss",
]
ODB_COLLATE_STATIC_MAX_ROWS = 2097152


class OdbError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{message} [status {status}]")
        self.status = status


class Window(ctypes.Structure):
    _fields_ = [
        ("num_ranks", ctypes.c_int32),
        ("reserved0", ctypes.c_int32),
        ("num_samples", ctypes.c_int64),
        ("rank_offsets", ctypes.c_void_p),
        ("d_token_offsets", ctypes.c_void_p),
        ("d_tokens", ctypes.c_void_p),
        ("d_identity", ctypes.c_void_p),
        ("num_identities", ctypes.c_int64),
    ]


class AlignParams(ctypes.Structure):
    _fields_ = [
        ("mode", ctypes.c_int32),
        ("reserved0", ctypes.c_int32),
        ("quota", ctypes.c_int64),
        ("slot_capacity", ctypes.c_void_p),
    ]


class PlanInfo(ctypes.Structure):
    _fields_ = [
        ("steps", ctypes.c_int64),
        ("rounds", ctypes.c_int32),
        ("stop_reason", ctypes.c_int32),
        ("emitted_samples", ctypes.c_int64),
        ("leftover_samples", ctypes.c_int64),
        ("real_tokens", ctypes.c_int64),
        ("padded_elems", ctypes.c_int64),
        ("max_step_samples", ctypes.c_int64),
        ("splits", ctypes.c_int64),
        ("overflow_groups", ctypes.c_int64),
        ("missing_ids", ctypes.c_int64),
        ("duplicate_ids", ctypes.c_int64),
        ("bad_views", ctypes.c_int64),
        ("pad_fraction", ctypes.c_double),
        ("required_slot_capacity", ctypes.c_int64),
        ("second_gather_rounds", ctypes.c_int64),
    ]

    def as_dict(self) -> dict:
        return {f: getattr(self, f) for f, _ in self._fields_}


class LengthSketch(ctypes.Structure):
    _fields_ = [
        ("samples", ctypes.c_int64),
        ("short_samples", ctypes.c_int64),
        ("sum_len", ctypes.c_int64),
        ("sum_sq_hi", ctypes.c_uint64),
        ("sum_sq_lo", ctypes.c_uint64),
        ("min_len", ctypes.c_int64),
        ("max_len", ctypes.c_int64),
        ("mean", ctypes.c_double),
        ("cv", ctypes.c_double),
        ("short_fraction", ctypes.c_double),
        ("high_roi", ctypes.c_int32),
        ("reserved0", ctypes.c_int32),
    ]


class StreamParams(ctypes.Structure):
    _fields_ = [
        ("mode", ctypes.c_int32),
        ("buffer_size", ctypes.c_int32),
        ("depth", ctypes.c_int32),
        ("reserved0", ctypes.c_int32),
        ("quota", ctypes.c_int64),
        ("rate", ctypes.c_void_p),
        ("slot_capacity", ctypes.c_void_p),
        ("max_rounds", ctypes.c_int64),
    ]


class StreamRound(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("reserved0", ctypes.c_int32), ("target", ctypes.c_int64),
                ("emitted", ctypes.c_int64), ("phi", ctypes.c_int64)]


class StreamInfo(ctypes.Structure):
    _fields_ = [
        ("steps", ctypes.c_int64),
        ("rounds", ctypes.c_int64),
        ("emit_rounds", ctypes.c_int64),
        ("skip_rounds", ctypes.c_int64),
        ("stop_reason", ctypes.c_int32),
        ("reserved0", ctypes.c_int32),
        ("views", ctypes.c_int64),
        ("emitted_views", ctypes.c_int64),
        ("undelivered_views", ctypes.c_int64),
        ("pending_views", ctypes.c_int64),
        ("real_tokens", ctypes.c_int64),
        ("padded_elems", ctypes.c_int64),
        ("max_step_samples", ctypes.c_int64),
        ("splits", ctypes.c_int64),
        ("overflow_groups", ctypes.c_int64),
        ("missing_ids", ctypes.c_int64),
        ("duplicate_ids", ctypes.c_int64),
        ("bad_views", ctypes.c_int64),
        ("second_gather_rounds", ctypes.c_int64),
        ("max_outstanding", ctypes.c_int64),
        ("pad_fraction", ctypes.c_double),
        ("required_slot_capacity", ctypes.c_int64),
    ]

    def as_dict(self) -> dict:
        return {f: getattr(self, f) for f, _ in self._fields_ if f != "reserved0"}


class Logits(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32),
        ("shift", ctypes.c_int32),
        ("rows", ctypes.c_int64),
        ("cols", ctypes.c_int64),
        ("vocab", ctypes.c_int64),
        ("row_stride", ctypes.c_int64),
        ("col_stride", ctypes.c_int64),
        ("scale", ctypes.c_double),
        ("d_logits", ctypes.c_void_p),
    ]


class TilesStruct(ctypes.Structure):
    _fields_ = [
        ("num_slots", ctypes.c_int64),
        ("num_rows", ctypes.c_int64),
        ("num_elems", ctypes.c_int64),
        ("d_slot_rows", ctypes.c_void_p),
        ("d_slot_maxlen", ctypes.c_void_p),
        ("d_slot_row_off", ctypes.c_void_p),
        ("d_slot_tile_off", ctypes.c_void_p),
        ("d_labels", ctypes.c_void_p),
        ("shift", ctypes.c_int32),
        ("reserved0", ctypes.c_int32),
    ]


class PolicyParams(ctypes.Structure):
    """Parameters of odb_policy_loss; keywords override the defaults below."""
    _fields_ = [
        ("kl", ctypes.c_int32),
        ("reduce", ctypes.c_int32),
        ("token_advantage", ctypes.c_int32),
        ("reserved0", ctypes.c_int32),
        ("clip_low", ctypes.c_double),
        ("clip_high", ctypes.c_double),
        ("dual_clip", ctypes.c_double),
        ("kl_coef", ctypes.c_double),
        ("entropy_coef", ctypes.c_double),
        ("loss_scale", ctypes.c_double),
    ]

    def __init__(self, **kw):
        super().__init__(**{**dict(clip_low=0.2, clip_high=0.2, loss_scale=1.0), **kw})


class PreferenceParams(ctypes.Structure):
    """Parameters of odb_preference_loss; keywords override the defaults below."""
    _fields_ = [
        ("kind", ctypes.c_int32),
        ("normalize", ctypes.c_int32),
        ("beta", ctypes.c_double),
        ("margin", ctypes.c_double),
        ("label_smoothing", ctypes.c_double),
        ("loss_scale", ctypes.c_double),
    ]

    def __init__(self, **kw):
        super().__init__(**{**dict(beta=0.1, loss_scale=1.0), **kw})


class DistillParams(ctypes.Structure):
    """Parameters of odb_distill_loss; keywords override the defaults below."""
    _fields_ = [
        ("kind", ctypes.c_int32),
        ("support", ctypes.c_int32),
        ("reduce", ctypes.c_int32),
        ("reserved0", ctypes.c_int32),
        ("mix", ctypes.c_double),
        ("loss_scale", ctypes.c_double),
    ]

    def __init__(self, **kw):
        super().__init__(**{**dict(mix=0.5, loss_scale=1.0), **kw})


_lib = None


def load():
    """Load libodb.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                               "or python -m paper_2606_19989_amd.build")
        lib = ctypes.CDLL(LIB_PATH)
        P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        W = ctypes.POINTER(Window)
        lib.odb_status_string.restype = ctypes.c_char_p
        lib.odb_status_string.argtypes = [ctypes.c_int]
        lib.odb_last_error_message.restype = ctypes.c_char_p
        lib.odb_last_error_message.argtypes = []
        lib.odb_workspace_size.restype = SZ
        lib.odb_workspace_size.argtypes = [W]
        lib.odb_form_groups.restype = ctypes.c_int
        lib.odb_form_groups.argtypes = [W, I64, P, P, P, P, P, SZ, P]
        lib.odb_align_groups.restype = ctypes.c_int
        lib.odb_align_groups.argtypes = [W, I64, ctypes.POINTER(AlignParams), P, P, P, P, I64,
                                         P, P, P, P, P, P, P, P, P, P, P, ctypes.POINTER(PlanInfo), P, SZ, P]
        lib.odb_collate.restype = ctypes.c_int
        lib.odb_collate.argtypes = [W, I64, P, P, P, P, P, P, P, I32, I64, P, P, P, P, P, SZ, P]
        lib.odb_collate_static.restype = ctypes.c_int
        lib.odb_collate_static.argtypes = [W, I64, P, P, P, P, P, P, P, I32, I64, P, P, P, P, P, P]
        lib.odb_collate_status.restype = ctypes.c_int
        lib.odb_collate_status.argtypes = [P, SZ, P]
        lib.odb_check_coverage.restype = ctypes.c_int
        lib.odb_check_coverage.argtypes = [W, P, I64, P, I64, ctypes.POINTER(PlanInfo), P, SZ, P]
        lib.odb_loss_weights.restype = ctypes.c_int
        lib.odb_loss_weights.argtypes = [I32, I64, I32, P, P, P, P, P, P, P]
        lib.odb_length_sketch.restype = ctypes.c_int
        lib.odb_length_sketch.argtypes = [W, P, I64, I64, ctypes.POINTER(LengthSketch), P, SZ, P]
        lib.odb_stream_workspace_size.restype = SZ
        lib.odb_stream_workspace_size.argtypes = [W, I32, I64, I64]
        lib.odb_stream_plan.restype = ctypes.c_int
        lib.odb_stream_plan.argtypes = [W, P, I64, ctypes.POINTER(StreamParams), I64, P, P, P, P, P, P, P, P, P, P, P, P,
                                        P, ctypes.POINTER(StreamInfo), P, SZ, P]
        T = ctypes.POINTER(TilesStruct)
        lib.odb_token_logprobs.restype = ctypes.c_int
        lib.odb_token_logprobs.argtypes = [ctypes.POINTER(Logits), P, P, P, P, P, P]
        lib.odb_token_logprobs_backward.restype = ctypes.c_int
        lib.odb_token_logprobs_backward.argtypes = [ctypes.POINTER(Logits), P, P, P, P, P, P, I64, I64, P, P]
        lib.odb_token_top_workspace_size.restype = SZ
        lib.odb_token_top_workspace_size.argtypes = [ctypes.POINTER(Logits), I32]
        lib.odb_token_top_logprobs.restype = ctypes.c_int
        lib.odb_token_top_logprobs.argtypes = [ctypes.POINTER(Logits), P, I32, P, P, P, P, P, P, P, P, SZ, P]
        lib.odb_token_list_logprobs.restype = ctypes.c_int
        lib.odb_token_list_logprobs.argtypes = [ctypes.POINTER(Logits), P, I32, P, P, P, P, P]
        lib.odb_token_list_logprobs_backward.restype = ctypes.c_int
        lib.odb_token_list_logprobs_backward.argtypes = [ctypes.POINTER(Logits), P, I32, P, P, P, P, I64, I64, P, P]
        lib.odb_loss_workspace_size.restype = SZ
        lib.odb_loss_workspace_size.argtypes = [T, I64]
        lib.odb_policy_loss.restype = ctypes.c_int
        lib.odb_policy_loss.argtypes = [T, ctypes.POINTER(PolicyParams), P, P, P, P, P, P, P, P, P, P, P, P, P, SZ, P]
        lib.odb_preference_loss.restype = ctypes.c_int
        lib.odb_preference_loss.argtypes = [T, ctypes.POINTER(PreferenceParams), P, P, P, I64, P, P, P, P, P, P, P, P,
                                            SZ, P]
        lib.odb_distill_workspace_size.restype = SZ
        lib.odb_distill_workspace_size.argtypes = [T, I32]
        lib.odb_distill_loss.restype = ctypes.c_int
        lib.odb_distill_loss.argtypes = [T, ctypes.POINTER(DistillParams), I32, P, P, P, P, P, P, P, P, P, SZ, P]
        _lib = lib
    return _lib


def _check(status: int):
    if status != ODB_OK:
        lib = load()
        raise OdbError(status, f"{lib.odb_status_string(status).decode()}: "
                               f"{lib.odb_last_error_message().decode()}")


def _dptr(t) -> Optional[int]:
    """Device pointer of a contiguous torch tensor on a GPU (None passes NULL)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    """Handle of a torch stream (default: the current one).  The current stream's handle is
    asked for directly: torch.cuda.current_stream() builds a Stream object around it, 2.9 us of
    a call that takes 15."""
    if stream is not None:
        return stream.cuda_stream
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _sync_current(device):
    """Waits for the current stream of a GPU device (no-op elsewhere)."""
    import torch
    if torch.device(device).type == "cuda":
        torch.cuda.current_stream(device).synchronize()


class DeviceWindow:
    """A window resident in device memory, with its C descriptor.

    rank_offsets stays on the host (int64 numpy, W+1 entries); token_offsets (int64,
    n+1), tokens (int32) and the optional identity map (int64, n) are device tensors.
    """

    def __init__(self, rank_offsets, token_offsets, tokens, identity=None, num_identities: int = 0):
        self.rank_offsets = np.ascontiguousarray(rank_offsets, dtype=np.int64)
        self.token_offsets = token_offsets
        self.tokens = tokens
        self.identity = identity
        self.num_ranks = len(self.rank_offsets) - 1
        self.num_samples = int(self.rank_offsets[-1])
        self.struct = Window(self.num_ranks, 0, self.num_samples,
                             self.rank_offsets.ctypes.data_as(ctypes.c_void_p).value,
                             _dptr(token_offsets), _dptr(tokens), _dptr(identity),
                             int(num_identities) if identity is not None else 0)

    @property
    def ref(self):
        return ctypes.byref(self.struct)


def odb_workspace_size(win: DeviceWindow) -> int:
    v = load().odb_workspace_size(win.ref)
    if v == 0:
        _check(ODB_E_INVALID_ARG)
    return int(v)


def odb_form_groups(win, budget, order, sorted_len, group_index, groups_per_rank, ws, stream=None):
    _check(load().odb_form_groups(win.ref, int(budget), _dptr(order), _dptr(sorted_len), _dptr(group_index),
                                  _dptr(groups_per_rank), _dptr(ws), ws.numel() * ws.element_size(),
                                  _stream(stream)))


def odb_align_groups(win, budget, mode, quota, slot_capacity_per_rank, order, sorted_len, group_index,
                     groups_per_rank, slot_capacity, emit_order, slot_rows, slot_maxlen, slot_row_off,
                     slot_tile_off, slot_tokens, leftover, leftover_off, ws, stream=None, raise_on_capacity=True,
                     slot_tokens_approx=None, row_token_start=None, row_len=None):
    cap = None
    if slot_capacity_per_rank is not None:
        cap = np.ascontiguousarray(slot_capacity_per_rank, dtype=np.int64)
    params = AlignParams(int(mode), 0, int(quota), None if cap is None else cap.ctypes.data_as(ctypes.c_void_p).value)
    info = PlanInfo()
    st = load().odb_align_groups(win.ref, int(budget), ctypes.byref(params), _dptr(order), _dptr(sorted_len),
                                 _dptr(group_index), _dptr(groups_per_rank), int(slot_capacity), _dptr(emit_order),
                                 _dptr(row_token_start), _dptr(row_len), _dptr(slot_rows), _dptr(slot_maxlen), _dptr(slot_row_off), _dptr(slot_tile_off),
                                 _dptr(slot_tokens), _dptr(slot_tokens_approx), _dptr(leftover), _dptr(leftover_off),
                                 ctypes.byref(info),
                                 _dptr(ws), ws.numel() * ws.element_size(), _stream(stream))
    if st == ODB_E_CAPACITY and not raise_on_capacity:
        return st, info.as_dict()
    _check(st)
    return st, info.as_dict()


def odb_collate(win, num_slots, emit_order, slot_rows, slot_maxlen, slot_row_off, slot_tile_off, pad_id,
                out_capacity, input_ids, labels, attention_mask, position_ids, ws, stream=None, row_token_start=None,
                row_len=None):
    _check(load().odb_collate(win.ref, int(num_slots), _dptr(emit_order), _dptr(row_token_start), _dptr(row_len),
                              _dptr(slot_rows), _dptr(slot_maxlen),
                              _dptr(slot_row_off), _dptr(slot_tile_off), int(pad_id), int(out_capacity),
                              _dptr(input_ids), _dptr(labels), _dptr(attention_mask), _dptr(position_ids),
                              _dptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def odb_collate_static(win, num_slots, emit_order, slot_rows, slot_maxlen, slot_row_off, slot_tile_off, pad_id,
                       out_capacity, input_ids, labels, attention_mask, position_ids, status, stream=None,
                       row_token_start=None, row_len=None):
    """odb_collate without a workspace (the library's fixed scratch); ``status`` is a
    device int32 tensor of one element that receives 0 or the plan-error flag."""
    _check(load().odb_collate_static(win.ref, int(num_slots), _dptr(emit_order), _dptr(row_token_start),
                                     _dptr(row_len), _dptr(slot_rows), _dptr(slot_maxlen), _dptr(slot_row_off),
                                     _dptr(slot_tile_off), int(pad_id), int(out_capacity), _dptr(input_ids),
                                     _dptr(labels), _dptr(attention_mask), _dptr(position_ids), _dptr(status),
                                     _stream(stream)))


def odb_collate_status(ws, stream=None):
    _check(load().odb_collate_status(_dptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def odb_check_coverage(win, emitted, num_emitted, leftover, num_leftover, ws, stream=None) -> dict:
    info = PlanInfo()
    _check(load().odb_check_coverage(win.ref, _dptr(emitted), int(num_emitted), _dptr(leftover), int(num_leftover),
                                     ctypes.byref(info), _dptr(ws), ws.numel() * ws.element_size(),
                                     _stream(stream)))
    return info.as_dict()


def odb_loss_weights(num_ranks, steps, mode, slot_rows, slot_tokens, slot_tokens_approx, weight,
                     step_tokens=None, step_samples=None, stream=None):
    _check(load().odb_loss_weights(int(num_ranks), int(steps), int(mode), _dptr(slot_rows), _dptr(slot_tokens),
                                   _dptr(slot_tokens_approx), _dptr(weight), _dptr(step_tokens), _dptr(step_samples),
                                   _stream(stream)))


def odb_length_sketch(win, ids, count, budget, ws, stream=None) -> dict:
    """CV, f_s and exact length moments of a sketch (ids: device int32 tensor or None for
    samples 0 .. count-1); ``sum_sq`` is returned as one Python integer."""
    out = LengthSketch()
    _check(load().odb_length_sketch(win.ref, _dptr(ids), int(count), int(budget), ctypes.byref(out), _dptr(ws),
                                    ws.numel() * ws.element_size(), _stream(stream)))
    d = {f: getattr(out, f) for f, _ in out._fields_ if f != "reserved0"}
    d["sum_sq"] = (int(d.pop("sum_sq_hi")) << 32) + int(d.pop("sum_sq_lo"))
    return d


# The loss operators take microseconds on small tiles, so their wrappers ask for little: torch and the
# types are looked up once and the current device once a call (14 us a call before, 6 now).
_types = None


def _torch_types():
    """(torch, float32, float64, int32, int64, {logits type: odb_dtype_t})."""
    global _types
    if _types is None:
        import torch
        _types = (torch, torch.float32, torch.float64, torch.int32, torch.int64,
                  {torch.float32: ODB_FLOAT32, torch.bfloat16: ODB_BFLOAT16, torch.float16: ODB_FLOAT16})
    return _types


def _current(torch) -> int:
    """Index of the current device (-2 before the first use of one: no tensor lies there)."""
    return torch._C._cuda_getDevice() if torch.cuda.is_initialized() else -2


def _refuse(t, dtype, least, name, current):
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.numel() < least:
        raise ValueError(f"{name}: {t.numel()} elements, {least} needed")
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a device tensor")
    if t.get_device() != current:
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{current}")
    raise ValueError(f"{name}: expected a contiguous tensor")


def _array(t, dtype, least: int, name: str, current: int):
    """Device pointer of an argument of the loss operators, its type, size and device checked
    (None passes NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() < least or t.get_device() != current or not t.is_contiguous():
        _refuse(t, dtype, least, name, current)
    return t.data_ptr()


def _tile_array(t, dtype, x, name: str, current: int, each: int = 1):
    """The same for an array parallel to the tile of the logits: flat, or of the tile's shape."""
    if t is None:
        return None
    rows, cols = x.rows, x.cols
    if t.shape != ((rows, cols) if each == 1 else (rows, cols, each)):    # one comparison where the shape is the tile's
        n = rows * cols * each
        # the first size tells [cols, rows] apart; [1, rows, cols] and [rows * cols, each] are as flat
        if t.dim() > 1 and (t.numel() != n or t.size(0) not in (rows, 1, rows * cols)):
            raise ValueError(f"{name}: shape {tuple(t.shape)} beside a tile of {rows} x {cols}")
        return _array(t, dtype, n, name, current)
    if t.dtype is not dtype or t.get_device() != current or not t.is_contiguous():
        _refuse(t, dtype, 0, name, current)
    return t.data_ptr()


def _loss_stream(torch, stream, current):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(current)
    if stream.device_index != current:
        raise ValueError(f"the stream is on cuda:{stream.device_index}, the current device is cuda:{current}")
    return stream.cuda_stream


def _logits(x, kinds, shift, scale, current, name="logits"):
    """Descriptor of a [rows, cols, vocab] tensor of logits; rows and columns may have any stride."""
    kind = kinds.get(x.dtype)
    if kind is None:
        raise ValueError(f"{name}: expected float32, bfloat16 or float16, got {x.dtype}")
    if x.dim() != 3:
        raise ValueError(f"{name}: expected [rows, cols, vocab], got {tuple(x.shape)}")
    rows, cols, vocab = x.shape
    rs, cs, vs = x.stride()
    if vs != 1 and vocab > 1:
        raise ValueError(f"{name}: the vocabulary must be contiguous")
    if x.get_device() != current:
        _refuse(x, None, 0, name, current)
    return Logits(kind, shift, rows, cols, vocab, rs, cs, scale, x.data_ptr())


def odb_token_logprobs(logits, labels, logprob, stats=None, entropy=None, status=None, shift=1, scale=1.0,
                       stream=None):
    """Log-probabilities of a tile's labels (int32, [rows, cols]) from its logits [rows, cols,
    vocab]; ``stats`` (float32, [rows, cols, 2]) is what the backward call takes."""
    torch, f32, _, i32, _, kinds = _torch_types()
    cur = _current(torch)
    x = _logits(logits, kinds, shift, scale, cur)
    a = _tile_array
    _check(load().odb_token_logprobs(ctypes.byref(x), a(labels, i32, x, "labels", cur),
                                     a(logprob, f32, x, "logprob", cur), a(stats, f32, x, "stats", cur, 2),
                                     a(entropy, f32, x, "entropy", cur), _array(status, i32, 1, "status", cur),
                                     _loss_stream(torch, stream, cur)))


def odb_token_logprobs_backward(logits, labels, stats, grad_logprob, grad_logits, entropy=None, grad_entropy=None,
                                status=None, shift=1, scale=1.0, stream=None):
    """Gradient of :func:`odb_token_logprobs` with respect to the logits, written to
    ``grad_logits`` (the logits' shape and type; may be the logits themselves)."""
    torch, f32, _, i32, _, kinds = _torch_types()
    cur = _current(torch)
    x = _logits(logits, kinds, shift, scale, cur)
    g = _logits(grad_logits, kinds, shift, scale, cur, "grad_logits")
    if (g.dtype, g.rows, g.cols, g.vocab) != (x.dtype, x.rows, x.cols, x.vocab):
        raise ValueError("grad_logits must have the shape and type of the logits")
    a = _tile_array
    _check(load().odb_token_logprobs_backward(ctypes.byref(x), a(labels, i32, x, "labels", cur),
                                              a(stats, f32, x, "stats", cur, 2),
                                              a(grad_logprob, f32, x, "grad_logprob", cur),
                                              a(entropy, f32, x, "entropy", cur),
                                              a(grad_entropy, f32, x, "grad_entropy", cur), g.d_logits,
                                              g.row_stride, g.col_stride, _array(status, i32, 1, "status", cur),
                                              _loss_stream(torch, stream, cur)))


def _list_length(t, x, name: str) -> int:
    """Entries of the lists of an array [rows, cols, k] beside a tile."""
    if t.dim() != 3 or t.size(0) != x.rows or t.size(1) != x.cols:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected [{x.rows}, {x.cols}, k]")
    return t.size(2)


def odb_token_top_workspace_size(logits, k: int) -> int:
    """Bytes of workspace for the ``k`` likeliest tokens of logits [rows, cols, vocab]."""
    torch, _, _, _, _, kinds = _torch_types()
    v = load().odb_token_top_workspace_size(ctypes.byref(_logits(logits, kinds, 0, 1.0, _current(torch))), int(k))
    if v == 0:
        _check(ODB_E_INVALID_ARG)
    return int(v)


def odb_token_top_logprobs(logits, top_ids, top_logprob, ws, labels=None, logprob=None, rank=None, stats=None,
                           entropy=None, status=None, shift=1, scale=1.0, stream=None):
    """The likeliest tokens at every position of a tile: ``top_ids`` (int32) and ``top_logprob`` (float32), both
    [rows, cols, k], from its logits [rows, cols, vocab].  ``labels`` says which tokens count (default: all) and
    is what ``logprob`` and ``rank`` are of."""
    torch, f32, _, i32, _, kinds = _torch_types()
    cur = _current(torch)
    x = _logits(logits, kinds, shift, scale, cur)
    k, a = _list_length(top_ids, x, "top_ids"), _tile_array
    _check(load().odb_token_top_logprobs(ctypes.byref(x), a(labels, i32, x, "labels", cur), k,
                                         a(top_ids, i32, x, "top_ids", cur, k),
                                         a(top_logprob, f32, x, "top_logprob", cur, k),
                                         a(logprob, f32, x, "logprob", cur), a(rank, i32, x, "rank", cur),
                                         a(stats, f32, x, "stats", cur, 2), a(entropy, f32, x, "entropy", cur),
                                         _array(status, i32, 1, "status", cur), _array(ws, ws.dtype, 0, "ws", cur),
                                         ws.numel() * ws.element_size(), _loss_stream(torch, stream, cur)))


def odb_token_list_logprobs(logits, ids, list_logprob, labels=None, stats=None, status=None, shift=1, scale=1.0,
                            stream=None):
    """Log-probabilities of the tokens ``ids`` (int32, [rows, cols, k]) at every position of a tile, from its
    logits [rows, cols, vocab]; ``ODB_LABEL_IGNORE`` is no entry.  ``labels`` says which tokens count (default:
    all); ``stats`` (float32, [rows, cols, 2]) is what the backward call takes."""
    torch, f32, _, i32, _, kinds = _torch_types()
    cur = _current(torch)
    x = _logits(logits, kinds, shift, scale, cur)
    k, a = _list_length(ids, x, "ids"), _tile_array
    _check(load().odb_token_list_logprobs(ctypes.byref(x), a(labels, i32, x, "labels", cur), k,
                                          a(ids, i32, x, "ids", cur, k),
                                          a(list_logprob, f32, x, "list_logprob", cur, k),
                                          a(stats, f32, x, "stats", cur, 2), _array(status, i32, 1, "status", cur),
                                          _loss_stream(torch, stream, cur)))


def odb_token_list_logprobs_backward(logits, ids, stats, grad_list, grad_logits, labels=None, status=None, shift=1,
                                     scale=1.0, stream=None):
    """Gradient of :func:`odb_token_list_logprobs` with respect to the logits, written to ``grad_logits`` (the
    logits' shape and type; may be the logits themselves)."""
    torch, f32, _, i32, _, kinds = _torch_types()
    cur = _current(torch)
    x = _logits(logits, kinds, shift, scale, cur)
    g = _logits(grad_logits, kinds, shift, scale, cur, "grad_logits")
    if (g.dtype, g.rows, g.cols, g.vocab) != (x.dtype, x.rows, x.cols, x.vocab):
        raise ValueError("grad_logits must have the shape and type of the logits")
    k, a = _list_length(ids, x, "ids"), _tile_array
    _check(load().odb_token_list_logprobs_backward(ctypes.byref(x), a(labels, i32, x, "labels", cur), k,
                                                   a(ids, i32, x, "ids", cur, k), a(stats, f32, x, "stats", cur, 2),
                                                   a(grad_list, f32, x, "grad_list", cur, k), g.d_logits, g.row_stride,
                                                   g.col_stride, _array(status, i32, 1, "status", cur),
                                                   _loss_stream(torch, stream, cur)))


class Tiles:
    """A run of a plan's slots and their labels, with its C descriptor.

    The slot arrays hold the run's slots (the offsets one entry more); ``labels`` and every array
    parallel to the tiles start at the run's first element, arrays parallel to the rows at its
    first row.  ``slots``, ``rows`` and ``elems`` are the run's ranges in the plan's arrays.
    """

    def __init__(self, slot_rows, slot_maxlen, slot_row_off, slot_tile_off, labels, num_rows: int, shift: int = 1,
                 slots=None, rows=None, elems=None):
        torch, _, _, i32, i64, _ = _torch_types()
        cur = _current(torch)
        K = slot_rows.numel()
        self.keep = (slot_rows, slot_maxlen, slot_row_off, slot_tile_off)
        self.num_slots, self.num_rows, self.num_elems = K, int(num_rows), labels.numel()
        self.slots = slice(0, K) if slots is None else slots
        self.rows = slice(0, self.num_rows) if rows is None else rows
        self.elems = slice(0, self.num_elems) if elems is None else elems
        self.labels = labels
        self.struct = TilesStruct(K, self.num_rows, self.num_elems, _array(slot_rows, i32, K, "slot_rows", cur),
                                  _array(slot_maxlen, i32, K, "slot_maxlen", cur),
                                  _array(slot_row_off, i64, K + 1, "slot_row_off", cur),
                                  _array(slot_tile_off, i64, K + 1, "slot_tile_off", cur),
                                  _array(labels, i32, 0, "labels", cur), int(shift), 0)
        self.device = slot_rows.get_device()

    @property
    def ref(self):
        return ctypes.byref(self.struct)


def odb_loss_workspace_size(tiles: Tiles, num_ids: int = 0) -> int:
    v = load().odb_loss_workspace_size(tiles.ref, int(num_ids))
    if v == 0:
        _check(ODB_E_INVALID_ARG)
    return int(v)


def _tiles_here(tiles, current):
    if tiles.device != current:
        raise ValueError(f"the tiles are on cuda:{tiles.device}, the current device is cuda:{current}")


def odb_policy_loss(tiles, params, logprob, advantage, slot_loss, slot_means, slot_counts, ws, old_logprob=None,
                    ref_logprob=None, entropy=None, slot_weight=None, grad_logprob=None, grad_entropy=None,
                    status=None, stream=None):
    torch, f32, f64, i32, i64, _ = _torch_types()
    cur = _current(torch)
    _tiles_here(tiles, cur)
    K, E, a = tiles.num_slots, tiles.num_elems, _array
    _check(load().odb_policy_loss(
        tiles.ref, ctypes.byref(params), a(logprob, f32, E, "logprob", cur), a(old_logprob, f32, E, "old_logprob", cur),
        a(ref_logprob, f32, E, "ref_logprob", cur), a(entropy, f32, E, "entropy", cur),
        a(advantage, f32, E if params.token_advantage else tiles.num_rows, "advantage", cur),
        a(slot_weight, f64, K, "slot_weight", cur), a(slot_loss, f32, K, "slot_loss", cur),
        a(slot_means, f32, 4 * K, "slot_means", cur), a(slot_counts, i64, 4 * K, "slot_counts", cur),
        a(grad_logprob, f32, E, "grad_logprob", cur), a(grad_entropy, f32, E, "grad_entropy", cur),
        a(status, i32, 1, "status", cur), a(ws, ws.dtype, 0, "ws", cur), ws.numel() * ws.element_size(),
        _loss_stream(torch, stream, cur)))


def odb_preference_loss(tiles, params, logprob, pair, loss, row_loss, row_reward, counts, ws, ref_logprob=None,
                        row_ids=None, grad_logprob=None, status=None, stream=None):
    torch, f32, _, i32, i64, _ = _torch_types()
    cur = _current(torch)
    _tiles_here(tiles, cur)
    R, E, a = tiles.num_rows, tiles.num_elems, _array
    ids = R if row_ids is None or R == 0 else pair.numel()    # an empty tensor has no address
    _check(load().odb_preference_loss(
        tiles.ref, ctypes.byref(params), a(logprob, f32, E, "logprob", cur), a(ref_logprob, f32, E, "ref_logprob", cur),
        a(row_ids, i32, R, "row_ids", cur), ids, a(pair, i32, ids, "pair", cur), a(loss, f32, 1, "loss", cur),
        a(row_loss, f32, R, "row_loss", cur), a(row_reward, f32, R, "row_reward", cur), a(counts, i64, 2, "counts", cur),
        a(grad_logprob, f32, E, "grad_logprob", cur), a(status, i32, 1, "status", cur), a(ws, ws.dtype, 0, "ws", cur),
        ws.numel() * ws.element_size(), _loss_stream(torch, stream, cur)))


def odb_distill_workspace_size(tiles: Tiles, k: int) -> int:
    v = load().odb_distill_workspace_size(tiles.ref, int(k))
    if v == 0:
        _check(ODB_E_INVALID_ARG)
    return int(v)


def odb_distill_loss(tiles, params, student, teacher, slot_loss, slot_mean, slot_count, ws, slot_weight=None,
                     grad_student=None, status=None, stream=None):
    """Divergence of the student's lists [num_elems, k] from the teacher's, reduced and weighted per slot, and
    its gradient."""
    torch, f32, f64, i32, i64, _ = _torch_types()
    cur = _current(torch)
    _tiles_here(tiles, cur)
    K, E, a = tiles.num_slots, tiles.num_elems, _array
    if student.dim() < 2:
        raise ValueError(f"student: shape {tuple(student.shape)}, expected [{E}, k]")
    k = student.size(-1)
    for name, t in (("student", student), ("teacher", teacher), ("grad_student", grad_student)):
        if t is not None and (t.numel() != E * k or t.size(-1) != k):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected [{E}, {k}]")
    _check(load().odb_distill_loss(
        tiles.ref, ctypes.byref(params), k, a(student, f32, E * k, "student", cur),
        a(teacher, f32, E * k, "teacher", cur), a(slot_weight, f64, K, "slot_weight", cur),
        a(slot_loss, f32, K, "slot_loss", cur), a(slot_mean, f32, K, "slot_mean", cur),
        a(slot_count, i64, K, "slot_count", cur), a(grad_student, f32, E * k, "grad_student", cur),
        a(status, i32, 1, "status", cur), a(ws, ws.dtype, 0, "ws", cur), ws.numel() * ws.element_size(),
        _loss_stream(torch, stream, cur)))


class _PlanLosses:
    """Losses over the tiles of a pipeline's plan.  Output buffers and workspaces are kept and
    reused, one set for each kind of loss, and views of them are returned: a
    call overwrites what the last one of its kind returned, and two of one kind must not be under
    way at once.  A call that needs larger ones than any before it waits for the device and
    replaces them, so it cannot be captured, and a graph captured before it is no longer valid.
    Inputs are checked on the host; what the device finds wrong with them is collected until
    :meth:`check_losses`."""

    _loss_buffers = None

    def tiles(self, labels=None, first: int = 0, count: Optional[int] = None, shift: int = 1) -> Tiles:
        """The run of `count` slots from `first` on (default: all of the plan's).  ``labels`` is
        parallel to the plan's tiles (default: the collate's).  A run that is not the whole plan
        reads its four bounds from the device (one synchronisation)."""
        K = self.num_slots
        a, b = int(first), K if count is None else int(first) + int(count)
        if not 0 <= a <= b <= K:
            raise ValueError(f"slots [{a}, {b}) of a plan of {K}")
        R = int(self.info["emitted_samples" if "emitted_samples" in self.info else "emitted_views"])
        e, r = (0, int(self.info["padded_elems"])), (0, R)
        if (a, b) != (0, K):
            v = self.torch.stack([self.slot_tile_off[a], self.slot_tile_off[b], self.slot_row_off[a],
                                  self.slot_row_off[b]]).tolist()
            e, r = (v[0], v[1]), (v[2], v[3])
        if labels is None:
            if self.outputs is None:
                raise ValueError("collate first, or pass labels")
            labels = self.outputs[1]
        if not labels.is_contiguous():
            raise ValueError("labels: expected a contiguous tensor")
        if labels.numel() < e[1]:
            raise ValueError(f"labels: {labels.numel()} elements, the plan's tiles have {int(self.info['padded_elems'])}")
        return Tiles(self.slot_rows[a:b], self.slot_maxlen[a:b], self.slot_row_off[a:b + 1],
                     self.slot_tile_off[a:b + 1], labels.reshape(-1)[e[0]:e[1]], r[1] - r[0], shift, slice(a, b),
                     slice(*r), slice(*e))

    def _loss_outputs(self, kind: str, sizes: dict):
        """Kept buffers of at least the given sizes: {name: (elements, type)}."""
        torch = self.torch
        if self._loss_buffers is None:
            self._loss_buffers = {"status": torch.zeros(1, dtype=torch.int32, device=self.device)}
            _sync_current(self.device)
        small = [name for name, (n, _) in sizes.items()
                 if (kind, name) not in self._loss_buffers or self._loss_buffers[kind, name].numel() < n]
        if small:
            if any((kind, name) in self._loss_buffers for name in small):
                torch.cuda.synchronize(self.device)     # a call on any stream may still use the old ones
            for name in small:
                n, dtype = sizes[name]
                self._loss_buffers[kind, name] = torch.empty(max(n, 1), dtype=getattr(torch, dtype), device=self.device)
            # buffers may be used on another stream than the one they were allocated on
            _sync_current(self.device)
        return [self._loss_buffers[kind, name][:n] for name, (n, _) in sizes.items()], self._loss_buffers["status"]

    def policy_loss(self, tiles: Tiles, logprob, advantage, params: Optional[PolicyParams] = None, old_logprob=None,
                    ref_logprob=None, entropy=None, slot_weight=None, stream=None):
        """odb_policy_loss of a run's tiles, usually weighted by
        ``loss_weights(mode)[0][tiles.slots]`` with ``params.loss_scale`` the number of ranks.
        Returns (loss per slot, means [K, 4], counts [K, 4], gradient of the log-probabilities,
        gradient of the entropies or None)."""
        K, E = tiles.num_slots, tiles.num_elems
        (ws, loss, means, counts, grad, gent), status = self._loss_outputs("policy", {
            "ws": (odb_loss_workspace_size(tiles), "uint8"), "loss": (K, "float32"), "means": (4 * K, "float32"),
            "counts": (4 * K, "int64"), "grad": (E, "float32"), "gent": (0 if entropy is None else E, "float32")})
        gent = None if entropy is None else gent
        odb_policy_loss(tiles, PolicyParams() if params is None else params, logprob, advantage, loss, means, counts,
                        ws, old_logprob, ref_logprob, entropy, slot_weight, grad, gent, status, stream)
        return loss, means.view(K, 4), counts.view(K, 4), grad, gent

    def preference_loss(self, tiles: Tiles, logprob, pair, params: Optional[PreferenceParams] = None,
                        ref_logprob=None, stream=None):
        """odb_preference_loss of a run's tiles; ``pair`` is by sample id (the plan's emitted
        ids).  Returns (loss, loss per row, reward per row, counts [2], gradient of the
        log-probabilities)."""
        R, E = tiles.num_rows, tiles.num_elems
        (ws, loss, row_loss, reward, counts, grad), status = self._loss_outputs("preference", {
            "ws": (odb_loss_workspace_size(tiles, pair.numel()), "uint8"), "loss": (1, "float32"),
            "row_loss": (R, "float32"), "reward": (R, "float32"), "counts": (2, "int64"), "grad": (E, "float32")})
        odb_preference_loss(tiles, PreferenceParams() if params is None else params, logprob, pair, loss, row_loss,
                            reward, counts, ws, ref_logprob, self.emit_order[tiles.rows], grad, status, stream)
        return loss, row_loss, reward, counts, grad

    def distill_loss(self, tiles: Tiles, student, teacher, params: Optional[DistillParams] = None, slot_weight=None,
                     stream=None):
        """odb_distill_loss of a run's tiles: the student's and the teacher's log-probabilities of each token's
        list, [elements, k].  Returns (loss per slot, divergence per slot, counted tokens per slot, gradient of the
        student's log-probabilities [elements, k])."""
        K, E, k = tiles.num_slots, tiles.num_elems, student.size(-1)
        (ws, loss, mean, count, grad), status = self._loss_outputs("distill", {
            "ws": (odb_distill_workspace_size(tiles, k), "uint8"), "loss": (K, "float32"), "mean": (K, "float32"),
            "count": (K, "int64"), "grad": (E * k, "float32")})
        grad = grad.view(E, k)
        odb_distill_loss(tiles, DistillParams() if params is None else params, student, teacher, loss, mean, count, ws,
                         slot_weight, grad, status, stream)
        return loss, mean, count, grad

    def check_losses(self, stream=None):
        """Synchronises `stream` and raises if a loss since the last check met bad tiles or pairs."""
        if self._loss_buffers is None:
            return
        st = self._loss_buffers["status"]
        with self.torch.cuda.stream(stream if stream is not None else self.torch.cuda.current_stream()):
            bad = int(st.item())
            if bad:
                st.zero_()
                _sync_current(self.device)
        if bad:
            raise OdbError(ODB_E_INVALID_DATA, f"a loss met inconsistent tiles or pairs (device flags {bad})")


class Pipeline(_PlanLosses):
    """Device buffers of one window and the three-stage call sequence.

    Slot arrays start at ``W * max_r n_r`` capacity unless ``slot_capacity`` is given;
    outputs of :meth:`collate` are allocated (or reused) at ``padded_elems``.
    """

    def __init__(self, win: DeviceWindow, budget: int, mode: str = "join", quota: int = 0,
                 capacity=None, pad_id: int = 0, slot_capacity: Optional[int] = None):
        import torch

        self.torch = torch
        self.win = win
        self.budget = int(budget)
        self.mode = ODB_MODE_NONJOIN_QUOTA if mode == "nonjoin" else ODB_MODE_JOIN
        self.quota = int(quota)
        self.capacity = capacity
        self.pad_id = int(pad_id)
        dev = win.token_offsets.device
        self.device = dev
        n, W = win.num_samples, win.num_ranks
        n1 = max(n, 1)
        i32 = dict(dtype=torch.int32, device=dev)
        i64 = dict(dtype=torch.int64, device=dev)
        self.ws = torch.empty(odb_workspace_size(win), dtype=torch.uint8, device=dev)
        self.order = torch.empty(n1, **i32)
        self.sorted_len = torch.empty(n1, **i32)
        self.group_index = torch.empty(n1, **i32)
        self.groups_per_rank = torch.empty(W, **i32)
        self.emit_order = torch.empty(n1, **i32)
        self.row_token_start = torch.empty(n1, **i64)
        self.row_len = torch.empty(n1, **i32)
        self.leftover = torch.empty(n1, **i32)
        self.leftover_off = torch.empty(W + 1, **i64)
        if slot_capacity is None:
            sizes = np.diff(win.rank_offsets)
            slot_capacity = int(W * (sizes.max() if len(sizes) else 0))
        self._alloc_slots(max(int(slot_capacity), 1))
        self.info = None
        self.outputs = None

    def _alloc_slots(self, cap: int):
        torch = self.torch
        self.slot_capacity = cap
        self.slot_rows = torch.empty(cap, dtype=torch.int32, device=self.device)
        self.slot_maxlen = torch.empty(cap, dtype=torch.int32, device=self.device)
        self.slot_tokens = torch.empty(cap, dtype=torch.int64, device=self.device)
        self.slot_tokens_approx = torch.empty(cap, dtype=torch.float64, device=self.device)
        self.slot_row_off = torch.empty(cap + 1, dtype=torch.int64, device=self.device)
        self.slot_tile_off = torch.empty(cap + 1, dtype=torch.int64, device=self.device)
        # buffers may be used on another stream than the one they were allocated on
        _sync_current(self.device)

    def form(self, stream=None):
        odb_form_groups(self.win, self.budget, self.order, self.sorted_len, self.group_index,
                        self.groups_per_rank, self.ws, stream)

    def align(self, stream=None) -> dict:
        args = lambda: (self.win, self.budget, self.mode, self.quota, self.capacity, self.order, self.sorted_len,
                        self.group_index, self.groups_per_rank, self.slot_capacity, self.emit_order,
                        self.slot_rows, self.slot_maxlen, self.slot_row_off, self.slot_tile_off, self.slot_tokens,
                        self.leftover, self.leftover_off, self.ws, stream)
        # both argument sets are read when the call is made: a retry after ODB_E_CAPACITY
        # must pass the reallocated slot arrays, every one of them
        rec = lambda: dict(slot_tokens_approx=self.slot_tokens_approx, row_token_start=self.row_token_start,
                           row_len=self.row_len)
        st, info = odb_align_groups(*args(), raise_on_capacity=False, **rec())
        if st == ODB_E_CAPACITY:
            self._alloc_slots(int(info["required_slot_capacity"]))
            st, info = odb_align_groups(*args(), **rec())
        self.info = info
        return info

    @property
    def num_slots(self) -> int:
        return self.win.num_ranks * int(self.info["steps"])

    def alloc_outputs(self, elems: int):
        torch = self.torch
        elems = max(int(elems), 1)
        if self.outputs is None or self.outputs[0].numel() < elems:
            self.outputs = tuple(torch.empty(elems, dtype=torch.int32, device=self.device) for _ in range(4))
            # the allocator may hand out memory freed by work still queued on the current
            # stream; the library may write it on another stream
            _sync_current(self.device)
        return self.outputs

    def collate(self, stream=None):
        P = int(self.info["padded_elems"])
        outs = self.alloc_outputs(P)
        odb_collate(self.win, self.num_slots, self.emit_order, self.slot_rows, self.slot_maxlen, self.slot_row_off,
                    self.slot_tile_off, self.pad_id, P, *outs, self.ws, stream, row_token_start=self.row_token_start,
                    row_len=self.row_len)
        return tuple(o[:P] for o in outs)

    def loss_weights(self, mode: int = ODB_WEIGHT_TOKEN_EXACT, stream=None):
        """Per-slot loss-scaling weights (rank-major, W * S) and the per-step sums of real
        tokens and samples over ranks, as device tensors."""
        torch = self.torch
        S = int(self.info["steps"])
        K = self.num_slots
        if getattr(self, "_weights", None) is None or self._weights[0].numel() < max(K, 1) \
                or self._weights[1].numel() < max(S, 1):
            self._weights = (torch.empty(max(K, 1), dtype=torch.float64, device=self.device),
                             torch.empty(max(S, 1), dtype=torch.int64, device=self.device),
                             torch.empty(max(S, 1), dtype=torch.int64, device=self.device))
        wt, st, ss = self._weights
        odb_loss_weights(self.win.num_ranks, S, mode, self.slot_rows, self.slot_tokens, self.slot_tokens_approx,
                         wt, st, ss, stream)
        return wt[:K], st[:S], ss[:S]

    def run(self, stream=None):
        self.form(stream)
        self.align(stream)
        return self.collate(stream)


def stream_round_bound(num_samples: int, num_ranks: int, buffer_size: int, rate) -> int:
    """Rounds one logical iteration can take: at most ceil(N/W) emitting rounds, between
    them at most ceil(buffer_size / min rate) fill rounds, and the stop round."""
    q = -(-int(num_samples) // int(num_ranks)) if num_samples else 0
    fill = -(-int(buffer_size) // int(np.min(rate)))
    return q + (q + 1) * fill + 2


class StreamPipeline(_PlanLosses):
    """Device buffers of one streaming iteration (odb_stream_plan) and its collate and
    loss weights (odb_collate / odb_loss_weights on the streaming plan)."""

    def __init__(self, win: DeviceWindow, perm, budget: int, buffer_size: int = 1024, depth: Optional[int] = None,
                 rate=None, mode: str = "join", quota: int = 0, capacity=None, pad_id: int = 0,
                 max_rounds: Optional[int] = None, slot_capacity: Optional[int] = None):
        import torch

        self.torch = torch
        self.win = win
        self.perm = perm
        self.budget = int(budget)
        W, N = win.num_ranks, win.num_samples
        self.W, self.N = W, N
        self.q = -(-N // W) if N else 0
        self.M = self.q * W
        depth = int(buffer_size if depth is None else depth)
        rate = np.full(W, buffer_size, np.int32) if rate is None else np.ascontiguousarray(rate, dtype=np.int32)
        self.rate = rate
        self.cap = None if capacity is None else np.ascontiguousarray(capacity, dtype=np.int64)
        if max_rounds is None:
            max_rounds = stream_round_bound(N, W, buffer_size, rate)
        self.params = StreamParams(ODB_MODE_NONJOIN_QUOTA if mode == "nonjoin" else ODB_MODE_JOIN, int(buffer_size),
                                   depth, 0, int(quota), rate.ctypes.data_as(ctypes.c_void_p).value,
                                   None if self.cap is None else self.cap.ctypes.data_as(ctypes.c_void_p).value,
                                   int(max_rounds))
        self.pad_id = int(pad_id)
        dev = win.token_offsets.device
        self.device = dev
        m1 = max(self.M, 1)
        self.emit_order = torch.empty(m1, dtype=torch.int32, device=dev)
        self.emit_views = torch.empty(m1, dtype=torch.int32, device=dev)
        self.row_token_start = torch.empty(m1, dtype=torch.int64, device=dev)
        self.row_len = torch.empty(m1, dtype=torch.int32, device=dev)
        self.left_views = torch.empty(m1, dtype=torch.int32, device=dev)
        self.left_off = torch.empty(W + 1, dtype=torch.int64, device=dev)
        self._alloc_slots(max(int(slot_capacity if slot_capacity is not None else W * max(self.q, 1)), W))
        self.trace = (StreamRound * max(int(max_rounds), 1))()
        self.info = None
        self.outputs = None

    def _alloc_slots(self, cap: int):
        torch = self.torch
        cap = (cap + self.W - 1) // self.W * self.W
        self.slot_capacity = cap
        d = self.device
        self.slot_rows = torch.empty(cap, dtype=torch.int32, device=d)
        self.slot_maxlen = torch.empty(cap, dtype=torch.int32, device=d)
        self.slot_tokens = torch.empty(cap, dtype=torch.int64, device=d)
        self.slot_tokens_approx = torch.empty(cap, dtype=torch.float64, device=d)
        self.slot_row_off = torch.empty(cap + 1, dtype=torch.int64, device=d)
        self.slot_tile_off = torch.empty(cap + 1, dtype=torch.int64, device=d)
        size = load().odb_stream_workspace_size(self.win.ref, self.params.depth, cap, self.params.max_rounds)
        if size == 0:
            _check(ODB_E_INVALID_ARG)
        self.ws = torch.empty(size, dtype=torch.uint8, device=d)
        # buffers may be used on another stream than the one they were allocated on
        _sync_current(d)

    def _call(self, stream):
        info = StreamInfo()
        st = load().odb_stream_plan(self.win.ref, _dptr(self.perm), self.budget, ctypes.byref(self.params),
                                    self.slot_capacity, _dptr(self.emit_order), _dptr(self.emit_views),
                                    _dptr(self.row_token_start), _dptr(self.row_len), _dptr(self.slot_rows), _dptr(self.slot_maxlen), _dptr(self.slot_row_off),
                                    _dptr(self.slot_tile_off), _dptr(self.slot_tokens),
                                    _dptr(self.slot_tokens_approx), _dptr(self.left_views), _dptr(self.left_off),
                                    ctypes.cast(self.trace, ctypes.c_void_p), ctypes.byref(info), _dptr(self.ws),
                                    self.ws.numel(), _stream(stream))
        return st, info.as_dict()

    def plan(self, stream=None) -> dict:
        st, info = self._call(stream)
        if st == ODB_E_CAPACITY and info["required_slot_capacity"] > self.slot_capacity:
            self._alloc_slots(int(info["required_slot_capacity"]))
            st, info = self._call(stream)
        _check(st)
        self.info = info
        return info

    def trace_array(self) -> np.ndarray:
        """Rounds as rows (kind, target, emitted, phi)."""
        n = int(self.info["rounds"])
        return np.array([(self.trace[i].kind, self.trace[i].target, self.trace[i].emitted, self.trace[i].phi)
                         for i in range(n)], dtype=np.int64).reshape(-1, 4)

    @property
    def num_slots(self) -> int:
        return self.W * int(self.info["steps"])

    def collate(self, stream=None):
        torch = self.torch
        P = int(self.info["padded_elems"])
        if self.outputs is None or self.outputs[0].numel() < max(P, 1):
            self.outputs = tuple(torch.empty(max(P, 1), dtype=torch.int32, device=self.device) for _ in range(4))
            _sync_current(self.device)
        odb_collate(self.win, self.num_slots, self.emit_order, self.slot_rows, self.slot_maxlen, self.slot_row_off,
                    self.slot_tile_off, self.pad_id, P, *self.outputs, self.ws, stream,
                    row_token_start=self.row_token_start, row_len=self.row_len)
        return tuple(o[:P] for o in self.outputs)

    def loss_weights(self, mode: int = ODB_WEIGHT_TOKEN_EXACT, stream=None):
        """As Pipeline.loss_weights; the output buffers are kept and reused (views of
        them are returned), so a call on another stream never writes freed memory."""
        torch = self.torch
        S, K = int(self.info["steps"]), self.num_slots
        if getattr(self, "_weights", None) is None or self._weights[0].numel() < max(K, 1) \
                or self._weights[1].numel() < max(S, 1):
            self._weights = (torch.empty(max(K, 1), dtype=torch.float64, device=self.device),
                             torch.empty(max(S, 1), dtype=torch.int64, device=self.device),
                             torch.empty(max(S, 1), dtype=torch.int64, device=self.device))
        wt, st, ss = self._weights
        odb_loss_weights(self.W, S, mode, self.slot_rows, self.slot_tokens, self.slot_tokens_approx, wt, st, ss,
                         stream)
        return wt[:K], st[:S], ss[:S]
