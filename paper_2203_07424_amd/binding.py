"""ctypes binding of the C boundary declared in include/rec.h and include/rec_history.h.

Argument marshalling only: every step of the forward pass, and of attention over
user histories, runs in the HIP library.  PyTorch supplies device memory and the stream.  Importing this
module raises if the library has not been built; there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import List, Optional, Sequence, Tuple

import torch  # loads the HIP runtime the library binds to

_PKG = os.path.dirname(os.path.abspath(__file__))
# REC_MI355X_LIBRARY: another build of the same library (the host-instrumented
# one of build.build_host_sanitized()); unset in normal use.
LIB_PATH = os.environ.get("REC_MI355X_LIBRARY") or os.path.join(_PKG, "librec_mi355x.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it first (python -m paper_2203_07424_amd.build "
        "or __graft_entry__.build()); there is no CPU fallback")

_lib = C.CDLL(LIB_PATH)
_F32, _I32 = torch.float32, torch.int32

REC_OK = 0
REC_ERR_ARG, REC_ERR_SHAPE, REC_ERR_STATE, REC_ERR_LENGTHS = 1, 2, 3, 4
REC_ERR_INDEX_RANGE, REC_ERR_OVERFLOW, REC_ERR_DEVICE, REC_ERR_CAPACITY = 5, 6, 7, 8
REC_ERR_VALUE = 9
REC_STATIC_SCRATCH_BYTES = 64 << 20
REC_STATIC_MAX_TABLES = 64
REC_F32, REC_F16, REC_BF16 = 0, 1, 2
REC_MX4, REC_MX8 = 0, 1
REC_FAULT_LENGTH, REC_FAULT_SLOT, REC_FAULT_PAGE, REC_FAULT_VALUE, REC_FAULT_WORDS = 0, 1, 2, 3, 4
REC_BOTTOM, REC_TOP = 0, 1          # REC_TOP + k: tower k of the Predict-FC
REC_INTERACT_DOT, REC_INTERACT_CONCAT = 0, 1
REC_MAX_TOWERS = 8
REC_DBG_OFFSETS, REC_DBG_POOLED, REC_DBG_BOTTOM_OUT, REC_DBG_INTERACT = 0, 1, 2, 3
REC_OPT_OVERLAP_DENSE = 0
REC_OPT_STREAM_ROWS = 1
REC_OPT_FUSE_MLP = 2
REC_OPT_PIPELINE = 3
REC_NUM_STAGES = 7
REC_FC_F32_ROWS, REC_FC_DOT, REC_FC_BESIDE_POOLING, REC_FC_ANY_ORDER = 1, 2, 4, 8
REC_FORM_TILES, REC_FORM_WIDE, REC_FORM_SPLIT = 0, 1, 2
REC_PLAN_RIDE, REC_PLAN_FRONT, REC_PLAN_LAYER, REC_PLAN_TAIL = 1, 2, 4, 8
(REC_POOL_BAG, REC_POOL_TWO, REC_POOL_SHORT, REC_POOL_HOT, REC_POOL_FRONT, REC_POOL_FRONT_LIGHT, REC_POOL_FEW_LOOKUPS,
 REC_POOL_MANY_LOOKUPS, REC_POOL_BESIDE_WIDE) = range(9)
STAGE_NAMES = ("scan", "pool", "bottom_first", "bottom_rest", "interact", "top_first", "top_rest")

EXPORTS = ("rec_create", "rec_destroy", "rec_workspace_bytes", "rec_bind_workspace",
           "rec_load_tables", "rec_load_hot_rows", "rec_mlp_packed_bytes", "rec_load_mlp", "rec_forward", "rec_forward_static", "rec_check",
           "rec_debug_get", "rec_set_option", "rec_set_dense_stream", "rec_set_pool_streams", "rec_drain", "rec_set_profiling", "rec_stage_ms", "rec_stage_shared", "rec_status_string",
           "rec_synth_fill_table", "rec_probe_mfma", "rec_probe_scan", "rec_probe_fc_form", "rec_probe_plan",
           "rec_probe_plan_joined", "rec_probe_plan_pooling", "rec_probe_dense_copy",
           "rec_history_bytes", "rec_history_write", "rec_history_read", "rec_history_attend_workspace_bytes",
           "rec_history_attend", "rec_window_attend", "rec_history_check", "rec_probe_clear_faults", "rec_probe_history_form")


class rec_config(C.Structure):
    _fields_ = [("num_tables", C.c_int32), ("emb_dim", C.c_int32),
                ("rows", C.POINTER(C.c_int64)), ("table_dtype", C.c_int32),
                ("num_dense", C.c_int32), ("n_bottom", C.c_int32),
                ("bottom_widths", C.POINTER(C.c_int32)), ("n_top", C.c_int32),
                ("top_widths", C.POINTER(C.c_int32)), ("max_batch", C.c_int32),
                ("max_nnz", C.c_int64), ("interaction", C.c_int32), ("num_towers", C.c_int32)]


class rec_history(C.Structure):
    _fields_ = [("dev_pages", C.c_void_p), ("num_pages", C.c_int64), ("page_tokens", C.c_int32),
                ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("format", C.c_int32), ("dev_fault", C.c_void_p)]


class rec_rows(C.Structure):
    _fields_ = [("dev", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class rec_query(C.Structure):
    _fields_ = [("dev_q", C.c_void_p), ("dev_out", C.c_void_p), ("batch_stride", C.c_int64),
                ("query_stride", C.c_int64), ("head_stride", C.c_int64), ("dtype", C.c_int32), ("batch", C.c_int32),
                ("queries", C.c_int32), ("heads", C.c_int32), ("dev_pages_of", C.c_void_p), ("table_stride", C.c_int64),
                ("table_width", C.c_int32), ("dev_lengths", C.c_void_p), ("scale", C.c_float), ("window", C.c_int32),
                ("sinks", C.c_int32), ("candidates", C.c_int32)]


class rec_window(C.Structure):
    _fields_ = [("q", rec_rows), ("k", rec_rows), ("v", rec_rows), ("dev_out", C.c_void_p), ("dtype", C.c_int32),
                ("batch", C.c_int32), ("tokens", C.c_int64), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dev_offsets", C.c_void_p), ("scale", C.c_float), ("window", C.c_int32),
                ("sinks", C.c_int32), ("dev_fault", C.c_void_p)]


_vp = C.c_void_p
_lib.rec_create.restype = C.c_int
_lib.rec_create.argtypes = [C.POINTER(rec_config), C.POINTER(_vp)]
_lib.rec_destroy.restype = None
_lib.rec_destroy.argtypes = [_vp]
_lib.rec_workspace_bytes.restype = C.c_size_t
_lib.rec_workspace_bytes.argtypes = [_vp]
_lib.rec_bind_workspace.restype = C.c_int
_lib.rec_bind_workspace.argtypes = [_vp, _vp, C.c_size_t, _vp]
_lib.rec_load_tables.restype = C.c_int
_lib.rec_load_tables.argtypes = [_vp, C.c_int32, _vp]
_lib.rec_load_hot_rows.restype = C.c_int
_lib.rec_load_hot_rows.argtypes = [_vp, C.c_int32, _vp, C.c_int32]
_lib.rec_mlp_packed_bytes.restype = C.c_size_t
_lib.rec_mlp_packed_bytes.argtypes = [_vp, C.c_int32, C.c_int32]
_lib.rec_load_mlp.restype = C.c_int
_lib.rec_load_mlp.argtypes = [_vp, C.c_int32, C.c_int32, _vp, _vp, _vp, _vp]
_lib.rec_forward.restype = C.c_int
_lib.rec_forward.argtypes = [_vp, _vp, _vp, _vp, C.c_int32, C.c_int64, _vp, _vp]
_lib.rec_forward_static.restype = C.c_int
_lib.rec_forward_static.argtypes = [_vp, _vp, _vp, _vp, C.c_int32, C.c_int64, _vp, _vp, _vp]
_lib.rec_check.restype = C.c_int
_lib.rec_check.argtypes = [_vp, _vp, C.POINTER(C.c_int64)]
_lib.rec_debug_get.restype = C.c_int
_lib.rec_debug_get.argtypes = [_vp, C.c_int32, C.POINTER(_vp), C.POINTER(C.c_int64)]
_lib.rec_set_option.restype = C.c_int
_lib.rec_set_option.argtypes = [_vp, C.c_int32, C.c_int32]
_lib.rec_set_dense_stream.restype = C.c_int
_lib.rec_set_dense_stream.argtypes = [_vp, _vp]
_lib.rec_set_pool_streams.restype = C.c_int
_lib.rec_set_pool_streams.argtypes = [_vp, _vp, _vp]
_lib.rec_drain.restype = C.c_int
_lib.rec_drain.argtypes = [_vp, _vp]
_lib.rec_set_profiling.restype = C.c_int
_lib.rec_set_profiling.argtypes = [_vp, C.c_int32, C.c_int32]
_lib.rec_stage_ms.restype = C.c_int
_lib.rec_stage_ms.argtypes = [_vp, C.c_int32, C.POINTER(C.c_float)]
_lib.rec_stage_shared.restype = C.c_int
_lib.rec_stage_shared.argtypes = [_vp, C.c_int32, C.POINTER(C.c_uint32)]
_lib.rec_status_string.restype = C.c_char_p
_lib.rec_status_string.argtypes = [C.c_int]
_lib.rec_synth_fill_table.restype = C.c_int
_lib.rec_synth_fill_table.argtypes = [_vp, C.c_int32, C.c_uint64, C.c_int32, C.c_int64, C.c_int32, _vp]


_lib.rec_probe_mfma.restype = C.c_int
_lib.rec_probe_mfma.argtypes = [C.c_int32, C.c_int32, C.c_int32, _vp, _vp]
_lib.rec_probe_scan.restype = C.c_int
_lib.rec_probe_scan.argtypes = [_vp, C.c_int32, C.c_int64, _vp, _vp, C.c_int32, _vp, _vp]
_lib.rec_probe_plan.restype = C.c_int
_lib.rec_probe_plan.argtypes = [_vp, C.c_int32, C.c_int64, C.POINTER(C.c_uint32), C.POINTER(C.c_int32)]
_lib.rec_probe_plan_joined.restype = C.c_int
_lib.rec_probe_plan_joined.argtypes = [_vp, C.c_int32, C.c_int64, C.POINTER(C.c_int32)]
_lib.rec_probe_plan_pooling.restype = C.c_int
_lib.rec_probe_plan_pooling.argtypes = [_vp, C.c_int32, C.c_int64, C.POINTER(C.c_int32)]
_lib.rec_probe_dense_copy.restype = C.c_int
_lib.rec_probe_dense_copy.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
_lib.rec_probe_fc_form.restype = C.c_int
_lib.rec_probe_fc_form.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_uint32, C.c_int32, C.POINTER(C.c_int32)]

# Structures go in by address: a ctypes structure by reference, or one packed into bytes.
_lib.rec_history_bytes.restype = C.c_size_t
_lib.rec_history_bytes.argtypes = [_vp]
_lib.rec_history_write.restype = C.c_int
_lib.rec_history_write.argtypes = [_vp, _vp, _vp, C.c_int32, _vp, C.c_int64, _vp]
_lib.rec_history_read.restype = C.c_int
_lib.rec_history_read.argtypes = [_vp, _vp, C.c_int64, C.c_int32, _vp, _vp, _vp]
_lib.rec_history_attend_workspace_bytes.restype = C.c_size_t
_lib.rec_history_attend_workspace_bytes.argtypes = [_vp, _vp]
_lib.rec_history_attend.restype = C.c_int
_lib.rec_history_attend.argtypes = [_vp, _vp, _vp, C.c_size_t, _vp]
_lib.rec_window_attend.restype = C.c_int
_lib.rec_window_attend.argtypes = [_vp, _vp]
_lib.rec_history_check.restype = C.c_int
_lib.rec_history_check.argtypes = [_vp, _vp, C.POINTER(C.c_int64), C.POINTER(C.c_int32)]
_lib.rec_probe_history_form.restype = C.c_int
_lib.rec_probe_history_form.argtypes = [_vp, _vp, C.POINTER(C.c_int32)]
_lib.rec_probe_clear_faults.restype = C.c_int
_lib.rec_probe_clear_faults.argtypes = [_vp, C.POINTER(C.c_uint64), _vp]
# The same layouts for one packing call, a quarter of the time of setting a structure's fields.
_ROWS, _QUERY, _WINDOW = struct.Struct("@Pqq"), struct.Struct("@PPqqqiiiiPqiPfiii"), struct.Struct("@PqqPqqPqqPiiqiiiPfiiP")
assert (_ROWS.size, _QUERY.size, _WINDOW.size) == (C.sizeof(rec_rows), C.sizeof(rec_query), C.sizeof(rec_window))


class RecError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def status_string(status: int) -> str:
    return _lib.rec_status_string(int(status)).decode()


def _stream() -> Optional[int]:
    # Behind the first use of the device its current stream is one cheap lookup; asking
    # whether there is a device and building a stream object took a third of a
    # forward's host time.
    if torch.cuda.is_initialized():
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    # Without a device only the host-side argument checks of the library can
    # run, and those never touch the stream.
    if not torch.cuda.is_available():
        return None
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# Raw entry points, same names as the C boundary; each returns the status.
def rec_create(num_tables: int, emb_dim: int, rows: Sequence[int], table_dtype: int,
               num_dense: int, bottom_widths: Sequence[int], top_widths: Sequence[int],
               max_batch: int, max_nnz: int, interaction: int = REC_INTERACT_DOT,
               num_towers: int = 1) -> Tuple[int, Optional[int]]:
    rows_a = (C.c_int64 * len(rows))(*rows)
    bw = (C.c_int32 * len(bottom_widths))(*bottom_widths)
    tw = (C.c_int32 * len(top_widths))(*top_widths)
    cfg = rec_config(num_tables, emb_dim, rows_a, table_dtype, num_dense, len(bottom_widths) - 1,
                     bw, len(top_widths) - 1, tw, max_batch, max_nnz, interaction, num_towers)
    out = _vp()
    st = _lib.rec_create(C.byref(cfg), C.byref(out))
    return st, out.value


def rec_destroy(m: int) -> None:
    _lib.rec_destroy(m)


def rec_workspace_bytes(m: int) -> int:
    return int(_lib.rec_workspace_bytes(m))


def rec_bind_workspace(m: int, ws: torch.Tensor) -> int:
    return _lib.rec_bind_workspace(m, ws.data_ptr(), ws.numel() * ws.element_size(), _stream())


def rec_load_tables(m: int, table: int, dev_rows: torch.Tensor) -> int:
    return _lib.rec_load_tables(m, table, dev_rows.data_ptr())


def rec_load_hot_rows(m: int, table: int, dev_ids: Optional[torch.Tensor]) -> int:
    n = 0 if dev_ids is None else dev_ids.numel()
    return _lib.rec_load_hot_rows(m, table, _ptr(dev_ids), n)


def rec_mlp_packed_bytes(m: int, which: int, layer: int) -> int:
    return int(_lib.rec_mlp_packed_bytes(m, which, layer))


def rec_load_mlp(m: int, which: int, layer: int, dev_W: torch.Tensor, dev_b: torch.Tensor,
                 dev_packed: torch.Tensor) -> int:
    return _lib.rec_load_mlp(m, which, layer, dev_W.data_ptr(), dev_b.data_ptr(),
                             dev_packed.data_ptr(), _stream())


def rec_forward(m: int, dev_dense, dev_indices, dev_lengths, batch: int, nnz: int, dev_logits) -> int:
    return _lib.rec_forward(m, _ptr(dev_dense), _ptr(dev_indices), _ptr(dev_lengths), batch, nnz,
                            _ptr(dev_logits), _stream())


def rec_forward_static(m: int, dev_dense, dev_indices, dev_lengths, batch: int, nnz: int, dev_logits,
                       dev_fault=None) -> int:
    return _lib.rec_forward_static(m, _ptr(dev_dense), _ptr(dev_indices), _ptr(dev_lengths), batch, nnz,
                                   _ptr(dev_logits), _ptr(dev_fault), _stream())


def rec_check(m: int) -> Tuple[int, int]:
    pos = C.c_int64(-1)
    st = _lib.rec_check(m, _stream(), C.byref(pos))
    return st, int(pos.value)


def rec_debug_get(m: int, what: int) -> Tuple[int, Optional[int], int]:
    p, ld = _vp(), C.c_int64(0)
    st = _lib.rec_debug_get(m, what, C.byref(p), C.byref(ld))
    return st, p.value, int(ld.value)


def rec_set_option(m: int, option: int, value: int) -> int:
    return _lib.rec_set_option(m, int(option), int(value))


def rec_set_dense_stream(m: int, stream: Optional["torch.cuda.Stream"]) -> int:
    return _lib.rec_set_dense_stream(m, None if stream is None else stream.cuda_stream)


def rec_set_pool_streams(m: int, a: Optional["torch.cuda.Stream"], b: Optional["torch.cuda.Stream"]) -> int:
    return _lib.rec_set_pool_streams(m, None if a is None else a.cuda_stream, None if b is None else b.cuda_stream)


def rec_drain(m: int) -> int:
    return _lib.rec_drain(m, _stream())


def rec_set_profiling(m: int, slots: int, period: int = 1) -> int:
    return _lib.rec_set_profiling(m, int(slots), int(period))


def rec_stage_ms(m: int, slot: int = 0) -> Tuple[int, List[float]]:
    ms = (C.c_float * REC_NUM_STAGES)()
    st = _lib.rec_stage_ms(m, slot, ms)
    return st, [float(v) for v in ms]


def rec_stage_shared(m: int, slot: int = 0) -> Tuple[int, int]:
    mask = C.c_uint32(0)
    st = _lib.rec_stage_shared(m, slot, C.byref(mask))
    return st, int(mask.value)


def rec_synth_fill_table(dev_rows: torch.Tensor, seed: int, table: int) -> int:
    dtype = REC_F16 if dev_rows.dtype == torch.float16 else REC_F32
    return _lib.rec_synth_fill_table(dev_rows.data_ptr(), dtype, seed, table, dev_rows.shape[0],
                                     dev_rows.shape[1], _stream())


def rec_probe_mfma(random_operands: bool, blocks: int, iters: int, dev_sink: Optional[torch.Tensor]) -> int:
    """One launch of nothing but bf16 matrix instructions (blocks * 8 * iters * 32 * 32768 flops)."""
    return _lib.rec_probe_mfma(int(bool(random_operands)), int(blocks), int(iters), _ptr(dev_sink), _stream())


def rec_probe_scan(dev_lengths: torch.Tensor, nnz: int, dev_offsets: torch.Tensor, dev_words: torch.Tensor,
                   polls: int, dev_err: torch.Tensor) -> int:
    """The offsets scan alone; dev_words int64, one per 2048 lengths, zero on entry; dev_err 64 bytes."""
    return _lib.rec_probe_scan(_ptr(dev_lengths), dev_lengths.numel(), int(nnz), _ptr(dev_offsets), _ptr(dev_words),
                               int(polls), _ptr(dev_err), _stream())


def rec_probe_fc_form(rows: int, inputs: int, outputs: int, stacks: int = 1, flags: int = 0,
                      compute_units: int = 256) -> Tuple[int, Tuple[int, int, int, int]]:
    """(status, (REC_FORM_*, rows and columns of a block's tile, waves that share its k))."""
    form = (C.c_int32 * 4)()
    st = _lib.rec_probe_fc_form(int(rows), int(inputs), int(outputs), int(stacks), int(flags), int(compute_units), form)
    return st, tuple(form)


def rec_probe_plan(m: int, batch: int, nnz: int) -> Tuple[int, int, int]:
    """(status, REC_PLAN_* bits, first Bottom-FC layer that the joint Predict-FC launch takes)."""
    mask, tail_from = C.c_uint32(0), C.c_int32(0)
    st = _lib.rec_probe_plan(m, int(batch), int(nnz), C.byref(mask), C.byref(tail_from))
    return st, mask.value, tail_from.value


def rec_probe_plan_joined(m: int, batch: int, nnz: int) -> Tuple[int, bool]:
    """(status, whether pooling shares the launch of scan and a first layer of large tiles)."""
    joined = C.c_int32(0)
    st = _lib.rec_probe_plan_joined(m, int(batch), int(nnz), C.byref(joined))
    return st, bool(joined.value)


def rec_probe_plan_pooling(m: int, batch: int, nnz: int) -> Tuple[int, int]:
    """(status, REC_POOL_*: the form of pooling that a forward takes)."""
    form = C.c_int32(-1)
    st = _lib.rec_probe_plan_pooling(m, int(batch), int(nnz), C.byref(form))
    return st, form.value


def rec_probe_dense_copy(rows: int, columns: int, pad: int, left: int = -1) -> Tuple[int, int, int, int]:
    """(status, blocks, waves of a block, units a wave) for the copy of a concatenation model's dense part."""
    deal = (C.c_int32 * 3)()
    st = _lib.rec_probe_dense_copy(int(rows), int(columns), int(pad), int(left), deal)
    return st, *deal


# User histories: same names, structures by reference.
def rec_history_bytes(h: rec_history) -> int:
    return int(_lib.rec_history_bytes(C.byref(h)))


def rec_history_write(h: rec_history, k: rec_rows, v: rec_rows, dtype: int, dev_slots, tokens: int) -> int:
    return _lib.rec_history_write(C.byref(h), C.byref(k), C.byref(v), int(dtype), _ptr(dev_slots), int(tokens), _stream())


def rec_history_read(h: rec_history, dev_slots, tokens: int, dtype: int, dev_k, dev_v) -> int:
    return _lib.rec_history_read(C.byref(h), _ptr(dev_slots), int(tokens), int(dtype), _ptr(dev_k), _ptr(dev_v), _stream())


def rec_history_attend_workspace_bytes(h: rec_history, q: rec_query) -> int:
    return int(_lib.rec_history_attend_workspace_bytes(C.byref(h), C.byref(q)))


def rec_history_attend(h: rec_history, q: rec_query, workspace=None) -> int:
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    return _lib.rec_history_attend(C.byref(h), C.byref(q), _ptr(workspace), nbytes, _stream())


def rec_window_attend(w: rec_window) -> int:
    return _lib.rec_window_attend(C.byref(w), _stream())


def _is_record(fault: torch.Tensor) -> bool:
    """Words next to each other: kernels write REC_FAULT_WORDS of them from the first on."""
    return fault.dtype is torch.int64 and fault.numel() >= REC_FAULT_WORDS and fault.is_contiguous()


def rec_history_check(dev_fault: torch.Tensor) -> Tuple[int, int, int]:
    """(status, position, REC_FAULT_* word) of a record on the current device; the last two -1 without a fault.
    Waits for the current stream: calls on others are counted once their work is done."""
    if not _is_record(dev_fault):
        raise ValueError(f"rec_history_check: a fault record is a contiguous int64 [{REC_FAULT_WORDS}]")
    pos, word = C.c_int64(-1), C.c_int32(-1)
    st = _lib.rec_history_check(_ptr(dev_fault), _stream_on(dev_fault.get_device(), "rec_history_check"), C.byref(pos), C.byref(word))
    return st, pos.value, word.value


def rec_probe_history_form(h: rec_history, q: rec_query) -> Tuple[int, int, int, int]:
    """(status, waves of a block, parts of a history, kv heads of a wave)."""
    form = (C.c_int32 * 3)()
    st = _lib.rec_probe_history_form(C.byref(h), C.byref(q), form)
    return (st, *form)


def rec_probe_clear_faults(dev_fault: torch.Tensor, seen: Sequence[int]) -> int:
    """seen: what was read of the record, a word each (-1: no fault)."""
    if not _is_record(dev_fault) or len(seen) != REC_FAULT_WORDS:
        raise ValueError(f"rec_probe_clear_faults: a fault record is a contiguous int64 [{REC_FAULT_WORDS}]")
    words = (C.c_uint64 * REC_FAULT_WORDS)(*(int(x) & (1 << 64) - 1 for x in seen))
    return _lib.rec_probe_clear_faults(_ptr(dev_fault), words, _stream_on(dev_fault.get_device(), "rec_probe_clear_faults"))


class RecModel:
    """Owns the device buffers of one model and forwards batches through the library."""

    def __init__(self, num_tables: int, emb_dim: int, rows: Sequence[int], table_dtype: str,
                 num_dense: int, bottom_widths: Sequence[int], top_widths: Sequence[int],
                 max_batch: int, max_nnz: int, device: str = "cuda:0", interaction: str = "dot",
                 towers: int = 1, pipeline: bool = False,
                 dense_stream: Optional["torch.cuda.Stream"] = None,
                 pool_streams: Sequence[Optional["torch.cuda.Stream"]] = (None, None)):
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the forward pass has no CPU path")
        self.device = torch.device(device)
        self.T, self.D, self.F = num_tables, emb_dim, num_dense
        self.table_dtype = {"f32": torch.float32, "f16": torch.float16}[table_dtype]
        self.width = top_widths[0]
        self.n_bottom, self.n_top = len(bottom_widths) - 1, len(top_widths) - 1
        self.towers, self.w0 = towers, bottom_widths[-1]
        code = REC_F16 if table_dtype == "f16" else REC_F32
        inter = {"dot": REC_INTERACT_DOT, "concat": REC_INTERACT_CONCAT}[interaction]
        st, self.handle = rec_create(num_tables, emb_dim, list(rows), code, num_dense,
                                     list(bottom_widths), list(top_widths), max_batch, max_nnz,
                                     inter, towers)
        if st != REC_OK:
            raise RecError(st, "rec_create")
        self.pipeline, self.dense_stream, self.pool_streams = bool(pipeline), dense_stream, tuple(pool_streams)
        if pipeline:      # decides the workspace size, so it is set before binding
            self._ok(rec_set_option(self.handle, REC_OPT_PIPELINE, 1), "rec_set_option")
            self._ok(rec_set_dense_stream(self.handle, dense_stream), "rec_set_dense_stream")
            self._ok(rec_set_pool_streams(self.handle, *self.pool_streams), "rec_set_pool_streams")
        self.ws = torch.empty(rec_workspace_bytes(self.handle), dtype=torch.uint8, device=self.device)
        self._ok(rec_bind_workspace(self.handle, self.ws), "rec_bind_workspace")
        self.tables: List[Optional[torch.Tensor]] = [None] * num_tables
        self.hot: List[Optional[torch.Tensor]] = [None] * num_tables
        self.packed: dict = {}
        self.last_batch = 0

    def _ok(self, st: int, where: str) -> None:
        if st != REC_OK:
            raise RecError(st, where)

    def close(self) -> None:
        if getattr(self, "handle", None):
            torch.cuda.synchronize(self.device)
            rec_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def load_table(self, t: int, dev_rows: torch.Tensor) -> None:
        assert dev_rows.is_cuda and dev_rows.is_contiguous() and dev_rows.dtype == self.table_dtype
        self._ok(rec_load_tables(self.handle, t, dev_rows), "rec_load_tables")
        self.tables[t] = dev_rows

    def load_hot_rows(self, t: int, ids) -> None:
        """ids: int32 row ids (tensor or array), or None / empty to remove the list."""
        dev_ids = None
        if ids is not None and len(ids) > 0:
            dev_ids = torch.as_tensor(ids, dtype=torch.int32).to(self.device).contiguous()
        self._ok(rec_load_hot_rows(self.handle, t, dev_ids), "rec_load_hot_rows")
        self.hot[t] = dev_ids

    def load_mlp(self, which: int, layer: int, W: torch.Tensor, b: torch.Tensor) -> None:
        W = W.to(self.device, torch.float32).contiguous()
        b = b.to(self.device, torch.float32).contiguous()
        packed = torch.empty(rec_mlp_packed_bytes(self.handle, which, layer), dtype=torch.uint8,
                             device=self.device)
        self._ok(rec_load_mlp(self.handle, which, layer, W, b, packed), "rec_load_mlp")
        torch.cuda.current_stream().synchronize()   # W and b may be freed after this
        self.packed[(which, layer)] = packed

    def forward(self, dense: torch.Tensor, indices: torch.Tensor, lengths: torch.Tensor,
                logits: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Returns fp32 logits: [batch] for one Predict-FC stack, [batch, towers] for several."""
        batch = dense.size(0)
        if logits is None:
            shape = (batch,) if self.towers == 1 else (batch, self.towers)
            logits = torch.empty(shape, dtype=torch.float32, device=self.device)
        nnz = self._check_buffers("rec_forward", dense, indices, lengths, logits, batch)
        st = _lib.rec_forward(self.handle, dense.data_ptr(), indices.data_ptr(), lengths.data_ptr(), batch, nnz,
                              logits.data_ptr(), _stream())
        if st:
            self._ok(st, "rec_forward")
        self.last_batch = batch
        return logits

    def _check_buffers(self, call: str, dense: torch.Tensor, indices: torch.Tensor, lengths: torch.Tensor,
                       logits: torch.Tensor, batch: int) -> int:
        """The library sees pointers only: check here that every buffer is as large as
        the call says, of the right type, contiguous and on the device.  Returns the
        id count."""
        nnz = indices.numel()
        if (dense.is_cuda and dense.dtype is _F32 and dense.numel() >= batch * self.F and dense.is_contiguous() and
                indices.is_cuda and indices.dtype is _I32 and indices.is_contiguous() and
                lengths.is_cuda and lengths.dtype is _I32 and lengths.numel() >= self.T * batch and lengths.is_contiguous() and
                logits.is_cuda and logits.dtype is _F32 and logits.numel() >= batch * self.towers and logits.is_contiguous()):
            return nnz
        for name, t, dt, n in (("dense", dense, _F32, batch * self.F), ("indices", indices, _I32, nnz),
                               ("lengths", lengths, _I32, self.T * batch), ("logits", logits, _F32, batch * self.towers)):
            if not (t.is_cuda and t.is_contiguous() and t.dtype == dt and t.numel() >= n):
                raise ValueError(f"{call}: {name} must be a contiguous {dt} device tensor of at least {n} elements")
        return nnz

    def forward_static(self, dense: torch.Tensor, indices: torch.Tensor, lengths: torch.Tensor,
                       logits: torch.Tensor, fault: Optional[torch.Tensor] = None) -> torch.Tensor:
        """rec_forward_static(): the same pass with the library's static scratch; the
        caller brings every buffer (logits fp32, fault int64 [2] or None)."""
        batch = dense.size(0)
        nnz = self._check_buffers("rec_forward_static", dense, indices, lengths, logits, batch)
        if fault is not None and not (fault.is_cuda and fault.dtype == torch.int64 and fault.numel() >= 2):
            raise ValueError("rec_forward_static: fault must be an int64 device tensor of 2 elements")
        self._ok(rec_forward_static(self.handle, dense, indices, lengths, batch, nnz, logits, fault),
                 "rec_forward_static")
        return logits

    def check(self) -> Tuple[int, int]:
        return rec_check(self.handle)

    def drain(self) -> None:
        """Pipelined models: orders every forward enqueued so far on the current stream."""
        self._ok(rec_drain(self.handle), "rec_drain")

    def set_option(self, option: int, value: int) -> None:
        self._ok(rec_set_option(self.handle, option, value), "rec_set_option")

    def set_profiling(self, slots: int, period: int = 1) -> None:
        self._ok(rec_set_profiling(self.handle, slots, period), "rec_set_profiling")

    def stage_ms(self, slot: int = 0) -> dict:
        st, ms = rec_stage_ms(self.handle, slot)
        self._ok(st, "rec_stage_ms")
        return dict(zip(STAGE_NAMES, ms))

    def stage_shared(self, slot: int = 0) -> set:
        """Names of the stages that had no launch of their own in the forward timed in `slot`."""
        st, mask = rec_stage_shared(self.handle, slot)
        self._ok(st, "rec_stage_shared")
        return {name for i, name in enumerate(STAGE_NAMES) if mask >> i & 1}

    def _view(self, what: int, nbytes: int) -> Tuple[torch.Tensor, int]:
        st, p, ld = rec_debug_get(self.handle, what)
        self._ok(st, "rec_debug_get")
        off = p - self.ws.data_ptr()
        return self.ws[off:off + nbytes], ld

    def debug_offsets(self) -> torch.Tensor:
        n = self.T * self.last_batch + 1
        raw, _ = self._view(REC_DBG_OFFSETS, 4 * n)
        return raw.view(torch.int32).clone()

    def debug_pooled(self) -> torch.Tensor:
        B = self.last_batch
        raw, _ = self._view(REC_DBG_POOLED, 4 * B * self.T * self.D)
        return raw.view(torch.float32).view(B, self.T, self.D).clone()

    def debug_bottom_out(self) -> torch.Tensor:
        B = self.last_batch
        st, p, ld = rec_debug_get(self.handle, REC_DBG_BOTTOM_OUT)
        raw, ld = self._view(REC_DBG_BOTTOM_OUT, 4 * B * ld)
        return raw.view(torch.float32).view(B, ld)[:, :self.w0].clone()

    def debug_interact(self) -> torch.Tensor:
        """The Predict-FC input, bf16 [B, ld]; columns beyond its width are zero padding."""
        B = self.last_batch
        st, p, ld = rec_debug_get(self.handle, REC_DBG_INTERACT)
        raw, ld = self._view(REC_DBG_INTERACT, 2 * B * ld)
        return raw.view(torch.bfloat16).view(B, ld).clone()


class CapturedForward:
    """One or more forwards recorded into a HIP graph and replayed with a single launch.

    rec_forward() only enqueues kernels (no allocation, no synchronisation, no
    memset), so it can be recorded under stream capture.  The graph replays the
    recorded pointers: callers keep `batches` and `logits` alive and refresh
    their contents in place.  Stage events must be off while recording."""

    def __init__(self, model: RecModel, batches, logits):
        self.model, self.batches, self.logits = model, list(batches), list(logits)
        assert len(self.batches) == len(self.logits) and self.batches
        for (d, i, l), out in zip(self.batches, self.logits):   # warm-up outside capture
            model.forward(d, i, l, out)
        model.drain()
        torch.cuda.synchronize(model.device)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            for (d, i, l), out in zip(self.batches, self.logits):
                model.forward(d, i, l, out)
            model.drain()       # a pipelined model's other streams join the capture here

    def replay(self) -> None:
        self.graph.replay()


_DTYPE_CODES = {torch.float32: REC_F32, torch.float16: REC_F16, torch.bfloat16: REC_BF16}
_ATTEND_CODES = {torch.float16: REC_F16, torch.bfloat16: REC_BF16}
_FORMATS = {"mx4": REC_MX4, "mx8": REC_MX8}
_I64 = torch.int64


def _faults(device) -> torch.Tensor:
    return torch.full((REC_FAULT_WORDS,), -1, dtype=torch.int64, device=device)


def _stream_on(index: int, call: str) -> int:
    """The current stream of device `index`, which has to be the current device: kernels start there."""
    if index < 0:
        raise ValueError(f"{call}: the tensors are not on a device")
    if torch._C._cuda_getDevice() != index:
        raise ValueError(f"{call}: the tensors are on cuda:{index}, the current device is another")
    return torch._C._cuda_getCurrentRawStream(index)


def _no_backward(call: str) -> None:
    """For a call with inputs that require grad: refused where a result without gradients would lose them unseen."""
    if torch.is_grad_enabled():
        raise ValueError(f"{call} has no backward pass: detach its inputs, or call it under torch.no_grad()")


class HistoryCache:
    """Keys and values of user histories in 4 or 8 bits a number (include/rec_history.h), and
    attention over them.

    The pages are one uint8 tensor, the cache's own or the caller's (`pages`, of
    [num_pages, kv_heads, page_tokens / 16, bytes of a group]); which page holds what is the
    caller's bookkeeping.  Calls go to the current stream and only enqueue.  They serve: there is no
    backward pass, and inputs that require grad are refused unless grad mode is off."""

    def __init__(self, num_pages: int, page_tokens: int, kv_heads: int, head_dim: int, fmt: str = "mx4",
                 device: str = "cuda:0", pages: Optional[torch.Tensor] = None):
        if fmt not in _FORMATS:
            raise ValueError(f"HistoryCache: format must be one of {sorted(_FORMATS)}, not {fmt!r}")
        self.page_tokens, self.kv_heads, self.head_dim, self.fmt = page_tokens, kv_heads, head_dim, fmt
        self._h = rec_history(None, num_pages, page_tokens, kv_heads, head_dim, _FORMATS[fmt], None)
        nbytes = rec_history_bytes(self._h)
        if nbytes == 0:
            raise RecError(REC_ERR_SHAPE, "HistoryCache")
        if pages is None:
            if not torch.cuda.is_available():
                raise RuntimeError("no GPU visible: a history cache has no CPU path")
            shape = (num_pages, kv_heads, page_tokens // 16, nbytes // (num_pages * kv_heads * (page_tokens // 16)))
            pages = torch.empty(shape, dtype=torch.uint8, device=device)
        elif not (pages.is_cuda and pages.dtype == torch.uint8 and pages.is_contiguous() and pages.numel() == nbytes):
            raise ValueError(f"HistoryCache: pages must be a contiguous uint8 device tensor of {nbytes} bytes")
        self.pages, self.device, self._index = pages, pages.device, pages.get_device()
        self.fault = _faults(self.device)
        self._h.dev_pages, self._h.dev_fault = pages.data_ptr(), self.fault.data_ptr()
        self._ref = C.byref(self._h)
        self._workspaces: dict = {}      # bytes by the shapes that decide them

    def _ok(self, st: int, where: str) -> None:
        if st != REC_OK:
            raise RecError(st, where)

    def _slots(self, call: str, slots: torch.Tensor) -> int:
        if slots.dtype is not _I64 or slots.get_device() != self._index or slots.dim() != 1 or not slots.is_contiguous():
            raise ValueError(f"{call}: slots must be a contiguous int64 vector on {self.device}")
        return slots.shape[0]

    def _rows(self, t: torch.Tensor, shape, dtype) -> bytes:
        if t.shape != shape or t.dtype is not dtype or t.get_device() != self._index:
            raise ValueError(f"rec_history_write: k and v must be {tuple(shape)} on {self.device}, both of one type")
        token, head, column = t.stride()
        if column != 1:
            raise ValueError("rec_history_write: rows of k and v must be contiguous")
        return _ROWS.pack(t.data_ptr(), token, head)

    def write(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
        """k, v: [tokens, kv_heads, head_dim] (any token and head strides), fp32, fp16 or bf16;
        slots: int64 [tokens], page * page_tokens + place, -1 for a row to leave out."""
        if k.requires_grad or v.requires_grad:
            _no_backward("rec_history_write")
        n = self._slots("rec_history_write", slots)
        code = _DTYPE_CODES.get(k.dtype)
        if code is None:
            raise ValueError(f"rec_history_write: unsupported type {k.dtype}")
        shape = (n, self.kv_heads, self.head_dim)
        st = _lib.rec_history_write(self._ref, self._rows(k, shape, k.dtype), self._rows(v, shape, k.dtype), code, slots.data_ptr(), n,
                                    _stream_on(self._index, "rec_history_write"))
        if st:
            self._ok(st, "rec_history_write")

    def read(self, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16) -> Tuple[torch.Tensor, torch.Tensor]:
        """Keys and values of `slots` as [tokens, kv_heads, head_dim]; zeros for slot -1."""
        n = self._slots("rec_history_read", slots)
        code = _DTYPE_CODES.get(dtype)
        if code is None:
            raise ValueError(f"rec_history_read: unsupported type {dtype}")
        k = torch.empty((n, self.kv_heads, self.head_dim), dtype=dtype, device=self.device)
        v = torch.empty_like(k)
        st = _lib.rec_history_read(self._ref, slots.data_ptr(), n, code, k.data_ptr(), v.data_ptr(),
                                   _stream_on(self._index, "rec_history_read"))
        if st:
            self._ok(st, "rec_history_read")
        return k, v

    def attend(self, q: torch.Tensor, pages_of: torch.Tensor, lengths: torch.Tensor, scale: Optional[float] = None,
               window: int = 0, sinks: int = 0, candidates: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """q: [batch, queries, heads, head_dim] or, one query each, [batch, heads, head_dim], fp16 or bf16
        (any strides but the last); pages_of: int32 [batch, width], a history's pages in order; lengths:
        int32 [batch].  scale: 1 / sqrt(head_dim) if None.  Returns attention outputs of q's shape, contiguous."""
        if q.requires_grad:
            _no_backward("rec_history_attend")
        index, code = self._index, _ATTEND_CODES.get(q.dtype)
        if q.dim() == 4:
            batch, queries, heads, dim = q.shape
            by_batch, by_query, by_head, by_column = q.stride()
        elif q.dim() == 3:
            (batch, heads, dim), queries = q.shape, 1
            (by_batch, by_head, by_column), by_query = q.stride(), 0
        else:
            code = None
        if code is None or dim != self.head_dim or q.get_device() != index or by_column != 1:
            raise ValueError(f"rec_history_attend: q must be fp16 or bf16 [batch, (queries,) heads, {self.head_dim}] on "
                             f"{self.device}, rows contiguous")
        if pages_of.dim() != 2 or pages_of.dtype is not _I32 or pages_of.get_device() != index or pages_of.shape[0] != batch \
                or (pages_of.stride(1) != 1 and pages_of.shape[1] > 1):
            raise ValueError(f"rec_history_attend: pages_of must be int32 [{batch}, width] on {self.device}, rows contiguous")
        if lengths.dtype is not _I32 or lengths.get_device() != index or lengths.shape != (batch,) or not lengths.is_contiguous():
            raise ValueError(f"rec_history_attend: lengths must be a contiguous int32 [{batch}] on {self.device}")
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif out.shape != q.shape or out.dtype is not q.dtype or out.get_device() != index or not out.is_contiguous():
            raise ValueError("rec_history_attend: out must be contiguous and of q's shape, type and device")
        width = pages_of.shape[1]
        query = _QUERY.pack(q.data_ptr(), out.data_ptr(), by_batch, by_query, by_head, code, batch, queries, heads, pages_of.data_ptr(),
                            pages_of.stride(0), width, lengths.data_ptr(), dim ** -0.5 if scale is None else scale, window, sinks,
                            1 if candidates else 0)
        shapes = (batch, queries, heads, width, window, sinks, candidates, code)
        need = self._workspaces.get(shapes)
        if need is None:
            need = _lib.rec_history_attend_workspace_bytes(self._ref, query)
            if len(self._workspaces) >= 1024:
                self._workspaces.clear()
            self._workspaces[shapes] = need
        workspace = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
        st = _lib.rec_history_attend(self._ref, query, workspace.data_ptr() if need else None, need,
                                     _stream_on(index, "rec_history_attend"))
        if st:
            self._ok(st, "rec_history_attend")
        return out

    def check(self) -> Tuple[int, int, int]:
        """(status, position, REC_FAULT_* word) of the first fault since the last check, of calls on the current stream
        (waited for) and of what others have done by now."""
        return rec_history_check(self.fault)


def attend_window(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor, scale: Optional[float] = None,
                  window: int = 0, sinks: int = 0, fault: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Whole histories attend to themselves (rec_window_attend()).  q: [tokens, heads, head_dim], k and v:
    [tokens, kv_heads, head_dim], fp16 or bf16, any token and head strides; offsets: int32 [batch + 1].
    fault: int64 [REC_FAULT_WORDS], contiguous, all -1, for rec_history_check(), or None.  No backward pass, as in HistoryCache."""
    if q.requires_grad or k.requires_grad or v.requires_grad:
        _no_backward("rec_window_attend")
    code, index = _ATTEND_CODES.get(q.dtype), q.get_device()
    if code is None or index < 0 or q.dim() != 3 or k.dim() != 3 or k.shape != v.shape:
        raise ValueError("rec_window_attend: q must be [tokens, heads, head_dim], k and v [tokens, kv_heads, head_dim] on a device, "
                         "fp16 or bf16")
    tokens, heads, dim = q.shape
    (q_token, q_head, q_column), (k_token, k_head, k_column), (v_token, v_head, v_column) = q.stride(), k.stride(), v.stride()
    if k.shape[0] != tokens or k.shape[2] != dim or k.dtype is not q.dtype or v.dtype is not q.dtype or k.get_device() != index \
            or v.get_device() != index or not q_column == k_column == v_column == 1:
        raise ValueError("rec_window_attend: q, k and v must agree in tokens, head_dim, type and device, rows contiguous")
    if offsets.dtype is not _I32 or offsets.get_device() != index or offsets.dim() != 1 or offsets.shape[0] < 1 or not offsets.is_contiguous():
        raise ValueError(f"rec_window_attend: offsets must be a contiguous int32 [batch + 1] on {q.device}")
    if fault is not None and (fault.get_device() != index or not _is_record(fault)):
        raise ValueError(f"rec_window_attend: fault must be a contiguous int64 [{REC_FAULT_WORDS}] on {q.device}")
    out = torch.empty_like(q, memory_format=torch.contiguous_format)
    st = _lib.rec_window_attend(
        _WINDOW.pack(q.data_ptr(), q_token, q_head, k.data_ptr(), k_token, k_head, v.data_ptr(), v_token, v_head, out.data_ptr(), code,
                     offsets.shape[0] - 1, tokens, heads, k.shape[1], dim, offsets.data_ptr(), dim ** -0.5 if scale is None else scale,
                     window, sinks, fault.data_ptr() if fault is not None else 0), _stream_on(index, "rec_window_attend"))
    if st:
        raise RecError(st, "rec_window_attend")
    return out
