"""ctypes binding of libfreescale_hip.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/freescale.h) and does
nothing but turn torch device tensors into pointers, allocate outputs through torch and pass
the current stream.  No step of the method is computed here, and there is no CPU fallback: if
the HIP library is missing, importing succeeds but the first call raises.
"""
from __future__ import annotations

import ctypes
import functools
import inspect
import os
import re
from typing import Dict, NamedTuple, Optional, Sequence, Union

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfreescale_hip.so")

FS_F32, FS_BF16 = 0, 1
FS_OK, FS_EINVAL, FS_ENOMEM, FS_EHIP, FS_ENOTIMPL, FS_ERANGE = 0, -1, -2, -3, -4, -5
FS_MAX_DIM = 256
FS_SHORT_SEGMENT = 8
FS_MAX_AHEAD_BATCH = 8
FS_MAX_STEP_TABLES = 16
SHORT_REC_INTS = 12

c_i64, c_i32, c_vp, c_f = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_float


class fs_step_args(ctypes.Structure):
    _fields_ = [
        ("table", c_vp), ("state", c_vp), ("num_rows", c_i64), ("dim", c_i32), ("dtype", c_i32),
        ("lr", c_f), ("eps", c_f),
        ("u_t", c_vp), ("seg_offsets_t", c_vp), ("perm_t", c_vp), ("inverse_t", c_vp), ("n_unique_t_dev", c_vp),
        ("grads_t", c_vp), ("n_t", c_i64),
        ("values_t1", c_vp), ("offsets_t1", c_vp), ("batch_t1", c_i64), ("n_t1", c_i64),
        ("u_t1", c_vp), ("seg_offsets_t1", c_vp), ("perm_t1", c_vp), ("inverse_t1", c_vp), ("n_unique_t1_dev", c_vp),
        ("co", c_vp), ("co_slot", c_vp), ("ex", c_vp), ("ex_slot", c_vp), ("ex_next", c_vp), ("ex_next_slot", c_vp),
        ("counts_dev", c_vp),
        ("cperm", c_vp), ("cslot", c_vp), ("cstart", c_vp), ("class_pos_dev", c_vp), ("short_rec", c_vp),
        ("reduced", c_vp), ("emb_t1", c_vp),
        ("co_flag_t1", c_vp),
        ("sorted_ids_t1", c_vp),
    ]


class fs_block_args(ctypes.Structure):
    _fields_ = [
        ("n", c_i64), ("dim", c_i32), ("rows_dt", c_i32), ("dt", c_i32), ("eps", c_f),
        ("x", c_vp), ("a", c_vp), ("g", c_vp), ("a_stride", c_i64), ("g_stride", c_i64),
        ("w_post", c_vp), ("scale", c_vp), ("w_pre", c_vp), ("y", c_vp), ("h", c_vp),
        ("a_codes", c_vp), ("g_codes", c_vp), ("y_codes", c_vp), ("a_exps", c_vp), ("g_exps", c_vp), ("y_exps", c_vp),
        ("dy", c_vp), ("dh", c_vp), ("dx", c_vp), ("da", c_vp), ("dg", c_vp), ("da_stride", c_i64), ("dg_stride", c_i64),
        ("dw_post", c_vp), ("dscale", c_vp), ("dw_pre", c_vp), ("work", c_vp), ("work_bytes", ctypes.c_size_t),
    ]


class fs_attention_args(ctypes.Structure):
    _fields_ = [
        ("q", c_vp), ("k", c_vp), ("v", c_vp), ("q_stride", c_i64), ("k_stride", c_i64), ("v_stride", c_i64),
        ("n_q", c_i64), ("n_kv", c_i64), ("batch", c_i64), ("q_offsets", c_vp), ("kv_offsets", c_vp), ("kv_lengths", c_vp),
        ("heads", c_i32), ("kv_heads", c_i32), ("head_dim", c_i32), ("dt", c_i32), ("causal", c_i32), ("max_q", c_i32),
        ("scale", c_f), ("num_buckets", c_i32), ("num_distances", c_i32), ("bias", c_vp), ("bucket_of", c_vp),
        ("out", c_vp), ("out_f32", c_vp), ("lse", c_vp),
        ("dout", c_vp), ("dq", c_vp), ("dk", c_vp), ("dv", c_vp), ("dq_stride", c_i64), ("dk_stride", c_i64), ("dv_stride", c_i64),
        ("dbias", c_vp), ("work", c_vp), ("work_bytes", ctypes.c_size_t),
    ]


class FreeScaleError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        super().__init__(f"{where} failed with status {code}" + (f": {detail}" if detail else ""))
        self.code = code


_lib: Optional[ctypes.CDLL] = None


def load_library() -> ctypes.CDLL:
    """Loads the in-tree HIP library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} is missing: build it with `python -m paper_2604_24073_amd.build` "
                                "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    S = c_vp  # stream
    sig = {
        "fs_version": (ctypes.c_int, []),
        "fs_ctx_create": (ctypes.c_int, [ctypes.POINTER(c_vp), ctypes.c_int, c_i64, c_i32]),
        "fs_ctx_destroy": (ctypes.c_int, [c_vp]),
        "fs_last_error": (ctypes.c_char_p, [c_vp]),
        "fs_check_async": (ctypes.c_int, [c_vp, S]),
        "fs_ctx_workspace_bytes": (ctypes.c_size_t, [c_vp]),
        "fs_gather_jagged": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i32, ctypes.c_int, c_vp, c_vp, c_i64, c_i64, c_vp, S]),
        "fs_gather_jagged_class": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i32, ctypes.c_int, c_vp, c_vp, c_i64, c_i64, c_vp,
                                                  c_vp, ctypes.c_int, c_vp, S]),
        "fs_unique_ids": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i64, c_vp, c_vp, c_vp, c_vp, c_vp, S]),
        "fs_jagged_keyed_transpose": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i32, c_vp, c_i64, c_i64, c_vp, c_vp, S]),
        "fs_jagged_ranged_dispatch": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i32, c_vp, c_i64, c_i64, c_vp, c_i32, c_vp,
                                                     c_vp, c_vp, S]),
        "fs_jagged_ranged_combine": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i32, c_vp, c_i64, c_i64, c_vp, c_i32, c_vp,
                                                    c_vp, S]),
        "fs_partition_vbs": (ctypes.c_int, [c_vp, c_vp, c_i64, c_vp, c_i64, c_i32, c_vp, c_vp, S]),
        "fs_partition_fbs": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i64, c_i32, c_vp, c_vp, S]),
        "fs_jagged_indexed_permute": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i32, c_vp, c_i64, c_vp, c_i64, c_vp, c_i64,
                                                     c_vp, S]),
        "fs_collision_split": (ctypes.c_int, [c_vp, c_vp, c_vp, c_vp, c_vp, c_i64, c_i64, c_vp, c_vp, c_vp, c_vp,
                                              c_vp, c_vp, c_vp, S]),
        "fs_collision_split_static": (ctypes.c_int, [c_vp, c_vp, c_vp, c_vp, c_i64, c_i64, c_vp, c_vp, c_vp, c_vp,
                                                     c_vp, c_vp, c_vp, S]),
        "fs_split_grads": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i32, c_vp, c_vp, c_vp, c_i64, c_vp, c_vp, c_vp, c_vp, c_vp,
                                          c_vp, S]),
        "fs_class_order_for_parts": (ctypes.c_int, [c_vp, c_vp, c_i64, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, S]),
        "fs_segment_reduce_grads": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i32, c_vp, c_vp, c_vp, c_vp, c_vp, S]),
        "fs_rowwise_adagrad_update": (ctypes.c_int, [c_vp, c_vp, ctypes.c_int, c_vp, c_i64, c_i32, c_vp, c_vp, c_vp,
                                                     c_i64, c_vp, c_f, c_f, S]),
        "fs_collision_split_classes": (ctypes.c_int, [c_vp, c_vp, c_vp, c_vp, c_vp, c_i64, c_i64, c_vp, c_vp, c_vp,
                                                      c_i64, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp,
                                                      c_vp, c_vp, c_vp, S]),
        "fs_reduce_update_class": (ctypes.c_int, [c_vp, ctypes.c_int, c_vp, ctypes.c_int, c_vp, c_i64, c_i32, c_f, c_f,
                                                  c_vp, c_i64, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, S]),
        "fs_unique_ids_ahead": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i64, c_vp, c_vp, c_vp, c_vp, c_vp, S]),
        "fs_prioritized_step": (ctypes.c_int, [c_vp, ctypes.POINTER(fs_step_args), S]),
        "fs_step_forward": (ctypes.c_int, [c_vp, ctypes.POINTER(fs_step_args), S]),
        "fs_step_forward_ahead": (ctypes.c_int, [c_vp, ctypes.POINTER(fs_step_args), S]),
        "fs_step_forward_ahead_batch": (ctypes.c_int, [c_vp, ctypes.POINTER(fs_step_args), ctypes.c_int, S]),
        "fs_prioritized_step_pipelined_multi": (ctypes.c_int, [c_vp, ctypes.POINTER(fs_step_args),
                                                                ctypes.POINTER(fs_step_args), ctypes.c_int, S]),
        "fs_prioritized_step_two_part_multi": (ctypes.c_int, [c_vp, ctypes.POINTER(fs_step_args),
                                                               ctypes.POINTER(fs_step_args), ctypes.c_int, S]),
        "fs_prioritized_step_pipelined": (ctypes.c_int, [c_vp, ctypes.POINTER(fs_step_args),
                                                         ctypes.POINTER(fs_step_args), S]),
        "fs_graph_capture_pipelined": (ctypes.c_int, [c_vp, ctypes.POINTER(fs_step_args), ctypes.POINTER(fs_step_args),
                                                      ctypes.POINTER(c_vp)]),
        "fs_ctx_set_threaded_enqueue": (ctypes.c_int, [c_vp, ctypes.c_int]),
        "fs_step_join": (ctypes.c_int, [c_vp, S]),
        "fs_two_part_forget": (ctypes.c_int, [c_vp]),
        "fs_ctx_host_times": (ctypes.c_int, [c_vp, ctypes.POINTER(ctypes.c_double), ctypes.c_int]),
        "fs_graph_launch": (ctypes.c_int, [c_vp, c_vp, S]),
        "fs_graph_destroy": (ctypes.c_int, [c_vp]),
        "fs_ctx_set_kernel_timing": (ctypes.c_int, [c_vp, ctypes.c_int, ctypes.c_int]),
        "fs_ctx_get_kernel_timing": (ctypes.c_int, [c_vp, ctypes.c_int, ctypes.POINTER(c_f), ctypes.c_int,
                                                    ctypes.POINTER(ctypes.c_int)]),
        "fs_rows_pack8": (ctypes.c_int, [c_vp, c_vp, c_i64, ctypes.c_int, c_i64, c_i32, c_vp, c_vp, S]),
        "fs_rows_unpack8": (ctypes.c_int, [c_vp, c_vp, c_vp, c_i64, c_i32, c_vp, c_i64, ctypes.c_int, S]),
        "fs_block_norm": (ctypes.c_int, [c_vp, ctypes.POINTER(fs_block_args), S]),
        "fs_block_norm_backward": (ctypes.c_int, [c_vp, ctypes.POINTER(fs_block_args), S]),
        "fs_block_norm_work_bytes": (ctypes.c_size_t, [c_i64, c_i32]),
        "fs_jagged_attention": (ctypes.c_int, [c_vp, ctypes.POINTER(fs_attention_args), S]),
        "fs_jagged_attention_work_bytes": (ctypes.c_size_t, [ctypes.POINTER(fs_attention_args)]),
        "fs_jagged_attention_backward": (ctypes.c_int, [c_vp, ctypes.POINTER(fs_attention_args), S]),
        "fs_jagged_attention_backward_work_bytes": (ctypes.c_size_t, [ctypes.POINTER(fs_attention_args)]),
        "fs_init_table_hash": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i32, ctypes.c_int, S]),
        "fs_stream_copy": (ctypes.c_int, [c_vp, c_vp, c_vp, c_i64, S]),
        "fs_stream_row_read": (ctypes.c_int, [c_vp, c_vp, c_i64, c_i32, c_vp, c_i64, c_vp, S]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    _lib = lib
    return lib


def declared_symbols(header_paths=None):
    """Names of the functions declared in include/*.h (what a -DFS_TRACE build adds is left out)."""
    if header_paths is None:
        inc = os.path.join(os.path.dirname(_HERE), "include")
        header_paths = sorted(os.path.join(inc, f) for f in os.listdir(inc) if f.endswith(".h"))
    names = set()
    for path in header_paths:
        text = open(path).read()
        text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
        text = re.sub(r"#ifdef FS_TRACE.*?#endif", "", text, flags=re.S)
        names.update(re.findall(r"\b(fs_[a-z0-9_]+)\s*\(", text))
    return sorted(names)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# The handle of the current stream without building a torch.cuda.Stream object for it, which takes 2.7 us of host
# time - as much as a kernel launch - where this takes 0.2; torch without the getter gets the object.
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _current_raw_stream is not None:
            return _current_raw_stream(torch.cuda.current_device()) or None
        stream = torch.cuda.current_stream()
    if isinstance(stream, torch.cuda.Stream):
        h = stream.cuda_stream
    else:
        h = int(stream)
    return h if h else None


def table_dtype_code(table: torch.Tensor) -> int:
    if table.dtype == torch.float32:
        return FS_F32
    if table.dtype == torch.bfloat16:
        return FS_BF16
    raise TypeError(f"table dtype {table.dtype}: fp32 or bf16 only")


class Context:
    """Owner of an fs_ctx (device workspace, side streams, events)."""

    def __init__(self, max_ids: int, max_dim: int = FS_MAX_DIM, device: Optional[int] = None):
        self.lib = load_library()
        if device is None:
            device = torch.cuda.current_device()
        self.device = device
        h = c_vp()
        rc = self.lib.fs_ctx_create(ctypes.byref(h), device, max_ids, max_dim)
        if rc != FS_OK:
            raise FreeScaleError(rc, "fs_ctx_create")
        self.handle = h
        self.max_ids, self.max_dim = max_ids, max_dim

    def close(self) -> None:
        if getattr(self, "handle", None):
            self.lib.fs_ctx_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def last_error(self) -> str:
        return self.lib.fs_last_error(self.handle).decode()

    def check(self, rc: int, where: str) -> None:
        if rc != FS_OK:
            raise FreeScaleError(rc, where, self.last_error())

    def workspace_bytes(self) -> int:
        return int(self.lib.fs_ctx_workspace_bytes(self.handle))


def fs_check_async(ctx: Context, stream=None) -> int:
    return ctx.lib.fs_check_async(ctx.handle, _stream(stream))


FS_TIME_REDUCE, FS_TIME_GATHER, FS_TIME_UPDATE_CO, FS_TIME_UPDATE_EX = 0, 1, 2, 3


def fs_ctx_set_kernel_timing(ctx: Context, slots: int, every: int = 1) -> None:
    ctx.check(ctx.lib.fs_ctx_set_kernel_timing(ctx.handle, slots, every), "fs_ctx_set_kernel_timing")


def fs_ctx_get_kernel_timing(ctx: Context, which: int, max_out: int = 65536):
    buf = (c_f * max_out)()
    n = ctypes.c_int(0)
    ctx.check(ctx.lib.fs_ctx_get_kernel_timing(ctx.handle, which, buf, max_out, ctypes.byref(n)),
              "fs_ctx_get_kernel_timing")
    return [buf[i] for i in range(n.value)]


def fs_gather_jagged(ctx: Context, table: torch.Tensor, values: torch.Tensor, offsets: Optional[torch.Tensor],
                     out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    n = values.numel()
    if out is None:
        out = torch.empty((n, table.shape[1]), dtype=table.dtype, device=table.device)
    batch = 0 if offsets is None else offsets.numel() - 1
    rc = ctx.lib.fs_gather_jagged(ctx.handle, _ptr(table), table.shape[0], table.shape[1], table_dtype_code(table),
                                  _ptr(values), _ptr(offsets), batch, n, _ptr(out), _stream(stream))
    ctx.check(rc, "fs_gather_jagged")
    return out


def fs_gather_jagged_class(ctx: Context, table: torch.Tensor, values: torch.Tensor, offsets: Optional[torch.Tensor],
                           inverse: torch.Tensor, co_flag: torch.Tensor, which: int, out: torch.Tensor,
                           stream=None) -> torch.Tensor:
    n = values.numel()
    batch = 0 if offsets is None else offsets.numel() - 1
    rc = ctx.lib.fs_gather_jagged_class(ctx.handle, _ptr(table), table.shape[0], table.shape[1],
                                        table_dtype_code(table), _ptr(values), _ptr(offsets), batch, n, _ptr(inverse),
                                        _ptr(co_flag), which, _ptr(out), _stream(stream))
    ctx.check(rc, "fs_gather_jagged_class")
    return out


def fs_partition_fbs(ctx: Context, lengths: torch.Tensor, max_len: int, n_ranks: int, stream=None, out=None):
    """(sample_of [B] int32, rank_offsets [n_ranks + 1] int64) of the FBS partitioner; `out`: the caller's pair."""
    B = lengths.numel()
    if out is not None:
        sample_of, rank_offsets = out
    else:
        sample_of = torch.empty(max(B, 1), dtype=torch.int32, device=lengths.device)
        rank_offsets = torch.empty(n_ranks + 1, dtype=torch.int64, device=lengths.device)
    rc = ctx.lib.fs_partition_fbs(ctx.handle, _ptr(lengths), B, max_len, n_ranks, _ptr(sample_of), _ptr(rank_offsets),
                                  _stream(stream))
    ctx.check(rc, "fs_partition_fbs")
    return sample_of[:B], rank_offsets


def fs_partition_vbs(ctx: Context, lengths: torch.Tensor, weight_of_len: torch.Tensor, n_ranks: int, stream=None):
    """(sample_of [B] int32 = the length-sorted order, rank_offsets [n_ranks + 1] int64) of the VBS partitioner;
    weight_of_len [max_len + 1] int64."""
    B = lengths.numel()
    sample_of = torch.empty(max(B, 1), dtype=torch.int32, device=lengths.device)
    rank_offsets = torch.empty(n_ranks + 1, dtype=torch.int64, device=lengths.device)
    rc = ctx.lib.fs_partition_vbs(ctx.handle, _ptr(lengths), B, _ptr(weight_of_len), weight_of_len.numel() - 1, n_ranks,
                                  _ptr(sample_of), _ptr(rank_offsets), _stream(stream))
    ctx.check(rc, "fs_partition_vbs")
    return sample_of[:B], rank_offsets


def fs_jagged_indexed_permute(ctx: Context, values: torch.Tensor, offsets: torch.Tensor, sample_of: torch.Tensor,
                              cap_out: int, stream=None, out=None):
    """(out_values [cap_out, ...], out_offsets [n_out + 1]); values is [n] or [n, width], any 4- or 8-byte dtype.
    `out`: the caller's (out_values, out_offsets)."""
    n_values = values.shape[0]
    elem = _elem_bytes(values)
    n_out = sample_of.numel()
    if out is not None:
        out, out_offsets = out
    else:
        out = torch.empty((cap_out,) + tuple(values.shape[1:]), dtype=values.dtype, device=values.device)
        out_offsets = torch.empty(n_out + 1, dtype=torch.int64, device=values.device)
    rc = ctx.lib.fs_jagged_indexed_permute(ctx.handle, _ptr(values), n_values, elem, _ptr(offsets), offsets.numel() - 1,
                                           _ptr(sample_of), n_out, _ptr(out), cap_out, _ptr(out_offsets),
                                           _stream(stream))
    ctx.check(rc, "fs_jagged_indexed_permute")
    return out, out_offsets


def _elem_bytes(values: torch.Tensor) -> int:
    elem = values.element_size()
    for d in values.shape[1:]:
        elem *= d
    return elem


def fs_jagged_keyed_transpose(ctx: Context, values: torch.Tensor, offsets: torch.Tensor, F: int, B: int, stream=None,
                              out=None):
    out, out_offsets = out if out is not None else (torch.empty_like(values), torch.empty_like(offsets))
    rc = ctx.lib.fs_jagged_keyed_transpose(ctx.handle, _ptr(values), values.shape[0], _elem_bytes(values), _ptr(offsets),
                                           F, B, _ptr(out), _ptr(out_offsets), _stream(stream))
    ctx.check(rc, "fs_jagged_keyed_transpose")
    return out, out_offsets


def fs_jagged_ranged_dispatch(ctx: Context, values: torch.Tensor, offsets: torch.Tensor, F: int, B: int,
                              rank_offsets: torch.Tensor, stream=None, out=None):
    """`out`: the caller's (out_values, out_offsets, splits [n_ranks])."""
    n_ranks = rank_offsets.numel() - 1
    if out is not None:
        out, out_offsets, splits = out
    else:
        out, out_offsets = torch.empty_like(values), torch.empty_like(offsets)
        splits = torch.empty(max(n_ranks, 1), dtype=torch.int64, device=values.device)
    rc = ctx.lib.fs_jagged_ranged_dispatch(ctx.handle, _ptr(values), values.shape[0], _elem_bytes(values), _ptr(offsets),
                                           F, B, _ptr(rank_offsets), n_ranks, _ptr(out), _ptr(out_offsets), _ptr(splits),
                                           _stream(stream))
    ctx.check(rc, "fs_jagged_ranged_dispatch")
    return out, out_offsets, splits[:n_ranks]


def fs_jagged_ranged_combine(ctx: Context, values: torch.Tensor, offsets: torch.Tensor, F: int, B: int,
                             rank_offsets: torch.Tensor, stream=None, out=None):
    out, out_offsets = out if out is not None else (torch.empty_like(values), torch.empty_like(offsets))
    rc = ctx.lib.fs_jagged_ranged_combine(ctx.handle, _ptr(values), values.shape[0], _elem_bytes(values), _ptr(offsets),
                                          F, B, _ptr(rank_offsets), rank_offsets.numel() - 1, _ptr(out),
                                          _ptr(out_offsets), _stream(stream))
    ctx.check(rc, "fs_jagged_ranged_combine")
    return out, out_offsets


def fs_unique_ids(ctx: Context, ids: torch.Tensor, num_rows: int, out: Optional[Dict[str, torch.Tensor]] = None,
                  stream=None) -> Dict[str, torch.Tensor]:
    n = ids.numel()
    dev = ids.device
    if out is None:
        out = {
            "unique": torch.empty(max(n, 1), dtype=torch.int64, device=dev),
            "seg_offsets": torch.empty(n + 1, dtype=torch.int32, device=dev),
            "perm": torch.empty(max(n, 1), dtype=torch.int32, device=dev),
            "inverse": torch.empty(max(n, 1), dtype=torch.int32, device=dev),
            "n_unique": torch.zeros(1, dtype=torch.int64, device=dev),
        }
    rc = ctx.lib.fs_unique_ids(ctx.handle, _ptr(ids), n, num_rows, _ptr(out["unique"]), _ptr(out["seg_offsets"]),
                               _ptr(out["perm"]), _ptr(out.get("inverse")), _ptr(out["n_unique"]), _stream(stream))
    ctx.check(rc, "fs_unique_ids")
    out["n"] = n
    return out


def fs_collision_split(ctx: Context, u_t: Optional[torch.Tensor], n_t_dev: Optional[torch.Tensor],
                       u_t1: Optional[torch.Tensor], n_t1_dev: Optional[torch.Tensor], cap_t: int, cap_t1: int,
                       out: Optional[Dict[str, torch.Tensor]] = None, stream=None) -> Dict[str, torch.Tensor]:
    dev = (u_t if u_t is not None else u_t1).device if (u_t is not None or u_t1 is not None) else torch.device("cuda")
    if out is None:
        i64 = lambda k: torch.empty(max(k, 1), dtype=torch.int64, device=dev)
        i32 = lambda k: torch.empty(max(k, 1), dtype=torch.int32, device=dev)
        out = {"co": i64(cap_t), "co_slot": i32(cap_t), "ex": i64(cap_t), "ex_slot": i32(cap_t),
               "ex_next": i64(cap_t1), "ex_next_slot": i32(cap_t1),
               "counts": torch.zeros(3, dtype=torch.int64, device=dev)}
    rc = ctx.lib.fs_collision_split(ctx.handle, _ptr(u_t), _ptr(n_t_dev), _ptr(u_t1), _ptr(n_t1_dev), cap_t, cap_t1,
                                    _ptr(out["co"]), _ptr(out["co_slot"]), _ptr(out["ex"]), _ptr(out["ex_slot"]),
                                    _ptr(out["ex_next"]), _ptr(out["ex_next_slot"]), _ptr(out["counts"]),
                                    _stream(stream))
    ctx.check(rc, "fs_collision_split")
    return out


FS_STATIC_SPLIT_MAX_ROWS = 1 << 20


def fs_collision_split_static(u_t: Optional[torch.Tensor], n_t_dev: Optional[torch.Tensor],
                              u_t1: Optional[torch.Tensor], n_t1_dev: Optional[torch.Tensor], cap_t: int, cap_t1: int,
                              out: Dict[str, torch.Tensor], stream=None) -> Dict[str, torch.Tensor]:
    """The split without a context and without any allocation: `out` (a bundle as fs_collision_split returns
    it) is the caller's."""
    lib = load_library()
    rc = lib.fs_collision_split_static(_ptr(u_t), _ptr(n_t_dev), _ptr(u_t1), _ptr(n_t1_dev), cap_t, cap_t1,
                                       _ptr(out["co"]), _ptr(out["co_slot"]), _ptr(out["ex"]), _ptr(out["ex_slot"]),
                                       _ptr(out["ex_next"]), _ptr(out["ex_next_slot"]), _ptr(out["counts"]),
                                       _stream(stream))
    if rc != FS_OK:
        raise FreeScaleError(rc, "fs_collision_split_static", lib.fs_last_error(None).decode())
    return out


def fs_collision_split_classes(ctx: Context, layout_t: Dict[str, torch.Tensor], u_t1: Optional[torch.Tensor],
                               n_t1_dev: Optional[torch.Tensor], cap_t1: int,
                               out: Optional[Dict[str, torch.Tensor]] = None, stream=None) -> Dict[str, torch.Tensor]:
    """layout_t: what fs_unique_ids returned for batch t (with its "n")."""
    n_t = layout_t["n"]
    dev = layout_t["unique"].device
    if out is None:
        out = alloc_split(n_t, cap_t1, dev)
    rc = ctx.lib.fs_collision_split_classes(
        ctx.handle, _ptr(layout_t["unique"]), _ptr(layout_t["n_unique"]), _ptr(u_t1), _ptr(n_t1_dev), n_t, cap_t1,
        _ptr(layout_t["seg_offsets"]), _ptr(layout_t["perm"]), _ptr(layout_t.get("inverse")), n_t,
        _ptr(out["co"]), _ptr(out["co_slot"]), _ptr(out["ex"]), _ptr(out["ex_slot"]), _ptr(out["ex_next"]),
        _ptr(out["ex_next_slot"]), _ptr(out["counts"]), _ptr(out["cperm"]), _ptr(out["cslot"]), _ptr(out["cstart"]),
        _ptr(out["class_pos"]), _ptr(out["short_rec"]), _stream(stream))
    ctx.check(rc, "fs_collision_split_classes")
    return out


def fs_split_grads(ctx: Context, grads: torch.Tensor, layout_t: Dict[str, torch.Tensor], split: Dict[str, torch.Tensor],
                   out: Optional[Dict[str, torch.Tensor]] = None, stream=None) -> Dict[str, torch.Tensor]:
    """split() of Algorithm 2's Backward.  layout_t: the batch's layout with its inverse map; split: its collision
    split (co_slot, counts).  Returns co_index, g_co, ex_index, g_ex, part_pos, counts ([2] occurrences per part)."""
    n, dim = grads.shape
    dev = grads.device
    if out is None:
        i32 = lambda: torch.empty(max(n, 1), dtype=torch.int32, device=dev)
        f32 = lambda: torch.empty((max(n, 1), dim), dtype=torch.float32, device=dev)
        out = {"co_index": i32(), "g_co": f32(), "ex_index": i32(), "g_ex": f32(), "part_pos": i32(),
               "counts": torch.zeros(2, dtype=torch.int64, device=dev)}
    rc = ctx.lib.fs_split_grads(ctx.handle, _ptr(grads), n, dim, _ptr(layout_t.get("inverse")), _ptr(split["co_slot"]),
                                _ptr(split["counts"]), n, _ptr(out["co_index"]), _ptr(out["g_co"]),
                                _ptr(out["ex_index"]), _ptr(out["g_ex"]), _ptr(out["part_pos"]), _ptr(out["counts"]),
                                _stream(stream))
    ctx.check(rc, "fs_split_grads")
    return out


def fs_class_order_for_parts(ctx: Context, parts: Dict[str, torch.Tensor], n_t: int, split: Dict[str, torch.Tensor],
                             stream=None) -> Dict[str, torch.Tensor]:
    """A copy of `split` whose class order and records address the packed parts of fs_split_grads."""
    out = dict(split)
    out["cperm"] = torch.empty_like(split["cperm"])
    out["short_rec"] = torch.empty_like(split["short_rec"])
    rc = ctx.lib.fs_class_order_for_parts(ctx.handle, _ptr(parts["part_pos"]), n_t, _ptr(split["cperm"]),
                                          _ptr(split["class_pos"]), _ptr(split["short_rec"]), _ptr(split["counts"]),
                                          _ptr(out["cperm"]), _ptr(out["short_rec"]), _stream(stream))
    ctx.check(rc, "fs_class_order_for_parts")
    return out


def fs_reduce_update_class(ctx: Context, cls: int, table: torch.Tensor, state: torch.Tensor, lr: float, eps: float,
                           grads: torch.Tensor, layout_t: Dict[str, torch.Tensor], split: Dict[str, torch.Tensor],
                           reduced: Optional[torch.Tensor] = None, stream=None) -> None:
    n, dim = grads.shape
    rc = ctx.lib.fs_reduce_update_class(
        ctx.handle, cls, _ptr(table), table_dtype_code(table), _ptr(state), table.shape[0], dim, lr, eps,
        _ptr(grads), n, _ptr(layout_t["unique"]), _ptr(layout_t["seg_offsets"]),
        split["short_rec"].data_ptr() + cls * 4 * SHORT_REC_INTS * n,
        split["counts"].data_ptr() + 8 * cls, _ptr(split["cperm"]),
        _ptr(split["cslot"]), _ptr(split["cstart"]), _ptr(split["class_pos"]), _ptr(reduced), _stream(stream))
    ctx.check(rc, "fs_reduce_update_class")


FS_STREAM_LAST_STEP = "last_step"


def fs_unique_ids_ahead(ctx: Context, ids: torch.Tensor, num_rows: int, out: Dict[str, torch.Tensor],
                        stream=None) -> Dict[str, torch.Tensor]:
    n = ids.numel()
    stream_arg = ctypes.c_void_p(-1) if stream == FS_STREAM_LAST_STEP else _stream(stream)
    rc = ctx.lib.fs_unique_ids_ahead(ctx.handle, _ptr(ids), n, num_rows, _ptr(out["unique"]),
                                     _ptr(out["seg_offsets"]), _ptr(out["perm"]), _ptr(out.get("inverse")),
                                     _ptr(out["n_unique"]), stream_arg)
    ctx.check(rc, "fs_unique_ids_ahead")
    out["n"] = n
    return out


def fs_segment_reduce_grads(ctx: Context, grads: torch.Tensor, perm: torch.Tensor, seg_offsets: torch.Tensor,
                            n_unique_dev: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None,
                            inverse: Optional[torch.Tensor] = None) -> torch.Tensor:
    n, dim = grads.shape
    if out is None:
        out = torch.empty((max(n, 1), dim), dtype=torch.float32, device=grads.device)
    rc = ctx.lib.fs_segment_reduce_grads(ctx.handle, _ptr(grads), n, dim, _ptr(perm), _ptr(seg_offsets),
                                         _ptr(inverse), _ptr(n_unique_dev), _ptr(out), _stream(stream))
    ctx.check(rc, "fs_segment_reduce_grads")
    return out


def fs_rowwise_adagrad_update(ctx: Context, table: torch.Tensor, state: torch.Tensor, rows: torch.Tensor,
                              slots: torch.Tensor, n_rows_dev: torch.Tensor, cap: int, reduced: torch.Tensor,
                              lr: float, eps: float, stream=None) -> None:
    rc = ctx.lib.fs_rowwise_adagrad_update(ctx.handle, _ptr(table), table_dtype_code(table), _ptr(state),
                                           table.shape[0], table.shape[1], _ptr(rows), _ptr(slots), _ptr(n_rows_dev),
                                           cap, _ptr(reduced), lr, eps, _stream(stream))
    ctx.check(rc, "fs_rowwise_adagrad_update")


def fs_prioritized_step(ctx: Context, args: fs_step_args, stream=None) -> None:
    rc = ctx.lib.fs_prioritized_step(ctx.handle, ctypes.byref(args), _stream(stream))
    ctx.check(rc, "fs_prioritized_step")


def fs_step_forward(ctx: Context, args: fs_step_args, stream=None) -> None:
    rc = ctx.lib.fs_step_forward(ctx.handle, ctypes.byref(args), _stream(stream))
    ctx.check(rc, "fs_step_forward")


def fs_step_forward_ahead(ctx: Context, args: fs_step_args, stream=None) -> None:
    stream_arg = ctypes.c_void_p(-1) if stream == FS_STREAM_LAST_STEP else _stream(stream)
    rc = ctx.lib.fs_step_forward_ahead(ctx.handle, ctypes.byref(args), stream_arg)
    ctx.check(rc, "fs_step_forward_ahead")


def fs_step_forward_ahead_batch(ctx: Context, args, stream=None) -> None:
    """args: sequence of 1..FS_MAX_AHEAD_BATCH argument records (copied into one contiguous array), or such an
    array from step_args_array (passed as it is)."""
    arr = args if isinstance(args, ctypes.Array) else (fs_step_args * len(args))(*args)
    stream_arg = ctypes.c_void_p(-1) if stream == FS_STREAM_LAST_STEP else _stream(stream)
    rc = ctx.lib.fs_step_forward_ahead_batch(ctx.handle, arr, len(args), stream_arg)
    ctx.check(rc, "fs_step_forward_ahead_batch")


def fs_prioritized_step_pipelined(ctx: Context, cur: fs_step_args, nxt: Optional[fs_step_args], stream=None) -> None:
    rc = ctx.lib.fs_prioritized_step_pipelined(ctx.handle, ctypes.byref(cur),
                                               ctypes.byref(nxt) if nxt is not None else None, _stream(stream))
    ctx.check(rc, "fs_prioritized_step_pipelined")


def step_args_array(records):
    """Contiguous copy of a sequence of argument records (for the calls that take several)."""
    return (fs_step_args * len(records))(*records)


def fs_prioritized_step_pipelined_multi(ctx: Context, cur, nxt, stream=None) -> None:
    """cur / nxt: fs_step_args arrays from step_args_array (nxt may be None), one record per table."""
    rc = ctx.lib.fs_prioritized_step_pipelined_multi(ctx.handle, cur, nxt, len(cur), _stream(stream))
    ctx.check(rc, "fs_prioritized_step_pipelined_multi")


def fs_prioritized_step_two_part_multi(ctx: Context, cur, nxt, stream=None) -> None:
    """As fs_prioritized_step_pipelined_multi, the lookup taken in its two parts (records need co_flag_t1)."""
    rc = ctx.lib.fs_prioritized_step_two_part_multi(ctx.handle, cur, nxt, len(cur), _stream(stream))
    ctx.check(rc, "fs_prioritized_step_two_part_multi")


def fs_two_part_forget(ctx: Context) -> None:
    ctx.check(ctx.lib.fs_two_part_forget(ctx.handle), "fs_two_part_forget")


def fs_ctx_host_times(ctx: Context, reset: bool = False):
    buf = (ctypes.c_double * 7)()
    ctx.check(ctx.lib.fs_ctx_host_times(ctx.handle, buf, 1 if reset else 0), "fs_ctx_host_times")
    return [buf[i] for i in range(7)]


def fs_step_join(ctx: Context, stream=None) -> None:
    ctx.check(ctx.lib.fs_step_join(ctx.handle, _stream(stream)), "fs_step_join")


def fs_graph_capture_pipelined(ctx: Context, cur: fs_step_args, nxt: Optional[fs_step_args]) -> c_vp:
    g = c_vp()
    rc = ctx.lib.fs_graph_capture_pipelined(ctx.handle, ctypes.byref(cur),
                                            ctypes.byref(nxt) if nxt is not None else None, ctypes.byref(g))
    ctx.check(rc, "fs_graph_capture_pipelined")
    return g


def fs_graph_launch(ctx: Context, graph: c_vp, stream=None) -> None:
    ctx.check(ctx.lib.fs_graph_launch(ctx.handle, graph, _stream(stream)), "fs_graph_launch")


def fs_graph_destroy(ctx: Context, graph: c_vp) -> None:
    ctx.lib.fs_graph_destroy(graph)


def fs_init_table_hash(ctx: Context, table: torch.Tensor, stream=None) -> None:
    rc = ctx.lib.fs_init_table_hash(ctx.handle, _ptr(table), table.shape[0], table.shape[1], table_dtype_code(table),
                                    _stream(stream))
    ctx.check(rc, "fs_init_table_hash")


def fs_stream_copy(ctx: Context, src: torch.Tensor, dst: torch.Tensor, stream=None) -> None:
    nbytes = src.numel() * src.element_size()
    rc = ctx.lib.fs_stream_copy(ctx.handle, _ptr(src), _ptr(dst), nbytes, _stream(stream))
    ctx.check(rc, "fs_stream_copy")


def fs_stream_row_read(ctx: Context, rows: torch.Tensor, index: torch.Tensor, sink: torch.Tensor, stream=None) -> None:
    """rows [num_rows, width] of any dtype with width * itemsize a multiple of 16; index int64; sink [1024] int32."""
    row_bytes = rows.shape[1] * rows.element_size()
    rc = ctx.lib.fs_stream_row_read(ctx.handle, _ptr(rows), rows.shape[0], row_bytes, _ptr(index), index.numel(),
                                    _ptr(sink), _stream(stream))
    ctx.check(rc, "fs_stream_row_read")


# ---- buffer bundles for the whole-iteration call (allocation only) -----------------------------
def alloc_layout(n: int, device, inverse: bool = True, sorted_ids: bool = False) -> Dict[str, torch.Tensor]:
    """inverse=False: no inverse map (the step calls do not need it; the two-part lookup does).
    sorted_ids=True: room for the ascending list of all IDs (the row-ordered lookup of the step calls reads it)."""
    out = {
        "unique": torch.empty(max(n, 1), dtype=torch.int64, device=device),
        "seg_offsets": torch.empty(n + 1, dtype=torch.int32, device=device),
        "perm": torch.empty(max(n, 1), dtype=torch.int32, device=device),
        "n_unique": torch.zeros(1, dtype=torch.int64, device=device),
        "n": n,
    }
    if inverse:
        out["inverse"] = torch.empty(max(n, 1), dtype=torch.int32, device=device)
    if sorted_ids:
        out["sorted_ids"] = torch.empty(max(n, 1), dtype=torch.int64, device=device)
    return out


def alloc_split(cap_t: int, cap_t1: int, device) -> Dict[str, torch.Tensor]:
    i64 = lambda k: torch.empty(max(k, 1), dtype=torch.int64, device=device)
    i32 = lambda k: torch.empty(max(k, 1), dtype=torch.int32, device=device)
    return {"co": i64(cap_t), "co_slot": i32(cap_t), "ex": i64(cap_t), "ex_slot": i32(cap_t),
            "ex_next": i64(cap_t1), "ex_next_slot": i32(cap_t1),
            "counts": torch.zeros(3, dtype=torch.int64, device=device),
            "cperm": i32(cap_t), "cslot": i32(cap_t), "cstart": i32(cap_t),
            "short_rec": i32(2 * SHORT_REC_INTS * cap_t),
            "co_flag_t1": torch.empty(max(cap_t1, 1), dtype=torch.uint8, device=device),
            "class_pos": torch.zeros(2, dtype=torch.int32, device=device)}


def make_step_args(table: torch.Tensor, state: torch.Tensor, lr: float, eps: float,
                   layout_t: Dict[str, torch.Tensor], grads_t: Optional[torch.Tensor],
                   values_t1: Optional[torch.Tensor], offsets_t1: Optional[torch.Tensor],
                   layout_t1: Optional[Dict[str, torch.Tensor]], split: Dict[str, torch.Tensor],
                   reduced: Optional[torch.Tensor], emb_t1: Optional[torch.Tensor]) -> fs_step_args:
    """Fills the argument record of fs_prioritized_step from tensors (pointers only)."""
    a = fs_step_args()
    a.table, a.state = _ptr(table), _ptr(state)
    a.num_rows, a.dim, a.dtype = table.shape[0], table.shape[1], table_dtype_code(table)
    a.lr, a.eps = lr, eps
    a.u_t, a.seg_offsets_t, a.perm_t = _ptr(layout_t["unique"]), _ptr(layout_t["seg_offsets"]), _ptr(layout_t["perm"])
    a.inverse_t = _ptr(layout_t.get("inverse"))
    a.n_unique_t_dev = _ptr(layout_t["n_unique"])
    a.grads_t = _ptr(grads_t)
    a.n_t = layout_t["n"]
    if values_t1 is not None:
        a.values_t1, a.offsets_t1 = _ptr(values_t1), _ptr(offsets_t1)
        a.batch_t1 = 0 if offsets_t1 is None else offsets_t1.numel() - 1
        a.n_t1 = values_t1.numel()
        a.u_t1, a.seg_offsets_t1 = _ptr(layout_t1["unique"]), _ptr(layout_t1["seg_offsets"])
        a.perm_t1, a.inverse_t1 = _ptr(layout_t1["perm"]), _ptr(layout_t1.get("inverse"))
        a.n_unique_t1_dev = _ptr(layout_t1["n_unique"])
        a.sorted_ids_t1 = _ptr(layout_t1.get("sorted_ids"))
        a.emb_t1 = _ptr(emb_t1)
    else:
        a.n_t1, a.batch_t1 = 0, 0
    a.co, a.co_slot, a.ex, a.ex_slot = _ptr(split["co"]), _ptr(split["co_slot"]), _ptr(split["ex"]), _ptr(split["ex_slot"])
    a.ex_next, a.ex_next_slot = _ptr(split["ex_next"]), _ptr(split["ex_next_slot"])
    a.counts_dev = _ptr(split["counts"])
    a.cperm, a.cslot, a.cstart = _ptr(split["cperm"]), _ptr(split["cslot"]), _ptr(split["cstart"])
    a.class_pos_dev = _ptr(split["class_pos"])
    a.short_rec = _ptr(split["short_rec"])
    a.co_flag_t1 = _ptr(split.get("co_flag_t1"))
    a.reduced = _ptr(reduced)
    return a


# ---- the history encoder (include/freescale_encoder.h) ----------------------------------------------------------------
FS_ROWS8_GROUP = 32
FS_MAX_BLOCK_DIM = 1024


class Rows8(NamedTuple):
    """Rows in 8 bits: codes int8 [n, dim], exps uint8 [n, dim / FS_ROWS8_GROUP]."""
    codes: torch.Tensor
    exps: torch.Tensor


def _ctx_stream(ctx: Context, stream):
    """The stream of a call: the current one of the context's GPU, which need not be the current GPU."""
    if stream is None and _current_raw_stream is not None:
        return _current_raw_stream(ctx.device) or None
    return _stream(torch.cuda.current_stream(ctx.device) if stream is None else stream)


def _on_its_stream(call):
    """A stream that a call names is the current one for as long as the call takes, so that torch takes scratch memory and
    results from that stream's pool: memory of the current stream's pool may still be in use by what that stream has ahead,
    which the named stream does not wait for.  Results belong to that stream as those of torch's own operators would: another
    stream that reads them waits for it, and is named to record_stream before they are dropped."""
    place = list(inspect.signature(call).parameters).index("stream") - 1          # behind ctx

    @functools.wraps(call)
    def run(ctx, *args, stream=None, **named):
        if len(args) > place:
            (stream,), args = args[place:], args[:place]
        handle = None if stream is None else _ctx_stream(ctx, stream)
        if stream is None or handle == _ctx_stream(ctx, None):
            return call(ctx, *args, **named)
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(handle or 0, device=ctx.device)
        elif stream.device_index != ctx.device:
            raise ValueError(f"stream: of cuda:{stream.device_index}, the context is on cuda:{ctx.device}")
        with torch.cuda.stream(stream):
            return call(ctx, *args, **named)
    return run


def _scratch(like: torch.Tensor, nbytes: int) -> torch.Tensor:
    """Scratch memory that is given back when the call has been enqueued on the current stream, whose pool it is from."""
    return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=like.device)


_DTYPE_CODES = {torch.float32: FS_F32, torch.bfloat16: FS_BF16}


def _code(what: str, dtype: torch.dtype) -> int:
    code = _DTYPE_CODES.get(dtype)
    if code is None:
        raise TypeError(f"{what}: {dtype}, fp32 or bf16 only")
    return code


def _addr(what: str, t: torch.Tensor, shape, dtype: torch.dtype, device: int) -> int:
    """The address of a contiguous tensor of that shape and type on that GPU; raises if it is not one.  (These checks are most
    of what a small call costs the host: one condition of four quick questions, and the explanation only where one fails.)"""
    if t is None or t.shape != shape or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        _refuse(what, t, shape, dtype, device)
    return t.data_ptr()


def _refuse(what, t, shape, dtype, device):
    if t is None:
        raise ValueError(f"{what}: is needed")
    if t.dtype != dtype:
        raise TypeError(f"{what}: {t.dtype}, {dtype} is needed")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, {tuple(shape)} is needed")
    if t.get_device() != device:
        raise ValueError(f"{what}: on {t.device}, the context is on cuda:{device}")
    raise ValueError(f"{what}: strides {t.stride()}, other than this call takes")


def _row_addr(what: str, t: torch.Tensor, shape, dtype: torch.dtype, device: int):
    """(address, elements from row to row) of a tensor whose rows may lie apart; a row itself may not."""
    if t is None or t.is_contiguous():
        stride = 1
        for k in shape[1:]:
            stride *= k
        return _addr(what, t, shape, dtype, device), stride
    strides, inner = t.stride(), 1
    for k in range(len(shape) - 1, 0, -1):
        if t.dim() != len(shape) or (shape[k] > 1 and strides[k] != inner):
            _refuse(what, t, shape, dtype, device)
        inner *= shape[k]
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        _refuse(what, t, shape, dtype, device)
    return t.data_ptr(), strides[0] if shape[0] > 1 else inner


def _pair_addr(what: str, t: Rows8, n: int, dim: int, device: int):
    return (_addr(what + ".codes", t.codes, (n, dim), torch.int8, device),
            _addr(what + ".exps", t.exps, (n, dim // FS_ROWS8_GROUP), torch.uint8, device))


def _alloc_rows8(n: int, dim: int, device) -> Rows8:
    return Rows8(torch.empty((n, dim), dtype=torch.int8, device=device),
                 torch.empty((n, dim // FS_ROWS8_GROUP), dtype=torch.uint8, device=device))


def _matrix(what: str, t: torch.Tensor):
    if t is None:
        raise ValueError(f"{what}: is needed")
    if t.dim() != 2:
        raise ValueError(f"{what}: shape {tuple(t.shape)}, two dimensions are needed")
    return tuple(t.shape)


@_on_its_stream
def fs_rows_pack8(ctx: Context, rows: torch.Tensor, out: Optional[Rows8] = None, stream=None) -> Rows8:
    n, dim = _matrix("rows", rows)
    address, stride = _row_addr("rows", rows, (n, dim), rows.dtype, ctx.device)
    if out is None:
        out = _alloc_rows8(n, dim, rows.device)
    codes, exps = _pair_addr("out", out, n, dim, ctx.device)
    rc = ctx.lib.fs_rows_pack8(ctx.handle, address, stride, _code("rows", rows.dtype), n, dim, codes, exps, _ctx_stream(ctx, stream))
    if rc:
        ctx.check(rc, "fs_rows_pack8")
    return out


@_on_its_stream
def fs_rows_unpack8(ctx: Context, packed: Rows8, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    n, dim = _matrix("packed.codes", packed.codes)
    codes, exps = _pair_addr("packed", packed, n, dim, ctx.device)
    if out is None:
        out = torch.empty((n, dim), dtype=dtype, device=packed.codes.device)
    address, stride = _row_addr("out", out, (n, dim), out.dtype, ctx.device)
    rc = ctx.lib.fs_rows_unpack8(ctx.handle, codes, exps, n, dim, address, stride, _code("out", out.dtype), _ctx_stream(ctx, stream))
    if rc:
        ctx.check(rc, "fs_rows_unpack8")
    return out


@_on_its_stream
def fs_block_norm(ctx: Context, x: torch.Tensor, a: Optional[torch.Tensor] = None, g: Optional[torch.Tensor] = None,
                  w_post: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                  w_pre: Optional[torch.Tensor] = None, eps: float = 1e-6, pack: Sequence[str] = (),
                  dtype: Optional[torch.dtype] = None, out: Optional[Dict] = None, stream=None) -> Dict:
    """y (where a is given) and h (where w_pre is given); pack: which of "a", "g", "y" are wanted in 8 bits too, as a8, g8,
    y8.  dtype: that of h where there is no a.  `out`: the caller's tensors under the same names."""
    n, dim = shape = _matrix("x", x)
    dev, rows_dt = ctx.device, x.dtype
    act = a.dtype if a is not None else dtype or rows_dt
    rec = fs_block_args()
    rec.n, rec.dim, rec.eps = n, dim, eps
    rec.rows_dt, rec.dt = _code("x", rows_dt), _code("a or h", act)
    rec.x = _addr("x", x, shape, rows_dt, dev)
    given, res = out or {}, {}
    if a is not None:
        rec.a, rec.a_stride = _row_addr("a", a, shape, act, dev)
        rec.g, rec.g_stride = _row_addr("g", g, shape, act, dev)
        rec.w_post = _addr("w_post", w_post, (dim,), torch.float32, dev)
        rec.scale = _addr("scale", scale, (dim,), torch.float32, dev)
        res["y"] = y = given["y"] if "y" in given else torch.empty_like(x)
        rec.y = _addr("y", y, shape, rows_dt, dev)
    if w_pre is not None:
        rec.w_pre = _addr("w_pre", w_pre, (dim,), torch.float32, dev)
        res["h"] = h = given["h"] if "h" in given else torch.empty(shape, dtype=act, device=x.device)
        rec.h = _addr("h", h, shape, act, dev)
    for name in pack:
        if name not in ("a", "g", "y") or (a is None and name != "y"):
            raise ValueError(f"pack: no {name!r} to pack")
        key = name + "8"
        res[key] = packed = given[key] if key in given else _alloc_rows8(n, dim, x.device)
        codes, exps = _pair_addr(key, packed, n, dim, dev)
        setattr(rec, name + "_codes", codes)
        setattr(rec, name + "_exps", exps)
    rc = ctx.lib.fs_block_norm(ctx.handle, rec, _ctx_stream(ctx, stream))
    if rc:
        ctx.check(rc, "fs_block_norm")
    return res


@_on_its_stream
def fs_block_norm_backward(ctx: Context, dy: Optional[torch.Tensor], dh: Optional[torch.Tensor],
                           a: Union[torch.Tensor, Rows8, None] = None, g: Union[torch.Tensor, Rows8, None] = None,
                           y: Union[torch.Tensor, Rows8, None] = None, w_post: Optional[torch.Tensor] = None,
                           scale: Optional[torch.Tensor] = None, w_pre: Optional[torch.Tensor] = None, eps: float = 1e-6,
                           dtype: Optional[torch.dtype] = None, rows_dtype: Optional[torch.dtype] = None,
                           out: Optional[Dict[str, torch.Tensor]] = None, stream=None) -> Dict[str, torch.Tensor]:
    """dx, and da, dg, dw_post, dscale where a is given, dw_pre where dh is given.  a, g, y: as the forward pass had or left
    them, or its a8, g8, y8.  dtype, rows_dtype: those of the block's rows and of the residual rows, where no tensor given
    tells."""
    some = dy if dy is not None else dh if dh is not None else a if a is not None else y
    if isinstance(some, Rows8):
        some = some.codes
    n, dim = shape = _matrix("dy, dh, a or y", some)
    dev, device, f32 = ctx.device, some.device, torch.float32
    plain = lambda *ts: next((t.dtype for t in ts if isinstance(t, torch.Tensor)), None)  # noqa: E731
    rows_dt = plain(dy, y) or rows_dtype or f32
    act = plain(dh, a, g) or dtype or rows_dt
    rec = fs_block_args()
    rec.n, rec.dim, rec.eps = n, dim, eps
    rec.rows_dt, rec.dt = _code("dy or y", rows_dt), _code("dh, a or g", act)
    given, res = out or {}, {}
    res["dx"] = t = given["dx"] if "dx" in given else torch.empty(shape, dtype=rows_dt, device=device)
    rec.dx = _addr("dx", t, shape, rows_dt, dev)
    if dy is not None:
        rec.dy = _addr("dy", dy, shape, rows_dt, dev)
    if dh is not None:
        rec.dh = _addr("dh", dh, shape, act, dev)
        rec.w_pre = _addr("w_pre", w_pre, (dim,), f32, dev)
        if isinstance(y, Rows8):
            rec.y_codes, rec.y_exps = _pair_addr("y", y, n, dim, dev)
        else:
            rec.y = _addr("y", y, shape, rows_dt, dev)
        res["dw_pre"] = t = given["dw_pre"] if "dw_pre" in given else torch.empty_like(w_pre)
        rec.dw_pre = _addr("dw_pre", t, (dim,), f32, dev)
    if a is not None:
        if isinstance(a, Rows8):
            rec.a_codes, rec.a_exps = _pair_addr("a", a, n, dim, dev)
        else:
            rec.a, rec.a_stride = _row_addr("a", a, shape, act, dev)
        if isinstance(g, Rows8):
            rec.g_codes, rec.g_exps = _pair_addr("g", g, n, dim, dev)
        else:
            rec.g, rec.g_stride = _row_addr("g", g, shape, act, dev)
        rec.w_post = _addr("w_post", w_post, (dim,), f32, dev)
        rec.scale = _addr("scale", scale, (dim,), f32, dev)
        res["da"] = t = given["da"] if "da" in given else torch.empty(shape, dtype=act, device=device)
        rec.da, rec.da_stride = _row_addr("da", t, shape, act, dev)
        res["dg"] = t = given["dg"] if "dg" in given else torch.empty(shape, dtype=act, device=device)
        rec.dg, rec.dg_stride = _row_addr("dg", t, shape, act, dev)
        res["dw_post"] = t = given["dw_post"] if "dw_post" in given else torch.empty_like(w_post)
        rec.dw_post = _addr("dw_post", t, (dim,), f32, dev)
        res["dscale"] = t = given["dscale"] if "dscale" in given else torch.empty_like(scale)
        rec.dscale = _addr("dscale", t, (dim,), f32, dev)
    work = _scratch(some, ctx.lib.fs_block_norm_work_bytes(n, dim))
    rec.work, rec.work_bytes = work.data_ptr(), work.numel()
    rc = ctx.lib.fs_block_norm_backward(ctx.handle, rec, _ctx_stream(ctx, stream))
    if rc:
        ctx.check(rc, "fs_block_norm_backward")
    return res


FS_MAX_HEAD_DIM, FS_MAX_BIAS_BUCKETS, FS_MAX_BIAS_DISTANCES, FS_MAX_ROW_STRIDE = 128, 1024, 4096, 1 << 22
FS_HIDDEN_BIAS = -40000.0      # a bias so low hides its pairs


def _attention_record(ctx, q, k, v, q_offsets, kv_offsets, bias, bucket_of, kv_lengths, causal, scale):
    """The record of a call but for what it writes; (shape of q, of k and v)."""
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError(f"q, k: shapes {tuple(q.shape)}, {tuple(k.shape)}, [rows, heads, head_dim] are needed")
    dev, dt, i64 = ctx.device, q.dtype, torch.int64
    shape, (n_kv, kv_heads, _) = tuple(q.shape), k.shape
    n_q, heads, width = shape
    keys, users = (n_kv, kv_heads, width), (q_offsets.numel(),)
    rec = fs_attention_args()
    rec.dt = _code("q", dt)
    rec.q, rec.q_stride = _row_addr("q", q, shape, dt, dev)
    rec.k, rec.k_stride = _row_addr("k", k, keys, dt, dev)
    rec.v, rec.v_stride = _row_addr("v", v, keys, dt, dev)
    rec.n_q, rec.n_kv, rec.batch, rec.heads, rec.kv_heads, rec.head_dim = n_q, n_kv, users[0] - 1, heads, kv_heads, width
    rec.q_offsets = _addr("q_offsets", q_offsets, users, i64, dev)
    rec.kv_offsets = _addr("kv_offsets", kv_offsets, users, i64, dev)
    rec.causal, rec.scale = 1 if causal else 0, width ** -0.5 if scale is None and width else scale or 0.0
    if kv_lengths is not None:
        rec.kv_lengths = _addr("kv_lengths", kv_lengths, (users[0] - 1,), i64, dev)
    if bias is not None:
        buckets, _ = _matrix("bias", bias)
        if bucket_of is None or buckets == 0:
            raise ValueError("bucket_of: is needed" if bucket_of is None else "bias: has no bucket")
        size = bucket_of.numel()
        if not causal and size % 2 == 0:
            raise ValueError(f"bucket_of: {size} entries, an odd number is needed for distances on both sides")
        rec.bias = _addr("bias", bias, (buckets, heads), torch.float32, dev)
        rec.bucket_of = _addr("bucket_of", bucket_of, (size,), torch.int32, dev)
        rec.num_buckets, rec.num_distances = buckets, size if causal else (size + 1) // 2
    return rec, shape, keys


@_on_its_stream
def fs_jagged_attention(ctx: Context, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_offsets: torch.Tensor,
                        kv_offsets: torch.Tensor, bias: Optional[torch.Tensor] = None, bucket_of: Optional[torch.Tensor] = None,
                        kv_lengths: Optional[torch.Tensor] = None, causal: bool = True, scale: Optional[float] = None,
                        max_q: int = 0, keep: bool = False, out: Optional[Dict[str, torch.Tensor]] = None,
                        stream=None) -> Dict[str, torch.Tensor]:
    """out [n_q, heads, head_dim]; keep: also what fs_jagged_attention_backward reads (lse, and out_f32 of bf16 rows).  scale:
    1 / sqrt(head_dim) unless given.  `out`: the caller's tensors under the same names."""
    rec, shape, _ = _attention_record(ctx, q, k, v, q_offsets, kv_offsets, bias, bucket_of, kv_lengths, causal, scale)
    rec.max_q = min(max_q, (1 << 31) - 1)                    # 32 bits there; no user has more rows than that
    given, res, dev, f32 = out or {}, {}, ctx.device, torch.float32
    res["out"] = t = given["out"] if "out" in given else torch.empty(shape, dtype=q.dtype, device=q.device)
    rec.out = _addr("out", t, shape, q.dtype, dev)
    if (keep or "out_f32" in given) and q.dtype != f32:
        res["out_f32"] = t = given["out_f32"] if "out_f32" in given else torch.empty(shape, dtype=f32, device=q.device)
        rec.out_f32 = _addr("out_f32", t, shape, f32, dev)
    if keep or "lse" in given:
        res["lse"] = t = given["lse"] if "lse" in given else torch.empty((shape[1], shape[0]), dtype=f32, device=q.device)
        rec.lse = _addr("lse", t, (shape[1], shape[0]), f32, dev)
    if max_q:
        nbytes = ctx.lib.fs_jagged_attention_work_bytes(rec)
        if nbytes:
            work = _scratch(q, nbytes)
            rec.work, rec.work_bytes = work.data_ptr(), work.numel()
    rc = ctx.lib.fs_jagged_attention(ctx.handle, rec, _ctx_stream(ctx, stream))
    if rc:
        ctx.check(rc, "fs_jagged_attention")
    return res


@_on_its_stream
def fs_jagged_attention_backward(ctx: Context, dout: torch.Tensor, kept: Dict[str, torch.Tensor], q: torch.Tensor, k: torch.Tensor,
                                 v: torch.Tensor, q_offsets: torch.Tensor, kv_offsets: torch.Tensor,
                                 bias: Optional[torch.Tensor] = None, bucket_of: Optional[torch.Tensor] = None,
                                 kv_lengths: Optional[torch.Tensor] = None, causal: bool = True, scale: Optional[float] = None,
                                 out: Optional[Dict[str, torch.Tensor]] = None, stream=None) -> Dict[str, torch.Tensor]:
    """dq, dk, dv, and dbias where there is a bias.  kept: what fs_jagged_attention(keep=True) returned.  `out`: the caller's
    tensors under the same names."""
    rec, shape, keys = _attention_record(ctx, q, k, v, q_offsets, kv_offsets, bias, bucket_of, kv_lengths, causal, scale)
    dev, dt, f32 = ctx.device, q.dtype, torch.float32
    rec.dout = _addr("dout", dout, shape, dt, dev)
    rec.out = _addr("kept['out']", kept["out"], shape, dt, dev)
    rec.lse = _addr("kept['lse']", kept["lse"], (shape[1], shape[0]), f32, dev)
    if kept.get("out_f32") is not None:
        rec.out_f32 = _addr("kept['out_f32']", kept["out_f32"], shape, f32, dev)
    given, res = out or {}, {}
    res["dq"] = t = given["dq"] if "dq" in given else torch.empty(shape, dtype=dt, device=q.device)
    rec.dq, rec.dq_stride = _row_addr("dq", t, shape, dt, dev)
    res["dk"] = t = given["dk"] if "dk" in given else torch.empty(keys, dtype=dt, device=q.device)
    rec.dk, rec.dk_stride = _row_addr("dk", t, keys, dt, dev)
    res["dv"] = t = given["dv"] if "dv" in given else torch.empty(keys, dtype=dt, device=q.device)
    rec.dv, rec.dv_stride = _row_addr("dv", t, keys, dt, dev)
    if bias is not None:
        res["dbias"] = t = given["dbias"] if "dbias" in given else torch.empty_like(bias)
        rec.dbias = _addr("dbias", t, bias.shape, f32, dev)
    work = _scratch(q, ctx.lib.fs_jagged_attention_backward_work_bytes(rec))
    rec.work, rec.work_bytes = work.data_ptr(), work.numel()
    rc = ctx.lib.fs_jagged_attention_backward(ctx.handle, rec, _ctx_stream(ctx, stream))
    if rc:
        ctx.check(rc, "fs_jagged_attention_backward")
    return res
