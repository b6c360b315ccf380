"""ctypes binding of libflexdraft.so: argument marshalling only.

Every function here has the name of the C entry point it forwards to
(include/flexdraft.h).  Torch is used for device memory and the current stream;
no arithmetic of the method happens in Python.  If the shared library has not
been built, loading raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# FLEXDRAFT_LIB names another build of the same library (same C ABI), e.g. one compiled with other tuning macros
LIB_PATH = os.environ.get("FLEXDRAFT_LIB") or os.path.join(_HERE, "libflexdraft.so")

FD_F32, FD_BF16 = 0, 1
FD_ATTN_FORCE_GENERIC = 1
FD_ATTN_PLANNED = 2
FD_OK = 0
STATUS_NAMES = {0: "FD_OK", 1: "FD_ERR_INVALID_ARG", 2: "FD_ERR_UNSUPPORTED",
                3: "FD_ERR_WORKSPACE_TOO_SMALL", 4: "FD_ERR_HIP"}


class fd_attn_args(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("num_q_heads", C.c_int32), ("num_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("page_size", C.c_int32), ("dtype", C.c_int32), ("sm_scale", C.c_float), ("flags", C.c_int32),
        ("total_rows", C.c_int32), ("max_kv_len", C.c_int32), ("max_new_rows", C.c_int32), ("num_pages", C.c_int32),
        ("kv_chunk", C.c_int32), ("page_indices_len", C.c_int32),
        ("k_cache", C.c_void_p), ("v_cache", C.c_void_p),
        ("cache_stride_page", C.c_int64), ("cache_stride_head", C.c_int64), ("cache_stride_token", C.c_int64),
        ("page_indptr", C.c_void_p), ("page_indices", C.c_void_p), ("kv_len", C.c_void_p),
        ("row_indptr", C.c_void_p), ("verify_len", C.c_void_p), ("mask_vis", C.c_void_p),
        ("mask_blocks", C.c_void_p),
        ("q", C.c_void_p), ("k_new", C.c_void_p), ("v_new", C.c_void_p),
        ("out", C.c_void_p), ("lse", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
        ("status", C.c_void_p),
    ]
    device, cache = -1, None     # of make_attn_args_q4: where the tensors are whose addresses these are, and the cache in 4 bits


class fd_table_args(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("page_size", C.c_int32), ("table_stride", C.c_int32), ("total_rows", C.c_int32),
        ("page_indices_len", C.c_int32), ("free_pages_len", C.c_int32),
        ("kv_len", C.c_void_p), ("verify_len", C.c_void_p), ("mask_rows", C.c_void_p), ("mask_vis", C.c_void_p),
        ("mask_blocks", C.c_void_p), ("block_table", C.c_void_p), ("table_len", C.c_void_p), ("table_len_out", C.c_void_p),
        ("free_pages", C.c_void_p), ("free_count", C.c_void_p), ("free_count_out", C.c_void_p),
        ("row_indptr", C.c_void_p), ("page_indptr", C.c_void_p), ("page_indices", C.c_void_p),
        ("positions", C.c_void_p), ("slot_map", C.c_void_p), ("status", C.c_void_p),
    ]
    device = -1                  # where the tensors are whose addresses these are


class fd_rope_args(C.Structure):
    _fields_ = [
        ("total_rows", C.c_int32), ("num_q_heads", C.c_int32), ("num_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("dtype", C.c_int32), ("eps", C.c_float),
        ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p),
        ("q_stride_row", C.c_int64), ("q_stride_head", C.c_int64), ("k_stride_row", C.c_int64), ("k_stride_head", C.c_int64),
        ("v_stride_row", C.c_int64), ("v_stride_head", C.c_int64),
        ("q_out", C.c_void_p), ("k_out", C.c_void_p), ("v_out", C.c_void_p),
        ("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("inv_freq", C.c_void_p), ("positions", C.c_void_p),
    ]


class fd_q4_cache(C.Structure):
    _fields_ = [
        ("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("v_scales", C.c_void_p),
        ("stride_page", C.c_int64), ("stride_head", C.c_int64),
    ]


class FlexDraftError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {msg}")
        self.code = code


_lib = None

EXPORTS = ["fd_verify_draft_attn_workspace", "fd_verify_draft_attn", "fd_accept_greedy", "fd_accept_sample",
           "fd_accept_workspace", "fd_draft_select", "fd_draft_select_workspace", "fd_append_kv", "fd_select_branch", "fd_last_error", "fd_version", "fd_verify_draft_attn_static",
           "fd_verify_draft_plan", "fd_step_tables", "fd_qk_norm_rope", "fd_verify_draft_attn_q4", "fd_verify_draft_attn_q4_workspace",
           "fd_append_kv_q4", "fd_read_kv_q4"]


def load() -> C.CDLL:
    """Load the HIP library; raises if it has not been built (python -m paper_2605_20022_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python paper_2605_20022_amd/build.py` "
                           "(hipcc, gfx950). There is no CPU fallback.")
    lib = C.CDLL(LIB_PATH)
    lib.fd_verify_draft_attn_workspace.restype = C.c_size_t
    lib.fd_verify_draft_attn_workspace.argtypes = [C.POINTER(fd_attn_args)]
    lib.fd_verify_draft_attn.restype = C.c_int
    lib.fd_verify_draft_attn.argtypes = [C.POINTER(fd_attn_args), C.c_void_p]
    lib.fd_accept_greedy.restype = C.c_int
    lib.fd_accept_greedy.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p,
                                     C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_void_p, C.c_size_t, C.c_void_p]
    lib.fd_accept_sample.restype = C.c_int
    lib.fd_accept_sample.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int32, C.c_float,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                     C.c_void_p, C.c_size_t, C.c_void_p]
    lib.fd_accept_workspace.restype = C.c_size_t
    lib.fd_accept_workspace.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32]
    lib.fd_draft_select.restype = C.c_int
    lib.fd_draft_select.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.c_int32, C.c_float, C.c_float, C.c_void_p,
                                    C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_size_t, C.c_void_p]
    lib.fd_draft_select_workspace.restype = C.c_size_t
    lib.fd_draft_select_workspace.argtypes = [C.c_int32, C.c_int32]
    lib.fd_append_kv.restype = C.c_int
    lib.fd_append_kv.argtypes = [C.POINTER(fd_attn_args), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.fd_verify_draft_plan.restype = C.c_int
    lib.fd_verify_draft_plan.argtypes = [C.POINTER(fd_attn_args), C.c_void_p]
    lib.fd_verify_draft_attn_static.restype = C.c_int
    lib.fd_verify_draft_attn_static.argtypes = [C.POINTER(fd_attn_args), C.c_void_p]
    lib.fd_select_branch.restype = C.c_int
    lib.fd_select_branch.argtypes = [C.c_void_p] * 6 + [C.c_int32] * 3 + [C.c_void_p] * 3
    lib.fd_step_tables.restype = C.c_int
    lib.fd_step_tables.argtypes = [C.POINTER(fd_table_args), C.c_void_p]
    lib.fd_qk_norm_rope.restype = C.c_int
    lib.fd_qk_norm_rope.argtypes = [C.POINTER(fd_rope_args), C.c_void_p]
    lib.fd_verify_draft_attn_q4_workspace.restype = C.c_size_t
    lib.fd_verify_draft_attn_q4_workspace.argtypes = [C.POINTER(fd_attn_args)]
    lib.fd_verify_draft_attn_q4.restype = C.c_int
    lib.fd_verify_draft_attn_q4.argtypes = [C.POINTER(fd_attn_args), C.POINTER(fd_q4_cache), C.c_void_p]
    lib.fd_append_kv_q4.restype = C.c_int
    lib.fd_append_kv_q4.argtypes = [C.POINTER(fd_attn_args), C.POINTER(fd_q4_cache), C.c_void_p, C.c_void_p, C.c_void_p]
    lib.fd_read_kv_q4.restype = C.c_int
    lib.fd_read_kv_q4.argtypes = [C.POINTER(fd_q4_cache)] + [C.c_int32] * 5 + [C.c_void_p] * 2 + [C.c_int32] + [C.c_void_p] * 2 + \
        [C.c_int32, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]
    lib.fd_last_error.restype = C.c_char_p
    lib.fd_version.restype = C.c_char_p
    _lib = lib
    return lib


def _check(code: int):
    if code != FD_OK:
        raise FlexDraftError(code, load().fd_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# The handle of the current device's current stream.  torch.cuda.current_stream() builds a Stream object for it, 2.2 us of
# a call's 8; thirteen calls of a decoding step take the host 107 us with it, 79 with the handle alone (76 with plain addresses too).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(torch._C._cuda_getDevice())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return FD_BF16
    if t.dtype == torch.float32:
        return FD_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _i32(t: torch.Tensor, name: str) -> torch.Tensor:
    if t.dtype != torch.int32 or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous int32 tensor")
    return t


def make_attn_args(q, k_new, v_new, k_cache, v_cache, page_indptr, page_indices, kv_len, row_indptr,
                   verify_len, mask_vis=None, mask_blocks=None, *, out, lse=None, max_kv_len: int, max_new_rows: int,
                   sm_scale: float = 0.0, flags: int = 0, kv_chunk: int = 0, workspace=None, status=None):
    """Fill an fd_attn_args from tensors.  k_cache / v_cache: [pages, Hkv, page_size, D] views
    (any strides with a contiguous last dimension)."""
    R, Hq, D = q.shape
    Hkv = k_new.shape[1]
    for name, t in (("q", q), ("k_new", k_new), ("v_new", v_new), ("out", out)):
        if not t.is_contiguous():
            raise TypeError(f"{name} must be contiguous")
    if k_cache.stride(3) != 1 or v_cache.stride() != k_cache.stride():
        raise TypeError("k_cache / v_cache need a contiguous last dimension and identical strides")
    a = fd_attn_args()
    a.batch = kv_len.shape[0]; a.num_q_heads = Hq; a.num_kv_heads = Hkv; a.head_dim = D
    a.page_size = k_cache.shape[2]; a.dtype = _dtype_code(q); a.sm_scale = sm_scale; a.flags = flags
    a.total_rows = R; a.max_kv_len = int(max_kv_len); a.max_new_rows = int(max_new_rows)
    a.num_pages = k_cache.shape[0]; a.kv_chunk = kv_chunk; a.page_indices_len = page_indices.numel()
    a.k_cache = k_cache.data_ptr(); a.v_cache = v_cache.data_ptr()
    a.cache_stride_page = k_cache.stride(0); a.cache_stride_head = k_cache.stride(1)
    a.cache_stride_token = k_cache.stride(2)
    a.page_indptr = _i32(page_indptr, "page_indptr").data_ptr()
    a.page_indices = _i32(page_indices, "page_indices").data_ptr()
    a.kv_len = _i32(kv_len, "kv_len").data_ptr()
    a.row_indptr = _i32(row_indptr, "row_indptr").data_ptr()
    a.verify_len = _i32(verify_len, "verify_len").data_ptr()
    a.mask_vis = None if mask_vis is None else _i32(mask_vis, "mask_vis").data_ptr()
    a.mask_blocks = None if mask_blocks is None else _i32(mask_blocks, "mask_blocks").data_ptr()
    a.q = q.data_ptr(); a.k_new = k_new.data_ptr(); a.v_new = v_new.data_ptr()
    a.out = out.data_ptr(); a.lse = None if lse is None else lse.data_ptr()
    if workspace is not None:
        a.workspace = workspace.data_ptr(); a.workspace_bytes = workspace.numel() * workspace.element_size()
    a.status = None if status is None else status.data_ptr()
    return a


def fd_verify_draft_attn_workspace(args: fd_attn_args) -> int:
    return int(load().fd_verify_draft_attn_workspace(C.byref(args)))


def fd_verify_draft_attn(args: fd_attn_args, stream=None) -> None:
    """Enqueue the attention call described by `args` on `stream` (default: torch's current stream)."""
    _check(load().fd_verify_draft_attn(C.byref(args), _stream(stream)))


def fd_verify_draft_plan(args: fd_attn_args, stream=None) -> None:
    """Write the plan for `args` into args.workspace; attention calls with FD_ATTN_PLANNED start from it."""
    _check(load().fd_verify_draft_plan(C.byref(args), _stream(stream)))


def fd_verify_draft_attn_static(args: fd_attn_args, stream=None) -> None:
    """The same call on the library's own static scratch buffer: args.workspace is ignored."""
    _check(load().fd_verify_draft_attn_static(C.byref(args), _stream(stream)))


FD_STATIC_SCRATCH_BYTES = 44 << 20


def fd_accept_workspace(batch: int, total_rows: int, vocab: int, sampling: bool) -> int:
    return int(load().fd_accept_workspace(batch, total_rows, vocab, 1 if sampling else 0))


def fd_accept_greedy(target_logits, row_indptr, input_tokens, accept_len, bonus_token, *, vocab=None,
                     max_rows_per_seq: int, row_argmax=None, workspace, stream=None) -> None:
    Rv = target_logits.shape[0]
    vocab = target_logits.shape[1] if vocab is None else vocab
    if target_logits.stride(1) != 1:
        raise TypeError("logits rows must be contiguous")
    _check(load().fd_accept_greedy(
        _ptr(target_logits), _dtype_code(target_logits), target_logits.stride(0), vocab,
        _ptr(_i32(row_indptr, "row_indptr")), _ptr(_i32(input_tokens, "input_tokens")),
        accept_len.shape[0], Rv, max_rows_per_seq,
        _ptr(_i32(accept_len, "accept_len")), _ptr(_i32(bonus_token, "bonus_token")),
        None if row_argmax is None else _ptr(_i32(row_argmax, "row_argmax")),
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def fd_accept_sample(target_logits, draft_logits, row_indptr, input_tokens, u_accept, u_resample,
                     accept_len, bonus_token, *, temperature: float, vocab=None, max_rows_per_seq: int,
                     workspace, stream=None) -> None:
    Rv = target_logits.shape[0]
    vocab = target_logits.shape[1] if vocab is None else vocab
    if target_logits.stride(1) != 1 or draft_logits.stride() != target_logits.stride() or \
            draft_logits.dtype != target_logits.dtype:
        raise TypeError("target / draft logits must share dtype and strides, rows contiguous")
    for name, t in (("u_accept", u_accept), ("u_resample", u_resample)):
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise TypeError(f"{name} must be contiguous float32")
    _check(load().fd_accept_sample(
        _ptr(target_logits), _ptr(draft_logits), _dtype_code(target_logits), target_logits.stride(0), vocab,
        float(temperature), _ptr(_i32(row_indptr, "row_indptr")), _ptr(_i32(input_tokens, "input_tokens")),
        _ptr(u_accept), _ptr(u_resample), accept_len.shape[0], Rv, max_rows_per_seq,
        _ptr(_i32(accept_len, "accept_len")), _ptr(_i32(bonus_token, "bonus_token")),
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def fd_draft_select_workspace(total_rows: int, vocab: int) -> int:
    return int(load().fd_draft_select_workspace(total_rows, vocab))


def fd_draft_select(draft_logits, row_indptr, draft_tokens, keep_len, *, temperature: float, threshold: float,
                    max_rows_per_seq: int, confidence=None, vocab=None, workspace, stream=None) -> None:
    R = draft_logits.shape[0]
    vocab = draft_logits.shape[1] if vocab is None else vocab
    if R and draft_logits.stride(1) != 1:
        raise TypeError("logits rows must be contiguous")
    _check(load().fd_draft_select(
        _ptr(draft_logits), _dtype_code(draft_logits), draft_logits.stride(0) if R else vocab, vocab,
        float(temperature), float(threshold), _ptr(_i32(row_indptr, "row_indptr")), keep_len.shape[0], R,
        int(max_rows_per_seq), _ptr(_i32(draft_tokens, "draft_tokens")),
        None if confidence is None else _ptr(confidence), _ptr(_i32(keep_len, "keep_len")),
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def fd_append_kv(args: fd_attn_args, k_cache, v_cache, accept_len, kv_len_out, stream=None) -> None:
    """Commit new rows 0 .. accept_len[i] of the call described by `args` to the paged cache
    k_cache / v_cache (written; laid out as args' strides say)."""
    _check(load().fd_append_kv(C.byref(args), _ptr(k_cache), _ptr(v_cache), _ptr(_i32(accept_len, "accept_len")),
                               _ptr(_i32(kv_len_out, "kv_len_out")), _stream(stream)))


def fd_select_branch(block_tokens, block_indptr, mask_blocks, accept_len, out_tokens, *, first_vis=None,
                     verify_len=None, out_block=None, stream=None) -> None:
    B = accept_len.shape[0]
    _check(load().fd_select_branch(
        _ptr(_i32(block_tokens, "block_tokens")), _ptr(_i32(block_indptr, "block_indptr")),
        _ptr(_i32(mask_blocks, "mask_blocks")), _ptr(_i32(accept_len, "accept_len")),
        None if first_vis is None else _ptr(_i32(first_vis, "first_vis")),
        None if verify_len is None else _ptr(_i32(verify_len, "verify_len")), B, block_tokens.numel(),
        out_tokens.shape[1], _ptr(_i32(out_tokens, "out_tokens")),
        None if out_block is None else _ptr(_i32(out_block, "out_block")), _stream(stream)))


def _opt_i32(t: Optional[torch.Tensor], name: str):
    return None if t is None else _i32(t, name).data_ptr()


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _one_device(*tensors: Optional[torch.Tensor]) -> int:
    """The index of the device on which all of them are, -1 for the CPU."""
    device = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise TypeError("the tensors are on different devices")
    return device


def _launchable(device: int) -> None:
    """A kernel runs on the current device, and what it is given has to be there."""
    if device < 0:
        raise TypeError("the tensors are on the CPU")
    if device != _current_device():
        raise TypeError(f"the tensors are on device {device}, the current device is {_current_device()}")


def make_table_args(kv_len, verify_len, block_table, table_len, free_pages, free_count, mask_rows=None, mask_vis=None, mask_blocks=None, *,
                    page_size: int, row_indptr, page_indptr, page_indices, positions=None, slot_map=None, table_len_out=None,
                    free_count_out=None, status=None):
    """Fill an fd_table_args from tensors.  table_len_out / free_count_out default to table_len / free_count, updated in place."""
    B = kv_len.shape[0]
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise TypeError("block_table must be [batch, entries]")
    sizes = [("verify_len", verify_len, B), ("table_len", table_len, B), ("mask_rows", mask_rows, B), ("mask_vis", mask_vis, B),
             ("mask_blocks", mask_blocks, B), ("table_len_out", table_len_out, B), ("row_indptr", row_indptr, B + 1), ("page_indptr", page_indptr, B + 1),
             ("free_count", free_count, 1), ("free_count_out", free_count_out, 1)]
    for name, t, n in sizes:
        if t is not None and t.numel() != n:
            raise TypeError(f"{name} must have {n} entries")
    if slot_map is not None and (slot_map.dtype != torch.int64 or not slot_map.is_contiguous()):
        raise TypeError("slot_map must be a contiguous int64 tensor")
    rows = [t.numel() for t in (positions, slot_map) if t is not None]
    a = fd_table_args()
    a.device = _one_device(kv_len, verify_len, block_table, table_len, free_pages, free_count, mask_rows, mask_vis, mask_blocks, row_indptr, page_indptr,
                           page_indices, positions, slot_map, table_len_out, free_count_out, status)
    a.batch = B; a.page_size = int(page_size); a.table_stride = block_table.shape[1]
    # without positions and slots there is nothing to bound the rows by but the call's own limit
    a.total_rows = min(rows) if rows else 1 << 20
    a.page_indices_len = page_indices.numel(); a.free_pages_len = free_pages.numel()
    a.kv_len = _i32(kv_len, "kv_len").data_ptr(); a.verify_len = _i32(verify_len, "verify_len").data_ptr()
    a.mask_rows = _opt_i32(mask_rows, "mask_rows"); a.mask_vis = _opt_i32(mask_vis, "mask_vis")
    a.mask_blocks = _opt_i32(mask_blocks, "mask_blocks")
    a.block_table = _i32(block_table, "block_table").data_ptr()
    a.table_len = _i32(table_len, "table_len").data_ptr()
    a.table_len_out = _i32(table_len if table_len_out is None else table_len_out, "table_len_out").data_ptr()
    a.free_pages = _i32(free_pages, "free_pages").data_ptr(); a.free_count = _i32(free_count, "free_count").data_ptr()
    a.free_count_out = _i32(free_count if free_count_out is None else free_count_out, "free_count_out").data_ptr()
    a.row_indptr = _i32(row_indptr, "row_indptr").data_ptr(); a.page_indptr = _i32(page_indptr, "page_indptr").data_ptr()
    a.page_indices = _i32(page_indices, "page_indices").data_ptr()
    a.positions = _opt_i32(positions, "positions"); a.slot_map = _ptr(slot_map)
    a.status = None if status is None else status.data_ptr()
    return a


def fd_step_tables(args: fd_table_args, stream=None) -> None:
    """Pages of a step change hands, then its row offsets, page lists, positions and slots are written."""
    _launchable(args.device)
    _check(load().fd_step_tables(C.byref(args), _stream(stream)))


def fd_qk_norm_rope(q, k, q_out, k_out, positions, inv_freq, *, q_weight=None, k_weight=None, v=None, v_out=None, eps: float = 1e-6,
                    interleaved: bool = False, stream=None) -> None:
    """q [R, Hq, D], k (and v) [R, Hkv, D]: any strides between rows and heads; outputs dense.  rotary_dim is twice the number of
    inv_freq's entries (None: no rotation)."""
    shape = q.shape
    R, Hq, D = shape
    kshape, dt, device = k.shape, q.dtype, q.get_device()
    Hkv = kshape[1]
    qs, ks = q.stride(), k.stride()
    vs = (0, 0, 1) if v is None else v.stride()
    if not (kshape == k_out.shape == (R, Hkv, D) and q_out.shape == shape and k.dtype is dt and q_out.dtype is dt and k_out.dtype is dt):
        raise TypeError(f"q, q_out must be [{R}, {Hq}, {D}] and k, k_out [{R}, {Hkv}, {D}], all of {dt}")
    if (qs[2] != 1 and R * Hq) or (ks[2] != 1 and R * Hkv) or (vs[2] != 1 and R * Hkv):
        raise TypeError("q, k and v need a contiguous last dimension")
    if not (q_out.is_contiguous() and k_out.is_contiguous()):
        raise TypeError("q_out and k_out must be contiguous")
    one = k.get_device() == q_out.get_device() == k_out.get_device() == device
    if v is not None:
        if not (v_out is not None and v.shape == v_out.shape == kshape and v.dtype is dt and v_out.dtype is dt and v_out.is_contiguous()):
            raise TypeError(f"v and v_out must be [{R}, {Hkv}, {D}] of {dt}, v_out contiguous")
        one = one and v.get_device() == v_out.get_device() == device
    if q_weight is not None:
        if q_weight.numel() != D or q_weight.dtype is not dt or not q_weight.is_contiguous():
            raise TypeError(f"q_weight must be {D} contiguous elements of {dt}")
        one = one and q_weight.get_device() == device
    if k_weight is not None:
        if k_weight.numel() != D or k_weight.dtype is not dt or not k_weight.is_contiguous():
            raise TypeError(f"k_weight must be {D} contiguous elements of {dt}")
        one = one and k_weight.get_device() == device
    half = 0
    if inv_freq is not None:
        half = inv_freq.numel()
        if inv_freq.dtype is not torch.float32 or not inv_freq.is_contiguous():
            raise TypeError("inv_freq must be contiguous float32")
        one = one and inv_freq.get_device() == device
        if half:
            if positions is None or positions.numel() != R:
                raise TypeError(f"positions must have {R} entries")
            one = one and positions.get_device() == device
    if not one:
        raise TypeError("the tensors are on different devices")
    _launchable(device)
    a = fd_rope_args(R, Hq, Hkv, D, 2 * half, 1 if interleaved else 0, _dtype_code(q), eps, q.data_ptr(), k.data_ptr(), _ptr(v), qs[0], qs[1], ks[0], ks[1],
                     vs[0], vs[1], q_out.data_ptr(), k_out.data_ptr(), _ptr(v_out), _ptr(q_weight), _ptr(k_weight), _ptr(inv_freq),
                     _i32(positions, "positions").data_ptr() if half else None)
    _check(load().fd_qk_norm_rope(C.byref(a), _stream(stream)))


class Q4Cache:
    """The four tensors of a cache held in 4 bits (fd_q4_cache has the layout) and the struct over them."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        P, H, ps, half = k_codes.shape
        D = 2 * half
        want = (("k_codes", k_codes, (P, H, ps, D // 2), torch.uint8), ("k_scales", k_scales, (P, H, ps, D // 32), torch.uint8),
                ("v_codes", v_codes, (P, H, ps // 16, 8 * D), torch.uint8), ("v_scales", v_scales, (P, H, ps), torch.bfloat16))
        for name, t, shape, dtype in want:
            if tuple(t.shape) != shape or t.dtype != dtype:
                raise TypeError(f"{name} must be {dtype} of shape {shape}")
            block = 1
            for n, st in zip(reversed(shape[2:]), reversed(t.stride()[2:])):
                if n > 1 and st != block:
                    raise TypeError(f"{name}: the block of a page and head must be contiguous")
                block *= n
            if t.numel() and (t.stride(0) % block or t.stride(1) % block or (t.stride(0) // block, t.stride(1) // block) !=
                              (k_codes.stride(0) // (ps * half), k_codes.stride(1) // (ps * half))):
                raise TypeError(f"{name}: pages and heads must lie as those of k_codes do, in blocks")
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales
        self.num_pages, self.num_kv_heads, self.page_size, self.head_dim = P, H, ps, D
        self.device = _one_device(k_codes, k_scales, v_codes, v_scales)
        self.c = fd_q4_cache(k_codes.data_ptr(), k_scales.data_ptr(), v_codes.data_ptr(), v_scales.data_ptr(),
                             k_codes.stride(0) // max(1, ps * half), k_codes.stride(1) // max(1, ps * half))


def alloc_q4_cache(num_pages: int, num_kv_heads: int, page_size: int, head_dim: int, device="cuda") -> Q4Cache:
    """A cache in 4 bits whose slots hold zeros."""
    z = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device=device)  # noqa: E731
    return Q4Cache(z(num_pages, num_kv_heads, page_size, head_dim // 2), z(num_pages, num_kv_heads, page_size, head_dim // 32),
                   z(num_pages, num_kv_heads, page_size // 16, 8 * head_dim),
                   torch.zeros(num_pages, num_kv_heads, page_size, dtype=torch.bfloat16, device=device))


def make_attn_args_q4(q, k_new, v_new, cache: Q4Cache, page_indptr, page_indices, kv_len, row_indptr, verify_len, mask_vis=None,
                      mask_blocks=None, *, out, lse=None, max_kv_len: int, max_new_rows: int, sm_scale: float = 0.0, flags: int = 0,
                      kv_chunk: int = 0, workspace=None, status=None):
    """make_attn_args for a cache in 4 bits: fd_verify_draft_attn_q4 and fd_append_kv_q4 take the cache beside the struct."""
    if cache.num_kv_heads != k_new.shape[1] or cache.head_dim != q.shape[2]:
        raise TypeError("the cache's heads or head dim are not those of the rows")
    R, B = q.shape[0], kv_len.shape[0]
    for name, t, shape in (("k_new", k_new, (R, cache.num_kv_heads, cache.head_dim)), ("v_new", v_new, k_new.shape), ("out", out, q.shape)):
        if t.shape != shape or t.dtype != q.dtype:
            raise TypeError(f"{name} must be {tuple(shape)} of {q.dtype}")
    if lse is not None and not (lse.shape == q.shape[:2] and lse.dtype == torch.float32 and lse.is_contiguous()):
        raise TypeError(f"lse must be {tuple(q.shape[:2])} of float32")
    for name, t, n in (("page_indptr", page_indptr, B + 1), ("row_indptr", row_indptr, B + 1), ("verify_len", verify_len, B), ("mask_vis", mask_vis, B),
                       ("mask_blocks", mask_blocks, B)):
        if t is not None and t.numel() != n:
            raise TypeError(f"{name} must have {n} entries")
    a = make_attn_args(q, k_new, v_new, cache.k_codes, cache.k_codes, page_indptr, page_indices, kv_len, row_indptr, verify_len, mask_vis,
                       mask_blocks, out=out, lse=lse, max_kv_len=max_kv_len, max_new_rows=max_new_rows, sm_scale=sm_scale, flags=flags,
                       kv_chunk=kv_chunk, workspace=workspace, status=status)
    a.device = _one_device(cache.k_codes, q, k_new, v_new, page_indptr, page_indices, kv_len, row_indptr, verify_len, mask_vis, mask_blocks, out, lse,
                           workspace, status)
    a.cache = cache
    a.k_cache = a.v_cache = None
    a.cache_stride_page = a.cache_stride_head = a.cache_stride_token = 0
    return a


def fd_verify_draft_attn_q4_workspace(args: fd_attn_args) -> int:
    return int(load().fd_verify_draft_attn_q4_workspace(C.byref(args)))


def _fits(args: fd_attn_args, cache: Q4Cache) -> None:
    """The call was made for this cache, or for one like it."""
    if cache is args.cache:
        return _launchable(cache.device)
    if (args.num_kv_heads, args.head_dim, args.page_size) != (cache.num_kv_heads, cache.head_dim, cache.page_size) or args.num_pages > cache.num_pages:
        raise TypeError("the cache is not of the shape that the call was made for")
    if args.device != cache.device:
        raise TypeError("the cache is on another device than the call's tensors")
    _launchable(cache.device)


def fd_verify_draft_attn_q4(args: fd_attn_args, cache: Q4Cache, stream=None) -> None:
    """Enqueue the attention call described by `args` (make_attn_args_q4) over the 4-bit `cache`."""
    _fits(args, cache)
    _check(load().fd_verify_draft_attn_q4(C.byref(args), C.byref(cache.c), _stream(stream)))


def fd_append_kv_q4(args: fd_attn_args, cache: Q4Cache, accept_len, kv_len_out, stream=None) -> None:
    """Round and commit new rows 0 .. accept_len[i] of the call described by `args` (make_attn_args_q4) to the 4-bit `cache`."""
    _fits(args, cache)
    B = args.batch
    if accept_len.numel() != B or kv_len_out.numel() != B:
        raise TypeError(f"accept_len and kv_len_out must have {B} entries")
    if not accept_len.get_device() == kv_len_out.get_device() == args.device:
        raise TypeError("accept_len and kv_len_out are on another device than the call's tensors")
    _check(load().fd_append_kv_q4(C.byref(args), C.byref(cache.c), _i32(accept_len, "accept_len").data_ptr(),
                                  _i32(kv_len_out, "kv_len_out").data_ptr(), _stream(stream)))


def fd_read_kv_q4(cache: Q4Cache, page_indptr, page_indices, start, out_indptr, k_out, v_out, *, status=None, stream=None) -> None:
    """Tokens start[i] .. of every sequence as rows out_indptr[i] .. of k_out / v_out [R, Hkv, D], float32 or bfloat16."""
    shape, dt, device = k_out.shape, k_out.dtype, cache.device
    if not (shape == v_out.shape and shape[1:] == (cache.num_kv_heads, cache.head_dim) and v_out.dtype is dt and k_out.is_contiguous() and
            v_out.is_contiguous()):
        raise TypeError(f"k_out and v_out must be contiguous, [rows, {cache.num_kv_heads}, {cache.head_dim}], both of one dtype")
    B = out_indptr.numel() - 1
    if B < 0 or page_indptr.numel() != B + 1 or (start is not None and start.numel() != B):
        raise TypeError("out_indptr and page_indptr must have one entry more than there are sequences, start one each")
    if not k_out.get_device() == v_out.get_device() == page_indptr.get_device() == page_indices.get_device() == out_indptr.get_device() == device or \
            (start is not None and start.get_device() != device) or (status is not None and status.get_device() != device):
        raise TypeError("the tensors are on different devices")
    _launchable(device)
    _check(load().fd_read_kv_q4(
        C.byref(cache.c), B, cache.num_kv_heads, cache.head_dim, cache.page_size, cache.num_pages,
        _i32(page_indptr, "page_indptr").data_ptr(), _i32(page_indices, "page_indices").data_ptr(), page_indices.numel(), _opt_i32(start, "start"),
        _i32(out_indptr, "out_indptr").data_ptr(), shape[0], k_out.data_ptr(), v_out.data_ptr(), _dtype_code(k_out), _ptr(status), _stream(stream)))


def fd_version() -> str:
    return load().fd_version().decode()


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """256-byte aligned device buffer of at least nbytes (torch allocations are 256-byte aligned)."""
    return torch.empty(max(256, (nbytes + 255) // 256 * 256), dtype=torch.uint8, device=device)
