"""ctypes binding of libpagedattn.so, the C ABI declared in include/pagedattn.h
and, for the caches held in 4 and in 8 bits and for rotary positions,
include/pagedattn_q4.h, include/pagedattn_q8.h and include/pa_rope.h.

Argument marshalling only: every step of the attention runs in the library's
HIP kernels.  Device buffers are passed as torch tensors (torch provides
device memory and streams here) or as raw integer device addresses.  The
library is loaded on first use; if it has not been built the call raises
instead of falling back to anything else.
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
# PAGEDATTN_LIB selects another build of the same library (e.g. one compiled
# with different tuning macros); default: the in-tree build.
LIB_PATH = os.environ.get("PAGEDATTN_LIB") or os.path.join(HERE, "_lib", "libpagedattn.so")

PA_OK, PA_EINVAL, PA_ENOTSUP, PA_ENOSPC, PA_EHIP = 0, -1, -2, -3, -4
PA_BF16, PA_FP32 = 0, 1
PAGE_SIZE = 16

EXPORTED = ("pa_workspace_size", "paged_attn", "paged_attn_varlen", "paged_attn_varlen_noalloc",
            "pa_gather_trace",
            "pa_kv_append", "pa_schedule_step", "pa_perf_model", "pa_read_probe", "pa_issue_probe",
            "pa_strerror",
            "pa_q4_tile_bytes", "pa_kv_append_q4", "pa_kv_read_q4", "pa_workspace_size_q4", "paged_attn_q4",
            "paged_attn_varlen_q4", "pa_kv_append_q8", "pa_kv_read_q8", "pa_workspace_size_q8", "paged_attn_q8",
            "paged_attn_varlen_q8", "pa_rope", "pa_rope_frequencies")


class PaDims(ctypes.Structure):
    """pa_dims_t"""
    _fields_ = [(n, ctypes.c_int32) for n in (
        "num_seqs", "num_q_heads", "num_kv_heads", "head_dim", "page_size", "num_pages",
        "max_pages_per_seq", "max_context_len", "pages_per_split", "dtype", "num_q_rows",
        "max_q_len")]


class PaTiming(ctypes.Structure):
    """pa_timing_t: three hipEvent_t handles (NULL = not recorded)."""
    _fields_ = [("attn_begin", ctypes.c_void_p), ("attn_end", ctypes.c_void_p),
                ("reduce_end", ctypes.c_void_p)]


SCHED_ARRAYS = ("free_pages", "hdr", "queue_seq", "queue_tok", "queue_fin", "slot_seq",
                "slot_order", "slot_fin", "context_lens", "block_table")


class PaSchedState(ctypes.Structure):
    """pa_sched_state_t: ten device array pointers, then four sizes."""
    _fields_ = [(n, ctypes.c_void_p) for n in SCHED_ARRAYS] + [
        (n, ctypes.c_int32) for n in ("num_slots", "num_pages", "max_pages_per_seq", "queue_cap")]


def make_sched_state(arrays) -> PaSchedState:
    """pa_sched_state_t from a mapping of the ten int32 device arrays (torch
    tensors or addresses); the sizes come from their shapes."""
    bt = arrays["block_table"]
    st = PaSchedState(**{n: _addr(arrays[n]) for n in SCHED_ARRAYS})
    st.num_slots, st.max_pages_per_seq = int(bt.shape[0]), int(bt.shape[1])
    st.num_pages = int(arrays["free_pages"].shape[0])
    st.queue_cap = int(arrays["queue_seq"].shape[0])
    return st


PM_INPUT_DOUBLES = ("num_experts", "top_k", "model_dim", "expert_dim", "gqa_group", "model_bytes",
                    "kv_bytes_per_token", "gemm_flops", "io_bw", "kv_capacity_bytes", "attn_bw",
                    "attn_intensity", "batch")
PM_INPUT_INTS = ("prompt", "gen", "block")
PM_OUTPUTS = ("intensity_per_token", "tokens_to_saturate", "pme", "delta", "kv_tokens", "t_gpu",
              "t_max", "mem_bw", "kv_bw", "attn_flops", "kv_effective", "kv_blocks", "q",
              "decode_seqs", "t1", "t_prefill", "iterations", "t2", "t", "attn_headroom",
              "delta_eff", "t_attn_bound")


class PaPmInput(ctypes.Structure):
    """pa_pm_input_t (include/pa_perf_model.h)"""
    _fields_ = [(n, ctypes.c_double) for n in PM_INPUT_DOUBLES] + [(n, ctypes.c_int32) for n in PM_INPUT_INTS]


class PaPmOutput(ctypes.Structure):
    """pa_pm_output_t"""
    _fields_ = [(n, ctypes.c_double) for n in PM_OUTPUTS]


class PaRope(ctypes.Structure):
    """pa_rope_t (include/pa_rope.h)"""
    _fields_ = [("inv_freq", ctypes.c_void_p), ("factor", ctypes.c_float), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("q_out_stride", ctypes.c_int64), ("k_out_stride", ctypes.c_int64)]


ROPE_KINDS = ("plain", "linear", "base", "turns", "pairs")


class PaRopeScaling(ctypes.Structure):
    """pa_rope_scaling_t"""
    _fields_ = [("kind", ctypes.c_int32), ("rot_dim", ctypes.c_int32)] + [(n, ctypes.c_double) for n in (
        "base", "stretch", "trained_context", "low_turns", "high_turns")]


class PagedAttnError(RuntimeError):
    def __init__(self, fn, code):
        super().__init__(f"{fn} returned {code}: {pa_strerror(code)}")
        self.code = code


_lib = None


def load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                           "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    P, SZ = ctypes.c_void_p, ctypes.c_size_t
    DP, TP = ctypes.POINTER(PaDims), ctypes.POINTER(PaTiming)
    lib.pa_workspace_size.argtypes = [DP, ctypes.POINTER(SZ)]
    lib.pa_workspace_size.restype = ctypes.c_int
    lib.paged_attn.argtypes = [P, P, P, P, P, ctypes.c_float, P, DP, P, SZ, P, TP]
    lib.paged_attn.restype = ctypes.c_int
    lib.paged_attn_varlen.argtypes = [P, P, P, P, P, P, ctypes.c_float, P, DP, P, SZ, P, TP]
    lib.paged_attn_varlen.restype = ctypes.c_int
    lib.paged_attn_varlen_noalloc.argtypes = [P, P, P, P, P, P, ctypes.c_float, P, DP, P, TP]
    lib.paged_attn_varlen_noalloc.restype = ctypes.c_int
    lib.pa_gather_trace.argtypes = [P, P, P, P, P, P, ctypes.c_float, P, DP, P, SZ, P, P]
    lib.pa_gather_trace.restype = ctypes.c_int
    lib.pa_kv_append.argtypes = [P, P, P, P, P, P, P, DP, P]
    lib.pa_kv_append.restype = ctypes.c_int
    lib.pa_schedule_step.argtypes = [ctypes.POINTER(PaSchedState), ctypes.c_int32, P, P, P,
                                     ctypes.c_int32, P, P, P, P]
    lib.pa_schedule_step.restype = ctypes.c_int
    lib.pa_perf_model.argtypes = [ctypes.POINTER(PaPmInput), ctypes.POINTER(PaPmOutput)]
    lib.pa_perf_model.restype = ctypes.c_int
    lib.pa_read_probe.argtypes = [P, ctypes.c_int64, P, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                  ctypes.c_int32, P, P]
    lib.pa_read_probe.restype = ctypes.c_int
    lib.pa_issue_probe.argtypes = [ctypes.c_int32] * 7 + [P, P, P]
    lib.pa_issue_probe.restype = ctypes.c_int
    lib.pa_strerror.argtypes = [ctypes.c_int]
    lib.pa_strerror.restype = ctypes.c_char_p
    lib.pa_q4_tile_bytes.argtypes = [ctypes.c_int32, ctypes.POINTER(SZ)]
    lib.pa_kv_append_q4.argtypes = [P, P, P, P, P, P, P, DP, P]
    lib.pa_kv_read_q4.argtypes = [P, P, P, P, P, P, P, DP, P]
    lib.pa_workspace_size_q4.argtypes = [DP, ctypes.POINTER(SZ)]
    lib.paged_attn_q4.argtypes = [P, P, P, P, P, ctypes.c_float, P, DP, P, SZ, P, TP]
    lib.paged_attn_varlen_q4.argtypes = [P, P, P, P, P, P, ctypes.c_float, P, DP, P, SZ, P, TP]
    lib.pa_kv_append_q8.argtypes = [P, P, P, P, P, P, P, P, DP, P]
    lib.pa_kv_read_q8.argtypes = [P, P, P, P, P, P, P, P, DP, P]
    lib.pa_rope.argtypes = [P, P, P, P, P, P, P, ctypes.POINTER(PaRope), DP, P]
    lib.pa_rope.restype = ctypes.c_int
    lib.pa_rope_frequencies.argtypes = [ctypes.POINTER(PaRopeScaling), ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_float)]
    lib.pa_rope_frequencies.restype = ctypes.c_int
    lib.pa_workspace_size_q8.argtypes = [DP, ctypes.POINTER(SZ)]
    lib.paged_attn_q8.argtypes = [P, P, P, P, P, P, ctypes.c_float, P, DP, P, SZ, P, TP]
    lib.paged_attn_varlen_q8.argtypes = [P, P, P, P, P, P, P, ctypes.c_float, P, DP, P, SZ, P, TP]
    for name in ("pa_q4_tile_bytes", "pa_kv_append_q4", "pa_kv_read_q4", "pa_workspace_size_q4", "paged_attn_q4",
                 "paged_attn_varlen_q4", "pa_kv_append_q8", "pa_kv_read_q8", "pa_workspace_size_q8", "paged_attn_q8",
                 "paged_attn_varlen_q8"):
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _addr(x):
    """Device address of a torch tensor, an int address, or None (NULL)."""
    if x is None:
        return None
    if isinstance(x, int):
        return x or None
    return x.data_ptr() or None


def _stream(stream, device=None):
    """Handle of a stream; None: the current one (device: the current device, if known)."""
    if stream is None:
        import torch
        # The current stream's handle without a Stream object around it, which takes 3 us,
        # where torch has this function (it is not among its documented ones).
        handle = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if handle is None:
            return torch.cuda.current_stream().cuda_stream or None
        return handle(torch.cuda.current_device() if device is None else device) or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _dtype_code(t):
    import torch
    if t.dtype == torch.bfloat16:
        return PA_BF16
    if t.dtype == torch.float32:
        return PA_FP32
    raise TypeError(f"unsupported dtype {t.dtype}")


def make_dims(q, k_pages, block_table, max_context_len, pages_per_split=0, num_q_rows=0,
              max_q_len=0, num_seqs=None) -> PaDims:
    """pa_dims_t from tensor shapes: q [rows][H_q][D], k_pages [N][H_kv][16][D],
    block_table [B][max_pages_per_seq]."""
    rows, H_q, D = q.shape
    N, H_kv, P, D2 = k_pages.shape
    B = block_table.shape[0] if num_seqs is None else num_seqs
    return PaDims(num_seqs=B, num_q_heads=H_q, num_kv_heads=H_kv, head_dim=D, page_size=P,
                  num_pages=N, max_pages_per_seq=block_table.shape[1],
                  max_context_len=int(max_context_len), pages_per_split=int(pages_per_split),
                  dtype=_dtype_code(q), num_q_rows=int(num_q_rows), max_q_len=int(max_q_len))


def pa_workspace_size(dims: PaDims) -> int:
    n = ctypes.c_size_t(0)
    rc = load().pa_workspace_size(ctypes.byref(dims), ctypes.byref(n))
    if rc != PA_OK:
        raise PagedAttnError("pa_workspace_size", rc)
    return int(n.value)


def pa_strerror(code: int) -> str:
    return load().pa_strerror(int(code)).decode()


def _workspace(dims, workspace, device, stream=None, size_of=pa_workspace_size):
    """The caller's workspace, or a temporary one of pa_workspace_size()
    bytes (size_of: of another call's size) on the device (None, of arrays given as
    addresses: the current GPU).  A temporary is allocated on torch's current stream;
    when the call runs on another stream, the allocation is also recorded on that
    stream, so torch's caching allocator does not hand the memory to other work before
    the call's kernels have finished with it."""
    need = size_of(dims)
    if workspace is None and need > 0:
        import torch
        if isinstance(stream, int) and stream:
            # torch cannot track work on a raw stream handle
            raise ValueError("pass a workspace (or a torch stream) when calling on a raw stream handle")
        workspace = torch.empty(need, dtype=torch.uint8, device="cuda" if device is None else device)
        if stream is not None and stream != torch.cuda.current_stream(workspace.device):
            workspace.record_stream(stream)
    size = 0 if workspace is None else (workspace.numel() * workspace.element_size()
                                        if hasattr(workspace, "numel") else need)
    return workspace, size


def paged_attn(q, k_pages, v_pages, block_table, context_lens, scale, out, dims: PaDims,
               workspace=None, stream=None, timing: PaTiming | None = None, check=True) -> int:
    """int paged_attn(...): decode attention; out is written in place."""
    ws, ws_bytes = _workspace(dims, workspace, getattr(q, "device", None), stream)
    rc = load().paged_attn(_addr(q), _addr(k_pages), _addr(v_pages), _addr(block_table),
                           _addr(context_lens), float(scale), _addr(out), ctypes.byref(dims),
                           _addr(ws), ws_bytes, _stream(stream),
                           ctypes.byref(timing) if timing is not None else None)
    if check and rc != PA_OK:
        raise PagedAttnError("paged_attn", rc)
    return rc


def paged_attn_varlen(q, k_pages, v_pages, block_table, context_lens, query_start_loc, scale, out,
                      dims: PaDims, workspace=None, stream=None, timing: PaTiming | None = None,
                      check=True) -> int:
    """int paged_attn_varlen(...): causal prefill chunks plus decode rows."""
    ws, ws_bytes = _workspace(dims, workspace, getattr(q, "device", None), stream)
    rc = load().paged_attn_varlen(_addr(q), _addr(k_pages), _addr(v_pages), _addr(block_table),
                                  _addr(context_lens), _addr(query_start_loc), float(scale),
                                  _addr(out), ctypes.byref(dims), _addr(ws), ws_bytes,
                                  _stream(stream),
                                  ctypes.byref(timing) if timing is not None else None)
    if check and rc != PA_OK:
        raise PagedAttnError("paged_attn_varlen", rc)
    return rc


def paged_attn_varlen_noalloc(q, k_pages, v_pages, block_table, context_lens, query_start_loc, scale, out,
                              dims: PaDims, stream=None, timing: PaTiming | None = None, check=True) -> int:
    """int paged_attn_varlen_noalloc(...): paged_attn_varlen with the library's
    fixed device scratch in place of a workspace (allocates nothing)."""
    rc = load().paged_attn_varlen_noalloc(_addr(q), _addr(k_pages), _addr(v_pages), _addr(block_table),
                                          _addr(context_lens), _addr(query_start_loc), float(scale),
                                          _addr(out), ctypes.byref(dims), _stream(stream),
                                          ctypes.byref(timing) if timing is not None else None)
    if check and rc != PA_OK:
        raise PagedAttnError("paged_attn_varlen_noalloc", rc)
    return rc


def pa_gather_trace(q, k_pages, v_pages, block_table, context_lens, scale, out, dims: PaDims,
                    rows_out, query_start_loc=None, workspace=None, stream=None, check=True) -> int:
    """int pa_gather_trace(...): the attention call (decode, or varlen when
    query_start_loc is given) through the kernels' trace instantiations;
    rows_out [H_kv][B][max_pages_per_seq * 16] int64 receives the pool row of
    every loaded token."""
    ws, ws_bytes = _workspace(dims, workspace, getattr(q, "device", None), stream)
    rc = load().pa_gather_trace(_addr(q), _addr(k_pages), _addr(v_pages), _addr(block_table),
                                _addr(context_lens), _addr(query_start_loc), float(scale),
                                _addr(out), ctypes.byref(dims), _addr(ws), ws_bytes,
                                _addr(rows_out), _stream(stream))
    if check and rc != PA_OK:
        raise PagedAttnError("pa_gather_trace", rc)
    return rc


def pa_kv_append(k_new, v_new, block_table, context_lens, k_pages, v_pages, dims: PaDims,
                 query_start_loc=None, stream=None, check=True) -> int:
    """int pa_kv_append(...): store the new tokens' K/V into the paged pools."""
    rc = load().pa_kv_append(_addr(k_new), _addr(v_new), _addr(block_table), _addr(context_lens),
                             _addr(query_start_loc), _addr(k_pages), _addr(v_pages),
                             ctypes.byref(dims), _stream(stream))
    if check and rc != PA_OK:
        raise PagedAttnError("pa_kv_append", rc)
    return rc


def pa_q4_tile_bytes(head_dim) -> int:
    """Bytes of a (page, KV head) tile of the 4-bit cache; a pool is uint8
    [num_pages][num_kv_heads][pa_q4_tile_bytes(head_dim)]."""
    n = ctypes.c_size_t(0)
    rc = load().pa_q4_tile_bytes(int(head_dim), ctypes.byref(n))
    if rc != PA_OK:
        raise PagedAttnError("pa_q4_tile_bytes", rc)
    return int(n.value)


_Q4_TILE = {64: 544, 128: 1088}  # pa_q4_tile_bytes (checked against it by the tests)
_Q8_TILE = {64: 1024, 128: 2048}


def make_dims_q4(rows, k_pages, block_table, max_context_len, num_q_rows=0, max_q_len=0, num_seqs=None) -> PaDims:
    """pa_dims_t of a call on the 4-bit cache from tensor shapes: rows
    [rows][H][D] (q, or k_new / k_out of the append and the read), k_pages uint8
    [N][H_kv][tile], block_table [B][max_pages_per_seq]."""
    _, H, D = rows.shape
    N, H_kv, tile = k_pages.shape
    B, width = block_table.shape
    if _Q4_TILE.get(D) != tile:
        raise ValueError(f"k_pages holds tiles of {tile} bytes, head_dim {D} takes {pa_q4_tile_bytes(D)}")
    return PaDims(B if num_seqs is None else num_seqs, H, H_kv, D, PAGE_SIZE, N, width, int(max_context_len), 0,
                  _dtype_code(rows), int(num_q_rows), int(max_q_len))


def pa_workspace_size_q4(dims: PaDims) -> int:
    n = ctypes.c_size_t(0)
    rc = load().pa_workspace_size_q4(ctypes.byref(dims), ctypes.byref(n))
    if rc != PA_OK:
        raise PagedAttnError("pa_workspace_size_q4", rc)
    return int(n.value)


def _is_address(t):
    return t is None or t.__class__ is int


def _take(t, kind, n, device):
    """Device address of a tensor of a call on a cache in few bits.  (Addresses are taken
    as they are.)"""
    if t is None:
        return None
    if t.__class__ is int:
        return t or None
    if t.dtype is not kind:
        raise TypeError(f"a tensor of {t.dtype} where {kind} is needed")
    if t.get_device() != device:
        raise ValueError(f"a tensor on {t.device}, not on the current device")
    if t.numel() < n or not t.is_contiguous():
        raise ValueError(f"a tensor of {t.numel()} elements{'' if t.is_contiguous() else ', not contiguous'}, "
                         f"where {n} in a row are needed")
    return t.data_ptr() or None


def _fit_q(tile, dims, heads, dense0, dense1, k_pages, v_pages, block_table):
    """Refuses arrays whose rows are not those that dims say: read with their strides
    they would be other values.  (Addresses, and arrays of other ranks, are taken by
    their elements.)"""
    H_kv, D = dims.num_kv_heads, dims.head_dim
    if D not in tile:  # (the library's to refuse)
        return
    tiles = (H_kv, tile[D])
    for t, row in ((dense0, (heads, D)), (dense1, (heads, D)), (k_pages, tiles), (v_pages, tiles),
                   (block_table, (dims.max_pages_per_seq,))):
        if not _is_address(t) and t.dim() == len(row) + 1 and tuple(t.shape[1:]) != row:
            raise ValueError(f"a tensor of shape {tuple(t.shape)} where dims say rows of {row}")


def _take_q(tile, dims, heads, varlen, dense0, dense1, k_pages, v_pages, block_table, context_lens, query_start_loc):
    """The addresses of a call's arrays, in this order.  Refuses a tensor that is not
    what dims and the format say: of another type or too few elements, not contiguous,
    not on the current device."""
    import torch
    i32, u8 = torch.int32, torch.uint8
    # (addresses alone need no device)
    dev = None
    if not _is_address(dense0) or not all(map(_is_address, (dense1, k_pages, v_pages, block_table, context_lens, query_start_loc))):
        dev = torch.cuda.current_device()
    B, D = dims.num_seqs, dims.head_dim
    kind = torch.bfloat16 if dims.dtype == PA_BF16 else torch.float32
    n = (dims.num_q_rows if varlen else B) * heads * D
    tiles = dims.num_pages * dims.num_kv_heads * tile.get(D, 0)
    return (_take(dense0, kind, n, dev), _take(dense1, kind, n, dev), _take(k_pages, u8, tiles, dev),
            _take(v_pages, u8, tiles, dev), _take(block_table, i32, B * dims.max_pages_per_seq, dev),
            _take(context_lens, i32, B, dev), _take(query_start_loc, i32, B + 1, dev))


def _take_q4(dims, *arrays):
    return _take_q(_Q4_TILE, dims, *arrays)


def _scales_q8(dims, scales):
    """Address of the scales, uint8 [num_pages][num_kv_heads][2]."""
    if _is_address(scales):
        return scales or None
    import torch
    if scales.dim() == 3 and tuple(scales.shape[1:]) != (dims.num_kv_heads, 2):
        raise ValueError(f"scales of shape {tuple(scales.shape)} where dims say rows of {(dims.num_kv_heads, 2)}")
    return _take(scales, torch.uint8, dims.num_pages * dims.num_kv_heads * 2, torch.cuda.current_device())


def _args_q(tile, dims, heads, varlen, dense0, dense1, k_pages, v_pages, block_table, context_lens, query_start_loc, scales=None):
    """_take_q, checked by _fit_q, the scales' address (None: a cache without), and the
    current device if it was looked up.  The usual call, tensors of just the shapes that
    dims say, is checked in one pass (one by one the checks take 1.3 us more, 2 us with
    scales)."""
    try:
        d, k, w = dense0.shape, k_pages.shape, block_table.shape
        import torch
        i32, u8 = torch.int32, torch.uint8
        kind = torch.bfloat16 if dims.dtype == PA_BF16 else torch.float32
        dev = torch.cuda.current_device()
        B, H_kv, D = dims.num_seqs, dims.num_kv_heads, dims.head_dim
        if (d[1] == heads and d[2] == D and d[0] >= (dims.num_q_rows if varlen else B) and dense1.shape == d
                and k[1] == H_kv and k[2] == tile.get(D) and k[0] >= dims.num_pages and v_pages.shape == k
                and w[1] == dims.max_pages_per_seq and w[0] >= B and context_lens.numel() >= B
                and dense0.dtype is kind and dense1.dtype is kind and k_pages.dtype is u8 and v_pages.dtype is u8
                and block_table.dtype is i32 and context_lens.dtype is i32
                and dense0.get_device() == dev == dense1.get_device() and k_pages.get_device() == dev == v_pages.get_device()
                and block_table.get_device() == dev == context_lens.get_device()
                and dense0.is_contiguous() and dense1.is_contiguous() and k_pages.is_contiguous() and v_pages.is_contiguous()
                and block_table.is_contiguous() and context_lens.is_contiguous()
                and len(d) == 3 and len(k) == 3 and len(w) == 2
                and (scales is None or (scales.shape == (k[0], H_kv, 2) and scales.dtype is u8 and scales.get_device() == dev
                                        and scales.is_contiguous()))):
            return (dense0.data_ptr(), dense1.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), block_table.data_ptr(),
                    context_lens.data_ptr(), None if query_start_loc is None else _take(query_start_loc, i32, B + 1, dev),
                    None if scales is None else scales.data_ptr(), dev)
    except (AttributeError, IndexError):  # (addresses, other ranks)
        pass
    taken = _take_q(tile, dims, heads, varlen, dense0, dense1, k_pages, v_pages, block_table, context_lens, query_start_loc)
    _fit_q(tile, dims, heads, dense0, dense1, k_pages, v_pages, block_table)
    return *taken, _scales_q8(dims, scales), None


def _workspace_q(size_of, dims, workspace, q, stream):
    """(address, bytes, owner) of the caller's workspace or of a temporary one.  A
    tensor of another device than the current one, or not contiguous, is refused."""
    if workspace is None or workspace.__class__ is int:
        ws, size = _workspace(dims, workspace, getattr(q, "device", None), stream, size_of)
        return _addr(ws), size, ws
    if _is_address(q):
        import torch
        device = torch.cuda.current_device()
    else:  # (which is on the current device: _take)
        device = q.get_device()
    if workspace.get_device() != device:
        raise ValueError(f"a workspace on {workspace.device}, not on the current device")
    if not workspace.is_contiguous():
        raise ValueError("a workspace that is not contiguous")
    return workspace.data_ptr() or None, workspace.numel() * workspace.element_size(), workspace


def pa_kv_append_q4(k_new, v_new, block_table, context_lens, k_pages, v_pages, dims: PaDims, query_start_loc=None,
                    stream=None, check=True) -> int:
    """int pa_kv_append_q4(...): quantise the new tokens' K/V into the 4-bit pools."""
    k, v, kp, vp, bt, cl, qsl, _, dev = _args_q(_Q4_TILE, dims, dims.num_kv_heads, query_start_loc is not None, k_new, v_new, k_pages,
                                              v_pages, block_table, context_lens, query_start_loc)
    rc = load().pa_kv_append_q4(k, v, bt, cl, qsl, kp, vp, ctypes.byref(dims), _stream(stream, dev))
    if check and rc != PA_OK:
        raise PagedAttnError("pa_kv_append_q4", rc)
    return rc


def pa_kv_read_q4(k_pages, v_pages, block_table, context_lens, k_out, v_out, dims: PaDims, query_start_loc=None,
                  stream=None, check=True) -> int:
    """int pa_kv_read_q4(...): the values that the 4-bit pools hold of the rows
    which pa_kv_append_q4 with the same arguments writes."""
    k, v, kp, vp, bt, cl, qsl, _, dev = _args_q(_Q4_TILE, dims, dims.num_kv_heads, query_start_loc is not None, k_out, v_out, k_pages,
                                              v_pages, block_table, context_lens, query_start_loc)
    rc = load().pa_kv_read_q4(kp, vp, bt, cl, qsl, k, v, ctypes.byref(dims), _stream(stream, dev))
    if check and rc != PA_OK:
        raise PagedAttnError("pa_kv_read_q4", rc)
    return rc


def paged_attn_q4(q, k_pages, v_pages, block_table, context_lens, scale, out, dims: PaDims, workspace=None,
                  stream=None, timing: PaTiming | None = None, check=True) -> int:
    """int paged_attn_q4(...): decode attention over the 4-bit cache; out is
    written in place."""
    qa, oa, kp, vp, bt, cl, _, _, dev = _args_q(_Q4_TILE, dims, dims.num_q_heads, False, q, out, k_pages, v_pages, block_table,
                                              context_lens, None)
    ws, ws_bytes, owner = _workspace_q(pa_workspace_size_q4, dims, workspace, q, stream)
    rc = load().paged_attn_q4(qa, kp, vp, bt, cl, scale, oa, ctypes.byref(dims), ws, ws_bytes, _stream(stream, dev),
                              ctypes.byref(timing) if timing is not None else None)
    if check and rc != PA_OK:
        raise PagedAttnError("paged_attn_q4", rc)
    return rc


def paged_attn_varlen_q4(q, k_pages, v_pages, block_table, context_lens, query_start_loc, scale, out, dims: PaDims,
                         workspace=None, stream=None, timing: PaTiming | None = None, check=True) -> int:
    """int paged_attn_varlen_q4(...): causal chunks plus decode rows over the
    4-bit cache."""
    qa, oa, kp, vp, bt, cl, qsl, _, dev = _args_q(_Q4_TILE, dims, dims.num_q_heads, True, q, out, k_pages, v_pages, block_table,
                                                context_lens, query_start_loc)
    ws, ws_bytes, owner = _workspace_q(pa_workspace_size_q4, dims, workspace, q, stream)
    rc = load().paged_attn_varlen_q4(qa, kp, vp, bt, cl, qsl, scale, oa, ctypes.byref(dims), ws, ws_bytes,
                                     _stream(stream, dev), ctypes.byref(timing) if timing is not None else None)
    if check and rc != PA_OK:
        raise PagedAttnError("paged_attn_varlen_q4", rc)
    return rc


def make_dims_q8(rows, k_pages, block_table, max_context_len, num_q_rows=0, max_q_len=0, num_seqs=None) -> PaDims:
    """pa_dims_t of a call on the 8-bit cache from tensor shapes: rows
    [rows][H][D] (q, or k_new / k_out of the append and the read), k_pages uint8
    [N][H_kv][16 D], block_table [B][max_pages_per_seq]."""
    _, H, D = rows.shape
    N, H_kv, tile = k_pages.shape
    B, width = block_table.shape
    if PAGE_SIZE * D != tile:
        raise ValueError(f"k_pages holds tiles of {tile} bytes, head_dim {D} takes {PAGE_SIZE * D}")
    return PaDims(B if num_seqs is None else num_seqs, H, H_kv, D, PAGE_SIZE, N, width, int(max_context_len), 0,
                  _dtype_code(rows), int(num_q_rows), int(max_q_len))


def pa_kv_append_q8(k_new, v_new, block_table, context_lens, k_pages, v_pages, scales, dims: PaDims, query_start_loc=None,
                    stream=None, check=True) -> int:
    """int pa_kv_append_q8(...): quantise the new tokens' K/V into the 8-bit pools."""
    k, v, kp, vp, bt, cl, qsl, sc, dev = _args_q(_Q8_TILE, dims, dims.num_kv_heads, query_start_loc is not None, k_new, v_new,
                                             k_pages, v_pages, block_table, context_lens, query_start_loc, scales)
    rc = load().pa_kv_append_q8(k, v, bt, cl, qsl, kp, vp, sc, ctypes.byref(dims), _stream(stream, dev))
    if check and rc != PA_OK:
        raise PagedAttnError("pa_kv_append_q8", rc)
    return rc


def pa_kv_read_q8(k_pages, v_pages, scales, block_table, context_lens, k_out, v_out, dims: PaDims, query_start_loc=None,
                  stream=None, check=True) -> int:
    """int pa_kv_read_q8(...): the values that the 8-bit pools hold of the rows
    which pa_kv_append_q8 with the same arguments writes."""
    k, v, kp, vp, bt, cl, qsl, sc, dev = _args_q(_Q8_TILE, dims, dims.num_kv_heads, query_start_loc is not None, k_out, v_out,
                                             k_pages, v_pages, block_table, context_lens, query_start_loc, scales)
    rc = load().pa_kv_read_q8(kp, vp, sc, bt, cl, qsl, k, v, ctypes.byref(dims), _stream(stream, dev))
    if check and rc != PA_OK:
        raise PagedAttnError("pa_kv_read_q8", rc)
    return rc


def pa_workspace_size_q8(dims: PaDims) -> int:
    n = ctypes.c_size_t(0)
    rc = load().pa_workspace_size_q8(ctypes.byref(dims), ctypes.byref(n))
    if rc != PA_OK:
        raise PagedAttnError("pa_workspace_size_q8", rc)
    return int(n.value)


def paged_attn_q8(q, k_pages, v_pages, scales, block_table, context_lens, scale, out, dims: PaDims, workspace=None,
                  stream=None, timing: PaTiming | None = None, check=True) -> int:
    """int paged_attn_q8(...): decode attention over the 8-bit cache; out is
    written in place."""
    qa, oa, kp, vp, bt, cl, _, sc, dev = _args_q(_Q8_TILE, dims, dims.num_q_heads, False, q, out, k_pages, v_pages, block_table,
                                             context_lens, None, scales)
    ws, ws_bytes, owner = _workspace_q(pa_workspace_size_q8, dims, workspace, q, stream)
    rc = load().paged_attn_q8(qa, kp, vp, sc, bt, cl, scale, oa, ctypes.byref(dims), ws, ws_bytes,
                              _stream(stream, dev), ctypes.byref(timing) if timing is not None else None)
    if check and rc != PA_OK:
        raise PagedAttnError("paged_attn_q8", rc)
    return rc


def paged_attn_varlen_q8(q, k_pages, v_pages, scales, block_table, context_lens, query_start_loc, scale, out, dims: PaDims,
                         workspace=None, stream=None, timing: PaTiming | None = None, check=True) -> int:
    """int paged_attn_varlen_q8(...): causal chunks plus decode rows over the
    8-bit cache."""
    qa, oa, kp, vp, bt, cl, qsl, sc, dev = _args_q(_Q8_TILE, dims, dims.num_q_heads, True, q, out, k_pages, v_pages, block_table,
                                               context_lens, query_start_loc, scales)
    ws, ws_bytes, owner = _workspace_q(pa_workspace_size_q8, dims, workspace, q, stream)
    rc = load().paged_attn_varlen_q8(qa, kp, vp, sc, bt, cl, qsl, scale, oa, ctypes.byref(dims), ws,
                                     ws_bytes, _stream(stream, dev), ctypes.byref(timing) if timing is not None else None)
    if check and rc != PA_OK:
        raise PagedAttnError("paged_attn_varlen_q8", rc)
    return rc


def pa_rope_frequencies(rot_dim, base=10000.0, kind="plain", stretch=1.0, trained_context=4096, low_turns=1.0, high_turns=32.0):
    """(inv_freq, factor) of a call to pa_rope: a CPU tensor of rot_dim / 2 float64 (move it to
    the GPU), and the factor.  kind: one of ROPE_KINDS (include/pa_rope.h)."""
    import torch
    if kind not in ROPE_KINDS:
        raise ValueError(f"kind {kind!r} is none of {ROPE_KINDS}")
    c = PaRopeScaling(ROPE_KINDS.index(kind), int(rot_dim), float(base), float(stretch), float(trained_context), float(low_turns), float(high_turns))
    out, factor = torch.empty(max(0, int(rot_dim)) // 2, dtype=torch.float64), ctypes.c_float(0)
    rc = load().pa_rope_frequencies(ctypes.byref(c), ctypes.cast(out.data_ptr(), ctypes.POINTER(ctypes.c_double)), ctypes.byref(factor))
    if rc != PA_OK:
        raise PagedAttnError("pa_rope_frequencies", rc)
    return out, float(factor.value)


def make_dims_rope(q, k, max_context_len, num_q_rows=0, num_seqs=None) -> PaDims:
    """pa_dims_t of a pa_rope call from tensor shapes: q [rows][H_q][D], k
    [rows][H_kv][D], of which one may be None."""
    one = q if q is not None else k
    rows, _, D = one.shape
    return PaDims(num_seqs=rows if num_seqs is None else num_seqs, num_q_heads=0 if q is None else q.shape[1],
                  num_kv_heads=0 if k is None else k.shape[1], head_dim=D, page_size=PAGE_SIZE, max_context_len=int(max_context_len),
                  dtype=_dtype_code(one), num_q_rows=int(num_q_rows))


def _rows_rope(t, kind, rows, heads, D, device):
    """(address, row stride) of rows [rows][heads][D]; the rows may lie apart."""
    if t is None:
        return None, 0
    if t.__class__ is int:
        return t or None, 0
    if t.dtype is not kind:
        raise TypeError(f"a tensor of {t.dtype} where {kind} is needed")
    if t.get_device() != device:
        raise ValueError(f"a tensor on {t.device}, not on the current device")
    shape = t.shape
    if len(shape) != 3 or shape[0] < rows or shape[1] != heads or shape[2] != D:
        raise ValueError(f"a tensor of shape {tuple(shape)} where {(rows, heads, D)} is needed")
    if t.is_contiguous():
        return t.data_ptr() or None, 0
    strides = t.stride()
    if strides[2] != 1 or (heads > 1 and strides[1] != D):
        raise ValueError(f"a tensor of strides {strides}, whose rows' heads do not lie one after the other")
    if rows <= 1:  # (a lone row's stride is any number: none is used)
        return t.data_ptr() or None, 0
    # (0, as broadcast rows have it, means packed rows to the library)
    if strides[0] < heads * D:
        raise ValueError(f"rows {strides[0]} elements apart, of {heads * D} each")
    return t.data_ptr() or None, strides[0]


def pa_rope(q, k, context_lens, inv_freq, q_out, k_out, dims: PaDims, interleaved=False, factor=1.0, positions=None, query_start_loc=None,
            rot_dim=None, stream=None, check=True) -> int:
    """int pa_rope(...): rotary positions of q and k (either may be None, with its
    output); rot_dim is twice the length of inv_freq (float64) unless given.  Rows of tensors
    may lie apart (q and k as parts of a joint projection's rows)."""
    import torch
    # (addresses alone need no device)
    dev = None
    if not all(map(_is_address, (q, k, context_lens, inv_freq, q_out, k_out, positions, query_start_loc))):
        dev = torch.cuda.current_device()
    if rot_dim is None:
        rot_dim = 2 * inv_freq.numel()
    kind, D, i32 = torch.bfloat16 if dims.dtype == PA_BF16 else torch.float32, dims.head_dim, torch.int32
    if positions is not None:
        rows = dims.num_q_rows or dims.num_seqs
    else:
        rows = dims.num_seqs if query_start_loc is None else dims.num_q_rows
    H_q, H_kv = dims.num_q_heads, dims.num_kv_heads
    qa, qs = _rows_rope(q, kind, rows, H_q, D, dev)
    qo, qos = _rows_rope(q_out, kind, rows, H_q, D, dev)
    ka, ks = _rows_rope(k, kind, rows, H_kv, D, dev)
    ko, kos = _rows_rope(k_out, kind, rows, H_kv, D, dev)
    if positions is None:
        B = dims.num_seqs
        pos, cl = None, _take(context_lens, i32, B, dev)
        qsl = None if query_start_loc is None else _take(query_start_loc, i32, B + 1, dev)
    else:  # (the others are not read)
        pos, cl, qsl = _take(positions, i32, rows, dev), None, None
    rope = PaRope(_take(inv_freq, torch.float64, rot_dim // 2, dev), float(factor), int(rot_dim), 1 if interleaved else 0, qs, ks, qos, kos)
    rc = load().pa_rope(qa, ka, pos, cl, qsl, qo, ko, ctypes.byref(rope), ctypes.byref(dims), _stream(stream, dev))
    if check and rc != PA_OK:
        raise PagedAttnError("pa_rope", rc)
    return rc


def pa_schedule_step(state: PaSchedState, n_real, new_seq, new_prompt, new_fin, n_new,
                     query_start_loc, finished_out, info, stream=None, check=True) -> int:
    """int pa_schedule_step(...): one scheduler step on the device-resident state."""
    rc = load().pa_schedule_step(ctypes.byref(state), int(n_real), _addr(new_seq),
                                 _addr(new_prompt), _addr(new_fin), int(n_new),
                                 _addr(query_start_loc), _addr(finished_out), _addr(info),
                                 _stream(stream))
    if check and rc != PA_OK:
        raise PagedAttnError("pa_schedule_step", rc)
    return rc


def pa_read_probe(buf, chunk_bytes, chunk_offsets, n_chunks, grid, waves, depth, non_temporal, sink, stream=None,
                  check=True) -> int:
    """int pa_read_probe(...): read n_chunks chunks of buf with the decode
    kernels' load pattern (include/pa_probe.h)."""
    rc = load().pa_read_probe(_addr(buf), int(chunk_bytes), _addr(chunk_offsets), int(n_chunks), int(grid),
                              int(waves), int(depth), int(non_temporal), _addr(sink), _stream(stream))
    if check and rc != PA_OK:
        raise PagedAttnError("pa_read_probe", rc)
    return rc


def pa_issue_probe(grid, waves, iters, big_mfma, valu_per_mfma, exp2, mode, sink, cycles=None, stream=None,
                   check=True) -> int:
    """int pa_issue_probe(...): matrix products beside vector work
    (include/pa_probe.h); the caller times the launch."""
    rc = load().pa_issue_probe(int(grid), int(waves), int(iters), int(big_mfma), int(valu_per_mfma), int(exp2),
                               int(mode), _addr(sink), _addr(cycles), _stream(stream))
    if check and rc != PA_OK:
        raise PagedAttnError("pa_issue_probe", rc)
    return rc


def pa_perf_model(**inputs) -> dict:
    """int pa_perf_model(...): the Sec. 5 performance model for one
    configuration; keyword names are the pa_pm_input_t fields (missing ones
    are 0).  Returns the pa_pm_output_t fields as a dict."""
    unknown = set(inputs) - set(PM_INPUT_DOUBLES) - set(PM_INPUT_INTS)
    if unknown:
        raise TypeError(f"unknown inputs {sorted(unknown)}")
    x = PaPmInput(**inputs)
    o = PaPmOutput()
    rc = load().pa_perf_model(ctypes.byref(x), ctypes.byref(o))
    if rc != PA_OK:
        raise PagedAttnError("pa_perf_model", rc)
    return {n: getattr(o, n) for n in PM_OUTPUTS}
