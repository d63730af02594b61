"""Thin ctypes binding of the C ABI in ``include/hybridgen_attn.h``.

Only argument marshalling happens here: torch tensors supply device (or host) pointers and the
current CUDA stream; every step of the attention path runs inside the library's kernels.  There is
no fallback: if the library has not been built, or a call returns a non-zero status, an exception
is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libhybridgen_attn.so"
_lib = None

HG_OK, HG_ERR_INVALID_ARG, HG_ERR_UNSUPPORTED, HG_ERR_CUDA, HG_ERR_WORKSPACE = 0, 1, 2, 3, 4
HG_DTYPE_F16, HG_DTYPE_BF16 = 0, 1
HG_DEV_OK, HG_DEV_WAIT_TIMEOUT, HG_DEV_BAD_PAGE, HG_DEV_RANGE, HG_DEV_NO_PAGE = 0, 1, 2, 4, 8
HG_MAX_MERGE_SRC = 8
HG_MAX_GROUPS = 512
HG_FLAG_TEST_STALL = 1
HG_FLAG_SPARSE_EMPTY = 2
HG_FLAG_COUNTER_CLEAN = 4
HG_STATIC_SCRATCH_BYTES = 8 << 20
(HG_TUNE_NO_PERSISTENT, HG_TUNE_NO_DYNAMIC, HG_TUNE_NO_PDL, HG_TUNE_NO_MERGE_CLUSTER, HG_TUNE_NO_MERGE_ROWS,
 HG_TUNE_NO_GQA16, HG_TUNE_NO_HOST_DIRECT, HG_TUNE_NO_SPEC_PREFETCH) = 1, 2, 4, 8, 16, 32, 64, 128
HG_LOGITS_TUNE_WARP_MMA, HG_LOGITS_TUNE_TCGEN05 = 1, 2


class HgError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {hg_status_string(status)} (hg_status {status})")


class HgAttnDesc(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32),
        ("batch", C.c_int32),
        ("num_q_heads", C.c_int32),
        ("num_kv_heads", C.c_int32),
        ("head_dim", C.c_int32),
        ("dtype", C.c_int32),
        ("page_size", C.c_int32),
        ("num_pages", C.c_int32),
        ("page_stride", C.c_int64),
        ("head_stride", C.c_int64),
        ("tok_stride", C.c_int64),
        ("block_table", C.c_void_p),
        ("max_pages", C.c_int32),
        ("chunk_tokens", C.c_int32),
        ("num_chunks", C.c_int32),
        ("scale", C.c_float),
        ("flags", C.c_uint32),
        ("status", C.c_void_p),
        ("sched_counter", C.c_void_p),
        ("tune", C.c_uint32),
        ("tune_stages", C.c_int32),
        ("tune_ctas_per_sm", C.c_int32),
    ]


class HgLogitsDesc(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32),
        ("batch", C.c_int32),
        ("num_q_heads", C.c_int32),
        ("num_kv_heads", C.c_int32),
        ("head_dim", C.c_int32),
        ("dtype", C.c_int32),
        ("max_selected", C.c_int32),
        ("chunk_tokens", C.c_int32),
        ("num_chunks", C.c_int32),
        ("status", C.c_void_p),
        ("tune", C.c_uint32),
        ("reserved", C.c_uint32),
    ]


class HgPrefixDesc(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32),
        ("num_groups", C.c_int32),
        ("seq_group", C.c_void_p),
        ("group_row", C.c_void_p),
        ("group_begin", C.c_void_p),
        ("group_end", C.c_void_p),
        ("chunk_tokens", C.c_int32),
        ("num_chunks", C.c_int32),
    ]


class HgPartialSrc(C.Structure):
    _fields_ = [("o", C.c_void_p), ("m", C.c_void_p), ("l", C.c_void_p), ("nc", C.c_int32), ("reserved", C.c_int32)]


def lib_path() -> str:
    return os.path.join(_PKG, _LIB_NAME)


def lib():
    """Load the CUDA library (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with `python -m paper_2604_18529_b200.build` "
                               "(there is no CPU or PyTorch fallback)")
        L = C.CDLL(path)
        vp, i32 = C.c_void_p, C.c_int32
        L.hg_attn_partial.argtypes = [vp] * 10 + [C.POINTER(HgAttnDesc)]
        L.hg_attn_partial.restype = C.c_int
        L.hg_attn_merge.argtypes = [C.POINTER(HgPartialSrc), i32, vp, vp, vp, C.POINTER(HgAttnDesc)]
        L.hg_attn_merge.restype = C.c_int
        L.hg_attn_workspace_bytes.argtypes = [C.POINTER(HgAttnDesc), i32]
        L.hg_attn_workspace_bytes.restype = C.c_size_t
        L.hg_attn_decode.argtypes = [vp] * 6 + [C.POINTER(HgPartialSrc), i32, vp, vp, vp, C.c_size_t, vp, C.POINTER(HgAttnDesc)]
        L.hg_attn_decode.restype = C.c_int
        L.hg_attn_decode_host.argtypes = L.hg_attn_decode.argtypes
        L.hg_attn_decode_host.restype = C.c_int
        L.hg_attn_decode_static.argtypes = [vp] * 6 + [C.POINTER(HgPartialSrc), i32, vp, vp, vp, C.POINTER(HgAttnDesc)]
        L.hg_attn_decode_static.restype = C.c_int
        L.hg_attn_partial_from_logits.argtypes = [vp] * 7 + [C.POINTER(HgLogitsDesc)]
        L.hg_attn_partial_from_logits.restype = C.c_int
        L.hg_kv_append.argtypes = [vp] * 7 + [C.POINTER(HgAttnDesc)]
        L.hg_kv_append.restype = C.c_int
        L.hg_kv_evict.argtypes = [vp] * 5 + [i32, vp, vp, vp, vp, i32, vp, C.POINTER(HgAttnDesc)]
        L.hg_kv_evict.restype = C.c_int
        L.hg_kv_evict_begin.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, C.POINTER(HgAttnDesc)]
        L.hg_kv_evict_begin.restype = C.c_int
        L.hg_kv_evict_copy.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, C.POINTER(HgAttnDesc)]
        L.hg_kv_evict_copy.restype = C.c_int
        L.hg_kv_evict_finish.argtypes = [vp, vp, vp, vp, i32, vp, C.POINTER(HgAttnDesc)]
        L.hg_kv_evict_finish.restype = C.c_int
        L.hg_attn_prefix_partial.argtypes = [vp] * 7 + [C.POINTER(HgAttnDesc), C.POINTER(HgPrefixDesc)]
        L.hg_attn_prefix_partial.restype = C.c_int
        L.hg_attn_prefix_suggest_chunk.argtypes = [C.c_int64] + [i32] * 5
        L.hg_attn_prefix_suggest_chunk.restype = i32
        L.hg_attn_shared_workspace_bytes.argtypes = [C.POINTER(HgAttnDesc), C.POINTER(HgPrefixDesc)]
        L.hg_attn_shared_workspace_bytes.restype = C.c_size_t
        L.hg_attn_decode_shared.argtypes = [vp] * 6 + [C.POINTER(HgPartialSrc), i32, vp, vp, vp, C.c_size_t, vp, C.POINTER(HgAttnDesc),
                                                       C.POINTER(HgPrefixDesc)]
        L.hg_attn_decode_shared.restype = C.c_int
        L.hg_kv_fork.argtypes = [vp] * 6 + [C.POINTER(HgAttnDesc)]
        L.hg_kv_fork.restype = C.c_int
        L.hg_kv_reserve.argtypes = [vp] * 8 + [C.POINTER(HgAttnDesc)]
        L.hg_kv_reserve.restype = C.c_int
        L.hg_kv_release.argtypes = [vp, i32, vp, vp, C.POINTER(HgAttnDesc)]
        L.hg_kv_release.restype = C.c_int
        L.hg_kv_compact.argtypes = [vp] * 4 + [i32, vp, vp, C.POINTER(HgAttnDesc)]
        L.hg_kv_compact.restype = C.c_int
        L.hg_kv_copy_pages.argtypes = [vp] * 3 + [i32] + [vp] * 4 + [C.POINTER(HgAttnDesc)]
        L.hg_kv_copy_pages.restype = C.c_int
        L.hg_kv_read_probe.argtypes = [vp] * 7 + [C.POINTER(HgAttnDesc)]
        L.hg_kv_read_probe.restype = C.c_int
        L.hg_status_string.argtypes = [C.c_int]
        L.hg_status_string.restype = C.c_char_p
        L.hg_version.argtypes = []
        L.hg_version.restype = C.c_uint32
        _lib = L
    return _lib


def hg_status_string(status: int) -> str:
    return lib().hg_status_string(int(status)).decode()


def hg_version() -> int:
    return int(lib().hg_version())


def _dev(t: Optional[torch.Tensor], name: str, dtype=None) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _host(t: Optional[torch.Tensor], name: str, dtype=None) -> Optional[int]:
    if t is None:
        return None
    if t.is_cuda:
        raise ValueError(f"{name} must be a host tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(status: int, where: str) -> None:
    if status != HG_OK:
        raise HgError(status, where)


_DTYPES = {torch.float16: HG_DTYPE_F16, torch.bfloat16: HG_DTYPE_BF16, "f16": HG_DTYPE_F16, "bf16": HG_DTYPE_BF16}


def attn_desc(*, batch: int, num_q_heads: int, num_kv_heads: int, head_dim: int, dtype, page_size: int,
              num_pages: int, page_stride: int, head_stride: int, tok_stride: int,
              block_table: Optional[torch.Tensor], max_pages: int, chunk_tokens: int, num_chunks: int,
              scale: float = 0.0, status: Optional[torch.Tensor] = None, flags: int = 0,
              sched_counter: Optional[torch.Tensor] = None, tune: int = 0, tune_stages: int = 0,
              tune_ctas_per_sm: int = 0) -> HgAttnDesc:
    """Fill an ``hg_attn_desc``.  ``block_table`` (int32 CUDA [B][max_pages]), ``status`` and
    ``sched_counter`` (int32 CUDA scalars) are kept alive by the returned object."""
    d = HgAttnDesc()
    d.struct_size = C.sizeof(HgAttnDesc)
    d.batch, d.num_q_heads, d.num_kv_heads, d.head_dim = batch, num_q_heads, num_kv_heads, head_dim
    d.dtype = _DTYPES[dtype]
    d.page_size, d.num_pages = page_size, num_pages
    d.page_stride, d.head_stride, d.tok_stride = page_stride, head_stride, tok_stride
    d.block_table = _dev(block_table, "block_table", torch.int32)
    d.max_pages, d.chunk_tokens, d.num_chunks = max_pages, chunk_tokens, num_chunks
    d.scale, d.flags = scale, flags
    d.status = _dev(status, "status", torch.int32)
    d.sched_counter = _dev(sched_counter, "sched_counter", torch.int32)
    d.tune, d.tune_stages, d.tune_ctas_per_sm = tune, tune_stages, tune_ctas_per_sm
    d._keep = (block_table, status, sched_counter)
    return d


def _src_array(partials: Sequence[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]], host: bool):
    arr = (HgPartialSrc * max(1, len(partials)))()
    conv = _host if host else _dev
    for i, (o, m, l) in enumerate(partials):
        arr[i].o = conv(o, "partial o", torch.float32)
        arr[i].m = conv(m, "partial m", torch.float32)
        arr[i].l = conv(l, "partial l", torch.float32)
        arr[i].nc = m.shape[-1]
        if o.numel() != m.numel() * o.shape[-1] or l.shape != m.shape:
            raise ValueError("partial source shapes must be o [B][Hq][nc][D], m and l [B][Hq][nc]")
    return arr


def hg_attn_partial(q, k_cache, v_cache, seq_lens, tok_begin, tok_end, o_part, m_part, l_part, desc: HgAttnDesc,
                    stream=None) -> None:
    """Chunk partials (o, m, l) of the GPU-resident slice; see ``hg_attn_partial`` in the header."""
    st = lib().hg_attn_partial(_dev(q, "q"), _dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"),
                               _dev(seq_lens, "seq_lens", torch.int32), _dev(tok_begin, "tok_begin", torch.int32),
                               _dev(tok_end, "tok_end", torch.int32), _dev(o_part, "o_part", torch.float32),
                               _dev(m_part, "m_part", torch.float32), _dev(l_part, "l_part", torch.float32),
                               _stream(stream), C.byref(desc))
    _check(st, "hg_attn_partial")


def logits_desc(*, batch: int, num_q_heads: int, num_kv_heads: int, head_dim: int, dtype, max_selected: int,
                chunk_tokens: int = 256, num_chunks: int = 0, status: Optional[torch.Tensor] = None,
                tune: int = 0) -> HgLogitsDesc:
    d = HgLogitsDesc()
    d.struct_size = C.sizeof(HgLogitsDesc)
    d.batch, d.num_q_heads, d.num_kv_heads, d.head_dim = batch, num_q_heads, num_kv_heads, head_dim
    d.dtype = _DTYPES[dtype]
    d.max_selected, d.chunk_tokens = max_selected, chunk_tokens
    d.num_chunks = num_chunks or -(-max_selected // chunk_tokens)
    d.status = _dev(status, "status", torch.int32)
    d.tune = tune
    d._keep = (status,)
    return d


def hg_attn_partial_from_logits(logits, v_rows, n_sel, o_part, m_part, l_part, desc: HgLogitsDesc, stream=None) -> None:
    """Partials (o, m, l) from host-computed logits [B][Hq][K] (fp32) and the matching V rows [B][Hkv][K][D]."""
    st = lib().hg_attn_partial_from_logits(_dev(logits, "logits", torch.float32), _dev(v_rows, "v_rows"),
                                           _dev(n_sel, "n_sel", torch.int32), _dev(o_part, "o_part", torch.float32),
                                           _dev(m_part, "m_part", torch.float32), _dev(l_part, "l_part", torch.float32),
                                           _stream(stream), C.byref(desc))
    _check(st, "hg_attn_partial_from_logits")


def hg_attn_merge(partials, out, lse, desc: HgAttnDesc, stream=None) -> None:
    """LSE-merge of partial sources [(o, m, l), ...] (device tensors) into out [B][Hq][D] and lse [B][Hq]."""
    arr = _src_array(partials, host=False)
    st = lib().hg_attn_merge(arr, len(partials), _dev(out, "out", torch.float32), _dev(lse, "lse", torch.float32),
                             _stream(stream), C.byref(desc))
    _check(st, "hg_attn_merge")


def hg_attn_suggest_chunk(total_tokens: int, num_q_heads: int, num_kv_heads: int, page_size: int) -> int:
    """A chunk size (tokens) for a problem with that many GPU-resident token positions in total."""
    f = lib().hg_attn_suggest_chunk
    f.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32]
    f.restype = C.c_int32
    n = int(f(total_tokens, num_q_heads, num_kv_heads, page_size))
    if n == 0:
        raise HgError(HG_ERR_INVALID_ARG, "hg_attn_suggest_chunk")
    return n


def hg_attn_workspace_bytes(desc: HgAttnDesc, n_host_partials: int = 0) -> int:
    n = int(lib().hg_attn_workspace_bytes(C.byref(desc), n_host_partials))
    if n == 0:
        raise HgError(HG_ERR_INVALID_ARG, "hg_attn_workspace_bytes")
    return n


def hg_attn_decode(q, k_cache, v_cache, seq_lens, tok_begin, tok_end, host_partials, out, lse, workspace,
                   desc: HgAttnDesc, stream=None) -> None:
    """partial + merge in one call; ``host_partials`` are device tensors holding the host-slice partials."""
    arr = _src_array(host_partials, host=False)
    st = lib().hg_attn_decode(_dev(q, "q"), _dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"),
                              _dev(seq_lens, "seq_lens", torch.int32), _dev(tok_begin, "tok_begin", torch.int32),
                              _dev(tok_end, "tok_end", torch.int32), arr, len(host_partials),
                              _dev(out, "out", torch.float32), _dev(lse, "lse", torch.float32),
                              _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(),
                              _stream(stream), C.byref(desc))
    _check(st, "hg_attn_decode")


def hg_attn_decode_static(q, k_cache, v_cache, seq_lens, tok_begin, tok_end, host_partials, out, lse,
                          desc: HgAttnDesc, stream=None) -> None:
    """``hg_attn_decode`` for callers that may not allocate device memory (fixed-budget plugins,
    allocator-free decode loops, components without an allocator): the chunk partials go to a fixed 8 MiB array inside the
    library instead of a caller workspace.  Raises ``HgError`` (workspace) if the problem's partials do
    not fit.  All calls on a device share that array, so calls that could overlap on the GPU must be
    serialised; make the first call on a device outside any stream capture."""
    arr = _src_array(host_partials, host=False)
    st = lib().hg_attn_decode_static(_dev(q, "q"), _dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"),
                                     _dev(seq_lens, "seq_lens", torch.int32), _dev(tok_begin, "tok_begin", torch.int32),
                                     _dev(tok_end, "tok_end", torch.int32), arr, len(host_partials),
                                     _dev(out, "out", torch.float32), _dev(lse, "lse", torch.float32),
                                     _stream(stream), C.byref(desc))
    _check(st, "hg_attn_decode_static")


def hg_attn_decode_host(q_host, k_cache, v_cache, seq_lens_host, tok_begin_host, tok_end_host, host_partials_host,
                        out_host, lse_host, workspace, desc: HgAttnDesc, stream=None) -> None:
    """The same pass with per-step data in host (ideally pinned) memory; results land in out_host / lse_host
    once the stream has been synchronised."""
    arr = _src_array(host_partials_host, host=True)
    st = lib().hg_attn_decode_host(_host(q_host, "q_host"), _dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"),
                                   _host(seq_lens_host, "seq_lens_host", torch.int32),
                                   _host(tok_begin_host, "tok_begin_host", torch.int32),
                                   _host(tok_end_host, "tok_end_host", torch.int32), arr, len(host_partials_host),
                                   _host(out_host, "out_host", torch.float32), _host(lse_host, "lse_host", torch.float32),
                                   _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(),
                                   _stream(stream), C.byref(desc))
    _check(st, "hg_attn_decode_host")


def _prepared(fn, args, keep, where: str):
    def call(_keep=keep) -> None:
        st = fn(*args)
        if st != HG_OK:
            _check(st, where)
    return call


def prepare_partial(q, k_cache, v_cache, seq_lens, tok_begin, tok_end, o_part, m_part, l_part, desc: HgAttnDesc, stream=None):
    """``hg_attn_partial`` with its arguments marshalled once: returns a callable for a decode loop that reuses the
    same buffers (and stream) every step.  The callable keeps the tensors alive."""
    args = (_dev(q, "q"), _dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"), _dev(seq_lens, "seq_lens", torch.int32),
            _dev(tok_begin, "tok_begin", torch.int32), _dev(tok_end, "tok_end", torch.int32),
            _dev(o_part, "o_part", torch.float32), _dev(m_part, "m_part", torch.float32), _dev(l_part, "l_part", torch.float32),
            _stream(stream), C.byref(desc))
    keep = (q, k_cache, v_cache, seq_lens, tok_begin, tok_end, o_part, m_part, l_part, desc)
    return _prepared(lib().hg_attn_partial, args, keep, "hg_attn_partial")


def prepare_merge(partials, out, lse, desc: HgAttnDesc, stream=None):
    """``hg_attn_merge`` with its arguments marshalled once (see ``prepare_partial``)."""
    arr = _src_array(partials, host=False)
    args = (arr, len(partials), _dev(out, "out", torch.float32), _dev(lse, "lse", torch.float32), _stream(stream), C.byref(desc))
    return _prepared(lib().hg_attn_merge, args, (partials, out, lse, desc, arr), "hg_attn_merge")


def prepare_decode_host(q_host, k_cache, v_cache, seq_lens_host, tok_begin_host, tok_end_host, host_partials_host,
                        out_host, lse_host, workspace, desc: HgAttnDesc, stream=None):
    """Marshal the arguments of ``hg_attn_decode_host`` once and return a callable that makes the call.

    For a decode loop that reuses the same buffers every step (the usual case): the per-call cost of
    checking and converting a dozen tensors is paid once.  The returned callable keeps the tensors alive.
    """
    arr = _src_array(host_partials_host, host=True)
    args = (_host(q_host, "q_host"), _dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"),
            _host(seq_lens_host, "seq_lens_host", torch.int32), _host(tok_begin_host, "tok_begin_host", torch.int32),
            _host(tok_end_host, "tok_end_host", torch.int32), arr, len(host_partials_host),
            _host(out_host, "out_host", torch.float32), _host(lse_host, "lse_host", torch.float32),
            _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(), _stream(stream), C.byref(desc))
    keep = (q_host, k_cache, v_cache, seq_lens_host, tok_begin_host, tok_end_host, host_partials_host, out_host, lse_host,
            workspace, desc, arr)
    return _prepared(lib().hg_attn_decode_host, args, keep, "hg_attn_decode_host")


def hg_kv_append(k_new, v_new, k_cache, v_cache, seq_lens, tok_end, desc: HgAttnDesc, stream=None) -> None:
    """Write this step's K/V rows [B][Hkv][D] at position seq_lens[b] and advance seq_lens (and tok_end)."""
    st = lib().hg_kv_append(_dev(k_new, "k_new"), _dev(v_new, "v_new"), _dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"),
                            _dev(seq_lens, "seq_lens", torch.int32), _dev(tok_end, "tok_end", torch.int32),
                            _stream(stream), C.byref(desc))
    _check(st, "hg_kv_append")


def hg_kv_evict(k_cache, v_cache, tok_begin, tok_end, n_evict, k_out, v_out, freed_pages, n_freed, desc: HgAttnDesc,
                stream=None) -> None:
    """Copy the oldest n_evict[b] tokens of every slice to k_out / v_out [B][max_evict][Hkv][D], advance tok_begin
    and un-map the pages that became empty (their ids go to freed_pages [B][max_freed])."""
    st = lib().hg_kv_evict(_dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"), _dev(tok_begin, "tok_begin", torch.int32),
                           _dev(tok_end, "tok_end", torch.int32), _dev(n_evict, "n_evict", torch.int32), k_out.shape[1],
                           _dev(k_out, "k_out"), _dev(v_out, "v_out"), _dev(freed_pages, "freed_pages", torch.int32),
                           _dev(n_freed, "n_freed", torch.int32), 0 if freed_pages is None else freed_pages.shape[1],
                           _stream(stream), C.byref(desc))
    _check(st, "hg_kv_evict")


def hg_kv_evict_begin(tok_begin, tok_end, n_evict, max_evict: int, max_freed: int, src_begin, n_moved, desc: HgAttnDesc,
                      stream=None) -> None:
    """Step 1 of an eviction that drains beside the attention: decide and record the rows that leave, advance tok_begin."""
    st = lib().hg_kv_evict_begin(_dev(tok_begin, "tok_begin", torch.int32), _dev(tok_end, "tok_end", torch.int32),
                                 _dev(n_evict, "n_evict", torch.int32), max_evict, max_freed,
                                 _dev(src_begin, "src_begin", torch.int32), _dev(n_moved, "n_moved", torch.int32),
                                 _stream(stream), C.byref(desc))
    _check(st, "hg_kv_evict_begin")


def hg_kv_evict_copy(k_cache, v_cache, src_begin, n_moved, k_out, v_out, desc: HgAttnDesc, stream=None) -> None:
    """Step 2: copy the recorded rows to k_out / v_out [B][max_evict][Hkv][D] (reads only)."""
    st = lib().hg_kv_evict_copy(_dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"), _dev(src_begin, "src_begin", torch.int32),
                                _dev(n_moved, "n_moved", torch.int32), k_out.shape[1], _dev(k_out, "k_out"),
                                _dev(v_out, "v_out"), _stream(stream), C.byref(desc))
    _check(st, "hg_kv_evict_copy")


def hg_kv_evict_finish(src_begin, n_moved, freed_pages, n_freed, desc: HgAttnDesc, stream=None) -> None:
    """Step 3: un-map and list the pages that lie wholly below the new beginning."""
    st = lib().hg_kv_evict_finish(_dev(src_begin, "src_begin", torch.int32), _dev(n_moved, "n_moved", torch.int32),
                                  _dev(freed_pages, "freed_pages", torch.int32), _dev(n_freed, "n_freed", torch.int32),
                                  0 if freed_pages is None else freed_pages.shape[1], _stream(stream), C.byref(desc))
    _check(st, "hg_kv_evict_finish")


def _here(t: Optional[torch.Tensor], name: str, dtype=None, numel: int = 0) -> Optional[int]:
    """``_dev`` for a tensor that must also live on the current device (where the call is launched) and hold at least
    ``numel`` elements."""
    p = _dev(t, name, dtype)
    if t is not None and t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{torch.cuda.current_device()}")
    if t is not None and t.numel() < numel:
        raise ValueError(f"{name} has {t.numel()} elements, {numel} are needed")
    return p


def _count(t: torch.Tensor, name: str) -> int:
    """The length of a list, which the C ABI takes as an int32 (ctypes would drop the bits above)."""
    if t.numel() > 0x7fffffff:
        raise ValueError(f"{name} has {t.numel()} entries, a call takes 2^31 - 1")
    return t.numel()


def _pool(t: torch.Tensor, name: str) -> int:
    """A KV pool, or a view of one: addressed through the description's strides, so it need not be contiguous."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{torch.cuda.current_device()}")
    return t.data_ptr()


def prefix_desc(*, seq_group: torch.Tensor, group_row: torch.Tensor, group_begin: torch.Tensor, group_end: torch.Tensor,
                chunk_tokens: int, num_chunks: int) -> HgPrefixDesc:
    """Fill an ``hg_prefix_desc`` (int32 CUDA tensors: seq_group [B], the others [num_groups]); keeps them alive."""
    d = HgPrefixDesc()
    d.struct_size = C.sizeof(HgPrefixDesc)
    d.num_groups = group_row.numel()
    d.seq_group = _dev(seq_group, "seq_group", torch.int32)
    d.group_row = _dev(group_row, "group_row", torch.int32)
    d.group_begin = _dev(group_begin, "group_begin", torch.int32)
    d.group_end = _dev(group_end, "group_end", torch.int32)
    if group_begin.numel() != d.num_groups or group_end.numel() != d.num_groups:
        raise ValueError("group_row, group_begin and group_end must have one element per group")
    d.chunk_tokens, d.num_chunks = chunk_tokens, num_chunks
    d._keep = (seq_group, group_row, group_begin, group_end)
    return d


def _check_groups(desc: HgAttnDesc, prefix: HgPrefixDesc) -> None:
    seq_group = prefix._keep[0]
    if seq_group.numel() < desc.batch:
        raise ValueError(f"seq_group has {seq_group.numel()} elements, the batch {desc.batch}")
    for t, name in zip(prefix._keep, ("seq_group", "group_row", "group_begin", "group_end")):
        if t.device.index != torch.cuda.current_device():
            raise ValueError(f"{name} is on {t.device}, the current device is cuda:{torch.cuda.current_device()}")


def hg_attn_prefix_partial(q, k_cache, v_cache, o_part, m_part, l_part, desc: HgAttnDesc, prefix: HgPrefixDesc, stream=None) -> None:
    """Chunk partials (o, m, l) of the groups' shared prefixes; one more source for ``hg_attn_merge``."""
    _check_groups(desc, prefix)
    n = desc.batch * desc.num_q_heads * prefix.num_chunks
    st = lib().hg_attn_prefix_partial(_here(q, "q", None, desc.batch * desc.num_q_heads * desc.head_dim), _pool(k_cache, "k_cache"), _pool(v_cache, "v_cache"),
                                      _here(o_part, "o_part", torch.float32, n * desc.head_dim),
                                      _here(m_part, "m_part", torch.float32, n), _here(l_part, "l_part", torch.float32, n),
                                      _stream(stream), C.byref(desc), C.byref(prefix))
    _check(st, "hg_attn_prefix_partial")


def hg_attn_prefix_suggest_chunk(shared_tokens: int, num_groups: int, num_members: int, num_q_heads: int, num_kv_heads: int,
                                 page_size: int) -> int:
    """A chunk size (tokens) for ``hg_attn_prefix_partial``; tokens and members are summed over the groups."""
    n = int(lib().hg_attn_prefix_suggest_chunk(shared_tokens, num_groups, num_members, num_q_heads, num_kv_heads, page_size))
    if n == 0:
        raise HgError(HG_ERR_INVALID_ARG, "hg_attn_prefix_suggest_chunk")
    return n


def hg_attn_shared_workspace_bytes(desc: HgAttnDesc, prefix: HgPrefixDesc) -> int:
    n = int(lib().hg_attn_shared_workspace_bytes(C.byref(desc), C.byref(prefix)))
    if n == 0:
        raise HgError(HG_ERR_INVALID_ARG, "hg_attn_shared_workspace_bytes")
    return n


def _decode_shared_args(q, k_cache, v_cache, seq_lens, tok_begin, tok_end, partials, out, lse, workspace, desc, prefix, stream):
    _check_groups(desc, prefix)
    B, rows = desc.batch, desc.batch * desc.num_q_heads
    arr = _src_array(partials, host=False)
    return (_here(q, "q", None, rows * desc.head_dim), _pool(k_cache, "k_cache"), _pool(v_cache, "v_cache"),
            _here(seq_lens, "seq_lens", torch.int32, B),
            _here(tok_begin, "tok_begin", torch.int32, B), _here(tok_end, "tok_end", torch.int32, B), arr, len(partials),
            _here(out, "out", torch.float32, rows * desc.head_dim), _here(lse, "lse", torch.float32, rows),
            _here(workspace, "workspace"), workspace.numel() * workspace.element_size(), _stream(stream), C.byref(desc),
            C.byref(prefix))


def hg_attn_decode_shared(q, k_cache, v_cache, seq_lens, tok_begin, tok_end, host_partials, out, lse, workspace, desc: HgAttnDesc,
                          prefix: HgPrefixDesc, stream=None) -> None:
    """One decode step over the groups' shared prefixes and every sequence's own tokens [tok_begin, tok_end), merged."""
    _check(lib().hg_attn_decode_shared(*_decode_shared_args(q, k_cache, v_cache, seq_lens, tok_begin, tok_end, host_partials, out, lse,
                                                            workspace, desc, prefix, stream)), "hg_attn_decode_shared")


def prepare_decode_shared(q, k_cache, v_cache, seq_lens, tok_begin, tok_end, host_partials, out, lse, workspace, desc: HgAttnDesc,
                          prefix: HgPrefixDesc, stream=None):
    """``hg_attn_decode_shared`` with its arguments marshalled once (see ``prepare_partial``)."""
    args = _decode_shared_args(q, k_cache, v_cache, seq_lens, tok_begin, tok_end, host_partials, out, lse, workspace, desc, prefix, stream)
    keep = (q, k_cache, v_cache, seq_lens, tok_begin, tok_end, host_partials, out, lse, workspace, desc, prefix)
    return _prepared(lib().hg_attn_decode_shared, args, keep, "hg_attn_decode_shared")


def _kv_fork_args(src_row, ref_count, seq_lens, tok_begin, tok_end, desc: HgAttnDesc, stream):
    B = desc.batch
    return (_here(src_row, "src_row", torch.int32, B), _here(ref_count, "ref_count", torch.int32, desc.num_pages),
            _here(seq_lens, "seq_lens", torch.int32, B), _here(tok_begin, "tok_begin", torch.int32, B),
            _here(tok_end, "tok_end", torch.int32, B), _stream(stream), C.byref(desc))


def hg_kv_fork(src_row, ref_count, seq_lens, tok_begin, tok_end, desc: HgAttnDesc, stream=None) -> None:
    """Row b of the block table takes the pages (and lengths) of row src_row[b], all rows at once; negative frees it."""
    _check(lib().hg_kv_fork(*_kv_fork_args(src_row, ref_count, seq_lens, tok_begin, tok_end, desc, stream)), "hg_kv_fork")


def prepare_kv_fork(src_row, ref_count, seq_lens, tok_begin, tok_end, desc: HgAttnDesc, stream=None):
    """``hg_kv_fork`` with its arguments marshalled once (see ``prepare_partial``)."""
    return _prepared(lib().hg_kv_fork, _kv_fork_args(src_row, ref_count, seq_lens, tok_begin, tok_end, desc, stream),
                     (src_row, ref_count, seq_lens, tok_begin, tok_end, desc), "hg_kv_fork")


def _kv_reserve_args(seq_lens, n_new, ref_count, copy_src, copy_dst, copy_rows, n_ready, desc: HgAttnDesc, stream):
    B = desc.batch
    return (_here(seq_lens, "seq_lens", torch.int32, B), _here(n_new, "n_new", torch.int32, B),
            _here(ref_count, "ref_count", torch.int32, desc.num_pages), _here(copy_src, "copy_src", torch.int32, B),
            _here(copy_dst, "copy_dst", torch.int32, B), _here(copy_rows, "copy_rows", torch.int32, B),
            _here(n_ready, "n_ready", torch.int32, B), _stream(stream), C.byref(desc))


def hg_kv_reserve(seq_lens, n_new, ref_count, copy_src, copy_dst, copy_rows, n_ready, desc: HgAttnDesc, stream=None) -> None:
    """Pages for the next n_new[b] positions of every row; shared pages are replaced (the copies to make are listed in
    copy_src / copy_dst / copy_rows, for ``hg_kv_copy_pages``)."""
    _check(lib().hg_kv_reserve(*_kv_reserve_args(seq_lens, n_new, ref_count, copy_src, copy_dst, copy_rows, n_ready, desc, stream)),
           "hg_kv_reserve")


def prepare_kv_reserve(seq_lens, n_new, ref_count, copy_src, copy_dst, copy_rows, n_ready, desc: HgAttnDesc, stream=None):
    """``hg_kv_reserve`` with its arguments marshalled once (see ``prepare_partial``)."""
    return _prepared(lib().hg_kv_reserve,
                     _kv_reserve_args(seq_lens, n_new, ref_count, copy_src, copy_dst, copy_rows, n_ready, desc, stream),
                     (seq_lens, n_new, ref_count, copy_src, copy_dst, copy_rows, n_ready, desc), "hg_kv_reserve")


def hg_kv_release(page_ids, ref_count, desc: HgAttnDesc, stream=None) -> None:
    """One reference less for every page id of the list (negative ones are skipped), as ``hg_kv_evict`` leaves it."""
    n = _count(page_ids, "page_ids")
    _check(lib().hg_kv_release(_here(page_ids, "page_ids", torch.int32), n,
                               _here(ref_count, "ref_count", torch.int32, desc.num_pages), _stream(stream), C.byref(desc)),
           "hg_kv_release")


def _kv_compact_args(ref_count, remap, move_src, move_dst, n_moves, desc: HgAttnDesc, stream):
    n = _count(move_src, "move_src")
    return (_here(ref_count, "ref_count", torch.int32, desc.num_pages), _here(remap, "remap", torch.int32, desc.num_pages),
            _here(move_src, "move_src", torch.int32), _here(move_dst, "move_dst", torch.int32, n), n,
            _here(n_moves, "n_moves", torch.int32, 1), _stream(stream), C.byref(desc))


def hg_kv_compact(ref_count, remap, move_src, move_dst, n_moves, desc: HgAttnDesc, stream=None) -> None:
    """Renames the pages in use to the low end of the pool (at most move_src.numel() of them); the moves to make are
    listed in move_src / move_dst, for ``hg_kv_copy_pages``."""
    _check(lib().hg_kv_compact(*_kv_compact_args(ref_count, remap, move_src, move_dst, n_moves, desc, stream)), "hg_kv_compact")


def prepare_kv_compact(ref_count, remap, move_src, move_dst, n_moves, desc: HgAttnDesc, stream=None):
    """``hg_kv_compact`` with its arguments marshalled once (see ``prepare_partial``)."""
    return _prepared(lib().hg_kv_compact, _kv_compact_args(ref_count, remap, move_src, move_dst, n_moves, desc, stream),
                     (ref_count, remap, move_src, move_dst, n_moves, desc), "hg_kv_compact")


def _kv_copy_pages_args(src, dst, rows, n_pairs, k_cache, v_cache, desc: HgAttnDesc, stream):
    n = _count(src, "src")
    return (_here(src, "src", torch.int32), _here(dst, "dst", torch.int32, n), _here(rows, "rows", torch.int32, n), n,
            _here(n_pairs, "n_pairs", torch.int32, 1), _pool(k_cache, "k_cache"), _pool(v_cache, "v_cache"), _stream(stream),
            C.byref(desc))


def hg_kv_copy_pages(src, dst, rows, n_pairs, k_cache, v_cache, desc: HgAttnDesc, stream=None) -> None:
    """Copies the first rows[i] token rows (None: all) of page src[i] to page dst[i], K and V; ``n_pairs`` (a device
    scalar or None) bounds how many pairs of the list count."""
    _check(lib().hg_kv_copy_pages(*_kv_copy_pages_args(src, dst, rows, n_pairs, k_cache, v_cache, desc, stream)), "hg_kv_copy_pages")


def prepare_kv_copy_pages(src, dst, rows, n_pairs, k_cache, v_cache, desc: HgAttnDesc, stream=None):
    """``hg_kv_copy_pages`` with its arguments marshalled once (see ``prepare_partial``)."""
    return _prepared(lib().hg_kv_copy_pages, _kv_copy_pages_args(src, dst, rows, n_pairs, k_cache, v_cache, desc, stream),
                     (src, dst, rows, n_pairs, k_cache, v_cache, desc), "hg_kv_copy_pages")


def hg_kv_read_probe(k_cache, v_cache, seq_lens, tok_begin, tok_end, sink, desc: HgAttnDesc, stream=None) -> None:
    """Stream the slice's K and V tiles and XOR-fold them into sink [B][Hkv][NC] (uint32 viewed as int32)."""
    st = lib().hg_kv_read_probe(_dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"),
                                _dev(seq_lens, "seq_lens", torch.int32), _dev(tok_begin, "tok_begin", torch.int32),
                                _dev(tok_end, "tok_end", torch.int32), _dev(sink, "sink", torch.int32),
                                _stream(stream), C.byref(desc))
    _check(st, "hg_kv_read_probe")
