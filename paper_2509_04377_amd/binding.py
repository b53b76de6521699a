"""Python front end of libpe.so: argument marshalling only.

Every function below has the name and argument order of the C-ABI entry point it calls
(include/pe.h), takes torch tensors that already live on the GPU, and enqueues the library's HIP
kernels on torch's current stream.  No step of the path is computed here or on the CPU and no
control flow of the method lives here (the host-side sequencing of calls is engine.py); if libpe.so
has not been built, the first call raises.  Without _pe_host.so, the native form of the same
marshalling, calls go through ctypes.
"""
import ctypes
import os
import warnings

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpe.so")
HOST_PATH = os.path.join(_HERE, "_pe_host.so")

PE_OK = 0
PE_ERR_INVALID_ARG, PE_ERR_UNSUPPORTED, PE_ERR_WORKSPACE, PE_ERR_HIP = -1, -2, -3, -4
PE_F32, PE_BF16 = 0, 1
PE_OP_SCORE_BLOCKS, PE_OP_PREFILL_PRUNE, PE_OP_EVICT_BLOCKS, PE_OP_PAGED_DECODE = 0, 1, 2, 3
PE_OP_APPEND_PAGED_DECODE = 4
PE_OP_TREE_DECODE, PE_OP_SELECT_PAGES, PE_OP_DECODE_WEIGHTS, PE_OP_QUANT_DECODE = 5, 6, 7, 8
PE_ROPE_HALF, PE_ROPE_INTERLEAVED = 0, 1
PE_ROPE_PLAIN, PE_ROPE_LINEAR, PE_ROPE_BY_PARTS = 0, 1, 2
PE_MAX_DRAFTS = 64
PE_STATIC_SCRATCH_BYTES = 8 * 1024 * 1024

EXPORTS = ["pe_workspace_bytes", "pe_status_string", "pe_version", "pe_decode_splits",
           "pe_score_blocks", "pe_prefill_prune", "pe_evict_blocks", "pe_paged_decode", "pe_append_kv",
           "pe_append_paged_decode", "pe_score_recent_blocks", "pe_evict_blocks_cached", "pe_evict_blocks_ex", "pe_score_evict",
           "pe_score_triggered_blocks", "pe_paged_decode_static", "pe_append_paged_decode_layers",
           "pe_tree_decode", "pe_append_path", "pe_page_bounds", "pe_select_pages",
           "pe_paged_decode_weights", "pe_plan_tokens", "pe_plan_tokens_ex", "pe_prefill_prune_admitted", "pe_quant_pages_admitted", "pe_rope_init", "pe_rotate",
           "pe_quant_pages", "pe_quant_append", "pe_quant_decode"]


class pe_cache_desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("num_seqs", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("num_q_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("max_blocks", ctypes.c_int32), ("num_phys_blocks", ctypes.c_int64), ("layout", ctypes.c_int32),
                ("decode_splits", ctypes.c_int32), ("decode_shape", ctypes.c_int32),
                ("decode_flat_order", ctypes.c_int32)]


class pe_evict_opts(ctypes.Structure):
    _fields_ = [("policy", ctypes.c_int32), ("protect_first", ctypes.c_int32), ("protect_last", ctypes.c_int32),
                ("share_heads", ctypes.c_int32), ("cached_scores", ctypes.c_int32)]


class pe_rope(ctypes.Structure):
    """Filled by make_rope()."""
    _fields_ = [("rotary_dim", ctypes.c_int32), ("pairs", ctypes.c_int32), ("magnitude", ctypes.c_float), ("filled", ctypes.c_int32),
                ("turns", ctypes.c_uint64 * 64)]


class pe_plan_opts(ctypes.Structure):
    _fields_ = [("admitted", ctypes.c_void_p), ("spare_used", ctypes.c_void_p), ("freed_phys", ctypes.c_void_p),
                ("only", ctypes.c_void_p), ("copies", ctypes.c_int32)]


class pe_quant_cache(ctypes.Structure):
    """Made by make_quant_cache(), which keeps the tensors alive beside it."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("k_tail", ctypes.c_void_p),
                ("v_tail", ctypes.c_void_p)]


PE_POLICY_LOWEST_SCORE, PE_POLICY_OLDEST = 0, 1
PE_LAYOUT_PER_HEAD, PE_LAYOUT_SHARED = 0, 1


class PeError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (where, status_string(status), status))


def _layout(structure):
    """Size, then name, offset and size of each field of a ctypes structure."""
    fields = ((name, getattr(structure, name).offset, getattr(structure, name).size) for name, _ in structure._fields_)
    return (ctypes.sizeof(structure),) + tuple(fields)


class _NoHost:
    """In place of the native marshalling: takes no call, so that every call goes through ctypes."""

    def __getattr__(self, name):
        return lambda *args: None


def _load_host():
    """The native marshalling, or, where it is not built or does not load, the reason as a warning and the way through ctypes."""
    why = "is not built"
    if os.path.exists(HOST_PATH):
        try:
            from . import _pe_host
            binds = ((_pe_host.bind_descriptor, pe_cache_desc), (_pe_host.bind_evict_opts, pe_evict_opts), (_pe_host.bind_rope, pe_rope),
                     (_pe_host.bind_quant_cache, pe_quant_cache))
            others = [of.__name__ for bind, of in binds if bind(of) != _layout(of)]
            if not others:
                return _pe_host
            why = "has another " + " and ".join(others)
        except (ImportError, AttributeError) as e:
            why = "does not load: %s" % e
    warnings.warn("_pe_host.so %s (%s): arguments are checked in Python, some 3 us more a call; build as for libpe.so" % (why, HOST_PATH),
                  RuntimeWarning, stacklevel=3)
    return _NoHost()


_lib = None
_host = None   # the native marshalling of the calls that come once a layer (csrc/pe_host.cpp), loaded with the library


def lib():
    """The loaded libpe.so.  Raises if it is missing: there is no fallback path."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libpe.so is not built (%s): run `python -c 'import __graft_entry__ as g; g.build()'` "
                               "or `python paper_2509_04377_amd/build.py`" % LIB_PATH)
        global _host
        _host = _load_host()
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        dp = ctypes.POINTER(pe_cache_desc)
        L.pe_workspace_bytes.restype = sz
        L.pe_workspace_bytes.argtypes = [ctypes.c_int, dp, i64]
        L.pe_status_string.restype = ctypes.c_char_p
        L.pe_status_string.argtypes = [ctypes.c_int]
        L.pe_version.restype = ctypes.c_int
        L.pe_version.argtypes = []
        L.pe_decode_splits.restype = ctypes.c_int
        L.pe_decode_splits.argtypes = [dp]
        L.pe_score_blocks.restype = ctypes.c_int
        L.pe_score_blocks.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.pe_prefill_prune.restype = ctypes.c_int
        L.pe_prefill_prune.argtypes = [dp, vp, vp, vp, i64, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.pe_evict_blocks.restype = ctypes.c_int
        L.pe_evict_blocks.argtypes = [dp, vp, vp, vp, i32, vp, vp, vp]
        L.pe_score_triggered_blocks.restype = ctypes.c_int
        L.pe_score_triggered_blocks.argtypes = [dp, vp, vp, vp, vp, i32, vp, vp]
        L.pe_score_evict.restype = ctypes.c_int
        L.pe_score_evict.argtypes = [dp, vp, vp, vp, vp, i32, vp, vp, vp, vp]
        L.pe_paged_decode.restype = ctypes.c_int
        L.pe_paged_decode.argtypes = [dp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]
        L.pe_paged_decode_static.restype = ctypes.c_int
        L.pe_paged_decode_static.argtypes = [dp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp]
        L.pe_append_kv.restype = ctypes.c_int
        L.pe_append_kv.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp]
        L.pe_append_paged_decode.restype = ctypes.c_int
        L.pe_append_paged_decode.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, ctypes.c_float, vp, vp, sz,
                                             vp]
        L.pe_append_paged_decode_layers.restype = ctypes.c_int
        L.pe_append_paged_decode_layers.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, ctypes.c_float,
                                                    vp, vp, sz, vp]
        L.pe_evict_blocks_ex.restype = ctypes.c_int
        L.pe_evict_blocks_ex.argtypes = [dp, ctypes.POINTER(pe_evict_opts), vp, vp, vp, i32, vp, vp, vp]
        L.pe_score_recent_blocks.restype = ctypes.c_int
        L.pe_score_recent_blocks.argtypes = [dp, vp, vp, vp, vp, i32, vp, vp]
        L.pe_evict_blocks_cached.restype = ctypes.c_int
        L.pe_evict_blocks_cached.argtypes = [dp, vp, vp, vp, i32, vp, vp, vp]
        L.pe_tree_decode.restype = ctypes.c_int
        L.pe_tree_decode.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]
        L.pe_append_path.restype = ctypes.c_int
        L.pe_append_path.argtypes = [dp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp]
        L.pe_page_bounds.restype = ctypes.c_int
        L.pe_page_bounds.argtypes = [dp, vp, vp, vp, i32, vp, vp]
        L.pe_select_pages.restype = ctypes.c_int
        L.pe_select_pages.argtypes = [dp, vp, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
        L.pe_paged_decode_weights.restype = ctypes.c_int
        L.pe_paged_decode_weights.argtypes = [dp, vp, vp, vp, vp, vp, ctypes.c_float, ctypes.c_float, vp, vp, vp, vp, sz, vp]
        dbl, rp, cp = ctypes.c_double, ctypes.POINTER(pe_rope), ctypes.POINTER(pe_quant_cache)
        L.pe_plan_tokens.restype = ctypes.c_int
        L.pe_plan_tokens.argtypes = [dp, vp, vp, vp, i64, i32, vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp]
        L.pe_plan_tokens_ex.restype = ctypes.c_int
        L.pe_plan_tokens_ex.argtypes = [dp, ctypes.POINTER(pe_plan_opts)] + L.pe_plan_tokens.argtypes[1:]
        L.pe_prefill_prune_admitted.restype = ctypes.c_int
        L.pe_prefill_prune_admitted.argtypes = [dp, vp, vp, vp, vp] + L.pe_prefill_prune.argtypes[4:]
        L.pe_rope_init.restype = ctypes.c_int
        L.pe_rope_init.argtypes = [rp, i32, i32, dbl, i32, dbl, dbl, dbl, dbl, dbl]
        L.pe_rotate.restype = ctypes.c_int
        L.pe_rotate.argtypes = [dp, rp, i32, i64, vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp]
        L.pe_quant_pages.restype = ctypes.c_int
        L.pe_quant_pages.argtypes = [dp, cp, vp, vp, vp, vp, vp, vp, vp]
        L.pe_quant_pages_admitted.restype = ctypes.c_int
        L.pe_quant_pages_admitted.argtypes = [dp, cp, vp] + L.pe_quant_pages.argtypes[2:]
        L.pe_quant_append.restype = ctypes.c_int
        L.pe_quant_append.argtypes = [dp, cp, rp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp]
        L.pe_quant_decode.restype = ctypes.c_int
        L.pe_quant_decode.argtypes = [dp, cp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]
        # addresses of the functions that are called through _pe_host
        for name in ("paged_decode", "append_paged_decode", "append_paged_decode_layers", "prefill_prune",
                     "score_triggered_blocks", "score_recent_blocks", "evict_blocks", "evict_blocks_cached", "evict_blocks_ex",
                     "tree_decode", "append_path", "paged_decode_weights", "page_bounds", "select_pages", "plan_tokens_ex", "prefill_prune_admitted", "rotate",
                     "quant_pages", "quant_pages_admitted", "quant_append", "quant_decode"):
            setattr(L, "addr_" + name, ctypes.cast(getattr(L, "pe_" + name), vp).value)
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().pe_status_string(int(status)).decode()


def pe_version() -> int:
    return int(lib().pe_version())


def pe_decode_splits(desc: pe_cache_desc) -> int:
    return int(lib().pe_decode_splits(ctypes.byref(desc)))


def make_desc(dtype, num_seqs, num_kv_heads, num_q_heads, head_dim, block_size, max_blocks, num_phys_blocks,
              layout=0, decode_splits=0, decode_shape=0, decode_flat_order=0):
    code = {torch.float32: PE_F32, torch.bfloat16: PE_BF16}.get(dtype, dtype if isinstance(dtype, int) else -1)
    return pe_cache_desc(int(code), int(num_seqs), int(num_kv_heads), int(num_q_heads), int(head_dim),
                         int(block_size), int(max_blocks), int(num_phys_blocks), int(layout), int(decode_splits),
                         int(decode_shape), int(decode_flat_order))


def check(status, where):
    if status != PE_OK:
        raise PeError(status, where)


def ptr(t, name, dtype=None, optional=False):
    if t is None:
        if optional:
            return None
        raise PeError(PE_ERR_INVALID_ARG, name + " is None")
    if not t.is_cuda:
        raise ValueError(name + " must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(name + " must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))
    return ctypes.c_void_p(t.data_ptr())


# What the calls below pass: the checks of ptr(), and the current stream and the workspace, as plain numbers (ctypes converts
# them by the declared argument types).  The calls of prompts and decode steps try _pe_host first, which does the same in native
# code: a small launch is over sooner than its arguments are put together here.  It returns None for anything out of the
# ordinary; the way through ctypes then accepts it or raises what is wrong.
def _addr(t, name, dtype=None):
    if t is not None and t.is_cuda and t.is_contiguous() and (dtype is None or t.dtype is dtype):
        return t.data_ptr()
    return ptr(t, name, dtype).value   # raises what is wrong


def _addr_opt(t, name, dtype=None):
    return None if t is None else _addr(t, name, dtype)


def _ws(workspace):
    if workspace is None:
        return None, 0
    if not workspace.is_cuda:
        raise ValueError("workspace must be a GPU tensor")
    # its bytes are its own only if nothing else lies between them, whatever the order of its dimensions
    if not workspace.is_contiguous():
        by_stride = sorted(range(workspace.dim()), key=workspace.stride, reverse=True)
        if not workspace.permute(by_stride).is_contiguous():
            raise ValueError("workspace must be dense")
    return workspace.data_ptr(), workspace.nbytes


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def pe_workspace_bytes(op: int, desc: pe_cache_desc, total_tokens: int = 0) -> int:
    return int(lib().pe_workspace_bytes(int(op), ctypes.byref(desc), int(total_tokens)))


def alloc_workspace(op: int, desc: pe_cache_desc, total_tokens: int = 0, device="cuda"):
    """A torch buffer of the size pe_workspace_bytes() asks for (None if the op needs none)."""
    n = pe_workspace_bytes(op, desc, total_tokens)
    if n == 0:
        return None
    return torch.empty((n + 255) // 256 * 256, dtype=torch.uint8, device=device)


def pe_score_blocks(desc, k_pool, v_pool, block_table, seq_lens, scores_out, workspace=None):
    # (the call needs no workspace; whatever is given is not looked at)
    check(lib().pe_score_blocks(ctypes.byref(desc), _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                 _addr(block_table, "block_table", torch.int32), _addr(seq_lens, "seq_lens", torch.int32),
                                 _addr(scores_out, "scores_out", torch.float32), None, 0, _stream()), "pe_score_blocks")


def pe_prefill_prune(desc, k_in, v_in, cu_seqlens, total_tokens, max_seqlen, budget_tokens, k_pool, v_pool,
                     block_table, seq_lens_out, kept_idx_out, workspace, admitted=None):
    """admitted: only the sequences that a plan of tokens let begin (pe_prefill_prune_admitted)."""
    L = lib()
    if admitted is None:
        status = _host.prefill_prune(L.addr_prefill_prune, desc, k_in, v_in, cu_seqlens, total_tokens, max_seqlen, budget_tokens,
                                     k_pool, v_pool, block_table, seq_lens_out, kept_idx_out, workspace)
    else:
        status = _host.prefill_prune_admitted(L.addr_prefill_prune_admitted, desc, k_in, v_in, cu_seqlens, admitted, total_tokens, max_seqlen,
                                              budget_tokens, k_pool, v_pool, block_table, seq_lens_out, kept_idx_out, workspace)
    if status is None:
        wp, wn = _ws(workspace)
        status = L.pe_prefill_prune_admitted(ctypes.byref(desc), _addr(k_in, "k_in"), _addr(v_in, "v_in"),
                                             _addr(cu_seqlens, "cu_seqlens", torch.int32), _addr_opt(admitted, "admitted", torch.int32),
                                             int(total_tokens), int(max_seqlen),
                                             int(budget_tokens), _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                             _addr(block_table, "block_table", torch.int32),
                                             _addr(seq_lens_out, "seq_lens_out", torch.int32),
                                             _addr_opt(kept_idx_out, "kept_idx_out", torch.int32), wp, wn, _stream())
    check(status, "pe_prefill_prune")


def pe_evict_blocks(desc, scores, block_table, seq_lens, budget_tokens, evicted_logical_out, freed_phys_out):
    L = lib()
    status = _host.evict_blocks(L.addr_evict_blocks, desc, scores, block_table, seq_lens, budget_tokens, evicted_logical_out,
                                freed_phys_out)
    if status is None:
        status = L.pe_evict_blocks(ctypes.byref(desc), _addr(scores, "scores", torch.float32),
                                   _addr(block_table, "block_table", torch.int32), _addr(seq_lens, "seq_lens", torch.int32),
                                   int(budget_tokens), _addr(evicted_logical_out, "evicted_logical_out", torch.int32),
                                   _addr(freed_phys_out, "freed_phys_out", torch.int32), _stream())
    check(status, "pe_evict_blocks")


def pe_score_triggered_blocks(desc, k_pool, v_pool, block_table, seq_lens, budget_tokens, scores_inout):
    L = lib()
    status = _host.score_triggered_blocks(L.addr_score_triggered_blocks, desc, k_pool, v_pool, block_table, seq_lens,
                                          budget_tokens, scores_inout)
    if status is None:
        status = L.pe_score_triggered_blocks(ctypes.byref(desc), _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                             _addr(block_table, "block_table", torch.int32),
                                             _addr(seq_lens, "seq_lens", torch.int32), int(budget_tokens),
                                             _addr(scores_inout, "scores_inout", torch.float32), _stream())
    check(status, "pe_score_triggered_blocks")


def pe_score_evict(desc, k_pool, v_pool, block_table, seq_lens, budget_tokens, scores_out, evicted_logical_out,
                   freed_phys_out):
    check(lib().pe_score_evict(ctypes.byref(desc), _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                _addr(block_table, "block_table", torch.int32), _addr(seq_lens, "seq_lens", torch.int32),
                                int(budget_tokens), _addr_opt(scores_out, "scores_out", torch.float32),
                                _addr(evicted_logical_out, "evicted_logical_out", torch.int32),
                                _addr(freed_phys_out, "freed_phys_out", torch.int32), _stream()), "pe_score_evict")


def pe_score_recent_blocks(desc, k_pool, v_pool, block_table, seq_lens, recent, scores_inout):
    L = lib()
    status = _host.score_recent_blocks(L.addr_score_recent_blocks, desc, k_pool, v_pool, block_table, seq_lens, recent,
                                       scores_inout)
    if status is None:
        status = L.pe_score_recent_blocks(ctypes.byref(desc), _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                          _addr(block_table, "block_table", torch.int32),
                                          _addr(seq_lens, "seq_lens", torch.int32), int(recent),
                                          _addr(scores_inout, "scores_inout", torch.float32), _stream())
    check(status, "pe_score_recent_blocks")


def pe_evict_blocks_cached(desc, scores_inout, block_table, seq_lens, budget_tokens, evicted_logical_out,
                           freed_phys_out):
    L = lib()
    status = _host.evict_blocks_cached(L.addr_evict_blocks_cached, desc, scores_inout, block_table, seq_lens, budget_tokens,
                                       evicted_logical_out, freed_phys_out)
    if status is None:
        status = L.pe_evict_blocks_cached(ctypes.byref(desc), _addr(scores_inout, "scores_inout", torch.float32),
                                          _addr(block_table, "block_table", torch.int32),
                                          _addr(seq_lens, "seq_lens", torch.int32), int(budget_tokens),
                                          _addr(evicted_logical_out, "evicted_logical_out", torch.int32),
                                          _addr(freed_phys_out, "freed_phys_out", torch.int32), _stream())
    check(status, "pe_evict_blocks_cached")


def pe_evict_blocks_ex(desc, opts, scores, block_table, seq_lens, budget_tokens, evicted_logical_out, freed_phys_out):
    L = lib()
    status = _host.evict_blocks_ex(L.addr_evict_blocks_ex, desc, opts, scores, block_table, seq_lens, budget_tokens,
                                   evicted_logical_out, freed_phys_out)
    if status is None:
        status = L.pe_evict_blocks_ex(ctypes.byref(desc), ctypes.byref(opts), _addr_opt(scores, "scores", torch.float32),
                                      _addr(block_table, "block_table", torch.int32), _addr(seq_lens, "seq_lens", torch.int32),
                                      int(budget_tokens), _addr(evicted_logical_out, "evicted_logical_out", torch.int32),
                                      _addr(freed_phys_out, "freed_phys_out", torch.int32), _stream())
    check(status, "pe_evict_blocks_ex")


def pe_paged_decode(desc, q, k_pool, v_pool, block_table, seq_lens, softmax_scale, out, workspace=None):
    L = lib()
    status = _host.paged_decode(L.addr_paged_decode, desc, q, k_pool, v_pool, block_table, seq_lens, softmax_scale, out,
                                workspace)
    if status is None:
        wp, wn = _ws(workspace)
        status = L.pe_paged_decode(ctypes.byref(desc), _addr(q, "q"), _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                   _addr(block_table, "block_table", torch.int32), _addr(seq_lens, "seq_lens", torch.int32),
                                   float(softmax_scale), _addr(out, "out"), wp, wn, _stream())
    check(status, "pe_paged_decode")


def pe_paged_decode_static(desc, q, k_pool, v_pool, block_table, seq_lens, softmax_scale, out):
    check(lib().pe_paged_decode_static(ctypes.byref(desc), _addr(q, "q"), _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                       _addr(block_table, "block_table", torch.int32),
                                       _addr(seq_lens, "seq_lens", torch.int32), float(softmax_scale),
                                       _addr(out, "out"), _stream()), "pe_paged_decode_static")


def pe_append_kv(desc, new_k, new_v, k_pool, v_pool, block_table, seq_lens, freed_phys, spare, spare_used):
    check(lib().pe_append_kv(ctypes.byref(desc), _addr(new_k, "new_k"), _addr(new_v, "new_v"), _addr(k_pool, "k_pool"),
                              _addr(v_pool, "v_pool"), _addr(block_table, "block_table", torch.int32),
                              _addr(seq_lens, "seq_lens", torch.int32), _addr(freed_phys, "freed_phys", torch.int32),
                              _addr(spare, "spare", torch.int32), _addr(spare_used, "spare_used", torch.int32),
                              int(spare.shape[-1]), _stream()), "pe_append_kv")


def pe_append_paged_decode(desc, new_k, new_v, q, k_pool, v_pool, block_table, seq_lens, seq_lens_out, freed_phys, spare,
                           spare_used, softmax_scale, out, workspace=None):
    L = lib()
    status = _host.append_paged_decode(L.addr_append_paged_decode, desc, new_k, new_v, q, k_pool, v_pool, block_table, seq_lens,
                                       seq_lens_out, freed_phys, spare, spare_used, spare, softmax_scale, out, workspace)
    if status is None:
        wp, wn = _ws(workspace)
        status = L.pe_append_paged_decode(ctypes.byref(desc), _addr(new_k, "new_k"), _addr(new_v, "new_v"), _addr(q, "q"),
                                          _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                          _addr(block_table, "block_table", torch.int32),
                                          _addr(seq_lens, "seq_lens", torch.int32),
                                          _addr(seq_lens_out, "seq_lens_out", torch.int32),
                                          _addr(freed_phys, "freed_phys", torch.int32), _addr(spare, "spare", torch.int32),
                                          _addr(spare_used, "spare_used", torch.int32), int(spare.shape[-1]),
                                          float(softmax_scale), _addr(out, "out"), wp, wn, _stream())
    check(status, "pe_append_paged_decode")


def pe_append_paged_decode_layers(desc, num_layers, new_k, new_v, q, k_pool, v_pool, block_table, seq_lens, seq_lens_out,
                                  freed_phys, spare, spare_used, softmax_scale, out, workspace=None):
    L = lib()
    status = _host.append_paged_decode_layers(L.addr_append_paged_decode_layers, desc, num_layers, new_k, new_v, q, k_pool,
                                              v_pool, block_table, seq_lens, seq_lens_out, freed_phys, spare, spare_used, spare,
                                              softmax_scale, out, workspace)
    if status is None:
        wp, wn = _ws(workspace)
        status = L.pe_append_paged_decode_layers(ctypes.byref(desc), int(num_layers), _addr(new_k, "new_k"), _addr(new_v, "new_v"),
                                                 _addr(q, "q"), _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                                 _addr(block_table, "block_table", torch.int32),
                                                 _addr(seq_lens, "seq_lens", torch.int32),
                                                 _addr(seq_lens_out, "seq_lens_out", torch.int32),
                                                 _addr(freed_phys, "freed_phys", torch.int32), _addr(spare, "spare", torch.int32),
                                                 _addr(spare_used, "spare_used", torch.int32), int(spare.shape[-1]),
                                                 float(softmax_scale), _addr(out, "out"), wp, wn, _stream())
    check(status, "pe_append_paged_decode_layers")


def pe_tree_decode(desc, num_drafts, q, k_draft, v_draft, draft_lens, tree_mask, k_pool, v_pool, block_table, seq_lens,
                   softmax_scale, out, workspace=None):
    """tree_mask: int64 (bit j of a word is draft j; bit 63 the sign)."""
    L = lib()
    status = _host.tree_decode(L.addr_tree_decode, desc, num_drafts, q, k_draft, v_draft, draft_lens, tree_mask, k_pool, v_pool,
                               block_table, seq_lens, softmax_scale, out, workspace)
    if status is None:
        wp, wn = _ws(workspace)
        status = L.pe_tree_decode(ctypes.byref(desc), int(num_drafts), _addr(q, "q"), _addr(k_draft, "k_draft"),
                                  _addr(v_draft, "v_draft"), _addr_opt(draft_lens, "draft_lens", torch.int32),
                                  _addr(tree_mask, "tree_mask", torch.int64), _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                  _addr(block_table, "block_table", torch.int32), _addr(seq_lens, "seq_lens", torch.int32),
                                  float(softmax_scale), _addr(out, "out"), wp, wn, _stream())
    check(status, "pe_tree_decode")


def pe_append_path(desc, k_draft, v_draft, path, path_lens, path_done, k_pool, v_pool, block_table, seq_lens, freed_phys, spare,
                   spare_used):
    L = lib()
    status = _host.append_path(L.addr_append_path, desc, k_draft, k_draft, v_draft, path, path, path_lens, path_done, k_pool, v_pool,
                               block_table, seq_lens, freed_phys, spare, spare_used, spare)
    if status is None:
        status = L.pe_append_path(ctypes.byref(desc), int(k_draft.shape[1]), _addr(k_draft, "k_draft"), _addr(v_draft, "v_draft"),
                                  _addr(path, "path", torch.int32), int(path.shape[-1]),
                                  _addr(path_lens, "path_lens", torch.int32), _addr(path_done, "path_done", torch.int32),
                                  _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                  _addr(block_table, "block_table", torch.int32), _addr(seq_lens, "seq_lens", torch.int32),
                                  _addr(freed_phys, "freed_phys", torch.int32), _addr(spare, "spare", torch.int32),
                                  _addr(spare_used, "spare_used", torch.int32), int(spare.shape[-1]), _stream())
    check(status, "pe_append_path")


def pe_page_bounds(desc, k_pool, block_table, seq_lens, recent, bounds_inout):
    L = lib()
    status = _host.page_bounds(L.addr_page_bounds, desc, k_pool, block_table, seq_lens, recent, bounds_inout)
    if status is None:
        status = L.pe_page_bounds(ctypes.byref(desc), _addr(k_pool, "k_pool"), _addr(block_table, "block_table", torch.int32),
                                  _addr(seq_lens, "seq_lens", torch.int32), int(recent), _addr(bounds_inout, "bounds_inout"),
                                  _stream())
    check(status, "pe_page_bounds")


def pe_select_pages(desc, q, bounds, block_table, seq_lens, num_pages, block_table_out, seq_lens_out, page_idx_out, workspace):
    L = lib()
    status = _host.select_pages(L.addr_select_pages, desc, q, bounds, block_table, seq_lens, num_pages, block_table_out, seq_lens_out,
                                page_idx_out, workspace)
    if status is None:
        wp, wn = _ws(workspace)
        status = L.pe_select_pages(ctypes.byref(desc), _addr(q, "q"), _addr(bounds, "bounds"),
                                   _addr(block_table, "block_table", torch.int32), _addr(seq_lens, "seq_lens", torch.int32),
                                   int(num_pages), _addr(block_table_out, "block_table_out", torch.int32),
                                   _addr(seq_lens_out, "seq_lens_out", torch.int32),
                                   _addr_opt(page_idx_out, "page_idx_out", torch.int32), wp, wn, _stream())
    check(status, "pe_select_pages")


def pe_paged_decode_weights(desc, q, k_pool, v_pool, block_table, seq_lens, softmax_scale, decay, weights_in, weights_out, out,
                            workspace=None):
    L = lib()
    status = _host.paged_decode_weights(L.addr_paged_decode_weights, desc, q, k_pool, v_pool, block_table, seq_lens, softmax_scale, decay,
                                        weights_in, weights_out, out, workspace)
    if status is None:
        wp, wn = _ws(workspace)
        status = L.pe_paged_decode_weights(ctypes.byref(desc), _addr(q, "q"), _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                           _addr(block_table, "block_table", torch.int32), _addr(seq_lens, "seq_lens", torch.int32),
                                           float(softmax_scale), float(decay), _addr_opt(weights_in, "weights_in", torch.float32),
                                           _addr(weights_out, "weights_out", torch.float32), _addr(out, "out"), wp, wn, _stream())
    check(status, "pe_paged_decode_weights")


def _with_room(address, t, name, room):
    if t.numel() < room:
        raise ValueError("%s must have room for %d numbers, got %s" % (name, room, tuple(t.shape)))
    return address


def pe_plan_tokens(desc, seq_lens, new_lens, first_positions, total_tokens, budget_tokens, free_pages, free_used, block_table, spare,
                   seq_lens_out, free_used_out, cu_seqlens_out, positions_out, slots_out, admitted=None,
                   spare_used=None, freed_phys=None, only=None, copies=1):
    """What is behind slots_out: the options of pe_plan_tokens_ex."""
    L = lib()
    status = _host.plan_tokens(L.addr_plan_tokens_ex, desc, seq_lens, new_lens, first_positions, total_tokens, budget_tokens, free_pages, free_used,
                               block_table, spare, seq_lens_out, free_used_out, cu_seqlens_out, positions_out, slots_out, admitted, spare_used,
                               freed_phys, only, copies)
    if status is None:
        S, T, n_spare = desc.num_seqs, int(total_tokens), 0 if spare is None else int(spare.shape[-1])
        of_seq = 1 if desc.layout == PE_LAYOUT_SHARED else desc.num_kv_heads
        rows = S * of_seq
        i32 = lambda t, name, room: _with_room(_addr(t, name, torch.int32), t, name, room)   # noqa: E731
        opt = lambda t, name, room: None if t is None else i32(t, name, room)   # noqa: E731
        o = pe_plan_opts(opt(admitted, "admitted", S), opt(spare_used, "spare_used", rows), opt(freed_phys, "freed_phys", rows), opt(only, "only", S),
                         int(copies))
        status = L.pe_plan_tokens_ex(ctypes.byref(desc), ctypes.byref(o), i32(seq_lens, "seq_lens", S), i32(new_lens, "new_lens", S),
                                     opt(first_positions, "first_positions", S), T, int(budget_tokens), i32(free_pages, "free_pages", 1),
                                     int(free_pages.numel()), i32(free_used, "free_used", 1), i32(block_table, "block_table", rows * desc.max_blocks),
                                     opt(spare, "spare", rows * n_spare), n_spare, i32(seq_lens_out, "seq_lens_out", S),
                                     i32(free_used_out, "free_used_out", 1), opt(cu_seqlens_out, "cu_seqlens_out", S + 1),
                                     opt(positions_out, "positions_out", T),
                                     None if slots_out is None else _with_room(_addr(slots_out, "slots_out", torch.int64), slots_out, "slots_out",
                                                                               T * of_seq),
                                     _stream())
    check(status, "pe_plan_tokens")


def make_rope(rotary_dim, base, interleaved=False, scaling=PE_ROPE_PLAIN, factor=1.0, low=1.0, high=4.0, original=8192.0, magnitude=1.0):
    """The frequencies of rotary positions (pe_rope_init), made once for a model."""
    rope = pe_rope()
    check(lib().pe_rope_init(ctypes.byref(rope), int(rotary_dim), PE_ROPE_INTERLEAVED if interleaved else PE_ROPE_HALF, float(base),
                             int(scaling), float(factor), float(low), float(high), float(original), float(magnitude)), "pe_rope_init")
    return rope


def _token_rows(t, name, tokens, heads, desc):
    """Address and token stride of [tokens, heads, D] whose tokens may lie apart (parts of one row a token side by side)."""
    if t is None:
        return None, 0
    if not t.is_cuda:
        raise ValueError(name + " must be a GPU tensor")
    if t.dtype != (torch.float32 if desc.dtype == PE_F32 else torch.bfloat16):
        raise ValueError("%s must be of the cache's dtype, got %s" % (name, t.dtype))
    if tuple(t.shape) != (tokens, heads, desc.head_dim):
        raise ValueError("%s must be [%d, %d, %d], got %s" % (name, tokens, heads, desc.head_dim, tuple(t.shape)))
    dense = heads * desc.head_dim
    if t.numel() and (t.stride(2) != 1 or (heads > 1 and t.stride(1) != desc.head_dim)):
        raise ValueError(name + ": a token's heads must be dense")
    return t.data_ptr(), (t.stride(0) if tokens > 1 else dense)


def pe_rotate(desc, rope, transpose, positions, q, k, v, q_out, k_out, slots=None, k_pool=None, v_pool=None):
    """q, k, v, q_out, k_out: [T, heads, D] with dense heads, tokens any stride apart."""
    L = lib()
    status = _host.rotate(L.addr_rotate, desc, rope, transpose, positions, q, k, v, q_out, k_out, slots, k_pool, v_pool)
    if status is None:
        T = int(positions.numel())
        qp, qs = _token_rows(q, "q", T, desc.num_q_heads, desc)
        kp, ks = _token_rows(k, "k", T, desc.num_kv_heads, desc)
        vp, vs = _token_rows(v if slots is not None else None, "v", T, desc.num_kv_heads, desc)
        qo, qos = _token_rows(q_out, "q_out", T, desc.num_q_heads, desc)
        ko, kos = _token_rows(k_out, "k_out", T, desc.num_kv_heads, desc)
        rows = 1 if desc.layout == PE_LAYOUT_SHARED else desc.num_kv_heads
        if slots is not None and slots.numel() != T * rows:
            raise ValueError("slots must be of %d tokens and %d rows, got %s" % (T, rows, tuple(slots.shape)))
        status = L.pe_rotate(ctypes.byref(desc), ctypes.byref(rope), 1 if transpose else 0, T, _addr(positions, "positions", torch.int32),
                             qp, qs, kp, ks, vp, vs, qo, qos, ko, kos, _addr_opt(slots, "slots", torch.int64),
                             _addr_opt(k_pool, "k_pool"), _addr_opt(v_pool, "v_pool"), _stream())
    check(status, "pe_rotate")


def make_quant_cache(desc, k, v, scales, k_tail, v_tail):
    """The descriptor of an 8-bit cache in these tensors (k, v: one byte an element, uint8 or float8_e4m3fn).  It holds them."""
    shared = desc.layout == PE_LAYOUT_SHARED
    heads = (desc.num_kv_heads,) if shared else ()
    pool = (desc.num_phys_blocks, desc.block_size) + heads + (desc.head_dim,)
    tail = (desc.num_seqs, desc.num_kv_heads, desc.block_size, desc.head_dim)
    wants = (("k", k, pool, None), ("v", v, pool, None), ("scales", scales, (desc.num_phys_blocks,) + heads + (2,), torch.float32),
             ("k_tail", k_tail, tail, torch.float32 if desc.dtype == PE_F32 else torch.bfloat16),
             ("v_tail", v_tail, tail, torch.float32 if desc.dtype == PE_F32 else torch.bfloat16))
    addresses = []
    for name, t, shape, dtype in wants:
        addresses.append(_addr(t, name, dtype))
        if dtype is None and t.dtype not in (torch.uint8, torch.float8_e4m3fn):
            raise ValueError("%s must be uint8 or float8_e4m3fn, got %s" % (name, t.dtype))
        if tuple(t.shape) != shape:
            raise ValueError("%s must be %s, got %s" % (name, shape, tuple(t.shape)))
    cache = pe_quant_cache(*addresses)
    cache.tensors = (k, v, scales, k_tail, v_tail)
    return cache


def pe_quant_pages(desc, cache, k_pool, v_pool, src_table, seq_lens, block_table, scores_out=None, admitted=None):
    """admitted: only the sequences that a plan of tokens let begin or go on (pe_quant_pages_admitted)."""
    L = lib()
    if admitted is None:
        status = _host.quant_pages(L.addr_quant_pages, desc, cache, k_pool, v_pool, src_table, seq_lens, block_table, scores_out)
    else:
        status = _host.quant_pages_admitted(L.addr_quant_pages_admitted, desc, cache, admitted, k_pool, v_pool, src_table, seq_lens, block_table,
                                            scores_out)
    if status is None:
        status = L.pe_quant_pages_admitted(ctypes.byref(desc), ctypes.byref(cache), _addr_opt(admitted, "admitted", torch.int32),
                                           _addr(k_pool, "k_pool"), _addr(v_pool, "v_pool"),
                                           _addr(src_table, "src_table", torch.int32), _addr(seq_lens, "seq_lens", torch.int32),
                                           _addr(block_table, "block_table", torch.int32), _addr_opt(scores_out, "scores_out", torch.float32),
                                           _stream())
    check(status, "pe_quant_pages")


def pe_quant_append(desc, cache, rope, positions, q, q_out, new_k, new_v, block_table, seq_lens, seq_lens_out, freed_phys, spare,
                    spare_used, scores=None):
    """rope None: positions, q and q_out are not looked at."""
    L = lib()
    turned = rope is not None
    if not turned:
        positions = q = q_out = None
    status = _host.quant_append(L.addr_quant_append, desc, cache, rope, positions, q, q_out, new_k, new_v, block_table, seq_lens, seq_lens_out,
                                freed_phys, spare, spare_used, spare, scores)
    if status is None:
        status = L.pe_quant_append(ctypes.byref(desc), ctypes.byref(cache), ctypes.byref(rope) if turned else None,
                                   _addr(positions, "positions", torch.int32) if turned else None, _addr(q, "q") if turned else None,
                                   _addr(q_out, "q_out") if turned else None, _addr(new_k, "new_k"), _addr(new_v, "new_v"),
                                   _addr(block_table, "block_table", torch.int32), _addr(seq_lens, "seq_lens", torch.int32),
                                   _addr(seq_lens_out, "seq_lens_out", torch.int32), _addr(freed_phys, "freed_phys", torch.int32),
                                   _addr(spare, "spare", torch.int32), _addr(spare_used, "spare_used", torch.int32), int(spare.shape[-1]),
                                   _addr_opt(scores, "scores", torch.float32), _stream())
    check(status, "pe_quant_append")


def pe_quant_decode(desc, cache, q, block_table, seq_lens, softmax_scale, out, workspace=None):
    L = lib()
    status = _host.quant_decode(L.addr_quant_decode, desc, cache, q, block_table, seq_lens, softmax_scale, out, workspace)
    if status is None:
        wp, wn = _ws(workspace)
        status = L.pe_quant_decode(ctypes.byref(desc), ctypes.byref(cache), _addr(q, "q"), _addr(block_table, "block_table", torch.int32),
                                   _addr(seq_lens, "seq_lens", torch.int32), float(softmax_scale), _addr(out, "out"), wp, wn, _stream())
    check(status, "pe_quant_decode")
