"""Thin ctypes binding of libchronostitch.so (argument marshalling only).

Every function has the name of the C entry point it calls.  Device buffers
are torch tensors (their data_ptr() is passed through); host arrays are numpy
arrays; the stream is torch's current stream unless one is given.  All the
computation happens in the library's HIP kernels: if the library cannot be
loaded, every call raises.
"""
import ctypes
import os

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "lib", "libchronostitch.so")

CS_OK, CS_ERR_INVALID_ARGUMENT, CS_ERR_UNSUPPORTED, CS_ERR_WORKSPACE_TOO_SMALL, CS_ERR_HIP = range(5)
CS_F32, CS_BF16 = 0, 1
EXPORTS = ("compose_rebase_k", "compose_rebase_k_tokens", "score_deviation_topk_workspace",
           "score_deviation_topk", "selective_attend_scatter_rope_workspace", "selective_attend_scatter_rope",
           "selective_attend_scatter_workspace", "selective_attend_scatter", "selective_attend_scatter_noalloc",
           "compose_rebase_k_paged", "compose_rebase_k_tokens_paged", "compose_load_rebase_k_paged",
           "score_deviation_topk_paged", "selective_attend_scatter_paged",
           "selective_attend_scatter_rope_paged", "batch_plan_pages", "qk_norm_rope_append",
           "tree_attend_paged_workspace", "tree_attend_paged", "tree_commit_paged", "packed_page_bytes", "pack_pages",
           "unpack_rebase_pages", "tree_attend_packed_workspace", "tree_attend_packed", "cs_last_error",
           "cs_trace_enable", "cs_trace_only", "cs_trace_collect", "cs_trace_count", "cs_trace_get",
           "cs_trace_reset")


class CsError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"chronostitch error {code}: {msg}")
        self.code = code


class Geometry(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("sections", ctypes.c_int32 * 3), ("dtype", ctypes.c_int32),
                ("rope_base", ctypes.c_double), ("inv_freq", ctypes.POINTER(ctypes.c_double)),
                ("n_tokens", ctypes.c_int64), ("n_chunks", ctypes.c_int32),
                ("chunk_start", ctypes.POINTER(ctypes.c_int64))]


class Rows(ctypes.Structure):
    """cs_rows: where the heads of rows lie (strides in elements).  Rows.of(t) describes a tensor
    [n_rows, heads, D] whose last dimension is contiguous; the calls take such a tensor too."""
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]

    @classmethod
    def of(cls, t):
        stride = t.stride()
        if len(stride) != 3 or stride[2] != 1:
            raise ValueError("rows are a tensor [n_rows, heads, D] with a contiguous last dimension")
        return cls(t.data_ptr(), stride[0], stride[1])


class _PagePool(ctypes.Structure):
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p), ("n_pages", ctypes.c_int64)]


class _PackedPool(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("n_pages", ctypes.c_int64)]


class _Batch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_requests", "n_rows", "max_blocks", "mask_words", "max_rows")] + [
        (n, ctypes.c_void_p) for n in ("cached_len", "row_start", "block_table", "slot", "coords", "tree_mask")]


class _PagePlan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("new_len", "n_blocks", "n_blocks_out", "free_pages")] + [
        ("n_free", ctypes.c_int32)] + [
        (n, ctypes.c_void_p) for n in ("free_head", "free_head_out", "parent", "coord_base", "status")]


_lib = None


def lib():
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        G = ctypes.POINTER(Geometry)
        L.compose_rebase_k.argtypes = [G, vp, vp, vp, vp, vp]
        L.compose_rebase_k_tokens.argtypes = [G, vp, vp, vp]
        L.score_deviation_topk_workspace.argtypes = [G, ctypes.POINTER(sz)]
        L.score_deviation_topk.argtypes = [G, vp, i32, vp, ctypes.c_double, vp, vp,
                                           ctypes.POINTER(i64), vp, sz, vp]
        L.selective_attend_scatter_workspace.argtypes = [G, i64, i32, ctypes.POINTER(sz)]
        L.selective_attend_scatter_rope_workspace.argtypes = [G, i64, i32, ctypes.POINTER(sz)]
        L.selective_attend_scatter_rope.argtypes = [G, vp, vp, i32, i32, vp, i64, vp, vp, vp, vp, vp, vp,
                                                    vp, sz, vp]
        L.selective_attend_scatter.argtypes = [G, vp, vp, i32, i32, vp, i64, vp, vp, vp, vp, vp,
                                               vp, sz, vp]
        L.selective_attend_scatter_noalloc.argtypes = [G, vp, vp, i32, i32, vp, i64, vp, vp, vp, vp, vp, vp]
        L.compose_rebase_k_paged.argtypes = [G, vp, vp, vp, vp, vp]
        L.compose_rebase_k_tokens_paged.argtypes = [G, vp, vp, vp]
        L.compose_load_rebase_k_paged.argtypes = [G, vp, vp, vp, vp, vp, vp, vp]
        L.score_deviation_topk_paged.argtypes = [G, vp, i32, vp, ctypes.c_double, vp, vp,
                                                 ctypes.POINTER(i64), vp, sz, vp]
        L.selective_attend_scatter_paged.argtypes = [G, vp, vp, i32, i32, vp, i64, vp, vp, vp, vp, vp,
                                                     vp, sz, vp]
        L.selective_attend_scatter_rope_paged.argtypes = [G, vp, vp, i32, i32, vp, i64, vp, vp, vp, vp, vp,
                                                          vp, vp, sz, vp]
        B, R = ctypes.POINTER(_Batch), ctypes.POINTER(Rows)
        L.batch_plan_pages.argtypes = [G, i64, B, ctypes.POINTER(_PagePlan), vp]
        L.qk_norm_rope_append.argtypes = [G, ctypes.POINTER(_PagePool), i32, B, R, R, R, vp, vp, ctypes.c_float, R, vp]
        L.tree_attend_paged_workspace.argtypes = [G, B, ctypes.POINTER(sz)]
        L.tree_attend_paged.argtypes = [G, ctypes.POINTER(_PagePool), i32, B, R, R, vp, vp, sz, vp]
        L.tree_commit_paged.argtypes = [G, ctypes.POINTER(_PagePool), i32, i32, B, vp, i32, vp, vp, vp]
        K = ctypes.POINTER(_PackedPool)
        L.packed_page_bytes.argtypes = [G, ctypes.POINTER(sz)]
        L.pack_pages.argtypes = [G, ctypes.POINTER(_PagePool), K, i32, i32, vp, vp, i32, vp]
        L.unpack_rebase_pages.argtypes = [G, K, ctypes.POINTER(_PagePool), i32, i32, vp, vp, vp, i32, vp]
        L.tree_attend_packed_workspace.argtypes = [G, B, ctypes.POINTER(sz)]
        L.tree_attend_packed.argtypes = [G, ctypes.POINTER(_PagePool), K, i32, B, vp, i32, i32, R, R, vp, vp, sz, vp]
        L.cs_last_error.restype = ctypes.c_char_p
        L.cs_trace_enable.argtypes = [i32]
        L.cs_trace_only.argtypes = [ctypes.c_char_p]
        L.cs_trace_get.argtypes = [i32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(i64),
                                   ctypes.POINTER(ctypes.c_double)]
        L.cs_trace_count.restype = i32
        for name in ("compose_rebase_k", "compose_rebase_k_tokens", "score_deviation_topk_workspace",
                     "score_deviation_topk",
                     "selective_attend_scatter_workspace", "selective_attend_scatter",
                     "selective_attend_scatter_noalloc",
                     "selective_attend_scatter_rope_workspace", "selective_attend_scatter_rope",
                     "compose_rebase_k_paged", "compose_rebase_k_tokens_paged", "score_deviation_topk_paged",
                     "compose_load_rebase_k_paged",
                     "selective_attend_scatter_paged", "selective_attend_scatter_rope_paged",
                     "batch_plan_pages", "qk_norm_rope_append", "tree_attend_paged_workspace",
                     "tree_attend_paged", "tree_commit_paged", "packed_page_bytes", "pack_pages",
                     "unpack_rebase_pages", "tree_attend_packed_workspace", "tree_attend_packed",
                     "cs_trace_enable", "cs_trace_only", "cs_trace_collect", "cs_trace_get"):
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(code):
    if code != CS_OK:
        raise CsError(code, lib().cs_last_error().decode())


def _int32(x, name):
    """x as an int of 32 bits (of a larger one ctypes would take the low bits without a word)."""
    if type(x) is not int:
        x = int(x)
    if -0x80000000 <= x <= 0x7fffffff:
        return x
    raise ValueError(f"{name} must be a whole number of 32 bits, got {x}")


def _layers(begin, end):
    if type(begin) is type(end) is int and 0 <= begin <= end <= 0x7fffffff:  # (0.1 us less than one by one)
        return begin, end
    return _int32(begin, "layer_begin"), _int32(end, "layer_end")


class Geo:
    """Owns a cs_geometry and the host arrays it points to."""

    def __init__(self, n_layers, n_q_heads, n_kv_heads, head_dim, sections, dtype, chunk_start,
                 rope_base=1.0e6, inv_freq=None):
        self.chunk_start = np.ascontiguousarray(chunk_start, dtype=np.int64)
        self.inv_freq = None if inv_freq is None else np.ascontiguousarray(inv_freq, dtype=np.float64)
        self.g = Geometry()
        self.g.n_layers, self.g.n_q_heads, self.g.n_kv_heads, self.g.head_dim = (
            n_layers, n_q_heads, n_kv_heads, head_dim)
        self.g.sections = (ctypes.c_int32 * 3)(*sections)
        self.g.dtype = {"bf16": CS_BF16, "f32": CS_F32}.get(dtype, dtype)
        self.g.rope_base = rope_base
        self.g.inv_freq = (self.inv_freq.ctypes.data_as(ctypes.POINTER(ctypes.c_double))
                           if self.inv_freq is not None else None)
        self.g.n_tokens = int(self.chunk_start[-1])
        self.g.n_chunks = len(self.chunk_start) - 1
        self.g.chunk_start = self.chunk_start.ctypes.data_as(ctypes.POINTER(ctypes.c_int64))

    @classmethod
    def from_workload(cls, w):
        return cls(w.n_layers, w.n_q_heads, w.n_kv_heads, w.head_dim, w.sections, w.dtype,
                   w.chunk_start, w.base)

    @property
    def ref(self):
        return ctypes.byref(self.g)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


_raw_stream = None  # torch's lookup of a device's current stream as an address


def _stream(stream, device=None):
    """The address of the stream given, or of torch's current one (looked up without making a
    Stream object where torch has that call: 0.3 us instead of 3)."""
    if stream is not None:
        return stream
    global _raw_stream
    import torch
    if _raw_stream is None:
        torch.cuda.current_stream()  # (initialises the runtime, and says why where it cannot)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)
    return _raw_stream(torch.cuda.current_device() if device is None else device)


def compose_rebase_k(geo, k_cache, chunk_offsets, local_coords=None, want_global=False, stream=None):
    """Re-base k_cache in place; returns global coords [T,3] (int32) when asked."""
    off = np.ascontiguousarray(chunk_offsets, dtype=np.int32)
    loc = None if local_coords is None else np.ascontiguousarray(local_coords, dtype=np.int32)
    glob = np.empty_like(loc) if (want_global and loc is not None) else None
    _check(lib().compose_rebase_k(geo.ref, _ptr(k_cache), off.ctypes.data_as(ctypes.c_void_p),
                                  None if loc is None else loc.ctypes.data_as(ctypes.c_void_p),
                                  None if glob is None else glob.ctypes.data_as(ctypes.c_void_p),
                                  _stream(stream)))
    return glob


def compose_rebase_k_tokens(geo, k_cache, token_offsets, stream=None):
    """Re-base k_cache in place by a per-token offset (DEVICE int32 [T, 3] tensor)."""
    _check(lib().compose_rebase_k_tokens(geo.ref, _ptr(k_cache), _ptr(token_offsets), _stream(stream)))


def score_deviation_topk_workspace(geo):
    n = ctypes.c_size_t(0)
    _check(lib().score_deviation_topk_workspace(geo.ref, ctypes.byref(n)))
    return n.value


def score_deviation_topk(geo, k_cache, score_layer, k_fresh, rho, scores, sel_idx, workspace=None,
                         stream=None):
    """Scores later-chunk tokens and selects the top rho; returns n_sel."""
    k = ctypes.c_int64(0)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().score_deviation_topk(geo.ref, _ptr(k_cache), _int32(score_layer, "score_layer"), _ptr(k_fresh),
                                      float(rho), _ptr(scores), _ptr(sel_idx), ctypes.byref(k),
                                      _ptr(workspace), ws_bytes, _stream(stream)))
    return k.value


def selective_attend_scatter_workspace(geo, n_sel, n_layers_per_call):
    n = ctypes.c_size_t(0)
    _check(lib().selective_attend_scatter_workspace(geo.ref, int(n_sel),
                                                    _int32(n_layers_per_call, "n_layers_per_call"), ctypes.byref(n)))
    return n.value


def selective_attend_scatter(geo, k_cache, v_cache, layer_begin, layer_end, sel_idx, n_sel, q_fresh,
                             k_fresh, v_fresh, out, lse=None, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().selective_attend_scatter(geo.ref, _ptr(k_cache), _ptr(v_cache), *_layers(layer_begin, layer_end),
                                          _ptr(sel_idx), int(n_sel), _ptr(q_fresh),
                                          _ptr(k_fresh), _ptr(v_fresh), _ptr(out), _ptr(lse),
                                          _ptr(workspace), ws_bytes, _stream(stream)))


def selective_attend_scatter_noalloc(geo, k_cache, v_cache, layer_begin, layer_end, sel_idx, n_sel, q_fresh,
                                     k_fresh, v_fresh, out, lse=None, stream=None):
    """selective_attend_scatter with the library's own per-GPU scratch array (no workspace)."""
    _check(lib().selective_attend_scatter_noalloc(geo.ref, _ptr(k_cache), _ptr(v_cache),
                                                  *_layers(layer_begin, layer_end), _ptr(sel_idx), int(n_sel), _ptr(q_fresh),
                                                  _ptr(k_fresh), _ptr(v_fresh), _ptr(out), _ptr(lse),
                                                  _stream(stream)))


# ---------------------------------------------------------------- tracing
def cs_trace_enable(on=True):
    _check(lib().cs_trace_enable(1 if on else 0))


def cs_trace_only(names=None):
    """Trace only the kernels named (an iterable of names, or None for all)."""
    _check(lib().cs_trace_only(None if names is None else ",".join(names).encode()))


def cs_trace_reset():
    lib().cs_trace_reset()


def cs_trace_collect():
    """Synchronises pending trace events; returns {kernel: (launches, total_ms)}."""
    L = lib()
    _check(L.cs_trace_collect())
    out = {}
    for i in range(L.cs_trace_count()):
        name = ctypes.c_char_p()
        n = ctypes.c_int64()
        ms = ctypes.c_double()
        _check(L.cs_trace_get(i, ctypes.byref(name), ctypes.byref(n), ctypes.byref(ms)))
        out[name.value.decode()] = (n.value, ms.value)
    return out


def selective_attend_scatter_rope_workspace(geo, n_sel, n_layers_per_call):
    n = ctypes.c_size_t(0)
    _check(lib().selective_attend_scatter_rope_workspace(geo.ref, int(n_sel),
                                                         _int32(n_layers_per_call, "n_layers_per_call"),
                                                         ctypes.byref(n)))
    return n.value


def selective_attend_scatter_rope(geo, k_cache, v_cache, layer_begin, layer_end, sel_idx, n_sel, q_pre, k_pre,
                                  v_fresh, coords, out, lse=None, workspace=None, stream=None):
    """selective_attend_scatter on pre-rotary fresh Q/K, rotated at the global coordinates (DEVICE int32 [T, 3])."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().selective_attend_scatter_rope(geo.ref, _ptr(k_cache), _ptr(v_cache), *_layers(layer_begin, layer_end),
                                               _ptr(sel_idx), int(n_sel), _ptr(q_pre), _ptr(k_pre),
                                               _ptr(v_fresh), _ptr(coords), _ptr(out), _ptr(lse), _ptr(workspace),
                                               ws_bytes, _stream(stream)))


# ---------------------------------------------------------------- paged cache
def _chunks(ts):
    """HOST array of the chunk tensors' device pointers (None stays NULL)."""
    if ts is None:
        return None
    arr = (ctypes.c_void_p * max(1, len(ts)))(*[None if t is None else t.data_ptr() for t in ts])
    return arr


def compose_rebase_k_paged(geo, k_chunks, chunk_offsets, local_coords=None, want_global=False, stream=None):
    """compose_rebase_k on a cache held as one tensor per chunk ([L, H_kv, len_c, D] each)."""
    off = np.ascontiguousarray(chunk_offsets, dtype=np.int32)
    loc = None if local_coords is None else np.ascontiguousarray(local_coords, dtype=np.int32)
    glob = np.empty_like(loc) if (want_global and loc is not None) else None
    _check(lib().compose_rebase_k_paged(geo.ref, _chunks(k_chunks), off.ctypes.data_as(ctypes.c_void_p),
                                        None if loc is None else loc.ctypes.data_as(ctypes.c_void_p),
                                        None if glob is None else glob.ctypes.data_as(ctypes.c_void_p),
                                        _stream(stream)))
    return glob


def compose_load_rebase_k_paged(geo, k_chunks, v_chunks, k_host, v_host, chunk_offsets, copy_stream=None,
                                stream=None):
    """Copy each chunk's K and V from host tensors (page-locked for overlap) into the device chunk
    tensors on copy_stream, re-basing each chunk's keys on stream as soon as they have landed."""
    off = np.ascontiguousarray(chunk_offsets, dtype=np.int32)
    _check(lib().compose_load_rebase_k_paged(geo.ref, _chunks(k_chunks), _chunks(v_chunks), _chunks(k_host),
                                             _chunks(v_host), off.ctypes.data_as(ctypes.c_void_p),
                                             None if copy_stream is None else ctypes.c_void_p(copy_stream),
                                             _stream(stream)))


def compose_rebase_k_tokens_paged(geo, k_chunks, token_offsets, stream=None):
    _check(lib().compose_rebase_k_tokens_paged(geo.ref, _chunks(k_chunks), _ptr(token_offsets), _stream(stream)))


def score_deviation_topk_paged(geo, k_chunks, score_layer, k_fresh, rho, scores, sel_idx, workspace=None,
                               stream=None):
    k = ctypes.c_int64(0)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().score_deviation_topk_paged(geo.ref, _chunks(k_chunks), _int32(score_layer, "score_layer"),
                                            _ptr(k_fresh),
                                            float(rho), _ptr(scores), _ptr(sel_idx), ctypes.byref(k),
                                            _ptr(workspace), ws_bytes, _stream(stream)))
    return k.value


def selective_attend_scatter_paged(geo, k_chunks, v_chunks, layer_begin, layer_end, sel_idx, n_sel, q_fresh,
                                   k_fresh, v_fresh, out, lse=None, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().selective_attend_scatter_paged(geo.ref, _chunks(k_chunks), _chunks(v_chunks),
                                                *_layers(layer_begin, layer_end), _ptr(sel_idx), int(n_sel), _ptr(q_fresh),
                                                _ptr(k_fresh), _ptr(v_fresh), _ptr(out), _ptr(lse),
                                                _ptr(workspace), ws_bytes, _stream(stream)))


def selective_attend_scatter_rope_paged(geo, k_chunks, v_chunks, layer_begin, layer_end, sel_idx, n_sel, q_pre,
                                        k_pre, v_fresh, coords, out, lse=None, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().selective_attend_scatter_rope_paged(geo.ref, _chunks(k_chunks), _chunks(v_chunks),
                                                     *_layers(layer_begin, layer_end), _ptr(sel_idx), int(n_sel),
                                                     _ptr(q_pre), _ptr(k_pre), _ptr(v_fresh), _ptr(coords),
                                                     _ptr(out), _ptr(lse), _ptr(workspace), ws_bytes,
                                                     _stream(stream)))


# ---------------------------------------------------------------- batches over a pool of pages
def _torch_dtype(dtype, _cache={}):
    """torch's type of a geometry's dtype, or of a type's name."""
    t = _cache.get(dtype)
    if t is None:
        import torch
        _cache.update({CS_F32: torch.float32, CS_BF16: torch.bfloat16, "int32": torch.int32, "int64": torch.int64,
                       "float32": torch.float32, "uint8": torch.uint8})
        t = _cache[dtype]
    return t


def _array(t, name, dtype, shape, device, optional=False):
    """Address of a dense tensor of the given type and shape (None in the shape: any size) on a device (None: any)."""
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is required")
    have = t.shape
    if t.dtype is not _torch_dtype(dtype) or not t.is_contiguous() or (have != shape and (
            len(have) != len(shape) or any(w is not None and w != h for h, w in zip(have, shape)))):
        raise ValueError(f"{name} must be a contiguous {_torch_dtype(dtype)} tensor of shape {shape}, got {t.dtype} "
                         f"{tuple(have)}")
    if not t.is_cuda or (device is not None and t.get_device() != device):
        raise ValueError(f"{name} must be in the memory of the batch's device")
    return t.data_ptr()


def _page_key(geo):
    return geo.g.n_layers, geo.g.n_kv_heads, geo.g.n_tokens, geo.g.head_dim, geo.g.dtype


class PagePool:
    """cs_page_pool: the key and value pages, tensors [n_pages, L, H_kv, P, D] of the page geometry's type."""

    def __init__(self, geo, k_pages, v_pages):
        shape = (None, geo.g.n_layers, geo.g.n_kv_heads, geo.g.n_tokens, geo.g.head_dim)
        self.tensors, self.geo = (k_pages, v_pages), geo
        self.c = _PagePool()
        self.c.k_pages = _array(k_pages, "k_pages", geo.g.dtype, shape, None)
        self.device = k_pages.get_device()
        self.c.v_pages = _array(v_pages, "v_pages", geo.g.dtype, (k_pages.shape[0],) + shape[1:], self.device)
        self.c.n_pages = k_pages.shape[0]


class Batch:
    """cs_batch: the arrays of a step.  int32 tensors cached_len [B], row_start [B + 1], block_table
    [B, max_blocks], slot [n_rows], coords [n_rows, 3]; tree_mask int64 [n_rows, mask_words] or None."""

    def __init__(self, cached_len, row_start, block_table, slot, coords, tree_mask=None, max_rows=0):
        n, rows = cached_len.shape[0], slot.shape[0]
        if tree_mask is not None and 0 in tree_mask.shape[1:]:  # (its address would be NULL: no mask)
            raise ValueError("tree_mask must have at least one word a row")
        self.tensors = (cached_len, row_start, block_table, slot, coords, tree_mask)
        c = self.c = _Batch()
        c.n_requests, c.n_rows = _int32(n, "n_requests"), _int32(rows, "n_rows")
        c.max_blocks, c.max_rows = _int32(block_table.shape[1], "max_blocks"), _int32(max_rows, "max_rows")
        c.mask_words = 0 if tree_mask is None else _int32(tree_mask.shape[1], "mask_words")
        c.cached_len = _array(cached_len, "cached_len", "int32", (n,), None)
        dev = self.device = cached_len.get_device()
        c.row_start = _array(row_start, "row_start", "int32", (n + 1,), dev)
        c.block_table = _array(block_table, "block_table", "int32", (n, None), dev)
        c.slot = _array(slot, "slot", "int32", (rows,), dev)
        c.coords = _array(coords, "coords", "int32", (rows, 3), dev)
        c.tree_mask = _array(tree_mask, "tree_mask", "int64", (rows, None), dev, optional=True)


class PagePlan:
    """cs_page_plan: what batch_plan_pages reads and writes beside the batch, int32 tensors new_len, n_blocks,
    n_blocks_out, coord_base [B], free_pages [n_free], free_head, free_head_out, status [1], parent [n_rows]."""

    def __init__(self, new_len, n_blocks, n_blocks_out, free_pages, free_head, free_head_out, status, parent=None,
                 coord_base=None):
        n = new_len.shape[0]
        self.tensors = (new_len, n_blocks, n_blocks_out, free_pages, free_head, free_head_out, status, parent,
                        coord_base)
        c = self.c = _PagePlan()
        c.new_len = _array(new_len, "new_len", "int32", (n,), None)
        dev = self.device = new_len.get_device()
        c.n_blocks = _array(n_blocks, "n_blocks", "int32", (n,), dev)
        c.n_blocks_out = _array(n_blocks_out, "n_blocks_out", "int32", (n,), dev)
        c.free_pages = _array(free_pages, "free_pages", "int32", (None,), dev)
        c.n_free = _int32(free_pages.shape[0], "n_free")
        c.free_head = _array(free_head, "free_head", "int32", (1,), dev)
        c.free_head_out = _array(free_head_out, "free_head_out", "int32", (1,), dev)
        c.status = _array(status, "status", "int32", (1,), dev)
        c.parent = _array(parent, "parent", "int32", (None,), dev, optional=True)
        c.coord_base = _array(coord_base, "coord_base", "int32", (n,), dev, optional=True)
        self.n_requests, self.n_parents = n, None if parent is None else parent.shape[0]


def _row_arg(t, name, geo, batch, heads):
    """A Rows, or a tensor that is checked and described."""
    if isinstance(t, Rows):
        return t
    shape, d = t.shape, geo.g.head_dim
    if t.dtype is not _torch_dtype(geo.g.dtype) or t.get_device() != batch.device or len(shape) != 3 or (
            shape[0] < batch.c.n_rows or shape[1] != heads or shape[2] != d):
        raise ValueError(f"{name} must be a {_torch_dtype(geo.g.dtype)} tensor [{batch.c.n_rows}, {heads}, {d}] on the "
                         f"batch's device, got {t.dtype} {tuple(shape)}")
    return Rows.of(t)


def _batch_stream(stream, batch, other, geo=None):
    """The stream, after a look at the devices (the batch's, the pool's or plan's, the current one) and at the
    pool's geometry, where one is given."""
    import torch
    device = torch.cuda.current_device()
    if batch.device != device or other.device != device:
        raise ValueError(f"the batch is on device {batch.device}, its pool or plan on {other.device}, and the current "
                         f"device is {device}")
    if geo is not None and geo is not other.geo and _page_key(geo) != _page_key(other.geo):
        raise ValueError("the pool's pages are of another geometry")
    return _stream(stream, device)


def batch_plan_pages(geo, n_pages, batch, plan, stream=None):
    """Block tables, slots, coordinates and tree masks of the step, into the batch's arrays and the plan's outputs."""
    if plan.n_requests != batch.c.n_requests or plan.n_parents not in (None, batch.c.n_rows):
        raise ValueError("the plan's tensors are of another batch")
    _check(lib().batch_plan_pages(geo.ref, int(n_pages), ctypes.byref(batch.c), ctypes.byref(plan.c),
                                  _batch_stream(stream, batch, plan)))


def qk_norm_rope_append(geo, pool, layer, batch, q, k, v, q_out, q_weight=None, k_weight=None, eps=1e-6,
                        stream=None):
    """Norm and rotation of the step's queries (to q_out) and keys; keys and values to their slots in `layer`."""
    hq, hkv = geo.g.n_q_heads, geo.g.n_kv_heads
    w = [_array(x, "a weight", geo.g.dtype, (geo.g.head_dim,), batch.device, optional=True)
         for x in (q_weight, k_weight)]
    _check(lib().qk_norm_rope_append(geo.ref, ctypes.byref(pool.c), _int32(layer, "layer"), ctypes.byref(batch.c),
                                     ctypes.byref(_row_arg(q, "q", geo, batch, hq)),
                                     ctypes.byref(_row_arg(k, "k", geo, batch, hkv)),
                                     ctypes.byref(_row_arg(v, "v", geo, batch, hkv)), w[0], w[1], float(eps),
                                     ctypes.byref(_row_arg(q_out, "q_out", geo, batch, hq)),
                                     _batch_stream(stream, batch, pool, geo)))


def tree_attend_paged_workspace(geo, batch):
    n = ctypes.c_size_t(0)
    _check(lib().tree_attend_paged_workspace(geo.ref, ctypes.byref(batch.c), ctypes.byref(n)))
    return n.value


def tree_attend_paged(geo, pool, layer, batch, q, out, lse=None, workspace=None, stream=None):
    """Attention of the step's rows over their requests' pages; lse: float32 [n_rows, H_q] or None."""
    hq = geo.g.n_q_heads
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if workspace is not None and (workspace.get_device() != batch.device or not workspace.is_contiguous()):
        raise ValueError("workspace must be contiguous memory of the batch's device")
    if lse is not None and lse.shape[0] < batch.c.n_rows:
        raise ValueError("lse has fewer rows than the batch")
    _check(lib().tree_attend_paged(geo.ref, ctypes.byref(pool.c), _int32(layer, "layer"), ctypes.byref(batch.c),
                                   ctypes.byref(_row_arg(q, "q", geo, batch, hq)),
                                   ctypes.byref(_row_arg(out, "out", geo, batch, hq)),
                                   _array(lse, "lse", "float32", (None, hq), batch.device, optional=True),
                                   _ptr(workspace), ws_bytes, _batch_stream(stream, batch, pool, geo)))


def tree_commit_paged(geo, pool, layer_begin, layer_end, batch, accepted, n_accepted, cached_len_out=None,
                      stream=None):
    """Moves the rows of accepted int32 [B, max_accept] (n_accepted [B] of them) behind the cached tokens."""
    n = batch.c.n_requests
    _check(lib().tree_commit_paged(geo.ref, ctypes.byref(pool.c), *_layers(layer_begin, layer_end),
                                   ctypes.byref(batch.c), _array(accepted, "accepted", "int32", (n, None), batch.device),
                                   _int32(accepted.shape[1], "max_accept"),
                                   _array(n_accepted, "n_accepted", "int32", (n,), batch.device),
                                   _array(cached_len_out, "cached_len_out", "int32", (n,), batch.device, optional=True),
                                   _batch_stream(stream, batch, pool, geo)))


# ---------------------------------------------------------------- memories held in 4 bits
def packed_page_bytes(geo):
    n = ctypes.c_size_t(0)
    _check(lib().packed_page_bytes(geo.ref, ctypes.byref(n)))
    return n.value


class PackedPool:
    """cs_packed_pool: uint8 tensor [n_pages, packed_page_bytes(geo)]."""

    def __init__(self, geo, pages):
        self.tensors, self.geo = (pages,), geo
        self.c = _PackedPool()
        self.c.pages = _array(pages, "pages", "uint8", (None, packed_page_bytes(geo)), None)
        self.device = pages.get_device()
        self.c.n_pages = pages.shape[0]


def _pages_stream(stream, geo, pool, packed):
    """The stream, after a look at the pools' geometries and devices (and the current one)."""
    for p in (pool, packed):
        if geo is not p.geo and _page_key(geo) != _page_key(p.geo):
            raise ValueError("the pool's pages are of another geometry")
    return _batch_stream(stream, pool, packed)


def pack_pages(geo, pool, packed, layer_begin, layer_end, src, dst, stream=None):
    """Pages src of the pool into pages dst of the packed pool (int32 tensors [n]), in layers of a range."""
    n = _int32(src.shape[0], "n")
    begin, end = _layers(layer_begin, layer_end)
    _check(lib().pack_pages(geo.ref, ctypes.byref(pool.c), ctypes.byref(packed.c), begin, end,
                            _array(src, "src", "int32", (n,), pool.device), _array(dst, "dst", "int32", (n,), pool.device),
                            n, _pages_stream(stream, geo, pool, packed)))


def unpack_rebase_pages(geo, packed, pool, layer_begin, layer_end, src, dst, offsets=None, stream=None):
    """Pages src of the packed pool into pages dst of the pool, keys turned by offsets (int32 tensor [n, 3])."""
    n = _int32(src.shape[0], "n")
    begin, end = _layers(layer_begin, layer_end)
    _check(lib().unpack_rebase_pages(geo.ref, ctypes.byref(packed.c), ctypes.byref(pool.c),
                                     begin, end, _array(src, "src", "int32", (n,), pool.device),
                                     _array(dst, "dst", "int32", (n,), pool.device),
                                     _array(offsets, "offsets", "int32", (n, 3), pool.device, optional=True), n,
                                     _pages_stream(stream, geo, pool, packed)))


def tree_attend_packed_workspace(geo, batch):
    n = ctypes.c_size_t(0)
    _check(lib().tree_attend_packed_workspace(geo.ref, ctypes.byref(batch.c), ctypes.byref(n)))
    return n.value


def tree_attend_packed(geo, pool, packed, layer, batch, packed_blocks, q, out, lse=None, workspace=None, sinks=0,
                       window=0, stream=None):
    """tree_attend_paged where the first packed_blocks (int32 [B], or None) pages of each request are pages of packed,
    and where, with window > 0, a row sees the first `sinks` and the last `window` of its tokens."""
    layer, sinks, window = _int32(layer, "layer"), _int32(sinks, "sinks"), _int32(window, "window")
    hq = geo.g.n_q_heads
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if workspace is not None and (workspace.get_device() != batch.device or not workspace.is_contiguous()):
        raise ValueError("workspace must be contiguous memory of the batch's device")
    if lse is not None and lse.shape[0] < batch.c.n_rows:
        raise ValueError("lse has fewer rows than the batch")
    if packed is None and packed_blocks is not None:
        raise ValueError("packed_blocks needs a packed pool")
    if packed is not None:
        _batch_stream(0, batch, packed, geo)
    _check(lib().tree_attend_packed(geo.ref, ctypes.byref(pool.c), None if packed is None else ctypes.byref(packed.c),
                                    layer, ctypes.byref(batch.c),
                                    _array(packed_blocks, "packed_blocks", "int32", (batch.c.n_requests,), batch.device,
                                           optional=True), sinks, window,
                                    ctypes.byref(_row_arg(q, "q", geo, batch, hq)),
                                    ctypes.byref(_row_arg(out, "out", geo, batch, hq)),
                                    _array(lse, "lse", "float32", (None, hq), batch.device, optional=True),
                                    _ptr(workspace), ws_bytes, _batch_stream(stream, batch, pool, geo)))
