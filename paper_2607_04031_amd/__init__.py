"""Tile-major GEMM for AMD MI355X (gfx950): Python binding over libtl's C ABI.

Every step of the path runs in libtl's HIP kernels; this module only marshals
arguments (torch tensors -> device pointers, the current torch stream -> a
hipStream_t) and turns status codes into exceptions.  The entry points carry
the C names and argument order of ``include/tl.h``:

    tl_tile_bytes(rows, cols, elem_bytes, G, block_rows) -> int
    tl_repack(src, dst, rows, cols, elem_bytes, G, block_rows, stream=None)
    tl_unpack(src_tm, dst, rows, cols, elem_bytes, G, block_rows, stream=None)
    tl_gemm(A, W, C, M, N, K, layout, fetch_mode, stream=None)
    tl_gemm_noalloc(A, W, C, M, N, K, layout, fetch_mode, stream=None)
    tl_gemm_plan(M, N, K, layout, fetch_mode) -> dict
    tl_gemm_grouped / tl_gemm_grouped_swiglu (..., layout, fetch_mode, stream=None)
    tl_read_amp(M, N, K, tile_m, tile_n, tile_k, layout, G) -> dict
    tl_kv_bytes / tl_kv_append / tl_kv_read / tl_kv_keep (a paged key/value cache)
    tl_attn (attention over it), tl_verify (drafted tokens)
    tl_fetch_counter_read(stream=None) -> int
    tl_release()
    tl_strerror(status) -> str

Pointer arguments accept a torch CUDA tensor or a raw integer address.
``layout`` is a :class:`LayoutDesc` (or a dict of its fields).  A few helpers
(``repack``, ``gemm``, ``layout``; ``kv_cache``, ``rope``, ``kv_append``,
``kv_read``, ``kv_keep``, ``attention``, ``verify``) build outputs and
descriptors for callers that just hold tensors.

If libtl.so has not been built the first call raises ``ImportError``; there is
no fallback path of any kind.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtl.so")
CALLS_PATH = os.path.join(_HERE, "_tl_torch.so")

TL_OK, TL_EINVAL, TL_EUNSUPPORTED, TL_EHIP, TL_ENOMEM, TL_ESCRATCH = 0, -1, -2, -3, -4, -5
TL_NOALLOC_SCRATCH_BYTES = 64 << 20
TL_LAYOUT_NK_ROW, TL_LAYOUT_KN_ROW, TL_LAYOUT_TILE = 0, 1, 2
TL_OUT_F32, TL_OUT_BF16 = 0, 1
TL_FETCH_NATIVE, TL_FETCH_BLOCK, TL_FETCH_COUNT = 0, 1, 0x100

EXPORTED = ("tl_tile_bytes", "tl_repack", "tl_unpack", "tl_gemm", "tl_gemm_noalloc", "tl_gemm_w8", "tl_gemm_plan", "tl_gemm_grouped", "tl_gemm_grouped_swiglu", "tl_read_amp",
            "tl_view_offsets", "tl_view_load", "tl_prefetch_degree", "tl_gemm_lgms", "tl_lgms_occupancy",
            "tl_kv_bytes", "tl_kv_append", "tl_kv_read", "tl_kv_keep", "tl_attn", "tl_verify",
            "tl_stream_read", "tl_fetch_counter_read", "tl_release", "tl_strerror")
TL_VIEW_MAX_RANK = 5
TL_IN_F32, TL_IN_BF16 = 0, 1


class View(ctypes.Structure):
    _fields_ = [("rank", ctypes.c_int32),
                ("box", ctypes.c_int32 * 5),
                ("strides", ctypes.c_int64 * 5),
                ("coords", ctypes.c_int64 * 5)]


def view(strides, coords, box) -> View:
    """tl_view of rank len(box); dimension 0 is the contiguous one."""
    v = View()
    v.rank = len(box)
    assert len(strides) == len(coords) == v.rank <= 5
    for d in range(v.rank):
        v.box[d], v.strides[d], v.coords[d] = int(box[d]), int(strides[d]), int(coords[d])
    return v


class LayoutDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32),
                ("elem_bytes", ctypes.c_int32),
                ("G", ctypes.c_int64),
                ("block_rows", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32),
                ("tile_m", ctypes.c_int32),
                ("tile_n", ctypes.c_int32),
                ("tile_k", ctypes.c_int32),
                ("split_k", ctypes.c_int32)]


class Amp(ctypes.Structure):
    _fields_ = [("compute_tiles", ctypes.c_int64),
                ("requests", ctypes.c_int64),
                ("fetched_bytes", ctypes.c_int64),
                ("useful_bytes", ctypes.c_int64),
                ("unique_blocks", ctypes.c_int64),
                ("min_blocks_per_tile", ctypes.c_int64),
                ("max_blocks_per_tile", ctypes.c_int64),
                ("amp", ctypes.c_double)]


class Plan(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32),
                ("tile_m", ctypes.c_int32),
                ("tile_n", ctypes.c_int32),
                ("tile_k", ctypes.c_int32),
                ("split_k", ctypes.c_int32),
                ("waves", ctypes.c_int32),
                ("workgroups", ctypes.c_int64),
                ("workspace_bytes", ctypes.c_int64)]


class KVCacheDesc(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p),
                ("k_exp", ctypes.c_void_p),
                ("v_exp", ctypes.c_void_p),
                ("num_pages", ctypes.c_int64),
                ("page_tokens", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32),
                ("elem_bytes", ctypes.c_int32)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p),
                ("inv_freq", ctypes.c_void_p),
                ("rot_dim", ctypes.c_int32),
                ("axes", ctypes.c_int32),
                ("sections", ctypes.c_int32 * 3),
                ("interleaved", ctypes.c_int32)]


class KVCache:
    """tl_kv_cache over tensors that it keeps alive: k and v [pages, kv_heads, page_tokens * head_dim] (uint8 holding
    E4M3, float8_e4m3fn or bfloat16), k_exp and v_exp uint8 [pages, kv_heads, page_tokens] (None for bfloat16)."""

    def __init__(self, k, v, k_exp, v_exp, page_tokens, kv_heads, head_dim):
        import torch
        if any(x.dtype not in (torch.uint8, torch.float8_e4m3fn, torch.bfloat16) for x in (k, v)) or \
                any(x is not None and x.dtype != torch.uint8 for x in (k_exp, v_exp)):
            raise ValueError("k and v are uint8 or float8_e4m3fn (E4M3), or bfloat16, exponents uint8")
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        self.page_tokens, self.kv_heads, self.head_dim = page_tokens, kv_heads, head_dim
        self.elem_bytes = k.element_size()
        block = page_tokens * kv_heads * head_dim
        self.num_pages = k.numel() // block
        if k.numel() != self.num_pages * block or v.numel() != k.numel() or v.element_size() != k.element_size():
            raise ValueError("k and v must hold whole pages of the same type")
        if (k_exp is None) != (self.elem_bytes == 2) or (v_exp is None) != (self.elem_bytes == 2):
            raise ValueError("8-bit caches have exponents, and only they")
        for x in (k_exp, v_exp):
            if x is not None and (x.numel() != self.num_pages * page_tokens * kv_heads):
                raise ValueError("one exponent byte per token and head")
        self.desc = KVCacheDesc(_ptr(k), _ptr(v), _ptr(k_exp), _ptr(v_exp), self.num_pages, page_tokens, kv_heads,
                                head_dim, self.elem_bytes)


class Rope:
    """tl_rope over tensors that it keeps alive."""

    def __init__(self, positions, inv_freq, sections, interleaved, rot_dim):
        self.positions, self.inv_freq, self.sections, self.interleaved = positions, inv_freq, sections, interleaved
        self.rot_dim = rot_dim

    @property
    def desc(self) -> RopeDesc:
        return RopeDesc(_ptr(self.positions), _ptr(self.inv_freq), self.rot_dim, len(self.sections),
                        (ctypes.c_int32 * 3)(*(list(self.sections) + [0] * (3 - len(self.sections)))), int(self.interleaved))


def _struct_dict(s):
    return {name: getattr(s, name) for name, _ in s._fields_}


class TLError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {tl_strerror(status)} ({status})")


_lib = None


def load_library():
    """Load libtl.so (after torch, so both share torch's HIP runtime)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libtl.so is not built ({LIB_PATH}); run python -m paper_2607_04031_amd.build")
    import torch  # noqa: F401  (binds libtl to torch's libamdhip64)
    lib = ctypes.CDLL(LIB_PATH)
    i32, i64, p = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
    lib.tl_tile_bytes.restype = ctypes.c_int
    lib.tl_tile_bytes.argtypes = [i64, i64, i32, i64, i32, ctypes.POINTER(i64)]
    lib.tl_repack.restype = ctypes.c_int
    lib.tl_repack.argtypes = [p, p, i64, i64, i32, i64, i32, p]
    lib.tl_unpack.restype = ctypes.c_int
    lib.tl_unpack.argtypes = [p, p, i64, i64, i32, i64, i32, p]
    lib.tl_gemm.restype = ctypes.c_int
    lib.tl_gemm.argtypes = [p, p, p, i64, i64, i64, ctypes.POINTER(LayoutDesc), i32, p]
    lib.tl_gemm_noalloc.restype = ctypes.c_int
    lib.tl_gemm_noalloc.argtypes = [p, p, p, i64, i64, i64, ctypes.POINTER(LayoutDesc), i32, p]
    lib.tl_gemm_w8.restype = ctypes.c_int
    lib.tl_gemm_w8.argtypes = [p, p, p, p, i64, i64, i64, ctypes.POINTER(LayoutDesc), i32, p]
    lib.tl_gemm_plan.restype = ctypes.c_int
    lib.tl_gemm_plan.argtypes = [i64, i64, i64, ctypes.POINTER(LayoutDesc), i32, ctypes.POINTER(Plan)]
    lib.tl_gemm_grouped.restype = ctypes.c_int
    lib.tl_gemm_grouped.argtypes = [p, i64, p, p, i32, i64, i64, p, i64, p, i64, i64,
                                    ctypes.POINTER(LayoutDesc), i32, p]
    lib.tl_gemm_grouped_swiglu.restype = ctypes.c_int
    lib.tl_gemm_grouped_swiglu.argtypes = [p, i64, p, p, i32, i64, i64, p, i64, p, i64, i64,
                                           ctypes.POINTER(LayoutDesc), i32, p]
    lib.tl_prefetch_degree.restype = ctypes.c_int
    lib.tl_prefetch_degree.argtypes = [ctypes.c_double, ctypes.c_double, ctypes.c_double, i64, ctypes.c_double,
                                       ctypes.POINTER(i64)]
    lib.tl_gemm_lgms.restype = ctypes.c_int
    lib.tl_gemm_lgms.argtypes = [p, p, p, i64, i64, i64, ctypes.POINTER(LayoutDesc), i64, i32, p]
    lib.tl_lgms_occupancy.restype = ctypes.c_int
    lib.tl_lgms_occupancy.argtypes = [i32, ctypes.POINTER(i32)]
    lib.tl_view_offsets.restype = ctypes.c_int
    lib.tl_view_offsets.argtypes = [ctypes.POINTER(View), i64, i64, i32, i64, i32, p, i64, ctypes.POINTER(i64)]
    lib.tl_view_load.restype = ctypes.c_int
    lib.tl_view_load.argtypes = [p, ctypes.POINTER(View), i64, i64, i32, i64, i32, p, p]
    lib.tl_read_amp.restype = ctypes.c_int
    lib.tl_read_amp.argtypes = [i64, i64, i64, i32, i32, i32, ctypes.POINTER(LayoutDesc), i64,
                                ctypes.POINTER(Amp)]
    f32, cache = ctypes.c_float, ctypes.POINTER(KVCacheDesc)
    lib.tl_kv_bytes.restype = ctypes.c_int
    lib.tl_kv_bytes.argtypes = [cache, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.tl_kv_append.restype = ctypes.c_int
    lib.tl_kv_append.argtypes = [p, i64, p, i64, p, i64, i32, i64, i32, p, ctypes.POINTER(RopeDesc), p, cache, p]
    lib.tl_kv_read.restype = ctypes.c_int
    lib.tl_kv_read.argtypes = [cache, p, i64, p, p, p]
    lib.tl_kv_keep.restype = ctypes.c_int
    lib.tl_kv_keep.argtypes = [cache, p, i64, p, p, i64, p, i32, p]
    lib.tl_attn.restype = ctypes.c_int
    lib.tl_attn.argtypes = [p, i64, cache, p, i64, p, p, p, i32, i32, i64, i64, i64, i32, f32, p, p]
    lib.tl_verify.restype = ctypes.c_int
    lib.tl_verify.argtypes = [p, i32, i64, p, p, p, i32, i64, i32, p, i32, p, p, p, p, p, p, p]
    lib.tl_stream_read.restype = ctypes.c_int
    lib.tl_stream_read.argtypes = [p, i64, p, p]
    lib.tl_fetch_counter_read.restype = ctypes.c_int
    lib.tl_fetch_counter_read.argtypes = [p, ctypes.POINTER(i64)]
    lib.tl_release.restype = ctypes.c_int
    lib.tl_release.argtypes = []
    lib.tl_strerror.restype = ctypes.c_char_p
    lib.tl_strerror.argtypes = [ctypes.c_int]
    _lib = lib
    return lib


def _ptr(x) -> int | None:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        if not x.is_cuda:
            raise ValueError("libtl needs device tensors")
        if not x.is_contiguous():
            raise ValueError("libtl needs contiguous tensors")
        return x.data_ptr()
    raise TypeError(f"cannot pass {type(x)!r} as a device pointer")


_raw_stream = None      # device index -> its current stream's handle


def _stream(stream) -> int | None:
    global _raw_stream
    if stream is None:
        import torch
        if _raw_stream is None:
            # the handle without the Stream object around it, which takes 2.7 us of a call
            _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
                (lambda device: torch.cuda.current_stream(device).cuda_stream)
        return _raw_stream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _desc(layout) -> LayoutDesc:
    if isinstance(layout, LayoutDesc):
        return layout
    d = LayoutDesc()
    d.kind, d.elem_bytes, d.G, d.block_rows = TL_LAYOUT_TILE, 2, 4096, 32
    for k, v in dict(layout).items():
        setattr(d, k, v)
    return d


def _check(rc: int, where: str):
    if rc != TL_OK:
        raise TLError(rc, where)


_calls = None


def _load_calls():
    """The extension module that takes tensors to the serving-step entry points; its functions return a status, or None
    for a call that needs the checks (or makes the outputs) below."""
    global _calls
    load_library()
    if not os.path.exists(CALLS_PATH):
        raise ImportError(f"_tl_torch.so is not built ({CALLS_PATH}); run python -m paper_2607_04031_amd.build")
    from . import _tl_torch
    _calls = _tl_torch
    return _calls


# ---------------------------------------------------------------------------
# C ABI, same names and argument order
# ---------------------------------------------------------------------------

def tl_tile_bytes(rows, cols, elem_bytes, G, block_rows) -> int:
    out = ctypes.c_int64()
    _check(load_library().tl_tile_bytes(rows, cols, elem_bytes, G, block_rows, ctypes.byref(out)), "tl_tile_bytes")
    return out.value


def tl_repack(src, dst, rows, cols, elem_bytes, G, block_rows, stream=None):
    _check(load_library().tl_repack(_ptr(src), _ptr(dst), rows, cols, elem_bytes, G, block_rows,
                                    _stream(stream)), "tl_repack")


def tl_unpack(src_tm, dst, rows, cols, elem_bytes, G, block_rows, stream=None):
    _check(load_library().tl_unpack(_ptr(src_tm), _ptr(dst), rows, cols, elem_bytes, G, block_rows,
                                    _stream(stream)), "tl_unpack")


def tl_gemm(A, W, C, M, N, K, layout, fetch_mode=TL_FETCH_BLOCK, stream=None):
    d = _desc(layout)
    _check(load_library().tl_gemm(_ptr(A), _ptr(W), _ptr(C), M, N, K, ctypes.byref(d), fetch_mode,
                                  _stream(stream)), "tl_gemm")


def tl_gemm_noalloc(A, W, C, M, N, K, layout, fetch_mode=TL_FETCH_BLOCK, stream=None):
    d = _desc(layout)
    _check(load_library().tl_gemm_noalloc(_ptr(A), _ptr(W), _ptr(C), M, N, K, ctypes.byref(d), fetch_mode,
                                          _stream(stream)), "tl_gemm_noalloc")


def tl_gemm_w8(A, W_fp8, scales, C, M, N, K, layout, fetch_mode=TL_FETCH_BLOCK, stream=None):
    """scales may be None (all 1)."""
    d = _desc(layout)
    _check(load_library().tl_gemm_w8(_ptr(A), _ptr(W_fp8), _ptr(scales), _ptr(C), M, N, K, ctypes.byref(d),
                                     fetch_mode, _stream(stream)), "tl_gemm_w8")


def tl_gemm_plan(M, N, K, layout, fetch_mode=TL_FETCH_BLOCK) -> dict:
    d = _desc(layout)
    out = Plan()
    _check(load_library().tl_gemm_plan(M, N, K, ctypes.byref(d), fetch_mode, ctypes.byref(out)),
           "tl_gemm_plan")
    return _struct_dict(out)


def tl_gemm_grouped(A, a_rows, token_ids, group_offsets, num_groups, total_rows, max_group_rows, W,
                    group_stride, C, N, K, layout, fetch_mode=TL_FETCH_BLOCK, stream=None):
    """token_ids may be None (row r of C reads row r of A)."""
    d = _desc(layout)
    _check(load_library().tl_gemm_grouped(_ptr(A), a_rows, _ptr(token_ids), _ptr(group_offsets), num_groups,
                                          total_rows, max_group_rows, _ptr(W), group_stride, _ptr(C), N, K,
                                          ctypes.byref(d), fetch_mode, _stream(stream)), "tl_gemm_grouped")


def tl_gemm_grouped_swiglu(A, a_rows, token_ids, group_offsets, num_groups, total_rows, max_group_rows, W_gate_up,
                           group_stride, H, I, K, layout, fetch_mode=TL_FETCH_BLOCK, stream=None):
    """H [total_rows, I] = silu(A W_gate^T) * (A W_up^T) per group; W_gate_up stacks [2I, K] per group."""
    d = _desc(layout)
    _check(load_library().tl_gemm_grouped_swiglu(_ptr(A), a_rows, _ptr(token_ids), _ptr(group_offsets), num_groups,
                                                 total_rows, max_group_rows, _ptr(W_gate_up), group_stride, _ptr(H),
                                                 I, K, ctypes.byref(d), fetch_mode, _stream(stream)),
           "tl_gemm_grouped_swiglu")


def tl_prefetch_degree(bandwidth, latency, bytes_per_iteration, k_iterations, collision_factor=1.0) -> int:
    d = ctypes.c_int64(0)
    _check(load_library().tl_prefetch_degree(float(bandwidth), float(latency), float(bytes_per_iteration),
                                             int(k_iterations), float(collision_factor), ctypes.byref(d)),
           "tl_prefetch_degree")
    return d.value


def tl_gemm_lgms(A, W, C, M, N, K, layout, latency_ns, steps_in_flight, stream=None):
    d = _desc(layout)
    _check(load_library().tl_gemm_lgms(_ptr(A), _ptr(W), _ptr(C), M, N, K, ctypes.byref(d), int(latency_ns),
                                       int(steps_in_flight), _stream(stream)), "tl_gemm_lgms")


def tl_lgms_occupancy(steps_in_flight) -> int:
    n = ctypes.c_int32(0)
    _check(load_library().tl_lgms_occupancy(int(steps_in_flight), ctypes.byref(n)), "tl_lgms_occupancy")
    return n.value


def tl_view_offsets(v: View, K, N, elem_bytes, G, block_rows):
    """numpy int64 byte offsets of the box's elements (view order)."""
    import numpy as np
    lib = load_library()
    n = ctypes.c_int64(0)
    _check(lib.tl_view_offsets(ctypes.byref(v), K, N, elem_bytes, G, block_rows, None, 0, ctypes.byref(n)),
           "tl_view_offsets")
    out = np.empty(n.value, dtype=np.int64)
    _check(lib.tl_view_offsets(ctypes.byref(v), K, N, elem_bytes, G, block_rows, out.ctypes.data, n.value,
                               ctypes.byref(n)), "tl_view_offsets")
    return out


def tl_view_load(src_tm, v: View, K, N, elem_bytes, G, block_rows, dst, stream=None):
    _check(load_library().tl_view_load(_ptr(src_tm), ctypes.byref(v), K, N, elem_bytes, G, block_rows, _ptr(dst),
                                       _stream(stream)), "tl_view_load")


def tl_read_amp(M, N, K, tile_m, tile_n, tile_k, layout, G) -> dict:
    d = _desc(layout)
    out = Amp()
    _check(load_library().tl_read_amp(M, N, K, tile_m, tile_n, tile_k, ctypes.byref(d), G,
                                      ctypes.byref(out)), "tl_read_amp")
    return _struct_dict(out)


def _cache_ref(cache):
    return ctypes.byref(cache.desc if isinstance(cache, KVCache) else cache)


def tl_kv_bytes(cache) -> tuple[int, int]:
    """(bytes of k and of v, bytes of k_exp and of v_exp) for a KVCacheDesc's sizes."""
    data, exps = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(load_library().tl_kv_bytes(_cache_ref(cache), ctypes.byref(data), ctypes.byref(exps)), "tl_kv_bytes")
    return data.value, exps.value


def tl_kv_append(Q, ldq, K, ldk, V, ldv, in_dtype, n, q_heads, slots, rope, Q_out, cache, stream=None):
    """rope: a Rope or None; Q, K, V: raw addresses where rows are not contiguous."""
    r = None if rope is None else ctypes.byref(rope.desc if isinstance(rope, Rope) else rope)
    _check(load_library().tl_kv_append(_ptr(Q), ldq, _ptr(K), ldk, _ptr(V), ldv, in_dtype, n, q_heads, _ptr(slots), r,
                                       _ptr(Q_out), _cache_ref(cache), _stream(stream)), "tl_kv_append")


def tl_kv_read(cache, slots, n, K_out, V_out, stream=None):
    _check(load_library().tl_kv_read(_cache_ref(cache), _ptr(slots), n, _ptr(K_out), _ptr(V_out), _stream(stream)),
           "tl_kv_read")


def tl_kv_keep(cache, page_table, max_pages, starts, path, max_path, counts, num_seqs, stream=None):
    _check(load_library().tl_kv_keep(_cache_ref(cache), _ptr(page_table), max_pages, _ptr(starts), _ptr(path), max_path,
                                     _ptr(counts), num_seqs, _stream(stream)), "tl_kv_keep")


def tl_attn(Q, ldq, cache, page_table, max_pages, lens, q_offsets, mask, mask_words, num_seqs, total_q, max_q, max_len,
            q_heads, scale, O, stream=None):
    """mask may be None (causal)."""
    _check(load_library().tl_attn(_ptr(Q), ldq, _cache_ref(cache), _ptr(page_table), max_pages, _ptr(lens),
                                  _ptr(q_offsets), _ptr(mask), mask_words, num_seqs, total_q, max_q, max_len, q_heads,
                                  scale, _ptr(O), _stream(stream)), "tl_attn")


def tl_verify(logits, logits_dtype, vocab, node_offsets, parents, tokens, num_seqs, total_nodes, max_nodes, draft,
              draft_dtype, temperature, uniform, noise, path, counts, next_token, stream=None):
    """draft may be None (drafted tokens were certain)."""
    _check(load_library().tl_verify(_ptr(logits), logits_dtype, vocab, _ptr(node_offsets), _ptr(parents), _ptr(tokens),
                                    num_seqs, total_nodes, max_nodes, _ptr(draft), draft_dtype, _ptr(temperature),
                                    _ptr(uniform), _ptr(noise), _ptr(path), _ptr(counts), _ptr(next_token),
                                    _stream(stream)), "tl_verify")


def tl_stream_read(src, nbytes, checksum, stream=None):
    """checksum: a device uint32/int32 tensor of one element; the XOR of src's 32-bit words is XORed into it."""
    _check(load_library().tl_stream_read(_ptr(src), nbytes, _ptr(checksum), _stream(stream)), "tl_stream_read")


def tl_fetch_counter_read(stream=None) -> int:
    v = ctypes.c_int64(0)
    _check(load_library().tl_fetch_counter_read(_stream(stream), ctypes.byref(v)),
           "tl_fetch_counter_read")
    return v.value


def tl_release():
    _check(load_library().tl_release(), "tl_release")


def tl_strerror(status: int) -> str:
    return load_library().tl_strerror(status).decode()


# ---------------------------------------------------------------------------
# Tensor helpers (allocation + the calls above)
# ---------------------------------------------------------------------------

def layout(kind=TL_LAYOUT_TILE, G=4096, block_rows=32, out_dtype=TL_OUT_F32, elem_bytes=2,
           tile_m=0, tile_n=0, tile_k=0, split_k=0) -> LayoutDesc:
    return _desc(dict(kind=kind, G=G, block_rows=block_rows, out_dtype=out_dtype,
                      elem_bytes=elem_bytes, tile_m=tile_m, tile_n=tile_n, tile_k=tile_k,
                      split_k=split_k))


def padded_shape(rows, cols, elem_bytes, G=4096, block_rows=32):
    """(rows, cols) rounded up to whole memory tiles: the shape of a tensor
    that holds the tile-major copy (tl_tile_bytes bytes)."""
    bc = G // (elem_bytes * block_rows)
    return (-(-rows // block_rows) * block_rows, -(-cols // bc) * bc)


def repack(w, G=4096, block_rows=32, out=None, stream=None):
    """Tile-major copy of a 2-D device tensor, same dtype, shape rounded up
    to whole memory tiles (the input's shape when the tile divides it)."""
    import torch
    rows, cols = w.shape
    if out is None:
        out = torch.empty(padded_shape(rows, cols, w.element_size(), G, block_rows), dtype=w.dtype, device=w.device)
    tl_repack(w, out, rows, cols, w.element_size(), G, block_rows, stream)
    return out


def unpack(w_tm, G=4096, block_rows=32, rows=None, cols=None, out=None, stream=None):
    """Row-major [rows, cols] (default: w_tm's shape) from a tile-major copy."""
    import torch
    rows = w_tm.shape[0] if rows is None else rows
    cols = w_tm.shape[1] if cols is None else cols
    out = torch.empty((rows, cols), dtype=w_tm.dtype, device=w_tm.device) if out is None else out
    tl_unpack(w_tm, out, rows, cols, w_tm.element_size(), G, block_rows, stream)
    return out


def gemm(A, W, N, desc: LayoutDesc, fetch_mode=TL_FETCH_BLOCK, out=None, stream=None):
    """C = A @ W^T for bf16 A [M, K] and a bf16 weight of logical shape [N, K]."""
    import torch
    M, K = A.shape
    dt = torch.bfloat16 if desc.out_dtype == TL_OUT_BF16 else torch.float32
    C = torch.empty((M, N), dtype=dt, device=A.device) if out is None else out
    tl_gemm(A, W, C, M, N, K, desc, fetch_mode, stream)
    return C


def kv_cache(num_pages, kv_heads, head_dim, page_tokens=64, elem_bytes=1, device="cuda") -> KVCache:
    """An empty cache: 8-bit (E4M3 with scales) or, with elem_bytes=2, bf16."""
    import torch
    dt = torch.uint8 if elem_bytes == 1 else torch.bfloat16
    data, exps = tl_kv_bytes(KVCacheDesc(None, None, None, None, num_pages, page_tokens, kv_heads, head_dim, elem_bytes))
    k, v = (torch.empty((num_pages, kv_heads, page_tokens * head_dim), dtype=dt, device=device) for _ in range(2))
    assert k.numel() * k.element_size() == data
    ke, ve = (torch.empty((num_pages, kv_heads, page_tokens), dtype=torch.uint8, device=device) if exps else None
              for _ in range(2))
    return KVCache(k, v, ke, ve, page_tokens, kv_heads, head_dim)


def rope(positions, inv_freq, sections=None, interleaved=False) -> Rope:
    """Rotary positions: int32 [axes, n] (or [n]) and float32 [rot_dim / 2]; sections: pairs of each axis (one axis: all)."""
    import torch
    if positions.dtype != torch.int32 or inv_freq.dtype != torch.float32:
        raise ValueError("positions are int32 and inv_freq float32")
    pairs = inv_freq.numel()
    sections = (pairs,) if sections is None else tuple(int(x) for x in sections)
    if positions.numel() and positions.numel() % len(sections):
        raise ValueError("positions need one row per axis")
    return Rope(positions, inv_freq, sections, interleaved, 2 * pairs)


def _rows(x, heads, head_dim):
    """(address, elements between rows) of [n, heads * head_dim] or [n, heads, head_dim] rows, each without gaps."""
    shape, stride, width = x.shape, x.stride(), heads * head_dim
    if not x.is_cuda:
        raise ValueError("libtl needs device tensors")
    if not (len(shape) == 2 and shape[1] == width and stride[1] == 1) and \
            not (len(shape) == 3 and shape[1] * shape[2] == width and stride[2] == 1 and (shape[1] == 1 or stride[1] == shape[2])):
        raise ValueError(f"rows of {heads} x {head_dim} elements without gaps are needed, not {tuple(shape)}")
    return x.data_ptr(), stride[0] if shape[0] > 1 else width


def _int32(*tensors):
    import torch
    for x in tensors:
        if x is not None and x.dtype is not torch.int32 and x.dtype is not torch.uint32:
            raise ValueError("indexes, offsets and masks are int32")


def _in_dtype(x):
    import torch
    if x.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("float32 or bfloat16 is needed")
    return TL_IN_BF16 if x.dtype == torch.bfloat16 else TL_IN_F32


def kv_append(q, k, v, cache: KVCache, slots, rope=None, q_out=None, stream=None):
    """Rows of a QKV projection (tensors, or column ranges of one) into the cache at slots; returns the queries, turned by
    rope, as bf16 [n, q_heads, head_dim].  q may be None, and so may k and v."""
    rc = (_calls or _load_calls()).kv_append(q, k, v, cache.desc, slots, rope, q_out, stream)
    if rc is not None:
        return q_out if rc == TL_OK else _check(rc, "tl_kv_append")
    import torch
    some = q if q is not None else k
    n, D, H = some.shape[0], cache.head_dim, cache.kv_heads
    heads = 0 if q is None else q.shape[1] if q.dim() == 3 else q.shape[1] // D
    if k is not None:
        _int32(slots)
    for x in (q, k, v):
        if x is not None and (x.dtype != some.dtype or x.shape[0] != n):
            raise ValueError("queries, keys and values are rows of one type")
    if k is not None and slots.numel() != n:
        raise ValueError("one slot per row")
    if rope is not None and rope.positions.numel() != n * len(rope.sections):
        raise ValueError("one position per axis and row")
    (qp, ldq), (kp, ldk), (vp, ldv) = ((None, 0) if x is None else _rows(x, h, D) for x, h in ((q, heads), (k, H), (v, H)))
    if q is not None and q_out is None:
        q_out = torch.empty((n, heads, D), dtype=torch.bfloat16, device=q.device)
    if q is not None and (q_out.dtype != torch.bfloat16 or q_out.numel() != n * heads * D):
        raise ValueError("q_out is bfloat16 [n, q_heads, head_dim]")
    tl_kv_append(qp, ldq, kp, ldk, vp, ldv, _in_dtype(some), n, heads, slots, rope, q_out, cache, stream)
    return q_out


def kv_read(cache: KVCache, slots, k_out=None, v_out=None, stream=None):
    """bf16 keys and values [n, kv_heads, head_dim] of the given slots."""
    rc = (_calls or _load_calls()).kv_read(cache.desc, slots, k_out, v_out, stream)
    if rc is not None:
        return (k_out, v_out) if rc == TL_OK else _check(rc, "tl_kv_read")
    import torch
    _int32(slots)
    n = slots.numel()
    shape = (n, cache.kv_heads, cache.head_dim)
    k_out = torch.empty(shape, dtype=torch.bfloat16, device=slots.device) if k_out is None else k_out
    v_out = torch.empty(shape, dtype=torch.bfloat16, device=slots.device) if v_out is None else v_out
    for x in (k_out, v_out):
        if x.dtype != torch.bfloat16 or x.numel() != n * cache.kv_heads * cache.head_dim:
            raise ValueError("outputs are bfloat16 [n, kv_heads, head_dim]")
    tl_kv_read(cache, slots, n, k_out, v_out, stream)
    return k_out, v_out


def kv_keep(cache: KVCache, page_table, starts, path, counts, stream=None):
    """Moves the entries of every sequence's accepted path (as verify returns it) to the front of its new tokens."""
    rc = (_calls or _load_calls()).kv_keep(cache.desc, page_table, starts, path, counts, stream)
    if rc is not None:
        return _check(rc, "tl_kv_keep")
    _int32(page_table, starts, path, counts)
    B = page_table.shape[0]
    if starts.numel() != B or counts.numel() != B or path.shape[0] != B:
        raise ValueError("one row per sequence")
    tl_kv_keep(cache, page_table, page_table.shape[1], starts, path, path.shape[1], counts, B, stream)


def attention(q, cache: KVCache, page_table, lens, q_offsets, max_q, max_len, scale, mask=None, out=None, stream=None):
    """Attention of the new tokens q [total_q, q_heads, head_dim] (bf16) over the cache: bf16 of q's shape.  mask: int32
    [total_q, words] of the new tokens that each new token sees, or None (causal)."""
    rc = (_calls or _load_calls()).attention(q, cache.desc, page_table, lens, q_offsets, max_q, max_len, scale, mask, out,
                                             stream)
    if rc is not None:
        return out if rc == TL_OK else _check(rc, "tl_attn")
    import torch
    if q.dtype != torch.bfloat16:
        raise ValueError("queries are bfloat16")
    _int32(page_table, lens, q_offsets, mask)
    total, B, D = q.shape[0], lens.numel(), cache.head_dim
    heads = q.shape[1] if q.dim() == 3 else q.shape[1] // D
    if page_table.shape[0] != B or q_offsets.numel() != B + 1 or (mask is not None and mask.shape[0] != total):
        raise ValueError("one row per sequence, one more offset, one mask row per query row")
    qp, ldq = _rows(q, heads, D)
    if out is None:
        out = torch.empty((total, heads, D), dtype=torch.bfloat16, device=q.device)
    if out.dtype != torch.bfloat16 or out.numel() != total * heads * D:
        raise ValueError("out is bfloat16 [total_q, q_heads, head_dim]")
    tl_attn(qp, ldq, cache, page_table, page_table.shape[1], lens, q_offsets, mask, 0 if mask is None else mask.shape[1],
            B, total, max_q, max_len, heads, scale, out, stream)
    return out


def verify(logits, node_offsets, parents, tokens, temperature, uniform, noise, max_nodes, draft=None, out=None,
           stream=None):
    """(path int32 [sequences, max_nodes], counts, next): the drafted tokens that stay, and the token after them."""
    path, count, after = out if out is not None else (None, None, None)
    rc = (_calls or _load_calls()).verify(logits, node_offsets, parents, tokens, temperature, uniform, noise, max_nodes,
                                          draft, path, count, after, stream)
    if rc is not None:
        return out if rc == TL_OK else _check(rc, "tl_verify")
    import torch
    _int32(node_offsets, parents, tokens)
    total, vocab = logits.shape
    B = temperature.numel()
    if any(x.dtype != torch.float32 for x in (temperature, uniform, noise)):
        raise ValueError("temperature, uniform and noise are float32")
    if node_offsets.numel() != B + 1 or any(x.numel() != total for x in (parents, tokens, uniform)) or \
            noise.numel() != B * vocab or (draft is not None and draft.shape != logits.shape):
        raise ValueError("sizes of logits, nodes and sequences do not agree")
    if out is None:
        out = (torch.empty((B, max_nodes), dtype=torch.int32, device=logits.device),
               torch.empty(B, dtype=torch.int32, device=logits.device),
               torch.empty(B, dtype=torch.int32, device=logits.device))
    _int32(*out)
    if [x.numel() for x in out] != [B * max_nodes, B, B]:
        raise ValueError("out is (path, counts, next)")
    tl_verify(logits, _in_dtype(logits), vocab, node_offsets, parents, tokens, B, total, max_nodes, draft,
              TL_IN_F32 if draft is None else _in_dtype(draft), temperature, uniform, noise, *out, stream)
    return out
