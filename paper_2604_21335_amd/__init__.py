"""Python binding of libstc (HIP, MI355X): decode attention over a Quest-selected,
group-packed KV cache.  The functions below have the names of the C entry
points in include/stc.h and only marshal arguments, through csrc/binding.cpp; every step of the
path runs in the HIP kernels.  PyTorch is used for device memory and the current stream.

There is no CPU fallback: if libstc.so cannot be loaded the calls raise.
"""
import ctypes
import os

import torch

from . import workloads  # noqa: F401  (seeded synthetic inputs)

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libstc.so")
BINDING_PATH = os.path.join(_PKG_DIR, "_binding.so")   # unpacks tensors for libstc.so

STC_OK = 0
STC_ERR_NULL, STC_ERR_SHAPE, STC_ERR_ALIGN, STC_ERR_WORKSPACE, STC_ERR_LAUNCH = -1, -2, -3, -4, -5
STC_WS_ROUTE, STC_WS_SELECT, STC_WS_ATTENTION, STC_WS_ATTENTION_TAIL = 1, 2, 3, 4
STC_WS_SELECT_PER_HEAD, STC_WS_ATTENTION_PER_HEAD, STC_WS_STEP, STC_WS_STEP_TAIL = 5, 6, 7, 8
STC_ROUTE_MASK, STC_ROUTE_TOPK, STC_ROUTE_GLOBAL = 0, 1, 2
STC_ROUTE_SHARED = 0x100        # flag: one set of routing inputs per batch element
STC_OUT_F32, STC_OUT_BF16 = 0, 1
STC_ROTARY_HALVES, STC_ROTARY_INTERLEAVED, STC_ROTARY_INVERSE = 0, 1, 0x100
STC_ROTARY_SCALE_NONE, STC_ROTARY_SCALE_LINEAR, STC_ROTARY_SCALE_BASE = 0, 1, 2
STC_ROTARY_SCALE_CHANNELS, STC_ROTARY_SCALE_WAVELENGTHS = 3, 4
STC_TAIL_FREED, STC_TAIL_EMPTY = -1, -2     # in the map of stc_fork_tail

EXPORTS = ["stc_version", "stc_status_string", "stc_workspace_bytes", "stc_bounds_bytes",
           "stc_build_page_bounds",
           "stc_route_and_pack_values", "stc_select_pages", "stc_score_pages", "stc_decode_attention", "stc_decode_attention_tail", "stc_append_tail",
           "stc_select_pages_per_head", "stc_decode_attention_per_head", "stc_router_logits",
           "stc_union_pages", "stc_decode_attention_union", "stc_flush_tail",
           "stc_compact_tokens", "stc_decode_step", "stc_decode_step_tail",
           "stc_decode_step_static", "stc_rotary_turns", "stc_rotary", "stc_rotary_append",
           "stc_shared_workspace_bytes", "stc_decode_attention_shared",
           "stc_rotary_append_tree", "stc_tree_workspace_bytes", "stc_decode_attention_tree",
           "stc_accept_tail", "stc_fork_tail", "stc_rotary_append_drafts", "stc_accept_drafts"]


class StcError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s failed: %d (%s)" % (where, status, status_string(status)))


class stc_shape_t(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("D", ctypes.c_int32), ("N", ctypes.c_int32), ("P", ctypes.c_int32),
                ("G", ctypes.c_int32), ("N_cap", ctypes.c_int32),
                ("v_cap_groups", ctypes.c_int64)]


def make_shape(B, Hq, Hkv, D, N, G, v_cap_groups, P=16, N_cap=0):
    """N_cap: token capacity (stride) of K, mask, tok_off and bounds; 0 = exactly N."""
    return stc_shape_t(B, Hq, Hkv, D, N, P, G, N_cap, v_cap_groups)


class stc_rotary_scaling_t(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("original_len", ctypes.c_int32),
                ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("slow", ctypes.c_double), ("fast", ctypes.c_double)]


_lib = None
_native = None


def load_library():
    """dlopen libstc.so from the package directory; build it first only if it is
    absent.  Raises if it can neither be found nor built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH) or not os.path.exists(BINDING_PATH):
        from .build import build_library
        build_library()
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    shp = ctypes.POINTER(stc_shape_t)
    lib.stc_version.restype = ctypes.c_int
    lib.stc_version.argtypes = []
    lib.stc_status_string.restype = ctypes.c_char_p
    lib.stc_status_string.argtypes = [ctypes.c_int]
    lib.stc_workspace_bytes.restype = sz
    lib.stc_workspace_bytes.argtypes = [shp, ctypes.c_int, ctypes.c_int]
    lib.stc_bounds_bytes.restype = ctypes.c_size_t
    lib.stc_bounds_bytes.argtypes = [shp]
    lib.stc_build_page_bounds.restype = ctypes.c_int
    lib.stc_build_page_bounds.argtypes = [shp, vp, vp, vp]
    lib.stc_route_and_pack_values.restype = ctypes.c_int
    lib.stc_route_and_pack_values.argtypes = [shp, ctypes.c_int, vp, vp, vp, ctypes.c_int, vp, vp,
                                              vp, vp, vp, vp, sz, vp]
    lib.stc_select_pages.restype = ctypes.c_int
    lib.stc_select_pages.argtypes = [shp, vp, vp, ctypes.c_int, vp, vp, vp, sz, vp]
    lib.stc_score_pages.restype = ctypes.c_int
    lib.stc_score_pages.argtypes = [shp, vp, vp, vp, vp]
    lib.stc_decode_attention.restype = ctypes.c_int
    lib.stc_decode_attention.argtypes = [shp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp, vp, sz, vp]
    lib.stc_select_pages_per_head.restype = ctypes.c_int
    lib.stc_select_pages_per_head.argtypes = lib.stc_select_pages.argtypes
    lib.stc_decode_attention_per_head.restype = ctypes.c_int
    lib.stc_decode_attention_per_head.argtypes = lib.stc_decode_attention.argtypes
    lib.stc_flush_tail.restype = ctypes.c_int
    lib.stc_flush_tail.argtypes = [shp, vp, vp, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                   ctypes.c_int, vp, vp,
                                   ctypes.c_int, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.stc_union_pages.restype = ctypes.c_int
    lib.stc_union_pages.argtypes = [shp, vp, ctypes.c_int, vp, vp, ctypes.c_int, vp]
    lib.stc_decode_attention_union.restype = ctypes.c_int
    lib.stc_decode_attention_union.argtypes = [shp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp, vp,
                                               sz, vp]
    lib.stc_decode_attention_tail.restype = ctypes.c_int
    lib.stc_decode_attention_tail.argtypes = [shp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp, vp,
                                              ctypes.c_int, ctypes.c_int, vp, vp, sz, vp]
    lib.stc_decode_step.restype = ctypes.c_int
    lib.stc_decode_step.argtypes = [shp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp, vp, vp, sz, vp]
    lib.stc_decode_step_static.restype = ctypes.c_int
    lib.stc_decode_step_static.argtypes = [shp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp, vp, vp]
    lib.stc_decode_step_tail.restype = ctypes.c_int
    lib.stc_decode_step_tail.argtypes = [shp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp, vp,
                                         ctypes.c_int, ctypes.c_int, vp, vp, vp, sz, vp]
    lib.stc_append_tail.restype = ctypes.c_int
    lib.stc_append_tail.argtypes = [shp, vp, vp, vp, vp, ctypes.c_int, ctypes.c_int, vp]
    lib.stc_router_logits.restype = ctypes.c_int
    lib.stc_router_logits.argtypes = [i32, i32, i32, i32, i32, vp, vp, vp, i32, vp, vp]
    i64, f32 = ctypes.c_int64, ctypes.c_float
    lib.stc_rotary_turns.restype = ctypes.c_int
    lib.stc_rotary_turns.argtypes = [i32, ctypes.POINTER(stc_rotary_scaling_t),
                                     ctypes.POINTER(ctypes.c_double)]
    strides = ctypes.POINTER(i64)
    lib.stc_rotary.restype = ctypes.c_int
    lib.stc_rotary.argtypes = [i32, i32, i32, i32, i32, i32, vp, f32, vp, i32, vp, strides, vp,
                               strides, vp]
    lib.stc_rotary_append.restype = ctypes.c_int
    lib.stc_rotary_append.argtypes = [shp, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp,
                                      ctypes.c_int, ctypes.c_int, ctypes.c_int, vp, f32, vp, i32, vp,
                                      vp]
    lib.stc_shared_workspace_bytes.restype = sz
    lib.stc_shared_workspace_bytes.argtypes = [shp, ctypes.c_int, ctypes.c_int]
    lib.stc_decode_attention_shared.restype = ctypes.c_int
    lib.stc_decode_attention_shared.argtypes = [shp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp, vp, vp,
                                                ctypes.c_int, ctypes.c_int, vp, vp, sz, vp]
    ci, ptrs = ctypes.c_int, ctypes.POINTER(vp)
    lib.stc_rotary_append_tree.restype = ci
    lib.stc_rotary_append_tree.argtypes = [shp, ci, vp, strides, vp, strides, vp, strides, vp, vp, vp, vp,
                                           vp, ci, vp, ci, ci, ci, vp, f32, vp, i32, vp, vp]
    lib.stc_rotary_append_drafts.restype = ci
    lib.stc_rotary_append_drafts.argtypes = [shp, ci, vp, strides, vp, strides, vp, strides, vp, vp, vp, vp,
                                             vp, ci, vp, ci, ci, ci, vp, f32, vp, i32, vp, vp, vp]
    lib.stc_tree_workspace_bytes.restype = sz
    lib.stc_tree_workspace_bytes.argtypes = [shp, ci, ci, ci, ci]
    lib.stc_decode_attention_tree.restype = ci
    lib.stc_decode_attention_tree.argtypes = [shp, ci, ci, vp, vp, vp, vp, vp, vp, ci, vp, vp, vp, vp, ci,
                                              vp, ci, ci, vp, vp, sz, vp]
    lib.stc_accept_tail.restype = ci
    lib.stc_accept_tail.argtypes = [shp, ci, ci, ptrs, ptrs, ptrs, ptrs, ci, vp, vp]
    lib.stc_accept_drafts.restype = ci
    lib.stc_accept_drafts.argtypes = [shp, ci, ci, ptrs, ptrs, ptrs, ptrs, ci, vp, vp, vp]
    lib.stc_fork_tail.restype = ci
    lib.stc_fork_tail.argtypes = [shp, ci, ptrs, ptrs, ptrs, ptrs, ci, vp, vp, vp, vp]
    lib.stc_compact_tokens.restype = ctypes.c_int
    lib.stc_compact_tokens.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, vp, vp]
    _lib = lib
    return lib


def status_string(status):
    return load_library().stc_status_string(int(status)).decode()


def _current_stream():
    return torch.cuda.current_stream().cuda_stream


def _load_native():
    """The module that unpacks the tensors of a call (csrc/binding.cpp)."""
    global _native
    if _native is None:
        load_library()
        from . import _binding
        _native = _binding
    return _native


def stc_version():
    return load_library().stc_version()


def stc_workspace_bytes(shape, which_call, k_pages=0):
    return int(load_library().stc_workspace_bytes(ctypes.byref(shape), which_call, k_pages))


def stc_bounds_bytes(shape):
    return int(load_library().stc_bounds_bytes(ctypes.byref(shape)))


def bounds_rows(bounds, shape):
    """The tiled bounds buffer as a [B, Hkv, NP, 2, D] tensor (row 0 = minima, row 1 = maxima):
    a pure re-ordering of its elements, for inspection and tests."""
    B, Hkv, D = shape.B, shape.Hkv, shape.D
    NP = (shape.N + shape.P - 1) // shape.P
    cap = shape.N_cap or shape.N
    nt = ((cap + shape.P - 1) // shape.P + 7) // 8          # tiles per stream in memory
    # dwords [s][t][j][g][e][col][w], each (min, max)
    t = bounds.reshape(B, Hkv, nt, D // 32, 2, 8, 4, 4, 2)
    # -> [B, Hkv, t, g, col, (min|max), e, j, w]
    t = t.permute(0, 1, 2, 4, 6, 8, 5, 3, 7)
    return t.reshape(B, Hkv, nt * 8, 2, D)[:, :, :NP].contiguous()


def stc_build_page_bounds(shape, K, bounds):
    (_native or _load_native()).build_page_bounds(shape, K, bounds)


def stc_route_and_pack_values(shape, mode, V, logits, kcount, fixed_k, mask_in, mask, tok_off,
                              vpacked, dev_status, ws):
    (_native or _load_native()).route_and_pack_values(
        shape, mode, V, logits, kcount, fixed_k, mask_in, mask, tok_off, vpacked, dev_status, ws)


def stc_select_pages(shape, q, bounds, k_pages, page_idx, page_score, ws):
    (_native or _load_native()).select_pages(shape, q, bounds, k_pages, page_idx, page_score, ws)


def stc_score_pages(shape, q, bounds, page_score):
    (_native or _load_native()).score_pages(shape, q, bounds, page_score)


def stc_decode_attention(shape, q, K, vpacked, mask, tok_off, page_idx, k_pages, out, ws):
    (_native or _load_native()).decode_attention(shape, q, K, vpacked, mask, tok_off, page_idx,
                                                 k_pages, out, ws)


def stc_select_pages_per_head(shape, q, bounds, k_pages, page_idx, page_score, ws):
    (_native or _load_native()).select_pages_per_head(shape, q, bounds, k_pages, page_idx,
                                                      page_score, ws)


def stc_decode_attention_per_head(shape, q, K, vpacked, mask, tok_off, page_idx, k_pages, out, ws):
    (_native or _load_native()).decode_attention_per_head(shape, q, K, vpacked, mask, tok_off,
                                                          page_idx, k_pages, out, ws)


def stc_flush_tail(shape, K_tail, V_tail, n_flush, n_tail, tail_cap, mode, logits, kcount, fixed_k, mask_in,
                   K, bounds, mask, tok_off, vpacked, dev_status):
    (_native or _load_native()).flush_tail(
        shape, K_tail, V_tail, n_flush, n_tail, tail_cap, mode, logits, kcount, fixed_k, mask_in, K,
        bounds, mask, tok_off, vpacked, dev_status)


def stc_union_pages(shape, page_idx_per_head, k_pages, union_idx, union_heads):
    (_native or _load_native()).union_pages(shape, page_idx_per_head, k_pages, union_idx,
                                            union_heads, union_idx.shape[-1])


def stc_decode_attention_union(shape, q, K, vpacked, mask, tok_off, union_idx, union_heads, out,
                               ws):
    (_native or _load_native()).decode_attention_union(
        shape, q, K, vpacked, mask, tok_off, union_idx, union_heads, union_idx.shape[-1], out, ws)


def stc_decode_step(shape, q, bounds, K, vpacked, mask, tok_off, k_pages, page_idx, out, ws):
    (_native or _load_native()).decode_step(shape, q, bounds, K, vpacked, mask, tok_off, k_pages,
                                            page_idx, out, ws)


STC_STATIC_SCRATCH_BYTES = 8 * 1024 * 1024


def stc_decode_step_static(shape, q, bounds, K, vpacked, mask, tok_off, k_pages, page_idx, out):
    """stc_decode_step over the library's own static scratch array: no workspace argument."""
    (_native or _load_native()).decode_step_static(shape, q, bounds, K, vpacked, mask, tok_off,
                                                   k_pages, page_idx, out)


def stc_decode_step_tail(shape, q, bounds, K, vpacked, mask, tok_off, k_pages, K_tail, V_tail,
                         n_tail, tail_cap, page_idx, out, ws):
    (_native or _load_native()).decode_step_tail(
        shape, q, bounds, K, vpacked, mask, tok_off, k_pages, K_tail, V_tail, n_tail, tail_cap,
        page_idx, out, ws)


def stc_decode_attention_tail(shape, q, K, vpacked, mask, tok_off, page_idx, k_pages, K_tail,
                              V_tail, n_tail, tail_cap, out, ws):
    (_native or _load_native()).decode_attention_tail(
        shape, q, K, vpacked, mask, tok_off, page_idx, k_pages, K_tail, V_tail, n_tail, tail_cap,
        out, ws)


def stc_append_tail(shape, k_new, v_new, K_tail, V_tail, n_tail, tail_cap):
    (_native or _load_native()).append_tail(shape, k_new, v_new, K_tail, V_tail, n_tail, tail_cap)


def stc_router_logits(h, W, bias, logits, Hkv):
    """h [B, N, d_model] bf16, W [G, d_model] bf16, bias [G] or [B, G] float32 or None ->
    logits [B, Hkv, N, G] float32 (the same for every KV head).  A [B, G] bias is one vector
    per batch element (the query term of a query-conditioned router)."""
    B, N, dm = h.shape
    G = W.shape[0]
    per_batch = 0
    if bias is not None and bias.dim() == 2:
        if tuple(bias.shape) != (B, G):
            raise ValueError("a per-element bias must be [B, G]")
        per_batch = 1
    (_native or _load_native()).router_logits(B, Hkv, N, dm, G, h, W, bias, per_batch, logits)


def stc_compact_tokens(src, token_idx, dst, B, Hkv, N_src, n_keep, D, dev_status=None):
    (_native or _load_native()).compact_tokens(src, token_idx, dst, B, Hkv, N_src, n_keep, D,
                                               dev_status)


def stc_rotary_turns(rot_dim, base=10000.0, kind=STC_ROTARY_SCALE_NONE, factor=1.0, original_len=0,
                     slow=0.0, fast=0.0):
    """Revolutions per position of the rot_dim/2 pairs: a float64 tensor in host memory, to be
    copied to the device once."""
    scaling = stc_rotary_scaling_t(kind, original_len, base, factor, slow, fast)
    out = (ctypes.c_double * (max(rot_dim, 2) // 2))()
    status = load_library().stc_rotary_turns(rot_dim, ctypes.byref(scaling), out)
    if status != STC_OK:
        raise StcError(status, "stc_rotary_turns")
    return torch.tensor(list(out), dtype=torch.float64)


def stc_rotary(x, y, turns, rot_dim, layout, pos=None, pos0=0, amplitude=1.0, inverse=False):
    """x, y [B, H, N, D] bf16, any strides that are multiples of 8 (y may be x); turns [rot_dim/2]
    float64; pos [B, N] int32, or None: token n stands at pos0 + n.  inverse: the rotation's
    transpose, which is its gradient."""
    if inverse:
        layout |= STC_ROTARY_INVERSE
    (_native or _load_native()).rotary(x, y, turns, rot_dim, layout, pos, pos0, amplitude)


def stc_rotary_append(shape, q, k_new, v_new, q_out, K_tail, V_tail, n_tail, tail_cap, turns, rot_dim,
                      layout, amplitude=1.0, pos=None, pos0=0, n_out=None, dev_status=None):
    """q [B, Hq, D], k_new, v_new [B, Hkv, D] (slices of one projection's output will do): rotated q
    to q_out, rotated k_new and v_new to row n_tail[b] of sequence b's tails.  n_out (n_tail itself
    will do) receives the tails' new lengths."""
    (_native or _load_native()).rotary_append(shape, q, k_new, v_new, q_out, K_tail, V_tail, n_tail,
                                              tail_cap, turns, rot_dim, layout, amplitude, pos, pos0,
                                              n_out, dev_status)


def stc_shared_workspace_bytes(shape, k_pages, tail_cap):
    return int(load_library().stc_shared_workspace_bytes(ctypes.byref(shape), k_pages, tail_cap))


def stc_decode_attention_shared(shape, q, K, vpacked, mask, tok_off, page_idx, k_pages, K_tail, V_tail,
                                n_tail, tail_cap, out, ws):
    """B sequences over one prefix (K, vpacked, mask, tok_off of a cache with B = 1), each with its own
    tail of n_tail[b] tokens; out [B, Hq, D] float32 or bfloat16."""
    (_native or _load_native()).decode_attention_shared(shape, q, K, vpacked, mask, tok_off, page_idx,
                                                        k_pages, K_tail, V_tail, n_tail, tail_cap, out,
                                                        ws)


def stc_rotary_append_tree(shape, q, k_new, v_new, q_out, K_tail, V_tail, n_tail, tail_cap, turns, rot_dim,
                           layout, tree=None, n_draft=None, amplitude=1.0, pos=None, pos0=0,
                           dev_status=None, n_have=None):
    """T drafted tokens of every sequence, q [B, T, Hq, D], k_new, v_new [B, T, Hkv, D] (slices of one
    projection's output will do): rotated q to q_out, rotated k_new and v_new to rows n_tail[b] .. of sequence
    b's tails, whose lengths stay.  tree [T] or [B, T] int64: the nodes that a node sees, as bits; None: a chain.
    n_draft [B] int32: nodes that a sequence has; None: T.  n_have [B] int32, out: nodes that it has now, none where there
    was no room for all (stc_rotary_append_drafts); the n_draft of the calls below."""
    (_native or _load_native()).rotary_append_tree(shape, q, k_new, v_new, q_out, K_tail, V_tail, n_tail,
                                                   tail_cap, turns, rot_dim, layout, tree, n_draft, amplitude,
                                                   pos, pos0, n_have, dev_status)


def stc_tree_workspace_bytes(shape, T, k_pages, tail_cap, n_prefix=1):
    return int(load_library().stc_tree_workspace_bytes(ctypes.byref(shape), T, n_prefix, k_pages, tail_cap))


def stc_decode_attention_tree(shape, q, K, vpacked, mask, tok_off, page_idx, k_pages, K_tail, V_tail, n_tail,
                              tail_cap, out, ws, tree=None, n_draft=None, n_prefix=1):
    """The nodes' queries q [B, T, Hq, D] over the listed pages of a prefix (n_prefix 1: the batch's; B: one for
    each sequence), the sequence's tail and the nodes that they see; out [B, T, Hq, D] float32 or bfloat16."""
    (_native or _load_native()).decode_attention_tree(shape, n_prefix, q.shape[1], q, K, vpacked, mask, tok_off,
                                                      page_idx, k_pages, K_tail, V_tail, n_tail, tail_cap, tree,
                                                      n_draft, out, ws)


def stc_accept_tail(shape, T, K_tails, V_tails, n_tails, tail_cap, keep, n_outs=None, n_draft=None):
    """Of the T nodes behind sequence b's tail, those whose bits keep[b] (int64) has move together, and the tail
    grows by them, in all layers: K_tails, V_tails, n_tails are lists of the layers' tensors.  n_outs: where the new
    lengths go; None: n_tails.  n_draft [B] int32: nodes that a sequence has (stc_accept_drafts); None: T."""
    (_native or _load_native()).accept_tail(shape, T, tail_cap, K_tails, V_tails, n_tails,
                                            n_tails if n_outs is None else n_outs, keep, n_draft)


def stc_fork_tail(shape, K_tails, V_tails, n_tails, tail_cap, src, n_keep=None, n_outs=None, dev_status=None):
    """Sequence b goes on with the tail of src[b] (int32; STC_TAIL_FREED: ends, STC_TAIL_EMPTY: starts anew), its
    first n_keep[b] tokens where given, in all layers: lists of tensors as for stc_accept_tail."""
    (_native or _load_native()).fork_tail(shape, tail_cap, K_tails, V_tails, n_tails,
                                          n_tails if n_outs is None else n_outs, src, n_keep, dev_status)


def tree_from_parents(parents, device="cuda:0"):
    """Bits of the nodes that each node of a tree of drafted tokens sees, its ancestors and itself: parents is a
    list of T numbers (or B such lists), the place of a node's parent, smaller than its own, or -1 for nodes that
    follow the sequence's last token.  -> int64 tensor [T] (or [B, T]), the `tree` of the calls below."""
    many = len(parents) > 0 and hasattr(parents[0], "__len__")
    out = []
    for one in (parents if many else [parents]):
        if not 1 <= len(one) <= 64:
            raise ValueError("a tree has 1 to 64 nodes")
        seen = []
        for t, p in enumerate(one):
            if not -1 <= p < t:
                raise ValueError("a node's parent stands in front of it")
            seen.append((seen[int(p)] if p >= 0 else 0) | 1 << t)
        out.append([x - (1 << 64) if x >> 63 else x for x in seen])
    return torch.tensor(out if many else out[0], dtype=torch.int64, device=device)


class Rotary:
    """A model's rotary positions: the frequencies on the device and how they are applied."""

    def __init__(self, rot_dim, layout=STC_ROTARY_HALVES, amplitude=1.0, device="cuda:0", **scaling):
        """scaling: base, kind, factor, original_len, slow, fast of stc_rotary_turns."""
        self.rot_dim, self.layout, self.amplitude = rot_dim, layout, amplitude
        self.turns = stc_rotary_turns(rot_dim, **scaling).to(device)

    def apply(self, x, y, pos=None, pos0=0, inverse=False):
        stc_rotary(x, y, self.turns, self.rot_dim, self.layout, pos, pos0, self.amplitude, inverse)


class RoutedCache:
    """Device buffers of one layer's compressed cache plus per-step outputs.

    Allocation (through torch, all of it in the constructor, sized for the token capacity) and
    nothing else: every computation is one of the stc_* calls above.
    """

    def __init__(self, B, Hq, Hkv, D, N, G, k_pages, v_cap_groups=None, device="cuda:0",
                 keep_scores=True, tail_cap=0, n_cap=0):
        """n_cap > N: room for n_cap tokens, so that tail tokens can be moved into the cache
        (flush); the cache then keeps its own copy of K."""
        self.device = torch.device(device)
        self.B, self.Hq, self.Hkv, self.D, self.N, self.G = B, Hq, Hkv, D, N, G
        self.n_cap = n_cap
        self.next_pos = N                   # position of the token behind the cache's last
        self.keep_scores = keep_scores
        self.k_pages = k_pages
        cap = (n_cap or N) * G if v_cap_groups is None else v_cap_groups
        self.shape = make_shape(B, Hq, Hkv, D, N, G, cap, N_cap=n_cap)
        dev = self.device
        Nc = n_cap or N                     # strides of mask and tok_off; most tokens ever held
        NPc = (Nc + 15) // 16
        k_max = min(k_pages, NPc)
        tail_pages = (tail_cap + 15) // 16
        self.bounds = torch.empty(stc_bounds_bytes(self.shape) // 2, dtype=torch.bfloat16,
                                  device=dev)
        self.mask = torch.empty(B, Hkv, Nc, dtype=torch.int16, device=dev)
        self.tok_off = torch.empty(B, Hkv, Nc + 1, dtype=torch.int32, device=dev)
        self.vpacked = torch.empty(B, Hkv, cap, D // G, dtype=torch.bfloat16, device=dev)
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=dev)
        self._page_idx_buf = torch.empty(B * Hkv * k_max, dtype=torch.int32, device=dev)
        self.out = torch.empty(B, Hq, D, dtype=torch.float32, device=dev)
        self.K = (torch.empty(B, Hkv, n_cap, D, dtype=torch.bfloat16, device=dev)
                  if n_cap else None)
        # uncompressed tail of recent tokens (tail_cap = 0: none)
        self.tail_cap, self.n_tail = tail_cap, 0
        if tail_cap:
            self.K_tail = torch.empty(B, Hkv, tail_cap, D, dtype=torch.bfloat16, device=dev)
            self.V_tail = torch.empty_like(self.K_tail)
        # workspaces for the largest shape the cache can reach (sizes grow with N and k)
        big = make_shape(B, Hq, Hkv, D, Nc, G, cap, N_cap=n_cap)

        def ws(which, k):
            return torch.empty(max(stc_workspace_bytes(big, which, k), 16), dtype=torch.uint8,
                               device=dev)
        self._ws_route = ws(STC_WS_ROUTE, 0)
        self._ws_select = ws(STC_WS_SELECT, 1)
        self._ws_attn = ws(STC_WS_ATTENTION_TAIL if tail_cap else STC_WS_ATTENTION,
                           k_max + tail_pages)
        self._ws_step = ws(STC_WS_STEP_TAIL, k_max + tail_pages)
        self._scores_all = (torch.empty(B * Hkv * NPc, dtype=torch.float32, device=dev)
                            if keep_scores else None)    # scores when every page is kept
        self._resize()

    def _resize(self):
        """Views for the current token count (no allocation): page list, page scores."""
        self.NP = (self.N + 15) // 16
        self.k_eff = min(self.k_pages, self.NP)
        B, Hkv = self.B, self.Hkv
        self.page_idx = self._page_idx_buf[:B * Hkv * self.k_eff].view(B, Hkv, self.k_eff)
        if self.k_pages >= self.NP:      # every page is kept: the list is 0 .. NP-1
            stc_select_pages(self.shape, None, None, self.k_pages, self.page_idx, None, None)
        # the page scores sit at the front of the workspace of stc_decode_step: page_score is a
        # view of them, so that both forms of step() leave the scores there
        self.page_score = None
        if self.keep_scores:
            n = B * Hkv * self.NP
            if self.k_pages < self.NP or self.tail_cap:
                src = self._ws_step[:4 * n].view(torch.float32)
            else:
                src = self._scores_all[:n]
            self.page_score = src.view(B, Hkv, self.NP)

    def build(self, K, V, logits=None, kcount=None, fixed_k=0, mask_in=None, global_k=None,
              shared=False, rotary=None, pos=None, pos0=0):
        """Cache construction: page bounds of K, routing mask + packed store of V.  The mask
        comes from mask_in, from a global budget of N*global_k token-group pairs per stream,
        or from the per-token top kcount[t] / fixed_k of the logits.  shared: the routing
        inputs are [B, 1, ...], one set per batch element for all its KV heads.  rotary: K comes
        without positions, [B, Hkv, N, D] with any strides (a projection's output, transposed), and
        gets them (pos, pos0 as in stc_rotary) on its way into the cache, which needs its own copy
        (n_cap).  pos0 says where the first token stands also for keys that have their positions."""
        if rotary is not None:
            if not self.n_cap:
                raise ValueError("keys that get positions need a cache with a copy of its own (n_cap)")
            rotary.apply(K, self.K[:, :, :self.N], pos, pos0)
        elif self.n_cap:
            self.K[:, :, :self.N].copy_(K)
        else:
            self.K = K
        self.next_pos = pos0 + self.N if pos is None else None      # (given ones lie on the device)
        stc_build_page_bounds(self.shape, self.K, self.bounds)
        mode = STC_ROUTE_MASK if mask_in is not None else STC_ROUTE_TOPK
        if global_k is not None:
            mode, fixed_k, kcount = STC_ROUTE_GLOBAL, int(global_k), None
        if shared:
            mode |= STC_ROUTE_SHARED
        stc_route_and_pack_values(self.shape, mode, V, logits, kcount, fixed_k, mask_in, self.mask,
                                  self.tok_off, self.vpacked, self.dev_status, self._ws_route)

    def bounds_rows(self):
        return bounds_rows(self.bounds, self.shape)

    def select(self, q):
        stc_select_pages(self.shape, q, self.bounds, self.k_pages, self.page_idx, self.page_score,
                         self._ws_select)

    def score(self, q, page_score):
        stc_score_pages(self.shape, q, self.bounds, page_score)

    def append(self, k_new, v_new):
        """New token of every stream ([B, Hkv, D] each) into the uncompressed tail."""
        stc_append_tail(self.shape, k_new, v_new, self.K_tail, self.V_tail, self.n_tail,
                        self.tail_cap)
        self.n_tail += 1

    def flush(self, n, logits=None, kcount=None, fixed_k=0, mask_in=None):
        """Move the oldest n tail tokens into the compressed cache (routing them by mask_in,
        or by the top kcount[t] / fixed_k of logits); the call moves the rest of the tail to
        its front."""
        mode = STC_ROUTE_MASK if mask_in is not None else STC_ROUTE_TOPK
        stc_flush_tail(self.shape, self.K_tail, self.V_tail, n, self.n_tail, self.tail_cap, mode,
                       logits, kcount, fixed_k, mask_in, self.K, self.bounds, self.mask,
                       self.tok_off, self.vpacked, self.dev_status)
        self.n_tail -= n
        self.N += n
        if self.next_pos is not None:
            self.next_pos += n
        self.shape.N = self.N
        self._resize()

    def attend(self, q):
        page_idx = self.page_idx if self.k_pages < self.NP else None
        if self.tail_cap:
            stc_decode_attention_tail(self.shape, q, self.K, self.vpacked, self.mask, self.tok_off,
                                      page_idx, self.k_eff, self.K_tail, self.V_tail,
                                      self.n_tail, self.tail_cap, self.out, self._ws_attn)
            return
        stc_decode_attention(self.shape, q, self.K, self.vpacked, self.mask, self.tok_off,
                             page_idx, self.k_eff, self.out, self._ws_attn)

    def step(self, q, one_call=True):
        """One decode step: page selection, then routed attention.  When every page is kept
        there is nothing to select: the attention call takes "all pages" as a missing list.
        one_call: through stc_decode_step (the page scores then stay in its workspace)
        instead of stc_select_pages + stc_decode_attention."""
        if self.k_pages < self.NP:
            if one_call:
                if self.tail_cap:
                    stc_decode_step_tail(self.shape, q, self.bounds, self.K, self.vpacked,
                                         self.mask, self.tok_off, self.k_eff, self.K_tail,
                                         self.V_tail, self.n_tail, self.tail_cap, self.page_idx,
                                         self.out, self._ws_step)
                else:
                    stc_decode_step(self.shape, q, self.bounds, self.K, self.vpacked, self.mask,
                                    self.tok_off, self.k_eff, self.page_idx, self.out,
                                    self._ws_step)
                return self.out
            self.select(q)
        self.attend(q)
        return self.out


class SharedPrefix:
    """B sequences that continue one prefix: a RoutedCache with B = 1 that holds the prefix, and the
    sequences' own uncompressed tails, per-step outputs and workspace.  As in RoutedCache, allocation
    and nothing else; the lengths of the tails lie on the device (n_tail; a negative one marks an
    element of the batch as padding), so that a step can be captured and replayed.  The prefix is
    whole when the object is made: its own tail is empty (flush moves it into the cache), and it
    does not grow while sequences continue it.  A sequence whose tail is full takes no more tokens:
    append() leaves its tail, length and query as they are and sets dev_status to 1, and attend() then
    answers the query of the step before once more.  The lengths are not known to the host, so nothing
    is raised: who does not stop a sequence in time looks at dev_status, which stays 1 until cleared."""

    n_prefix = 1        # prefixes of the batch

    def __init__(self, prefix, B, tail_cap, rotary=None, out_dtype=torch.float32, pos0=None, nodes=()):
        """rotary: positions for the queries and keys given to append().  pos0: position of a tail's first
        token; None: the one behind the prefix's last, which the prefix knows unless it was built from
        given positions.  nodes: the numbers of nodes that drafts have (one, or several in a tuple)."""
        if prefix.B != self.n_prefix:
            raise ValueError("the prefix is a cache of one batch element")
        self.prefix, self.B, self.tail_cap, self.rotary = prefix, B, tail_cap, rotary
        self.pos0 = pos0
        self.N = prefix.N
        self._whole()
        p, dev = prefix, prefix.device
        self.shape = make_shape(B, p.Hq, p.Hkv, p.D, p.N, p.G, p.shape.v_cap_groups, N_cap=p.n_cap)
        self.n_tail = torch.zeros(B, dtype=torch.int32, device=dev)
        self.K_tail = torch.empty(B, p.Hkv, tail_cap, p.D, dtype=torch.bfloat16, device=dev)
        self.V_tail = torch.empty_like(self.K_tail)
        self.q = torch.zeros(B, p.Hq, p.D, dtype=torch.bfloat16, device=dev)
        self.out = torch.zeros(B, p.Hq, p.D, dtype=out_dtype, device=dev)
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.nodes = (nodes,) if isinstance(nodes, int) else tuple(nodes)
        most = max(self.nodes, default=0)
        self._q_tree = torch.zeros(B * most * p.Hq * p.D, dtype=torch.bfloat16, device=dev)
        self._out_tree = torch.zeros(B * most * p.Hq * p.D, dtype=out_dtype, device=dev)
        # nodes that sequences have, of the last draft; before it, as many as a call says
        self.n_nodes = torch.full((B,), 64, dtype=torch.int32, device=dev)
        self._same = torch.arange(B, dtype=torch.int32, device=dev)
        # the workspace covers every choice of pages
        need = max(self._need(k) for k in range(1, p.NP + 1))
        self._ws = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)

    def _need(self, k):
        return max([stc_shared_workspace_bytes(self.shape, k, self.tail_cap)] +
                   [stc_tree_workspace_bytes(self.shape, T, k, self.tail_cap) for T in self.nodes])

    def _whole(self):
        if self.prefix.n_tail or self.prefix.N != self.N:
            raise ValueError("the prefix has a tail of its own or has grown")

    def _first(self, pos):
        """Position of a tail's first token, for calls that are not given positions."""
        self._whole()
        pos0 = self.prefix.next_pos if self.pos0 is None else self.pos0
        if pos0 is None:
            if self.rotary and pos is None:
                raise ValueError("the prefix was built from given positions: pos0 or pos has to say where "
                                 "its sequences go on")
            pos0 = 0
        return pos0

    def append(self, q, k_new, v_new, pos=None):
        """The new token of every sequence: q [B, Hq, D], k_new, v_new [B, Hkv, D] (without positions
        where rotary is given).  Key and value go to the tails; returns the queries for attend().
        pos [B] int32: the tokens' positions; None: pos0 + n_tail."""
        pos0, r = self._first(pos), self.rotary
        stc_rotary_append(self.shape, q, k_new, v_new, self.q, self.K_tail, self.V_tail, self.n_tail,
                          self.tail_cap, r.turns if r else None, r.rot_dim if r else 0,
                          r.layout if r else STC_ROTARY_HALVES, amplitude=r.amplitude if r else 1.0,
                          pos=pos, pos0=pos0, n_out=self.n_tail, dev_status=self.dev_status)
        return self.q

    def attend(self, q, page_idx=None):
        """page_idx [Hkv, k]: the pages of the prefix to attend; None: all of it."""
        self._whole()
        p = self.prefix
        k = p.NP if page_idx is None else page_idx.shape[-1]
        stc_decode_attention_shared(self.shape, q, p.K, p.vpacked, p.mask, p.tok_off, page_idx, k,
                                    self.K_tail, self.V_tail, self.n_tail, self.tail_cap, self.out,
                                    self._ws)
        return self.out

    def step(self, q, k_new, v_new, page_idx=None, pos=None):
        return self.attend(self.append(q, k_new, v_new, pos), page_idx)

    # Drafted tokens, the nodes of a tree behind each tail: draft, attend_tree (or step_tree for both), and
    # accept for those that stay.  tree, n_draft as in stc_rotary_append_tree.
    def _tree_rows(self, buf, T):
        if T not in self.nodes:
            raise ValueError("drafts have %s nodes, not %d" % (list(self.nodes), T))
        return buf[:self.B * T * self.prefix.Hq * self.prefix.D].view(self.B, T, self.prefix.Hq, self.prefix.D)

    def draft(self, q, k_new, v_new, tree=None, n_draft=None, pos=None):
        """The nodes of every sequence: q [B, T, Hq, D], k_new, v_new [B, T, Hkv, D].  Keys and values go behind
        the tails, whose lengths stay; returns the queries for attend_tree().  Where a sequence has no room for
        all of its nodes, it has none: nothing of it is written, attend_tree() leaves its rows as they are, accept()
        its tail and length, and dev_status becomes 1."""
        pos0, r, out = self._first(pos), self.rotary, self._tree_rows(self._q_tree, q.shape[1])
        stc_rotary_append_tree(self.shape, q, k_new, v_new, out, self.K_tail, self.V_tail, self.n_tail,
                               self.tail_cap, r.turns if r else None, r.rot_dim if r else 0,
                               r.layout if r else STC_ROTARY_HALVES, tree=tree, n_draft=n_draft,
                               amplitude=r.amplitude if r else 1.0, pos=pos, pos0=pos0,
                               dev_status=self.dev_status, n_have=self.n_nodes)
        return out

    def attend_tree(self, q, tree=None, n_draft=None, page_idx=None):
        """The nodes that draft() wrote, or the first n_draft [B] of them.  page_idx as in attend().  Returns
        [B, T, Hq, D]; rows of nodes that are not there are what they were."""
        nodes = self.n_nodes
        if n_draft is not None:
            if n_draft.numel() != self.B:
                raise ValueError("n_draft has a number for each sequence")
            nodes = torch.minimum(n_draft.view(-1), nodes)
        return self._attend_tree(q, self._tree_rows(self._out_tree, q.shape[1]), tree, nodes, page_idx)

    def _attend_tree(self, q, out, tree, n_draft, page_idx):
        self._whole()
        p = self.prefix
        k = p.NP if page_idx is None else page_idx.shape[-1]
        stc_decode_attention_tree(self.shape, q, p.K, p.vpacked, p.mask, p.tok_off, page_idx, k, self.K_tail,
                                  self.V_tail, self.n_tail, self.tail_cap, out, self._ws, tree=tree,
                                  n_draft=n_draft, n_prefix=self.n_prefix)
        return out

    def step_tree(self, q, k_new, v_new, tree=None, n_draft=None, page_idx=None, pos=None):
        return self.attend_tree(self.draft(q, k_new, v_new, tree, n_draft, pos), tree, None, page_idx)

    def accept(self, keep, T, layers=()):
        """keep [B] int64: bits of the nodes (of T, and of those that draft() wrote) that stay, in order, behind the
        tails, which grow by them.  layers: the objects of the model's other layers, for the same in all of them."""
        every = (self,) + tuple(layers)
        stc_accept_tail(self.shape, T, [x.K_tail for x in every], [x.V_tail for x in every],
                        [x.n_tail for x in every], self.tail_cap, keep, n_draft=self.n_nodes)

    def fork(self, src=None, n_keep=None, layers=()):
        """src [B] int32: sequence b goes on with the tail of src[b] (STC_TAIL_FREED: it ends, STC_TAIL_EMPTY: it
        starts anew; None: with its own), the first n_keep[b] tokens of it where given.  layers as in accept()."""
        every = (self,) + tuple(layers)
        stc_fork_tail(self.shape, [x.K_tail for x in every], [x.V_tail for x in every],
                      [x.n_tail for x in every], self.tail_cap, self._same if src is None else src,
                      n_keep=n_keep, dev_status=self.dev_status)


class OwnPrefixes(SharedPrefix):
    """As SharedPrefix, for B sequences that continue a prefix of their own each: `prefix` is a RoutedCache of B
    elements, and page lists have a dimension for them, [B, Hkv, k] (RoutedCache.page_idx).  Sequences do not take
    over others' tails, which belong to other prefixes: fork() only shortens them (n_keep)."""

    def __init__(self, prefix, tail_cap, rotary=None, out_dtype=torch.float32, pos0=None, nodes=()):
        self.n_prefix = prefix.B
        self._blind = torch.zeros(1, dtype=torch.int64, device=prefix.device)
        super().__init__(prefix, prefix.B, tail_cap, rotary, out_dtype, pos0, nodes)

    def _need(self, k):
        return max(stc_tree_workspace_bytes(self.shape, T, k, self.tail_cap, self.n_prefix)
                   for T in (1,) + self.nodes)

    def attend(self, q, page_idx=None):
        # the token was appended: a query that stands behind the tail and sees nothing but it
        one = (self.B, 1, self.prefix.Hq, self.prefix.D)
        self._attend_tree(q.view(one), self.out.view(one), self._blind, None, page_idx)
        return self.out

    def fork(self, src=None, n_keep=None, layers=()):
        if src is not None:
            raise ValueError("sequences with prefixes of their own go on with their own tails")
        super().fork(None, n_keep, layers)
