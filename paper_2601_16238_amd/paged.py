"""Thin binding of the paged key/value cache of include/attn_paged.h: argument marshalling only (csrc/marshal.cpp),
every step runs in the HIP kernels of libmi355attn.so."""
import ctypes

from .binding import _call, lib, marshal

EXPORTS = ("attn_paged_params_contiguous", "attn_paged_append", "attn_paged_append_f16",
           "attn_fwd_paged_workspace_bytes", "attn_fwd_paged", "attn_fwd_paged_f16")


class AttnPagedParams(ctypes.Structure):
    """Mirror of attn_paged_params_t."""
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "B", "Hq", "Hkv", "D", "pages", "page_size", "table_width",
                                              "table_stride", "max_q", "causal", "rot", "table_rows")] + \
               [("scale", ctypes.c_float)] + \
               [(n, ctypes.c_int64) for n in ("q_stride_t", "q_stride_h", "out_stride_t",
                                              "out_stride_h", "kv_stride_t", "kv_stride_h",
                                              "cache_stride_p", "cache_stride_h", "cache_stride_s")]


_bound = False


def _lib():
    global _bound
    L = lib()
    if not _bound:
        vp, i32, pp = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(AttnPagedParams)
        L.attn_paged_params_contiguous.argtypes = [pp] + [i32] * 8 + [ctypes.c_float, i32]
        L.attn_paged_params_contiguous.restype = None
        L.attn_fwd_paged_workspace_bytes.argtypes = [pp]
        L.attn_fwd_paged_workspace_bytes.restype = ctypes.c_size_t
        for n in ("attn_paged_append", "attn_paged_append_f16"):
            getattr(L, n).argtypes = [vp] * 13 + [pp, vp]
            getattr(L, n).restype = ctypes.c_int
        for n in ("attn_fwd_paged", "attn_fwd_paged_f16"):
            getattr(L, n).argtypes = [vp] * 11 + [ctypes.c_size_t, pp, vp]
            getattr(L, n).restype = ctypes.c_int
        _bound = True
    return L


def make_paged_params(T, B, Hq, Hkv, D, pages, page_size, table_width, scale=1.0, causal=False):
    """attn_paged_params_t for contiguous tensors."""
    p = AttnPagedParams()
    _lib().attn_paged_params_contiguous(ctypes.byref(p), T, B, Hq, Hkv, D, pages, page_size, table_width,
                                        float(scale), int(bool(causal)))
    return p


def attn_paged_append(K, V, K_cache, V_cache, page_table, q_start, kv_lens, cos=None, sin=None, Q=None, Q_rot=None,
                      k_scale=None, v_scale=None, stream=None):
    """Appends the batch's rows of K and V [T,Hkv,D] (bf16 or fp16) to the caches [pages,Hkv,page_size,D], in place.
    Sequence b has the rows q_start[b] .. q_start[b+1]-1 (int32 [B+1]); they are the last ones of its kv_lens[b] keys
    (int32 [B], the new rows counted), whose pages page_table[b] lists (int32 [B,width]); all three lie on the GPU.
    cos, sin: fp32 tables [positions, rot/2] that rotate the first rot columns of K and of Q [T,Hq,D], which is
    returned rotated (in Q_rot, if given; it may be Q).  Without Q returns None.
    Caches of torch.float8_e4m3fn: k_scale, v_scale fp32 [pages,Hkv] are updated with them."""
    return _call(marshal().attn_paged_append, stream, K, V, K_cache, V_cache, page_table, q_start, kv_lens, cos, sin,
                 Q, Q_rot, k_scale, v_scale)


def attn_fwd_paged_workspace_bytes(T, B, Hq, Hkv, D, pages, page_size, table_width, max_q=None, causal=True):
    """Bytes attn_fwd_paged needs to spread this problem over the chip (0: none)."""
    p = make_paged_params(T, B, Hq, Hkv, D, pages, page_size, table_width, 1.0, causal)
    if max_q is not None:
        p.max_q = max_q
    return int(_lib().attn_fwd_paged_workspace_bytes(ctypes.byref(p)))


def attn_fwd_paged(Q, K_cache, V_cache, page_table, q_start, kv_lens, scale, causal, k_scale=None, v_scale=None,
                   max_q=None, O=None, LSE=None, workspace=None, split=True, stream=None):
    """O [T,Hq,D], LSE [T,Hq] = attention of the batch's rows Q over the caches; batch and caches as in
    attn_paged_append.  With causal=True the row at position p sees keys 0 .. p, otherwise all kv_lens[b]; a row that
    sees none gets O = 0 and LSE = -inf.  max_q: no sequence has more rows (1 when decoding; without it a
    call counts with sequences of many rows and takes the kernel for those); rows of one that has more are left as they were, as
    are those behind the last sequence.  `split=False` passes no workspace, which leaves every row's keys to one
    work-group.  e4m3 caches with their scales (any fp32 scale that is 0 or positive and normal)."""
    return _call(marshal().attn_fwd_paged, stream, Q, K_cache, V_cache, page_table, q_start, kv_lens, float(scale),
                 bool(causal), k_scale, v_scale, None if max_q is None else int(max_q), O, LSE, workspace, bool(split))
