"""Thin Python binding of libstom_oqm.so (argument marshalling only): ctypes, and for the calls of the paged cache, the
next token and the 4-bit products, which are made once per token, _stom_bind.so (written against torch's C++ tensors; only
those calls need it).

Every step of the path runs in the library's CUDA kernels; PyTorch is used for
device memory and streams.  There is no CPU fallback: if the library is not
built, importing `lib()` raises.
"""
from __future__ import annotations

import ctypes as C
from pathlib import Path

import torch

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libstom_oqm.so"

BF16, FP16, FP32 = 0, 1, 2
PER_LAYER, PER_HEAD = 0, 1
FLAG_BAD_INDEX = 1
FLAG_TIMEOUT = 2
FLAG_DIRTY_WORKSPACE = 4
FLAG_NO_PAGE = 8
FLAG_BAD_VALUE = 16

ROPE_HALF, ROPE_PAIRS = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_WAVES = 0, 1, 2, 3

_TORCH_DTYPE = {BF16: torch.bfloat16, FP16: torch.float16, FP32: torch.float32}
_DTYPE_CODE = {v: k for k, v in _TORCH_DTYPE.items()}

EXPORTS = (
    "stom_oqm_store_layout", "stom_oqm_store_bind", "stom_oqm_budget_to_k", "stom_oqm_score_workspace_bytes",
    "stom_status_string", "stom_last_cuda_error", "stom_oqm_quantize_frame", "stom_oqm_score_groups",
    "stom_oqm_topk", "stom_oqm_dequant_gather", "stom_oqm_retrieve",
    "stom_oqm_quantize_host_scratch_bytes", "stom_oqm_quantize_frame_host",
    "stom_oqm_retrieve_host_scratch_bytes", "stom_oqm_retrieve_host",
    "stom_oqm_score_groups_noalloc", "stom_oqm_attend_workspace_bytes", "stom_oqm_attend",
    "stom_oqm_retrieve_workspace_bytes",
    "stom_ctr_similarity", "stom_ctr_select", "stom_ctr_reduce", "stom_ctr_merge", "stom_ctr_reduce_tokens",
    "stom_kv_frequencies", "stom_kv_attend_workspace_bytes", "stom_kv_attend",
    "stom_kv_rotate", "stom_kv_append", "stom_kv_pages_workspace_bytes", "stom_kv_reserve", "stom_kv_fork",
    "stom_kv_free", "stom_kv_compact", "stom_sample_tokens",
    "stom_kv_attend_tree_workspace_bytes", "stom_kv_attend_tree", "stom_kv_accept", "stom_w4_workspace_bytes",
    "stom_w4_linear",
)


class Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_layers", "n_q_heads", "n_kv_heads", "head_dim", "group_tokens",
        "capacity_groups", "bits", "kv_dtype", "score_mode", "meta_dtype")]


class StoreDesc(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in (
        "codes_k", "codes_v", "scale_k", "zero_k", "scale_v", "zero_v", "rep_key", "rep_norm2")]


class Layout(C.Structure):
    _fields_ = [(n, C.c_int64) for n in (
        "bytes_total", "off_codes_k", "off_codes_v", "off_scale_k", "off_zero_k", "off_scale_v", "off_zero_v",
        "off_rep_key", "off_rep_norm2", "bytes_codes", "bytes_meta", "bytes_norm2")]


class KvPoolDesc(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p)] + [(n, C.c_int32) for n in (
        "dtype", "n_layers", "n_pages", "page_tokens", "n_kv_heads", "head_dim")] + [(n, C.c_int64) for n in (
            "stride_layer", "stride_page", "stride_token", "stride_head")]


class KvSeqsDesc(C.Structure):
    _fields_ = [("table", C.c_void_p), ("len", C.c_void_p), ("refs", C.c_void_p), ("n_seqs", C.c_int32),
                ("max_pages", C.c_int32), ("table_stride", C.c_int64)]


class RopeDesc(C.Structure):
    _fields_ = [("freq", C.c_void_p), ("rot_dim", C.c_int32), ("layout", C.c_int32), ("magnitude", C.c_float)]


class W4Desc(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scale", C.c_void_p), ("zero", C.c_void_p)] + [(n, C.c_int32) for n in (
        "n", "k", "group", "meta_dtype")] + [("code_stride", C.c_int64), ("meta_stride", C.c_int64)]


class StomError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().stom_status_string(code).decode()
        super().__init__(f"{where}: {msg} (status {code}, cuda error {lib().stom_last_cuda_error()})")


# Result and argument types of the calls for the paged cache and the next token, for those who make them through ctypes:
# p pointer, i int32, l int64, f float, d double.
_CTYPE = {"p": C.c_void_p, "i": C.c_int32, "l": C.c_int64, "f": C.c_float, "d": C.c_double}
_SIGNATURES = {
    "stom_kv_frequencies": (C.c_int32, "ididdddp"),
    "stom_kv_attend_workspace_bytes": (C.c_int64, "ppi"),
    "stom_kv_attend": (C.c_int32, "ppiipllffipllpplpp"),
    "stom_kv_rotate": (C.c_int32, "piiip" + 2 * "pillpllp" + "fp"),
    "stom_kv_append": (C.c_int32, "ppipippp" + "pillpllp" + "pllp" + "pll" + "fpp"),
    "stom_kv_pages_workspace_bytes": (C.c_int64, "pp"),
    "stom_kv_reserve": (C.c_int32, "pppplpp"),
    "stom_kv_fork": (C.c_int32, "ppppp"),
    "stom_kv_free": (C.c_int32, "ppppp"),
    "stom_kv_compact": (C.c_int32, "ppppppl" + "pp"),
    "stom_sample_tokens": (C.c_int32, "piiil" + "ppppp" + "ppp" + "pp"),
    "stom_kv_attend_tree_workspace_bytes": (C.c_int64, "ppii"),
    "stom_kv_attend_tree": (C.c_int32, "ppii" + "pp" + "ipllffi" + "pllp" + "plpp"),
    "stom_kv_accept": (C.c_int32, "ppi" + "pppp" + "ppp" + "pp"),
    "stom_w4_workspace_bytes": (C.c_int64, "pi"),
    "stom_w4_linear": (C.c_int32, "piipl" + "ppl" + "pl" + "plpp"),
}

_lib = None
_bind = None   # the binding of the calls that are made once per token, loaded by the first of them
_BOUND = ("stom_kv_attend", "stom_kv_rotate", "stom_kv_append", "stom_kv_reserve", "stom_kv_fork", "stom_kv_free",
          "stom_kv_compact", "stom_sample_tokens", "stom_kv_attend_tree", "stom_kv_accept", "stom_w4_linear",
          "stom_w4_workspace_bytes")


def lib():
    """The loaded C-ABI library.  Fails loudly when it has not been built."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2510_18269_b200.build` "
                "(there is no fallback path)")
        L = C.CDLL(str(LIB_PATH))
        L.stom_status_string.restype = C.c_char_p
        L.stom_status_string.argtypes = [C.c_int32]
        L.stom_oqm_score_workspace_bytes.restype = C.c_int64
        L.stom_oqm_score_workspace_bytes.argtypes = [C.POINTER(Config), C.c_int32]
        L.stom_oqm_budget_to_k.argtypes = [C.c_int64, C.c_int32, C.c_int32]
        L.stom_oqm_attend_workspace_bytes.restype = C.c_int64
        L.stom_oqm_retrieve_workspace_bytes.restype = C.c_int64
        L.stom_oqm_quantize_host_scratch_bytes.restype = C.c_int64
        L.stom_oqm_retrieve_host_scratch_bytes.restype = C.c_int64
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, [_CTYPE[a] for a in args]
        for name in EXPORTS:
            fn = getattr(L, name)
            if fn.restype is C.c_int:
                fn.restype = C.c_int32
        _lib = L
    return _lib


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def _check(rc: int, where: str):
    if rc != 0:
        raise StomError(rc, where)


def make_config(n_layers, n_q_heads, n_kv_heads, head_dim, group_tokens, capacity_groups,
                bits=4, kv_dtype=BF16, score_mode=PER_LAYER, meta_dtype=FP32) -> Config:
    return Config(n_layers, n_q_heads, n_kv_heads, head_dim, group_tokens, capacity_groups,
                  bits, kv_dtype, score_mode, meta_dtype)


def dtype_code(t: torch.dtype) -> int:
    return _DTYPE_CODE[t]


def stom_oqm_store_layout(cfg: Config) -> Layout:
    lay = Layout()
    _check(lib().stom_oqm_store_layout(C.byref(cfg), C.byref(lay)), "stom_oqm_store_layout")
    return lay


def stom_oqm_budget_to_k(budget_tokens: int, group_tokens: int, stored_groups: int) -> int:
    return int(lib().stom_oqm_budget_to_k(budget_tokens, group_tokens, stored_groups))


def stom_oqm_score_workspace_bytes(cfg: Config, layer_count: int) -> int:
    return int(lib().stom_oqm_score_workspace_bytes(C.byref(cfg), layer_count))


class Store:
    """One device arena holding the memory bank, plus typed tensor views of its arrays."""

    def __init__(self, cfg: Config, device="cuda", zero: bool = True):
        self.cfg = cfg
        self.layout = stom_oqm_store_layout(cfg)
        alloc = torch.zeros if zero else torch.empty
        self.arena = alloc(self.layout.bytes_total + 256, dtype=torch.uint8, device=device)
        shift = (-self.arena.data_ptr()) % 256
        self.base = self.arena[shift:shift + self.layout.bytes_total]
        self.desc = StoreDesc()
        _check(lib().stom_oqm_store_bind(C.byref(cfg), C.c_void_p(self.base.data_ptr()), C.byref(self.desc)),
               "stom_oqm_store_bind")
        L, T, H, G, d = cfg.n_layers, cfg.capacity_groups, cfg.n_kv_heads, cfg.group_tokens, cfg.head_dim
        lay = self.layout

        def view(off, nbytes, dtype, shape):
            return self.base[off:off + nbytes].view(dtype).view(*shape)

        self.codes_k = view(lay.off_codes_k, lay.bytes_codes, torch.uint8, (L, T, H, G, d * cfg.bits // 8))
        self.codes_v = view(lay.off_codes_v, lay.bytes_codes, torch.uint8, (L, T, H, G, d * cfg.bits // 8))
        mt = _TORCH_DTYPE[cfg.meta_dtype]  # element type of s, m and k-bar
        self.scale_k = view(lay.off_scale_k, lay.bytes_meta, mt, (L, T, H, d))
        self.zero_k = view(lay.off_zero_k, lay.bytes_meta, mt, (L, T, H, d))
        self.scale_v = view(lay.off_scale_v, lay.bytes_meta, mt, (L, T, H, d))
        self.zero_v = view(lay.off_zero_v, lay.bytes_meta, mt, (L, T, H, d))
        self.rep_key = view(lay.off_rep_key, lay.bytes_meta, mt, (L, T, H, d))
        self.rep_norm2 = view(lay.off_rep_norm2, lay.bytes_norm2, torch.float32, (L, T, H))


def stom_oqm_quantize_frame(cfg: Config, store: Store, layer_begin, layer_count, group_begin, group_count,
                            K, V, strides, K_summary=None, token_idx=None, tokens_per_frame_in=0,
                            dev_flags=None, stream=None):
    """strides = (layer, group, head, token) in elements of K / V."""
    sl, sg, sh, st = strides
    rc = lib().stom_oqm_quantize_frame(
        C.byref(cfg), C.byref(store.desc), C.c_int32(layer_begin), C.c_int32(layer_count),
        C.c_int32(group_begin), C.c_int32(group_count), _ptr(K), _ptr(V),
        C.c_int64(sl), C.c_int64(sg), C.c_int64(sh), C.c_int64(st), _ptr(K_summary), _ptr(token_idx),
        C.c_int32(tokens_per_frame_in), _ptr(dev_flags), _stream(stream))
    _check(rc, "stom_oqm_quantize_frame")


def stom_oqm_score_groups(cfg: Config, store: Store, layer_begin, layer_count, n_groups, Q, T_q, q_strides,
                          scores, workspace, stream=None):
    ql, qh, qt = q_strides
    rc = lib().stom_oqm_score_groups(
        C.byref(cfg), C.byref(store.desc), C.c_int32(layer_begin), C.c_int32(layer_count), C.c_int32(n_groups),
        _ptr(Q), C.c_int32(T_q), C.c_int64(ql), C.c_int64(qh), C.c_int64(qt), _ptr(scores), _ptr(workspace),
        C.c_int64(0 if workspace is None else workspace.numel() * workspace.element_size()), _stream(stream))
    _check(rc, "stom_oqm_score_groups")


NOALLOC_SCRATCH_BYTES = 512 * 1024


def stom_oqm_score_groups_noalloc(cfg: Config, store: Store, layer_begin, layer_count, n_groups, Q, T_q, q_strides,
                                  scores, stream=None):
    """Scores without caller scratch, for hosts that cannot allocate device memory (for example a server whose
    memory pool owns all of HBM, or code that may not call cudaMalloc because it would stall the device).

    Same result as stom_oqm_score_groups.  The intermediate question embeddings live in a NOALLOC_SCRATCH_BYTES
    array inside the library that all calls on a GPU share: keep such calls ordered on the GPU (one stream, or
    events), make the first call on each GPU outside of stream capture, and split the layer range when the call
    reports that the array is too small."""
    ql, qh, qt = q_strides
    rc = lib().stom_oqm_score_groups_noalloc(
        C.byref(cfg), C.byref(store.desc), C.c_int32(layer_begin), C.c_int32(layer_count), C.c_int32(n_groups),
        _ptr(Q), C.c_int32(T_q), C.c_int64(ql), C.c_int64(qh), C.c_int64(qt), _ptr(scores), _stream(stream))
    _check(rc, "stom_oqm_score_groups_noalloc")


def stom_oqm_topk(scores, rows, n, row_stride, k, idx_out, score_out=None, n_sel_out=None, stream=None):
    rc = lib().stom_oqm_topk(_ptr(scores), C.c_int32(rows), C.c_int32(n), C.c_int64(row_stride), C.c_int32(k),
                             _ptr(idx_out), _ptr(score_out), _ptr(n_sel_out), _stream(stream))
    _check(rc, "stom_oqm_topk")


def stom_oqm_dequant_gather(cfg: Config, store: Store, layer_begin, layer_count, idx, k, n_groups,
                            k_active, v_active, out_dtype, strides, token_offset, dev_flags=None, stream=None):
    """strides = (layer, head, token) in elements of the active cache."""
    sl, sh, st = strides
    rc = lib().stom_oqm_dequant_gather(
        C.byref(cfg), C.byref(store.desc), C.c_int32(layer_begin), C.c_int32(layer_count), _ptr(idx),
        C.c_int32(k), C.c_int32(n_groups), _ptr(k_active), _ptr(v_active), C.c_int32(out_dtype),
        C.c_int64(sl), C.c_int64(sh), C.c_int64(st), C.c_int32(token_offset), _ptr(dev_flags), _stream(stream))
    _check(rc, "stom_oqm_dequant_gather")


def stom_oqm_retrieve_workspace_bytes(cfg: Config, layer_count: int, n_groups: int, k: int) -> int:
    return int(lib().stom_oqm_retrieve_workspace_bytes(C.byref(cfg), C.c_int32(layer_count), C.c_int32(n_groups),
                                                       C.c_int32(k)))


def stom_oqm_retrieve(cfg: Config, store: Store, layer_begin, layer_count, n_groups, Q, T_q, q_strides, k,
                      scores, idx, k_active, v_active, out_dtype, strides, token_offset, workspace,
                      dev_flags=None, stream=None):
    ql, qh, qt = q_strides
    sl, sh, st = strides
    rc = lib().stom_oqm_retrieve(
        C.byref(cfg), C.byref(store.desc), C.c_int32(layer_begin), C.c_int32(layer_count), C.c_int32(n_groups),
        _ptr(Q), C.c_int32(T_q), C.c_int64(ql), C.c_int64(qh), C.c_int64(qt), C.c_int32(k), _ptr(scores),
        _ptr(idx), _ptr(k_active), _ptr(v_active), C.c_int32(out_dtype), C.c_int64(sl), C.c_int64(sh),
        C.c_int64(st), C.c_int32(token_offset), _ptr(workspace),
        C.c_int64(0 if workspace is None else workspace.numel() * workspace.element_size()), _ptr(dev_flags),
        _stream(stream))
    _check(rc, "stom_oqm_retrieve")


def stom_oqm_attend_workspace_bytes(cfg: Config, layer_count: int, k: int, sys_len: int) -> int:
    return int(lib().stom_oqm_attend_workspace_bytes(C.byref(cfg), C.c_int32(layer_count), C.c_int32(k),
                                                     C.c_int32(sys_len)))


def stom_oqm_attend(cfg: Config, store: Store, layer_begin, layer_count, idx, k, n_groups, q_dec, q_strides,
                    k_sys, v_sys, cache_dtype, sys_strides, sys_len, softmax_scale, out, out_strides, workspace,
                    dev_flags=None, stream=None):
    """q_strides = (layer, head); sys_strides = (layer, head, token); out_strides = (layer, head), all in elements.
    `workspace` is not used by the call (it may be None); the argument remains for callers of the earlier form."""
    rc = lib().stom_oqm_attend(
        C.byref(cfg), C.byref(store.desc), C.c_int32(layer_begin), C.c_int32(layer_count), _ptr(idx), C.c_int32(k),
        C.c_int32(n_groups), _ptr(q_dec), C.c_int64(q_strides[0]), C.c_int64(q_strides[1]), _ptr(k_sys), _ptr(v_sys),
        C.c_int32(cache_dtype), C.c_int64(sys_strides[0]), C.c_int64(sys_strides[1]), C.c_int64(sys_strides[2]),
        C.c_int32(sys_len), C.c_float(softmax_scale), _ptr(out), C.c_int64(out_strides[0]), C.c_int64(out_strides[1]),
        _ptr(workspace), C.c_int64(0 if workspace is None else workspace.numel() * workspace.element_size()),
        _ptr(dev_flags), _stream(stream))
    _check(rc, "stom_oqm_attend")


# ---------------------------------------------------------------- host-buffer entry points

def _hptr(t):
    """Address of a HOST tensor (pinned or pageable)."""
    if t is None:
        return None
    assert not t.is_cuda and t.is_contiguous()
    return C.c_void_p(t.data_ptr())


def stom_oqm_quantize_host_scratch_bytes(cfg: Config, layer_count: int, group_count: int) -> int:
    return int(lib().stom_oqm_quantize_host_scratch_bytes(C.byref(cfg), C.c_int32(layer_count), C.c_int32(group_count)))


def stom_oqm_quantize_frame_host(cfg: Config, store: Store, layer_begin, layer_count, group_begin, group_count,
                                 K_host, V_host, scratch, dev_flags=None, stream=None):
    rc = lib().stom_oqm_quantize_frame_host(
        C.byref(cfg), C.byref(store.desc), C.c_int32(layer_begin), C.c_int32(layer_count), C.c_int32(group_begin),
        C.c_int32(group_count), _hptr(K_host), _hptr(V_host), _ptr(scratch),
        C.c_int64(scratch.numel() * scratch.element_size()), _ptr(dev_flags), _stream(stream))
    _check(rc, "stom_oqm_quantize_frame_host")


def stom_oqm_retrieve_host_scratch_bytes(cfg: Config, layer_count, n_groups, T_q, k, out_dtype) -> int:
    return int(lib().stom_oqm_retrieve_host_scratch_bytes(
        C.byref(cfg), C.c_int32(layer_count), C.c_int32(n_groups), C.c_int32(T_q), C.c_int32(k), C.c_int32(out_dtype)))


def stom_oqm_retrieve_host(cfg: Config, store: Store, layer_begin, layer_count, n_groups, Q_host, T_q, k,
                           idx_host, k_active_host, v_active_host, out_dtype, scratch, dev_flags=None, stream=None):
    rc = lib().stom_oqm_retrieve_host(
        C.byref(cfg), C.byref(store.desc), C.c_int32(layer_begin), C.c_int32(layer_count), C.c_int32(n_groups),
        _hptr(Q_host), C.c_int32(T_q), C.c_int32(k), _hptr(idx_host), _hptr(k_active_host), _hptr(v_active_host),
        C.c_int32(out_dtype), _ptr(scratch), C.c_int64(scratch.numel() * scratch.element_size()), _ptr(dev_flags),
        _stream(stream))
    _check(rc, "stom_oqm_retrieve_host")


# ---------------------------------------------------------------- CTR (include/stom_ctr.h)

def stom_ctr_similarity(F, prev, T, N, D, strides, sim, stream=None):
    """F: device tensor of T x N x D features (strides = (frame, token) in elements); prev: [N][D] or None."""
    sf, st = strides
    _check(lib().stom_ctr_similarity(_ptr(F), _ptr(prev), C.c_int32(dtype_code(F.dtype)), C.c_int32(T), C.c_int32(N),
                                     C.c_int32(D), C.c_int64(sf), C.c_int64(st), _ptr(sim), _stream(stream)),
           "stom_ctr_similarity")


def stom_ctr_select(sim, alpha, T, N, G, tau_c, k_s, k_d, static_idx, dyn_idx, stream=None):
    _check(lib().stom_ctr_select(_ptr(sim), _ptr(alpha), C.c_int32(T), C.c_int32(N), C.c_int32(G), C.c_float(tau_c),
                                 _ptr(k_s), _ptr(k_d), _ptr(static_idx), _ptr(dyn_idx), _stream(stream)),
           "stom_ctr_select")


def stom_ctr_reduce(F, prev, T, N, D, strides, alpha, G, tau_c, sim, k_s, k_d, static_idx, dyn_idx, stream=None):
    sf, st = strides
    _check(lib().stom_ctr_reduce(_ptr(F), _ptr(prev), C.c_int32(dtype_code(F.dtype)), C.c_int32(T), C.c_int32(N),
                                 C.c_int32(D), C.c_int64(sf), C.c_int64(st), _ptr(alpha), C.c_int32(G),
                                 C.c_float(tau_c), _ptr(sim), _ptr(k_s), _ptr(k_d), _ptr(static_idx), _ptr(dyn_idx),
                                 _stream(stream)), "stom_ctr_reduce")


def stom_ctr_merge(F, T, N, D, strides, k_s, k_d, static_idx, dyn_idx, G, knn, retained, retained_pos, centre=None,
                   assign=None, dev_flags=None, stream=None):
    """Merge_{k_s} of the static tokens and the retained group [T][G][D] (see include/stom_ctr.h for the rule)."""
    sf, st = strides
    _check(lib().stom_ctr_merge(_ptr(F), C.c_int32(dtype_code(F.dtype)), C.c_int32(T), C.c_int32(N), C.c_int32(D),
                                C.c_int64(sf), C.c_int64(st), _ptr(k_s), _ptr(k_d), _ptr(static_idx), _ptr(dyn_idx),
                                C.c_int32(G), C.c_int32(knn), _ptr(retained), _ptr(retained_pos), _ptr(centre),
                                _ptr(assign), _ptr(dev_flags), _stream(stream)), "stom_ctr_merge")


def stom_ctr_reduce_tokens(F, prev, T, N, D, strides, alpha, G, tau_c, knn, sim, k_s, k_d, static_idx, dyn_idx, retained,
                           retained_pos, dev_flags=None, stream=None):
    sf, st = strides
    _check(lib().stom_ctr_reduce_tokens(_ptr(F), _ptr(prev), C.c_int32(dtype_code(F.dtype)), C.c_int32(T), C.c_int32(N),
                                        C.c_int32(D), C.c_int64(sf), C.c_int64(st), _ptr(alpha), C.c_int32(G),
                                        C.c_float(tau_c), C.c_int32(knn), _ptr(sim), _ptr(k_s), _ptr(k_d),
                                        _ptr(static_idx), _ptr(dyn_idx), _ptr(retained), _ptr(retained_pos),
                                        _ptr(dev_flags), _stream(stream)), "stom_ctr_reduce_tokens")


# ---------------------------------------------------------------- paged cache (include/stom_kv.h)

def _addr(t):
    return None if t is None else t.data_ptr()


def _dense(t, dtype, shape, name, dev):
    """Address of a contiguous tensor of this type and shape on device number `dev` (-1: the CPU), or None."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} on device {dev} is needed, not "
                     f"{t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _binding():
    """The loaded binding of the calls made once per token.  Fails loudly when it has not been built for this torch."""
    global _bind
    if _bind is None:
        L = lib()
        try:
            from . import _stom_bind
        except ImportError as e:
            raise ImportError(f"{_PKG / '_stom_bind.so'} is missing or does not fit: build it with "
                              "`python -m paper_2510_18269_b200.build`") from e
        _stom_bind.use(*(C.cast(getattr(L, n), C.c_void_p).value for n in _BOUND))
        _bind = _stom_bind
    return _bind


def _handle(stream):
    """What the binding takes for a stream: its handle, or None for the current one of the call's device."""
    return None if stream is None else stream.cuda_stream


class KvPool:
    """Pages of keys and values: two tensors [layers][pages][page_tokens][kv heads][d] of the same strides."""

    def __init__(self, k, v):
        if k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.device != v.device or k.dim() != 5:
            raise ValueError("k and v are two [layers][pages][page_tokens][heads][d] tensors of the same type and strides")
        if k.stride(4) != 1:
            raise ValueError("the channels of a head are adjacent")
        self.k, self.v, self.dev, self.dtype = k, v, k.get_device(), k.dtype
        L, P, n, H, d = k.shape
        self.n_layers, self.n_pages, self.page_tokens, self.n_kv_heads, self.head_dim = L, P, n, H, d
        self.desc = KvPoolDesc(k.data_ptr(), v.data_ptr(), dtype_code(k.dtype), L, P, n, H, d, *k.stride()[:4])
        self.ref = C.addressof(self.desc)


class KvSeqs:
    """The sequences of a pool: table [n_seqs][max_pages], len [n_seqs] and refs [pages], all int32."""

    def __init__(self, table, len, refs=None):
        n, width = table.shape
        if table.dtype is not torch.int32 or (width > 1 and table.stride(1) != 1):
            raise ValueError("table: int32 [n_seqs][max_pages] with adjacent entries")
        self.dev = table.get_device()
        _dense(len, torch.int32, (n,), "len", self.dev)
        if refs is not None:
            _dense(refs, torch.int32, (refs.numel(),), "refs", self.dev)
        self.table, self.len, self.refs, self.n_seqs, self.max_pages = table, len, refs, n, width
        self.n_refs = 0 if refs is None else refs.numel()
        stride = table.stride(0) if n > 1 else width
        self.desc = KvSeqsDesc(_addr(table), _addr(len), _addr(refs), n, width, stride)
        self.ref = C.addressof(self.desc)


class Rope:
    """Rotation of the first 2 * freq.numel() channels; freq: float64 tensor of radians per position."""

    def __init__(self, freq=None, layout=ROPE_HALF, magnitude=1.0):
        if freq is not None:
            _dense(freq, torch.float64, (freq.numel(),), "freq", freq.get_device())
        self.freq, self.rot_dim = freq, 0 if freq is None else 2 * freq.numel()
        self.dev = None if freq is None else freq.get_device()
        self.desc = RopeDesc(_addr(freq), self.rot_dim, layout, magnitude)
        self.ref = C.addressof(self.desc)


def stom_kv_frequencies(rot_dim, theta=1.0e6, scaling=ROPE_PLAIN, factor=1.0, trained=0.0, low=1.0, high=4.0):
    """Radians per position of every rotated pair, as a float64 CPU tensor (move it to the device once)."""
    out = torch.empty(max(rot_dim // 2, 0), dtype=torch.float64)
    _check(lib().stom_kv_frequencies(rot_dim, theta, scaling, factor, trained, low, high, out.data_ptr()),
           "stom_kv_frequencies")
    return out


def stom_kv_attend_workspace_bytes(pool: KvPool, seqs: KvSeqs, n_q_heads: int) -> int:
    n = lib().stom_kv_attend_workspace_bytes(pool.ref, seqs.ref, n_q_heads)
    if n < 0:
        _check(int(n), "stom_kv_attend_workspace_bytes")
    return int(n)


def _same_device(pool, seqs, rope=None):
    if seqs.dev != pool.dev or (rope is not None and rope.dev is not None and rope.dev != pool.dev):
        raise ValueError("pool, table and frequencies lie on the same device")


def stom_kv_attend(pool: KvPool, seqs: KvSeqs, layer, q, out, softmax_scale, workspace, lse=None, softcap=0.0, window=0,
                   dev_flags=None, stream=None):
    """q, out: [n_seqs][query heads][d] of the pool's type; lse: [n_seqs][query heads] float32 or None."""
    _same_device(pool, seqs)
    rc = _binding().attend(pool.ref, seqs.ref, pool.dev, layer, q, out, softmax_scale, softcap, window, lse, workspace,
                           dev_flags, _handle(stream))
    if rc:
        _check(rc, "stom_kv_attend")


def stom_kv_attend_tree_workspace_bytes(pool: KvPool, seqs: KvSeqs, n_tokens: int, n_q_heads: int) -> int:
    n = lib().stom_kv_attend_tree_workspace_bytes(pool.ref, seqs.ref, n_tokens, n_q_heads)
    if n < 0:
        _check(int(n), "stom_kv_attend_tree_workspace_bytes")
    return int(n)


def stom_kv_attend_tree(pool: KvPool, seqs: KvSeqs, layer, first, q, out, softmax_scale, workspace, parent=None, lse=None,
                        softcap=0.0, window=0, dev_flags=None, stream=None):
    """The last first[i + 1] - first[i] tokens of every sequence, rows first[i] ... of q and out ([n][query heads][d] of the
    pool's type) and of lse ([n][query heads] float32 or None); first: int32 [n_seqs + 1]; parent: int32 [n], the node of
    its sequence that each follows (-1: the context), or None: each follows the one before it."""
    _same_device(pool, seqs)
    rc = _binding().attend_tree(pool.ref, seqs.ref, pool.dev, layer, first, parent, q, out, softmax_scale, softcap, window, lse,
                                workspace, dev_flags, _handle(stream))
    if rc:
        _check(rc, "stom_kv_attend_tree")


def stom_kv_rotate(rope: Rope, pos, q=None, q_out=None, k=None, k_out=None, q_weight=None, k_weight=None, eps=1e-6,
                   stream=None):
    """q, k and their outputs: [n][heads][d], each with its own strides (an output may be its input); pos: int32 [n];
    weights: float32 [d] or None (no norm)."""
    rc = _binding().rotate(rope.ref, pos, q, q_out, k, k_out, q_weight, k_weight, eps, _handle(stream), rope.dev)
    if rc:
        _check(rc, "stom_kv_rotate")


def stom_kv_append(pool: KvPool, seqs: KvSeqs, layer, rope: Rope, pos, slot, k, v, q=None, q_out=None, seq=None,
                   q_weight=None, k_weight=None, eps=1e-6, dev_flags=None, stream=None):
    """k, v: [n][kv heads][d] of the pool's type; slot, pos, seq: int32 [n]; q and q_out: [n][query heads][d] or None."""
    _same_device(pool, seqs, rope)
    rc = _binding().append(pool.ref, seqs.ref, pool.dev, layer, rope.ref, pos, slot, k, v, q, q_out, seq, q_weight, k_weight,
                           eps, dev_flags, _handle(stream))
    if rc:
        _check(rc, "stom_kv_append")


def stom_kv_pages_workspace_bytes(pool: KvPool, seqs: KvSeqs) -> int:
    n = lib().stom_kv_pages_workspace_bytes(pool.ref, seqs.ref)
    if n < 0:
        _check(int(n), "stom_kv_pages_workspace_bytes")
    return int(n)


def _counts_of(pool, seqs):
    if seqs.refs is None or seqs.n_refs != pool.n_pages:
        raise ValueError("the sequences need refs, one count for each page of the pool")
    _same_device(pool, seqs)


def stom_kv_reserve(pool: KvPool, seqs: KvSeqs, want, workspace, dev_flags=None, stream=None):
    """want: int32 [n_seqs], the length each sequence grows to (at most its length: it stays)."""
    _counts_of(pool, seqs)
    _check(_binding().reserve(pool.ref, seqs.ref, pool.dev, want, workspace, dev_flags, _handle(stream)), "stom_kv_reserve")


def stom_kv_fork(pool: KvPool, seqs: KvSeqs, parent, dev_flags=None, stream=None):
    """parent: int32 [n_seqs], the sequence an empty one shares from now on, or -1."""
    _counts_of(pool, seqs)
    _check(_binding().fork(pool.ref, seqs.ref, pool.dev, parent, dev_flags, _handle(stream)), "stom_kv_fork")


def stom_kv_free(pool: KvPool, seqs: KvSeqs, drop, dev_flags=None, stream=None):
    """drop: int32 [n_seqs], not 0 for the sequences that give their pages back."""
    _counts_of(pool, seqs)
    _check(_binding().free(pool.ref, seqs.ref, pool.dev, drop, dev_flags, _handle(stream)), "stom_kv_free")


def stom_kv_compact(pool: KvPool, seqs: KvSeqs, table_out, refs_out, n_live, workspace, dev_flags=None, stream=None):
    """table_out, refs_out: like seqs.table and seqs.refs (or those themselves); n_live: int32 [1] or None."""
    _counts_of(pool, seqs)
    _check(_binding().compact(pool.ref, seqs.ref, pool.dev, table_out, refs_out, n_live, workspace, dev_flags,
                              _handle(stream)), "stom_kv_compact")


def stom_kv_accept(pool: KvPool, seqs: KvSeqs, first, draft, chosen, path=None, n_accepted=None, next=None, parent=None,
                   dev_flags=None, stream=None):
    """Keeps each sequence's longest drafted path that was chosen.  first, parent as in stom_kv_attend_tree; draft, chosen,
    path: int32 [n]; n_accepted, next: int32 [n_seqs]."""
    _counts_of(pool, seqs)
    _check(_binding().accept(pool.ref, seqs.ref, pool.dev, first, parent, draft, chosen, path, n_accepted, next, dev_flags,
                             _handle(stream)), "stom_kv_accept")


# ---------------------------------------------------------------- choice of the next token (include/stom_sample.h)

def stom_sample_tokens(logits, u, token, temperature=None, top_k=None, top_p=None, min_p=None, logprob=None, kept=None,
                       dev_flags=None, stream=None):
    """logits: [rows][n]; u, temperature, top_p, min_p, logprob: float32 [rows]; token, kept, top_k: int32 [rows]."""
    rc = _binding().sample(logits, u, token, temperature, top_k, top_p, min_p, logprob, kept, dev_flags, _handle(stream))
    if rc:
        _check(rc, "stom_sample_tokens")


# ---------------------------------------------------------------- products with 4-bit weights (include/stom_w4.h)

class W4Matrix:
    """[n][k] weights of 4 bits: codes uint8 [n][k / 2] (even columns in the low halves), scale and zero [n][k / group] of one
    type and the same strides; zero None: a code stands for (code - 8) * scale."""

    def __init__(self, codes, scale, zero=None):
        if codes.dtype is not torch.uint8 or codes.dim() != 2 or (codes.shape[1] > 1 and codes.stride(1) != 1):
            raise ValueError("codes: uint8 [n][k / 2] with adjacent entries")
        n, k = codes.shape[0], 2 * codes.shape[1]
        if (scale.dim() != 2 or scale.shape[0] != n or scale.shape[1] < 1 or k % scale.shape[1] or scale.dtype not in _DTYPE_CODE
                or (scale.shape[1] > 1 and scale.stride(1) != 1) or scale.device != codes.device):
            raise ValueError("scale: [n][k / group] with adjacent entries on the device of the codes")
        if zero is not None and (zero.shape != scale.shape or zero.stride() != scale.stride() or zero.dtype != scale.dtype
                                 or zero.device != scale.device):
            raise ValueError("zero: like scale")
        self.codes, self.scale, self.zero, self.dev = codes, scale, zero, codes.get_device()
        self.n, self.k, self.group = n, k, k // scale.shape[1]
        strides = [t.stride(0) if n > 1 else t.shape[1] for t in (codes, scale)]
        self.desc = W4Desc(_addr(codes), _addr(scale), _addr(zero), n, k, self.group, dtype_code(scale.dtype), *strides)
        self.ref = C.addressof(self.desc)


def stom_w4_workspace_bytes(w: W4Matrix, rows: int) -> int:
    with torch.cuda.device(w.dev):   # (what is needed goes by the device's size)
        n = lib().stom_w4_workspace_bytes(w.ref, rows)
    if n < 0:
        _check(int(n), "stom_w4_workspace_bytes")
    return int(n)


def stom_w4_linear(w: W4Matrix, x, y, bias=None, add=None, workspace=None, dev_flags=None, stream=None):
    """y = x W^T + bias + add; x: [rows][k], y and add: [rows][n], bias: [n], all bfloat16 or all float16; add may be y.
    workspace None: what is needed is taken from torch's allocator for the call."""
    rc = _binding().w4_linear(w.ref, w.dev, x, y, bias, add, workspace, dev_flags, _handle(stream))
    if rc:
        _check(rc, "stom_w4_linear")
