"""ctypes binding over the C ABI in include/entmaxkv.h -- argument marshalling only.

Every function has the name of the C entry point it calls and takes torch tensors (device memory
owned by the caller) where the C call takes device pointers.  No step of the method runs in Python.
The shared library is loaded on first use and its absence is an error: there is no fallback path.
"""
import ctypes
import os
from ctypes import c_float, c_int32, c_int64, c_size_t, c_void_p, POINTER, byref

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libentmaxkv.so")

EKV_OK = 0
EKV_F32, EKV_BF16 = 0, 1
_TYPES = {EKV_F32: torch.float32, EKV_BF16: torch.bfloat16}
EKV_SCORE_BOX, EKV_SCORE_GAUSS, EKV_SCORE_BOTH, EKV_SCORE_GROUP_MAX, EKV_SCORE_BOX8 = 1, 2, 3, 4, 8
EKV_STATIC_SCRATCH_BYTES = 32 << 20
EKV_OP_SELECT_TOPK, EKV_OP_SELECT_GAUSS, EKV_OP_DECODE_SPARSE, EKV_OP_DECODE_FULL, \
    EKV_OP_DECODE_SPARSE_SOFTMAX, EKV_OP_SELECT_BOX_THRESHOLD, EKV_OP_DECODE8_SPARSE_SOFTMAX, \
    EKV_OP_DECODE8_FULL_SOFTMAX, EKV_OP_TREE_SPARSE, EKV_OP_TREE_FULL, EKV_OP_TREE_SPARSE_SOFTMAX, \
    EKV_OP_TREE_FULL_SOFTMAX = range(12)

# every symbol the header declares
EXPORTS = ["ekv_stats_build", "ekv_stats_append", "ekv_score_pages", "ekv_append_score_pages", "ekv_select_topk",
           "ekv_select_gauss",
           "ekv_select_box_threshold", "ekv_decode_sparse", "ekv_decode_sparse_group", "ekv_decode_full",
           "ekv_decode_sparse_softmax", "ekv_workspace_bytes", "ekv_probe_read", "ekv_decode_sparse_static",
           "ekv_probe_handoff", "ekv_map_tokens", "ekv_release_pages", "ekv_cache8_append", "ekv_decode8_sparse",
           "ekv_decode8_sparse_group", "ekv_decode8_full", "ekv_decode8_sparse_softmax", "ekv_decode8_full_softmax",
           "ekv_norm_rotate", "ekv_cache_append", "ekv_tree_sparse", "ekv_tree_sparse_group", "ekv_tree_full",
           "ekv_tree_sparse_softmax", "ekv_tree_full_softmax", "ekv_tree8_sparse", "ekv_tree8_sparse_group", "ekv_tree8_full",
           "ekv_tree8_sparse_softmax", "ekv_tree8_full_softmax", "ekv_tree_workspace_bytes",
           "ekv_status_string", "ekv_last_hip_error", "ekv_version"]
_STATUS_CALLS = EXPORTS[:-3]      # entry points that return ekv_status


class ekv_config(ctypes.Structure):
    _fields_ = [("batch", c_int32), ("n_q_heads", c_int32), ("n_kv_heads", c_int32), ("head_dim", c_int32),
                ("page_size", c_int32), ("kv_dtype", c_int32), ("alpha", c_float), ("scale", c_float),
                ("max_pages_per_seq", c_int32), ("max_sel_pages", c_int32), ("pool_kv_heads", c_int32)]


class ekv_cache_view(ctypes.Structure):
    _fields_ = [("k_pool", c_void_p), ("v_pool", c_void_p), ("block_table", c_void_p), ("seq_lens", c_void_p),
                ("n_phys_pages", c_int32)]


class ekv_stats_view(ctypes.Structure):
    _fields_ = [("box", c_void_p), ("gauss", c_void_p), ("box8", c_void_p)]


class ekv_decode_extras(ctypes.Structure):
    _fields_ = [("support_tokens", c_void_p), ("support_cap", c_int32), ("tau_ref", c_void_p),
                ("kept_mass_ref", c_void_p), ("kept_supp_ref", c_void_p), ("lse", c_void_p),
                ("tau_seed", c_void_p), ("solve_evals", c_void_p), ("score_pass_only", c_int32)]


class ekv_cache8_view(ctypes.Structure):
    _fields_ = [("k_pool", c_void_p), ("v_pool", c_void_p), ("k_scale", c_void_p), ("v_scale", c_void_p),
                ("block_table", c_void_p), ("seq_lens", c_void_p), ("n_phys_pages", c_int32)]


class ekv_token_map(ctypes.Structure):
    _fields_ = [("slots", c_void_p), ("seq", c_void_p), ("pos", c_void_p), ("start", c_void_p), ("n_mapped", c_void_p),
                ("max_tokens", c_int32)]


class ekv_tree_view(ctypes.Structure):
    _fields_ = [("k_new", c_void_p), ("v_new", c_void_p), ("k_stride", c_int64), ("v_stride", c_int64), ("start", c_void_p),
                ("visible", c_void_p), ("max_tokens", c_int32), ("max_tree", c_int32)]


class EkvError(RuntimeError):
    pass


_lib = None


def load_library():
    """Load libentmaxkv.so (built in-tree by paper_2605_21649_amd.build).  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise EkvError(f"HIP library not built: {LIB_PATH} (run `python -m paper_2605_21649_amd.build`)")
    lib = ctypes.CDLL(LIB_PATH)
    P = POINTER
    lib.ekv_stats_build.argtypes = [P(ekv_config), P(ekv_cache_view), P(ekv_stats_view), c_void_p]
    lib.ekv_stats_append.argtypes = [P(ekv_config), P(ekv_cache_view), P(ekv_stats_view), c_void_p, c_void_p,
                                     c_void_p]
    lib.ekv_score_pages.argtypes = [P(ekv_config), c_void_p, P(ekv_stats_view), c_void_p, c_int32, c_void_p,
                                    c_void_p, c_void_p, c_void_p]
    lib.ekv_append_score_pages.argtypes = [P(ekv_config), P(ekv_cache_view), P(ekv_stats_view), c_void_p, c_void_p,
                                           c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.ekv_select_topk.argtypes = [P(ekv_config), c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p,
                                    c_size_t, c_void_p]
    lib.ekv_select_gauss.argtypes = [P(ekv_config), c_void_p, c_void_p, c_void_p, c_float, c_float, c_void_p,
                                     c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.ekv_decode_sparse.argtypes = [P(ekv_config), c_void_p, P(ekv_cache_view), c_void_p, c_void_p, c_void_p,
                                      c_void_p, c_void_p, P(ekv_decode_extras), c_void_p, c_size_t, c_void_p]
    lib.ekv_decode_sparse_group.argtypes = lib.ekv_decode_sparse.argtypes
    lib.ekv_decode_sparse_static.argtypes = [P(ekv_config), c_void_p, P(ekv_cache_view), c_void_p, c_void_p, c_void_p,
                                             c_void_p, c_void_p, P(ekv_decode_extras), c_void_p]
    lib.ekv_decode_full.argtypes = [P(ekv_config), c_void_p, P(ekv_cache_view), c_void_p, c_void_p, c_void_p,
                                    P(ekv_decode_extras), c_void_p, c_size_t, c_void_p]
    lib.ekv_decode_sparse_softmax.argtypes = [P(ekv_config), c_void_p, P(ekv_cache_view), c_void_p, c_void_p,
                                              c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.ekv_workspace_bytes.argtypes = [P(ekv_config), c_int32, P(c_size_t)]
    lib.ekv_status_string.argtypes = [c_int32]
    lib.ekv_status_string.restype = ctypes.c_char_p
    lib.ekv_last_hip_error.restype = c_int32
    lib.ekv_version.restype = c_int32
    lib.ekv_select_box_threshold.argtypes = [P(ekv_config), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                             c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.ekv_probe_read.argtypes = [c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p]
    lib.ekv_probe_handoff.argtypes = [c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_void_p]
    lib.ekv_map_tokens.argtypes = [P(ekv_config), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int32,
                                   P(ekv_token_map), c_void_p, c_void_p, c_void_p]
    lib.ekv_release_pages.argtypes = [P(ekv_config), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int32,
                                      c_void_p, c_void_p, c_void_p]
    lib.ekv_cache8_append.argtypes = [P(ekv_config), P(ekv_cache8_view), P(ekv_stats_view), P(ekv_token_map), c_void_p,
                                      c_int64, c_void_p, c_int64, c_void_p]
    lib.ekv_decode8_sparse.argtypes = [P(ekv_config), c_void_p, P(ekv_cache8_view), c_void_p, c_void_p, c_void_p,
                                       c_void_p, c_void_p, P(ekv_decode_extras), c_void_p, c_size_t, c_void_p]
    lib.ekv_decode8_sparse_group.argtypes = lib.ekv_decode8_sparse.argtypes
    lib.ekv_decode8_full.argtypes = [P(ekv_config), c_void_p, P(ekv_cache8_view), c_void_p, c_void_p, c_void_p,
                                     P(ekv_decode_extras), c_void_p, c_size_t, c_void_p]
    lib.ekv_decode8_sparse_softmax.argtypes = [P(ekv_config), c_void_p, P(ekv_cache8_view), c_void_p, c_void_p,
                                               c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.ekv_decode8_full_softmax.argtypes = [P(ekv_config), c_void_p, P(ekv_cache8_view), c_void_p, c_void_p, c_void_p,
                                             c_size_t, c_void_p]
    lib.ekv_norm_rotate.argtypes = [P(ekv_config), c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_float, c_void_p,
                                    c_int32, c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p]
    lib.ekv_cache_append.argtypes = [P(ekv_config), P(ekv_cache_view), P(ekv_stats_view), P(ekv_token_map), c_void_p, c_int32,
                                     c_void_p, c_int64, c_void_p, c_int64, c_void_p]
    for name, view in (("ekv_tree_", ekv_cache_view), ("ekv_tree8_", ekv_cache8_view)):
        head, tail = [P(ekv_config), c_void_p, P(view), P(ekv_tree_view)], [c_void_p, c_size_t, c_void_p]
        getattr(lib, name + "sparse").argtypes = head + [c_void_p] * 5 + tail
        getattr(lib, name + "sparse_group").argtypes = head + [c_void_p] * 5 + tail
        getattr(lib, name + "full").argtypes = head + [c_void_p] * 3 + tail
        getattr(lib, name + "sparse_softmax").argtypes = head + [c_void_p] * 4 + tail
        getattr(lib, name + "full_softmax").argtypes = head + [c_void_p] * 2 + tail
    lib.ekv_tree_workspace_bytes.argtypes = [P(ekv_config), c_int32, c_int32, c_int32, P(c_size_t)]
    for name in _STATUS_CALLS:
        getattr(lib, name).restype = c_int32
    _lib = lib
    return lib


def _check(status):
    if status != EKV_OK:
        lib = load_library()
        raise EkvError(f"{lib.ekv_status_string(status).decode()} (hip error {lib.ekv_last_hip_error()})")


def _ptr(t):
    if t is None:
        return None
    assert t.is_contiguous(), "tensors passed to the C ABI must be contiguous"
    return t.data_ptr()


# Handle of the current stream of a device: torch.cuda.current_stream() builds a Stream object for it (2.9 us per call,
# more than all other marshalling together; this: 0.35 us), and a step of a short sequence is three calls of 5 us of kernels.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(stream):
    if stream is not None:
        return stream
    return _raw_stream(torch.cuda.current_device())


def make_config(batch, n_q_heads, n_kv_heads, head_dim, page_size, kv_dtype, alpha, scale, max_pages_per_seq,
                max_sel_pages, pool_kv_heads=0):
    dt = {"f32": EKV_F32, "bf16": EKV_BF16}.get(kv_dtype, kv_dtype)
    return ekv_config(batch, n_q_heads, n_kv_heads, head_dim, page_size, dt, alpha, scale, max_pages_per_seq,
                      max_sel_pages, pool_kv_heads)


def cache_view(k_pool, v_pool, block_table, seq_lens):
    return ekv_cache_view(_ptr(k_pool), _ptr(v_pool), _ptr(block_table), _ptr(seq_lens), k_pool.shape[0])


def cache_view_heads(k_pool, v_pool, block_table, seq_lens, first_kv_head):
    """Cache view of the KV heads from `first_kv_head` on (pools [n_phys][Hkv][P][d]): the pool pointers are
    advanced to that head; use it with a config whose pool_kv_heads is the cache's head count."""
    off = first_kv_head * k_pool.shape[2] * k_pool.shape[3] * k_pool.element_size()
    assert k_pool.is_contiguous() and v_pool.is_contiguous()
    return ekv_cache_view(k_pool.data_ptr() + off, v_pool.data_ptr() + off, _ptr(block_table), _ptr(seq_lens),
                          k_pool.shape[0])


def stats_view(box, gauss, box8=None):
    return ekv_stats_view(_ptr(box), _ptr(gauss), _ptr(box8))


def cache8_view(k_pool, v_pool, k_scale, v_scale, block_table=None, seq_lens=None):
    assert k_pool.element_size() == 1 and v_pool.element_size() == 1 and k_pool.shape == v_pool.shape, "pools of one shape, a byte per element"
    for t in (k_scale, v_scale):
        assert t.dtype == torch.float32 and t.shape == k_pool.shape[:2], "scales: float32, one for every page and head of the pools"
    for t in (block_table, seq_lens):
        assert t is None or t.dtype == torch.int32, "block_table and seq_lens are int32"
    return ekv_cache8_view(_ptr(k_pool), _ptr(v_pool), _ptr(k_scale), _ptr(v_scale), _ptr(block_table), _ptr(seq_lens),
                           k_pool.shape[0])


def token_map(slots, seq=None, pos=None, start=None, n_mapped=None):
    assert slots.dtype == torch.int64, "slots are int64"
    for t in (seq, pos):
        assert t is None or (t.dtype == torch.int32 and t.numel() == slots.numel()), "seq and pos: int32, one for every slot"
    for t in (start, n_mapped):
        assert t is None or t.dtype == torch.int32, "start and n_mapped are int32"
    return ekv_token_map(_ptr(slots), _ptr(seq), _ptr(pos), _ptr(start), _ptr(n_mapped), slots.numel())


def decode_extras(support_tokens=None, tau_ref=None, kept_mass_ref=None, kept_supp_ref=None, lse=None,
                  tau_seed=None, solve_evals=None, score_pass_only=False):
    cap = support_tokens.shape[-1] if support_tokens is not None else 0
    return ekv_decode_extras(_ptr(support_tokens), cap, _ptr(tau_ref), _ptr(kept_mass_ref), _ptr(kept_supp_ref),
                             _ptr(lse), _ptr(tau_seed), _ptr(solve_evals), 1 if score_pass_only else 0)


def ekv_workspace_bytes(cfg, op):
    n = c_size_t(0)
    _check(load_library().ekv_workspace_bytes(byref(cfg), op, byref(n)))
    return n.value


def ekv_stats_build(cfg, cache, stats, stream=None):
    _check(load_library().ekv_stats_build(byref(cfg), byref(cache), byref(stats), _stream(stream)))


def ekv_stats_append(cfg, cache, stats, k_new, v_new=None, stream=None):
    _check(load_library().ekv_stats_append(byref(cfg), byref(cache), byref(stats), _ptr(k_new), _ptr(v_new),
                                           _stream(stream)))


def ekv_score_pages(cfg, q, stats, seq_lens, mode, box=None, mu=None, sigma=None, stream=None):
    _check(load_library().ekv_score_pages(byref(cfg), _ptr(q), byref(stats), _ptr(seq_lens), mode, _ptr(box),
                                          _ptr(mu), _ptr(sigma), _stream(stream)))


def ekv_append_score_pages(cfg, cache, stats, k_new, v_new, q, mode, box=None, mu=None, sigma=None, stream=None):
    _check(load_library().ekv_append_score_pages(byref(cfg), byref(cache), byref(stats), _ptr(k_new), _ptr(v_new),
                                                 _ptr(q), mode, _ptr(box), _ptr(mu), _ptr(sigma), _stream(stream)))


def ekv_select_topk(cfg, box, seq_lens, k_pages, page_idx, n_sel, workspace, stream=None):
    nbytes = workspace.numel() * workspace.element_size()
    _check(load_library().ekv_select_topk(byref(cfg), _ptr(box), _ptr(seq_lens), k_pages, _ptr(page_idx),
                                          _ptr(n_sel), _ptr(workspace), nbytes, _stream(stream)))


def ekv_select_gauss(cfg, mu, sigma, seq_lens, q_page, margin, tau_hat, page_idx, n_sel, overflow, workspace,
                     stream=None):
    nbytes = workspace.numel() * workspace.element_size()
    _check(load_library().ekv_select_gauss(byref(cfg), _ptr(mu), _ptr(sigma), _ptr(seq_lens), q_page, margin,
                                           _ptr(tau_hat), _ptr(page_idx), _ptr(n_sel), _ptr(overflow),
                                           _ptr(workspace), nbytes, _stream(stream)))


def ekv_select_box_threshold(cfg, box, seq_lens, tau_lo, page_idx_in, n_sel_in, page_idx_out, n_sel_out, n_added,
                             overflow, workspace, stream=None):
    nbytes = workspace.numel() * workspace.element_size()
    _check(load_library().ekv_select_box_threshold(byref(cfg), _ptr(box), _ptr(seq_lens), _ptr(tau_lo),
                                                   _ptr(page_idx_in), _ptr(n_sel_in), _ptr(page_idx_out),
                                                   _ptr(n_sel_out), _ptr(n_added), _ptr(overflow), _ptr(workspace),
                                                   nbytes, _stream(stream)))


def ekv_decode_sparse(cfg, q, cache, page_idx, n_sel, out, tau, supp, workspace, extras=None, stream=None):
    nbytes = workspace.numel() * workspace.element_size()
    ex = byref(extras) if extras is not None else None
    _check(load_library().ekv_decode_sparse(byref(cfg), _ptr(q), byref(cache), _ptr(page_idx), _ptr(n_sel),
                                            _ptr(out), _ptr(tau), _ptr(supp), ex, _ptr(workspace), nbytes,
                                            _stream(stream)))


def ekv_decode_sparse_group(cfg, q, cache, page_idx, n_sel, out, tau, supp, workspace, extras=None, stream=None):
    nbytes = workspace.numel() * workspace.element_size()
    ex = byref(extras) if extras is not None else None
    _check(load_library().ekv_decode_sparse_group(byref(cfg), _ptr(q), byref(cache), _ptr(page_idx), _ptr(n_sel),
                                                  _ptr(out), _ptr(tau), _ptr(supp), ex, _ptr(workspace), nbytes,
                                                  _stream(stream)))


def ekv_decode_full(cfg, q, cache, out, tau, supp, workspace, extras=None, stream=None):
    nbytes = workspace.numel() * workspace.element_size()
    ex = byref(extras) if extras is not None else None
    _check(load_library().ekv_decode_full(byref(cfg), _ptr(q), byref(cache), _ptr(out), _ptr(tau), _ptr(supp), ex,
                                          _ptr(workspace), nbytes, _stream(stream)))


def ekv_decode_sparse_softmax(cfg, q, cache, page_idx, n_sel, out, lse_sel, workspace, stream=None):
    nbytes = workspace.numel() * workspace.element_size()
    _check(load_library().ekv_decode_sparse_softmax(byref(cfg), _ptr(q), byref(cache), _ptr(page_idx),
                                                    _ptr(n_sel), _ptr(out), _ptr(lse_sel), _ptr(workspace), nbytes,
                                                    _stream(stream)))


def ekv_probe_read(base, page_ids, n_pages, page_bytes, sink, lookup=None, out=None, stream=None):
    _check(load_library().ekv_probe_read(_ptr(base), _ptr(page_ids), _ptr(lookup), n_pages, page_bytes, _ptr(out),
                                         _ptr(sink), _stream(stream)))


def ekv_decode_sparse_static(cfg, q, cache, page_idx, n_sel, out, tau, supp, extras=None, stream=None):
    ex = byref(extras) if extras is not None else None
    _check(load_library().ekv_decode_sparse_static(byref(cfg), _ptr(q), byref(cache), _ptr(page_idx), _ptr(n_sel),
                                                   _ptr(out), _ptr(tau), _ptr(supp), ex, _stream(stream)))


def ekv_probe_handoff(data, counter, out, n_workgroups, mode, stream=None):
    _check(load_library().ekv_probe_handoff(_ptr(data), _ptr(counter), _ptr(out), n_workgroups, mode, _stream(stream)))


def ekv_map_tokens(cfg, seq_lens, n_new, block_table, free_pages, n_free, tokens, new_lens, n_left, stream=None):
    _check(load_library().ekv_map_tokens(byref(cfg), _ptr(seq_lens), _ptr(n_new), _ptr(block_table), _ptr(free_pages),
                                         _ptr(n_free), free_pages.numel(), byref(tokens), _ptr(new_lens), _ptr(n_left),
                                         _stream(stream)))


def ekv_release_pages(cfg, release, seq_lens, block_table, free_pages, n_free, new_lens, n_left, stream=None):
    _check(load_library().ekv_release_pages(byref(cfg), _ptr(release), _ptr(seq_lens), _ptr(block_table),
                                            _ptr(free_pages), _ptr(n_free), free_pages.numel(), _ptr(new_lens),
                                            _ptr(n_left), _stream(stream)))


def _rows(t, shape=None):
    """Pointer and row stride of [tokens][Hkv][d] rows that may be parts of longer ones."""
    n, st = shape or t.shape, t.stride()         # asked for once: an attribute of a tensor is a tenth of a microsecond
    assert len(n) == 3 and st[2] == 1 and (n[1] == 1 or st[1] == n[2]), "the heads of a row must follow each other"
    return t.data_ptr(), st[0] if n[0] > 1 else n[1] * n[2]


def ekv_cache8_append(cfg, cache, stats, tokens, k_new, v_new, stream=None):
    kn, vn, rows, t = k_new.shape, v_new.shape, tokens.max_tokens, _TYPES.get(cfg.kv_dtype)
    (k, ks), (v, vs) = _rows(k_new, kn), _rows(v_new, vn)
    assert kn[0] >= rows and vn[0] >= rows, "a row for every token of the map"
    assert kn[1] == vn[1] == cfg.n_kv_heads and kn[2] == vn[2] == cfg.head_dim, "rows of the config's KV heads and head size"
    assert k_new.dtype is t and v_new.dtype is t, "rows of the config's type"
    _check(load_library().ekv_cache8_append(byref(cfg), byref(cache), byref(stats) if stats is not None else None,
                                            byref(tokens), k, ks, v, vs, _stream(stream)))


def _query(cfg, q):
    assert q.dtype is _TYPES.get(cfg.kv_dtype), "queries of the config's type"
    assert q.numel() >= cfg.batch * cfg.n_q_heads * cfg.head_dim, "a query for every sequence and head"
    return _ptr(q)


def ekv_decode8_sparse(cfg, q, cache, page_idx, n_sel, out, tau, supp, workspace, extras=None, stream=None):
    nbytes = workspace.numel() * workspace.element_size()
    ex = byref(extras) if extras is not None else None
    _check(load_library().ekv_decode8_sparse(byref(cfg), _query(cfg, q), byref(cache), _ptr(page_idx), _ptr(n_sel), _ptr(out),
                                             _ptr(tau), _ptr(supp), ex, _ptr(workspace), nbytes, _stream(stream)))


def ekv_decode8_sparse_group(cfg, q, cache, page_idx, n_sel, out, tau, supp, workspace, extras=None, stream=None):
    nbytes = workspace.numel() * workspace.element_size()
    ex = byref(extras) if extras is not None else None
    _check(load_library().ekv_decode8_sparse_group(byref(cfg), _query(cfg, q), byref(cache), _ptr(page_idx), _ptr(n_sel),
                                                   _ptr(out), _ptr(tau), _ptr(supp), ex, _ptr(workspace), nbytes,
                                                   _stream(stream)))


def ekv_decode8_full(cfg, q, cache, out, tau, supp, workspace, extras=None, stream=None):
    nbytes = workspace.numel() * workspace.element_size()
    ex = byref(extras) if extras is not None else None
    _check(load_library().ekv_decode8_full(byref(cfg), _query(cfg, q), byref(cache), _ptr(out), _ptr(tau), _ptr(supp), ex,
                                           _ptr(workspace), nbytes, _stream(stream)))


def ekv_decode8_sparse_softmax(cfg, q, cache, page_idx, n_sel, out, lse_sel, workspace, stream=None):
    nbytes = workspace.numel() * workspace.element_size()
    _check(load_library().ekv_decode8_sparse_softmax(byref(cfg), _query(cfg, q), byref(cache), _ptr(page_idx), _ptr(n_sel),
                                                     _ptr(out), _ptr(lse_sel), _ptr(workspace), nbytes, _stream(stream)))


def ekv_decode8_full_softmax(cfg, q, cache, out, lse, workspace, stream=None):
    nbytes = workspace.numel() * workspace.element_size()
    _check(load_library().ekv_decode8_full_softmax(byref(cfg), _query(cfg, q), byref(cache), _ptr(out), _ptr(lse),
                                                   _ptr(workspace), nbytes, _stream(stream)))


def ekv_norm_rotate(cfg, x_q, x_k, w_q, w_k, eps, freq, pos, q_out, k_out, pairs=False, stream=None):
    t, d = _TYPES.get(cfg.kv_dtype), cfg.head_dim
    qn, kn = x_q.shape, x_k.shape
    (q, qs), (k, ks) = _rows(x_q, qn), _rows(x_k, kn)
    n, hq, hk = qn[0], qn[1], kn[1]
    assert kn[0] == n and hq == cfg.n_q_heads and hk == cfg.n_kv_heads and qn[2] == d == kn[2], "rows of the config's heads and head size"
    assert x_q.dtype is t and x_k.dtype is t and q_out.dtype is t and k_out.dtype is t, "rows and outputs of the config's type"
    assert q_out.numel() == n * hq * d and k_out.numel() == n * hk * d, "an output row for every token"
    assert w_q is None or (w_q.dtype is t and w_q.numel() == d), "weights of the config's type and head size"
    assert w_k is None or (w_k.dtype is t and w_k.numel() == d), "weights of the config's type and head size"
    turned = 0
    if freq is not None:
        turned = freq.numel()
        assert freq.dtype is torch.float32, "frequencies are float32"
    assert pos is None or (pos.dtype is torch.int32 and pos.numel() >= n), "positions: int32, one for every token"
    status = load_library().ekv_norm_rotate(byref(cfg), q, qs, k, ks, _ptr(w_q), _ptr(w_k), eps, _ptr(freq), turned, _ptr(pos), n,
                                            1 if pairs else 0, _ptr(q_out), _ptr(k_out), _stream(stream))
    if status:
        _check(status)


def ekv_cache_append(cfg, cache, stats, tokens, k_new, v_new, rows=None, stream=None):
    kn, vn, n, t = k_new.shape, v_new.shape, tokens.max_tokens, _TYPES.get(cfg.kv_dtype)
    (k, ks), (v, vs) = _rows(k_new, kn), _rows(v_new, vn)
    if rows is None:
        assert kn[0] >= n and vn[0] >= n, "a row for every token of the map"
    else:
        assert rows.dtype is torch.int32 and rows.numel() >= n and vn[0] == kn[0], "rows: int32, one for every token of the map"
    assert kn[1] == vn[1] == cfg.n_kv_heads and kn[2] == vn[2] == cfg.head_dim, "rows of the config's KV heads and head size"
    assert k_new.dtype is t and v_new.dtype is t, "rows of the config's type"
    _check(load_library().ekv_cache_append(byref(cfg), byref(cache), byref(stats) if stats is not None else None, byref(tokens),
                                           _ptr(rows), kn[0], k, ks, v, vs, _stream(stream)))


def tree_view(start, visible, k_new, v_new, max_tree):
    """Drafted rows: k_new, v_new [max_tokens][Hkv][d] (may be parts of longer rows), start int32 [B + 1], visible int64 [max_tokens],
    the 64 bits of a row's mask.  The view holds the tensors: it is used in several calls, and masks are made for it alone."""
    kn, vn = k_new.shape, v_new.shape
    (k, ks), (v, vs) = _rows(k_new, kn), _rows(v_new, vn)
    assert kn == vn and k_new.dtype is v_new.dtype, "drafted keys and values of one shape and type"
    assert start.dtype is torch.int32 and visible.element_size() == 8 and not visible.is_floating_point(), "start int32, masks of 64 bits"
    assert visible.numel() == kn[0], "a mask for every drafted row"
    tree = ekv_tree_view(k, v, ks, vs, _ptr(start), _ptr(visible), kn[0], max_tree)
    tree.of = (kn[1], kn[2], k_new.dtype, start.numel())      # what the calls check against their config
    tree.holds = (start, visible, k_new, v_new)
    return tree


def ekv_tree_workspace_bytes(cfg, op, max_tokens, max_tree):
    n = c_size_t(0)
    _check(load_library().ekv_tree_workspace_bytes(byref(cfg), op, max_tokens, max_tree, byref(n)))
    return n.value


def _tree(call, cfg, q, cache, tree, page_idx, n_sel, heads, outs, workspace, stream):
    t, hq, d, batch, n = _TYPES.get(cfg.kv_dtype), cfg.n_q_heads, cfg.head_dim, cfg.batch, tree.max_tokens
    rows = n * hq
    assert q.dtype is t and q.numel() == rows * d, "a query of the config's type for every row and head"
    kv_heads, size, dtype, starts = tree.of
    assert kv_heads == cfg.n_kv_heads and size == d and dtype is t, "drafted rows of the config's type, KV heads and head size"
    assert starts == batch + 1, "start has an entry for every sequence and one more"
    out, norm = outs[0], outs[1]
    assert out.dtype is torch.float32 and out.numel() == rows * d, "out: float32, like q"
    assert norm.dtype is torch.float32 and norm.numel() == rows, "tau or lse: float32, one for every row and head"
    args = [byref(cfg), _ptr(q), byref(cache), byref(tree)]
    if heads:
        assert page_idx.dtype is torch.int32 and n_sel.dtype is torch.int32, "page lists are int32"
        assert n_sel.numel() == batch * heads and page_idx.numel() == batch * heads * cfg.max_sel_pages, "a list of cap pages for every sequence and head"
        args += (_ptr(page_idx), _ptr(n_sel))
    args += (_ptr(out), _ptr(norm))
    if len(outs) > 2:
        supp = outs[2]
        assert supp.dtype is torch.int32 and supp.numel() == rows, "supp: int32, one for every row and head"
        args.append(_ptr(supp))
    status = call(*args, _ptr(workspace), workspace.nbytes, _stream(stream))
    if status:
        _check(status)


def ekv_tree_sparse(cfg, q, cache, tree, page_idx, n_sel, out, tau, supp, workspace, stream=None):
    _tree(load_library().ekv_tree_sparse, cfg, q, cache, tree, page_idx, n_sel, cfg.n_q_heads, (out, tau, supp), workspace, stream)


def ekv_tree_sparse_group(cfg, q, cache, tree, page_idx, n_sel, out, tau, supp, workspace, stream=None):
    _tree(load_library().ekv_tree_sparse_group, cfg, q, cache, tree, page_idx, n_sel, cfg.n_kv_heads, (out, tau, supp), workspace, stream)


def ekv_tree_full(cfg, q, cache, tree, out, tau, supp, workspace, stream=None):
    _tree(load_library().ekv_tree_full, cfg, q, cache, tree, None, None, 0, (out, tau, supp), workspace, stream)


def ekv_tree_sparse_softmax(cfg, q, cache, tree, page_idx, n_sel, out, lse, workspace, stream=None):
    _tree(load_library().ekv_tree_sparse_softmax, cfg, q, cache, tree, page_idx, n_sel, cfg.n_q_heads, (out, lse), workspace, stream)


def ekv_tree_full_softmax(cfg, q, cache, tree, out, lse, workspace, stream=None):
    _tree(load_library().ekv_tree_full_softmax, cfg, q, cache, tree, None, None, 0, (out, lse), workspace, stream)


def ekv_tree8_sparse(cfg, q, cache, tree, page_idx, n_sel, out, tau, supp, workspace, stream=None):
    _tree(load_library().ekv_tree8_sparse, cfg, q, cache, tree, page_idx, n_sel, cfg.n_q_heads, (out, tau, supp), workspace, stream)


def ekv_tree8_sparse_group(cfg, q, cache, tree, page_idx, n_sel, out, tau, supp, workspace, stream=None):
    _tree(load_library().ekv_tree8_sparse_group, cfg, q, cache, tree, page_idx, n_sel, cfg.n_kv_heads, (out, tau, supp), workspace, stream)


def ekv_tree8_full(cfg, q, cache, tree, out, tau, supp, workspace, stream=None):
    _tree(load_library().ekv_tree8_full, cfg, q, cache, tree, None, None, 0, (out, tau, supp), workspace, stream)


def ekv_tree8_sparse_softmax(cfg, q, cache, tree, page_idx, n_sel, out, lse, workspace, stream=None):
    _tree(load_library().ekv_tree8_sparse_softmax, cfg, q, cache, tree, page_idx, n_sel, cfg.n_q_heads, (out, lse), workspace, stream)


def ekv_tree8_full_softmax(cfg, q, cache, tree, out, lse, workspace, stream=None):
    _tree(load_library().ekv_tree8_full_softmax, cfg, q, cache, tree, None, None, 0, (out, lse), workspace, stream)
