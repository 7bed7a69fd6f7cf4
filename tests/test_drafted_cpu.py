"""Refusals of the entry points for drafted tokens, before anything is launched (no GPU is needed)."""
import ctypes

import pytest
import torch

from paper_2605_21649_amd import binding as ekv

D = 128
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


def config(**kw):
    base = dict(batch=3, n_q_heads=8, n_kv_heads=2, head_dim=D, page_size=16, kv_dtype="bf16", alpha=1.5, scale=0.1,
                max_pages_per_seq=64, max_sel_pages=8)
    base.update(kw)
    return ekv.make_config(**base)


NORM = dict(x_q=0x1000, q_stride=1536, x_k=0x2000, k_stride=1536, w_q=0x3000, w_k=0x4000, eps=1e-6, freq=0x5000, n_freq=64, pos=0x6000,
            n=5, pairs=0, q_out=0x7000, k_out=0x8000)


@pytest.mark.parametrize("change,code", [
    (dict(x_q=None), INVALID), (dict(x_k=0x2004), INVALID), (dict(w_q=0x3002), INVALID), (dict(q_stride=1023), INVALID),
    (dict(q_stride=1028), INVALID), (dict(k_stride=248), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(eps=float("inf")), INVALID), (dict(freq=None), INVALID), (dict(pos=None), INVALID), (dict(pos=0x6002), INVALID),
    (dict(n_freq=-8), INVALID), (dict(n_freq=12), UNSUPPORTED), (dict(n_freq=72), UNSUPPORTED), (dict(n=0), INVALID),
    (dict(n=1 << 28), UNSUPPORTED), (dict(q_out=0x1000), INVALID), (dict(k_out=0x7000), INVALID), (dict(k_out=None), INVALID),
])
def test_norm_rotate_refuses(change, code):
    a = dict(NORM, **change)
    cfg = config()
    assert ekv.load_library().ekv_norm_rotate(ctypes.byref(cfg), *list(a.values()), None) == code


def append_args(**kw):
    cache = ekv.ekv_cache_view(kw.get("k_pool", 0x1000), kw.get("v_pool", 0x2000), None, None, kw.get("n_phys", 9))
    stats = ekv.ekv_stats_view(kw.get("box", 0x3000), kw.get("gauss", 0x4000), kw.get("box8"))
    tokens = ekv.ekv_token_map(kw.get("slots", 0x5000), kw.get("seq", 0x6000), kw.get("pos", 0x7000), None, None, kw.get("n", 4))
    return [ctypes.byref(cache) if kw.get("cache", True) else None, ctypes.byref(stats) if kw.get("stats", True) else None,
            ctypes.byref(tokens) if kw.get("tokens", True) else None, kw.get("rows"), kw.get("n_rows", 0), kw.get("k", 0x8000),
            kw.get("ks", 256), kw.get("v", 0x9000), kw.get("vs", 256), None], (cache, stats, tokens)


@pytest.mark.parametrize("change,code", [
    (dict(cache=False), INVALID), (dict(tokens=False), INVALID), (dict(k_pool=None), INVALID), (dict(v_pool=0x2008), INVALID),
    (dict(n_phys=0), INVALID), (dict(slots=None), INVALID), (dict(slots=0x5004), INVALID), (dict(n=0), INVALID), (dict(k=None), INVALID),
    (dict(ks=255), INVALID), (dict(vs=260), INVALID), (dict(rows=0xa002, n_rows=4), INVALID), (dict(rows=0xa000, n_rows=0), INVALID),
    (dict(box=None), INVALID), (dict(gauss=None), INVALID), (dict(seq=None), INVALID), (dict(pos=None), INVALID),
    (dict(box8=0xb008), INVALID), (dict(n=1 << 28), UNSUPPORTED), (dict(n=(1 << 31) - 1), UNSUPPORTED),
])
def test_cache_append_refuses(change, code):
    cfg = config()
    args, keep = append_args(**change)
    assert ekv.load_library().ekv_cache_append(ctypes.byref(cfg), *args) == code


def test_cache_append_refuses_8_bit_bounds_of_float32_caches_and_too_many_heads():
    lib = ekv.load_library()
    args, keep = append_args(box8=0xb000)
    assert lib.ekv_cache_append(ctypes.byref(config(kv_dtype="f32")), *args) == UNSUPPORTED
    args, keep = append_args(n=1 << 26, ks=1024, vs=1024, stats=False)
    assert lib.ekv_cache_append(ctypes.byref(config(n_q_heads=8, n_kv_heads=8)), *args) == UNSUPPORTED


def test_the_binding_refuses_tensors_of_other_types_and_sizes():
    cfg = config()
    q, k = torch.zeros(4, 8, D).bfloat16(), torch.zeros(4, 2, D).bfloat16()
    w, freq, pos = torch.zeros(D).bfloat16(), torch.zeros(64), torch.zeros(4, dtype=torch.int32)
    good = dict(x_q=q, x_k=k, w_q=w, w_k=w, eps=1e-6, freq=freq, pos=pos, q_out=q.clone(), k_out=k.clone())
    for bad in (dict(x_q=q.float()), dict(x_q=q[:, :7]), dict(x_k=k[:3]), dict(w_q=w[:64]), dict(w_k=w.float()), dict(freq=freq.double()),
                dict(pos=pos.long()), dict(pos=pos[:3]), dict(q_out=q[:3].clone()), dict(k_out=k.float()), dict(x_q=q.transpose(1, 2))):
        with pytest.raises(AssertionError):
            ekv.ekv_norm_rotate(cfg, **dict(good, **bad), stream=0)
    cache = ekv.cache_view(torch.zeros(3, 2, 16, D).bfloat16(), torch.zeros(3, 2, 16, D).bfloat16(), None, None)
    tokens = ekv.token_map(torch.zeros(4, dtype=torch.int64), pos, pos)
    for kn, vn, rows in ((k.float(), k, None), (k[:3], k, None), (k, k[:, :1], None), (k, k, pos.long()), (k, k, pos[:3]), (k, k[:3], pos)):
        with pytest.raises(AssertionError):
            ekv.ekv_cache_append(cfg, cache, None, tokens, kn, vn, rows=rows, stream=0)


CALLS = [(c8, name) for c8 in (False, True) for name in ("sparse", "sparse_group", "full", "sparse_softmax", "full_softmax")]


def tree_call(c8, name, cfg, **kw):
    """Status of ekv_tree(8)_`name` with made-up pointers, one of them changed; a good call is never made."""
    lib = ekv.load_library()
    if c8:
        cache = ekv.ekv_cache8_view(kw.get("k_pool", 0x1000), kw.get("v_pool", 0x2000), kw.get("k_scale", 0x3000), kw.get("v_scale", 0x4000),
                                    kw.get("table", 0x5000), kw.get("lens", 0x6000), kw.get("n_phys", 99))
    else:
        cache = ekv.ekv_cache_view(kw.get("k_pool", 0x1000), kw.get("v_pool", 0x2000), kw.get("table", 0x5000), kw.get("lens", 0x6000),
                                   kw.get("n_phys", 99))
    tree = ekv.ekv_tree_view(kw.get("k_new", 0x7000), kw.get("v_new", 0x8000), kw.get("ks", 256), kw.get("vs", 768), kw.get("start", 0x9000),
                             kw.get("visible", 0xa000), kw.get("max_tokens", 20), kw.get("max_tree", 9))
    args = [ctypes.byref(cfg), kw.get("q", 0xb000), ctypes.byref(cache) if kw.get("cache", True) else None,
            ctypes.byref(tree) if kw.get("tree", True) else None]
    if "sparse" in name:
        args += [kw.get("page_idx", 0xc000), kw.get("n_sel", 0xd000)]
    args += [kw.get("out", 0xe000), kw.get("norm", 0xf000)] + ([] if "softmax" in name else [kw.get("supp", 0x10000)])
    args += [kw.get("ws", 0x11000), kw.get("ws_bytes", 0), None]
    return getattr(lib, ("ekv_tree8_" if c8 else "ekv_tree_") + name)(*args)


@pytest.mark.parametrize("c8,name", CALLS)
def test_tree_calls_refuse(c8, name):
    cfg = config()
    assert tree_call(c8, name, cfg) == WORKSPACE                           # all good but the workspace
    assert tree_call(c8, name, cfg, ws=None, ws_bytes=1 << 40) == WORKSPACE and tree_call(c8, name, cfg, ws=0x11008, ws_bytes=1 << 40) == WORKSPACE
    for bad in (dict(cache=False), dict(tree=False), dict(k_pool=None), dict(v_pool=0x2004), dict(table=None), dict(lens=0x6001), dict(n_phys=0),
                dict(k_new=None), dict(v_new=0x8008), dict(ks=255), dict(ks=260), dict(vs=248), dict(start=None), dict(start=0x9002),
                dict(visible=None), dict(visible=0xa004), dict(max_tokens=0), dict(max_tree=0), dict(q=None), dict(q=0xb008), dict(out=None),
                dict(out=0xe004), dict(norm=None)):
        assert tree_call(c8, name, cfg, **bad) == INVALID, bad
    if "sparse" in name:
        assert tree_call(c8, name, cfg, page_idx=None) == INVALID and tree_call(c8, name, cfg, n_sel=0xd002) == INVALID
    if "softmax" not in name:
        assert tree_call(c8, name, cfg, supp=None) == INVALID
    if c8:
        assert tree_call(c8, name, cfg, k_scale=None) == INVALID and tree_call(c8, name, cfg, v_scale=0x4002) == INVALID
    for bad in (dict(max_tree=65), dict(max_tokens=1 << 21), dict(n_phys=1 << 26)):
        assert tree_call(c8, name, cfg, **bad) == UNSUPPORTED, bad
    many = config(batch=1 << 21, max_pages_per_seq=1 << 16)
    assert tree_call(c8, name, many) == UNSUPPORTED


def test_tree_workspace_sizes():
    cfg = config()
    rows = 20 * 8
    full = ekv.ekv_tree_workspace_bytes(cfg, ekv.EKV_OP_TREE_FULL, 20, 9)
    groups = 64 * 16 // 64 + 1                                             # of 64 positions, and one of drafted keys
    assert rows * groups * 65 * 4 <= full <= rows * groups * 65 * 4 + 1024
    sparse = ekv.ekv_tree_workspace_bytes(cfg, ekv.EKV_OP_TREE_SPARSE, 20, 9)
    assert rows * 3 * 65 * 4 <= sparse <= rows * 3 * 65 * 4 + 1024
    assert ekv.ekv_tree_workspace_bytes(cfg, ekv.EKV_OP_TREE_FULL_SOFTMAX, 20, 64) >= 1024 * 64 * 130 * 4
    assert ekv.ekv_tree_workspace_bytes(cfg, ekv.EKV_OP_TREE_SPARSE_SOFTMAX, 20, 9) >= 1024 * 16 * 130 * 4
    lib, n = ekv.load_library(), ctypes.c_size_t(0)
    ask = lambda op, tokens, most: lib.ekv_tree_workspace_bytes(ctypes.byref(cfg), op, tokens, most, ctypes.byref(n))  # noqa: E731
    assert ask(ekv.EKV_OP_DECODE_FULL, 20, 9) == INVALID and ask(12, 20, 9) == INVALID and ask(8, 0, 9) == INVALID and ask(8, 20, 0) == INVALID
    assert ask(8, 20, 65) == UNSUPPORTED and ask(8, 1 << 22, 9) == UNSUPPORTED
    assert lib.ekv_tree_workspace_bytes(ctypes.byref(cfg), 8, 20, 9, None) == INVALID
    assert lib.ekv_workspace_bytes(ctypes.byref(cfg), ekv.EKV_OP_TREE_FULL, ctypes.byref(n)) == INVALID


def test_the_binding_refuses_trees_that_do_not_fit_their_config():
    cfg = config()
    k = torch.zeros(5, 2, D).bfloat16()
    start, visible = torch.zeros(4, dtype=torch.int32), torch.zeros(5, dtype=torch.int64)
    for bad in (dict(start=start.long()), dict(visible=visible.int()), dict(visible=visible.double()), dict(visible=visible[:4]), dict(v_new=k[:4]),
                dict(v_new=k.float()), dict(k_new=k.transpose(0, 1))):
        with pytest.raises(AssertionError):
            ekv.tree_view(**dict(dict(start=start, visible=visible, k_new=k, v_new=k, max_tree=5), **bad))
    cache = ekv.cache_view(torch.zeros(3, 2, 16, D).bfloat16(), torch.zeros(3, 2, 16, D).bfloat16(), torch.zeros(3, 64, dtype=torch.int32), start[:3])
    tree, q = ekv.tree_view(start, visible, k, k, 5), torch.zeros(5, 8, D).bfloat16()
    out, tau, supp, ws = torch.zeros(5, 8, D), torch.zeros(5, 8), torch.zeros(5, 8, dtype=torch.int32), torch.zeros(4, dtype=torch.uint8)
    lists = dict(page_idx=torch.zeros(3, 8, 8, dtype=torch.int32), n_sel=torch.zeros(3, 8, dtype=torch.int32))
    good = dict(cfg=cfg, q=q, cache=cache, tree=tree, out=out, tau=tau, supp=supp, workspace=ws, **lists)
    with pytest.raises(ekv.EkvError, match="WORKSPACE"):
        ekv.ekv_tree_sparse(**good, stream=0)
    for bad in (dict(q=q.float()), dict(q=q[:4]), dict(out=out.double()), dict(out=out[:4]), dict(tau=tau.int()), dict(supp=supp.float()), dict(supp=supp[:4]),
                dict(n_sel=lists["n_sel"].long()), dict(page_idx=lists["page_idx"][:, :4].contiguous()), dict(n_sel=lists["n_sel"][:2]),
                dict(cfg=config(batch=4)), dict(cfg=config(n_kv_heads=8)), dict(cfg=config(kv_dtype="f32"))):
        with pytest.raises(AssertionError):
            ekv.ekv_tree_sparse(**dict(good, **bad), stream=0)
