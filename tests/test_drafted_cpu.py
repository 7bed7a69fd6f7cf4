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
    (dict(box8=0xb008), INVALID), (dict(n=1 << 30), UNSUPPORTED),
])
def test_cache_append_refuses(change, code):
    cfg = config()
    args, keep = append_args(**change)
    assert ekv.load_library().ekv_cache_append(ctypes.byref(cfg), *args) == code


def test_cache_append_refuses_8_bit_bounds_of_float32_caches_and_too_many_heads():
    lib = ekv.load_library()
    args, keep = append_args(box8=0xb000)
    assert lib.ekv_cache_append(ctypes.byref(config(kv_dtype="f32")), *args) == UNSUPPORTED
    args, keep = append_args(n=1 << 29, ks=1024, vs=1024, stats=False)
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
