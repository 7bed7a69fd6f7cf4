"""What the entry points of the 8-bit cache refuse, on the host and before anything is launched."""
import ctypes

import pytest
import torch

from paper_2605_21649_amd import binding as ekv
from tests.test_abi_cpu import good_cfg

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
A = [0x1000 * i for i in range(1, 20)]


def tokens(**kw):
    base = dict(slots=A[0], seq=A[1], pos=A[2], start=A[3], n_mapped=A[4], max_tokens=64)
    base.update(kw)
    return ekv.ekv_token_map(**base)


def cache(**kw):
    base = dict(k_pool=A[0], v_pool=A[1], k_scale=A[2], v_scale=A[3], block_table=A[4], seq_lens=A[5], n_phys_pages=100)
    base.update(kw)
    return ekv.ekv_cache8_view(**base)


def status(name, *args):
    lib = ekv.load_library()
    return getattr(lib, name)(*(ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args))


MAP = dict(cfg=good_cfg(batch=3), seq_lens=A[5], n_new=A[6], block_table=A[7], free_pages=A[8], n_free=A[9], capacity=10,
           tok=tokens(), new_lens=A[10], n_left=A[11], stream=None)


@pytest.mark.parametrize("bad,code", [
    (dict(cfg=None), INVALID), (dict(cfg=good_cfg(page_size=6)), UNSUPPORTED), (dict(seq_lens=None), INVALID),
    (dict(n_new=0x1002), INVALID), (dict(block_table=None), INVALID), (dict(free_pages=None), INVALID), (dict(n_free=None), INVALID),
    (dict(capacity=0), INVALID), (dict(capacity=-1), INVALID), (dict(tok=None), INVALID), (dict(tok=tokens(slots=None)), INVALID),
    (dict(tok=tokens(slots=0x1004)), INVALID), (dict(tok=tokens(seq=None)), INVALID), (dict(tok=tokens(pos=None)), INVALID),
    (dict(tok=tokens(start=None)), INVALID), (dict(tok=tokens(n_mapped=None)), INVALID), (dict(tok=tokens(max_tokens=0)), INVALID),
    (dict(tok=tokens(max_tokens=-5)), INVALID), (dict(tok=tokens(max_tokens=1 << 30)), UNSUPPORTED), (dict(new_lens=None), INVALID),
    (dict(n_left=None), INVALID), (dict(new_lens=A[5]), INVALID), (dict(n_left=A[9]), INVALID), (dict(new_lens=A[6]), INVALID),
    (dict(cfg=good_cfg(batch=4097)), UNSUPPORTED), (dict(free_pages=A[7]), INVALID),
])
def test_map_tokens_refuses(bad, code):
    assert status("ekv_map_tokens", *dict(MAP, **bad).values()) == code


RELEASE = dict(cfg=good_cfg(batch=3), release=A[4], seq_lens=A[5], block_table=A[7], free_pages=A[8], n_free=A[9], capacity=10,
               new_lens=A[10], n_left=A[11], stream=None)


@pytest.mark.parametrize("bad,code", [
    (dict(cfg=None), INVALID), (dict(release=None), INVALID), (dict(seq_lens=None), INVALID), (dict(block_table=None), INVALID),
    (dict(free_pages=None), INVALID), (dict(n_free=None), INVALID), (dict(capacity=0), INVALID), (dict(new_lens=None), INVALID),
    (dict(n_left=None), INVALID), (dict(new_lens=A[5]), INVALID), (dict(new_lens=A[4]), INVALID), (dict(n_left=A[9]), INVALID),
    (dict(free_pages=A[7]), INVALID), (dict(cfg=good_cfg(batch=5000)), UNSUPPORTED),
])
def test_release_pages_refuses(bad, code):
    assert status("ekv_release_pages", *dict(RELEASE, **bad).values()) == code


APPEND = dict(cfg=good_cfg(), cache=cache(), stats=None, tok=tokens(seq=None, pos=None, start=None, n_mapped=None), k_new=A[10],
              k_stride=1024, v_new=A[11], v_stride=1024, stream=None)


@pytest.mark.parametrize("bad,code", [
    (dict(cfg=None), INVALID), (dict(cache=None), INVALID), (dict(cache=cache(k_pool=None)), INVALID),
    (dict(cache=cache(v_pool=0x1008)), INVALID), (dict(cache=cache(k_scale=None)), INVALID), (dict(cache=cache(v_scale=0x1001)), INVALID),
    (dict(cache=cache(n_phys_pages=0)), INVALID), (dict(cache=cache(n_phys_pages=1 << 23)), UNSUPPORTED),
    (dict(tok=None), INVALID), (dict(tok=tokens(slots=None)), INVALID), (dict(tok=tokens(max_tokens=0)), INVALID),
    (dict(tok=tokens(max_tokens=1 << 30)), UNSUPPORTED), (dict(k_new=None), INVALID), (dict(v_new=None), INVALID),
    (dict(k_new=0x1008), INVALID), (dict(k_stride=1016), INVALID), (dict(v_stride=1028), INVALID), (dict(k_stride=-1024), INVALID),
    (dict(stats=ekv.ekv_stats_view(A[12], None, None)), INVALID), (dict(stats=ekv.ekv_stats_view(A[12], A[13], None)), INVALID),
    (dict(stats=ekv.ekv_stats_view(A[12], A[13], 0x1008), tok=tokens()), INVALID),
    (dict(cfg=good_cfg(kv_dtype="f32"), stats=ekv.ekv_stats_view(A[12], A[13], A[14]), tok=tokens()), UNSUPPORTED),
])
def test_append_refuses(bad, code):
    assert status("ekv_cache8_append", *dict(APPEND, **bad).values()) == code


SPARSE = dict(cfg=good_cfg(), q=A[6], cache=cache(), page_idx=A[7], n_sel=A[8], out=A[9], tau=A[10], supp=A[11], extras=None,
              ws=A[12], nbytes=1 << 40, stream=None)
ATTENTION = [(dict(cfg=None), INVALID), (dict(q=None), INVALID), (dict(cache=None), INVALID), (dict(cache=cache(block_table=None)), INVALID),
             (dict(cache=cache(seq_lens=None)), INVALID), (dict(cache=cache(k_scale=None)), INVALID), (dict(cache=cache(n_phys_pages=-3)), INVALID),
             (dict(cache=cache(n_phys_pages=1 << 24)), UNSUPPORTED), (dict(cfg=good_cfg(head_dim=64)), UNSUPPORTED), (dict(out=None), INVALID),
             (dict(tau=None), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=0x1004), WORKSPACE), (dict(nbytes=16), WORKSPACE)]


@pytest.mark.parametrize("name", ["ekv_decode8_sparse", "ekv_decode8_sparse_group", "ekv_decode8_full", "ekv_decode8_sparse_softmax",
                                  "ekv_decode8_full_softmax"])
@pytest.mark.parametrize("bad,code", ATTENTION + [(dict(page_idx=None), INVALID), (dict(n_sel=None), INVALID), (dict(supp=None), INVALID)])
def test_attention_refuses(name, bad, code):
    args = dict(SPARSE, **bad)
    if "full" in name:
        if "page_idx" in bad or "n_sel" in bad:
            pytest.skip("no lists")
        del args["page_idx"], args["n_sel"]
    if "softmax" in name:
        if "supp" in bad:
            pytest.skip("no support")
        del args["supp"], args["extras"]
    assert status(name, *args.values()) == code


def test_workspaces_of_the_softmax_do_not_grow_with_the_lists():
    small, large = good_cfg(max_sel_pages=16), good_cfg(max_sel_pages=65536)
    for op, rows in ((ekv.EKV_OP_DECODE8_SPARSE_SOFTMAX, 1), (ekv.EKV_OP_DECODE8_FULL_SOFTMAX, 4)):
        assert 0 < ekv.ekv_workspace_bytes(small, op) <= ekv.ekv_workspace_bytes(large, op) <= (1024 + 64) * rows * 130 * 4


def test_the_binding_takes_rows_of_a_longer_projection_and_no_other_strides():
    rows = torch.zeros(5, 3, 2, 128)
    assert ekv._rows(rows[:, 1]) == (rows.data_ptr() + 2 * 128 * 4, 3 * 2 * 128)
    assert ekv._rows(rows[:1, 0])[1] == 256
    for bad in (rows[:, 0].transpose(0, 1), rows[..., ::2][:, 0], rows[:, :, 0].transpose(1, 2)):
        with pytest.raises(AssertionError):
            ekv._rows(bad)
    with pytest.raises(AssertionError):                      # fewer rows than the map has tokens
        ekv.ekv_cache8_append(good_cfg(), cache(), None, tokens(max_tokens=6), rows[:, 0], rows[:, 1])


def test_the_binding_takes_maps_of_the_right_types_only():
    slots, i32 = torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.int32)
    assert ekv.token_map(slots, i32, i32, i32, i32).max_tokens == 4
    for bad in ((i32,), (slots, slots, i32), (slots, i32, torch.zeros(3, dtype=torch.int32)), (slots, i32, i32, slots), (slots, i32, i32, i32, slots)):
        with pytest.raises(AssertionError):
            ekv.token_map(*bad)


def test_softmax_refuses_capacities_of_more_steps_than_it_counts():
    """128 units (512 lists) of 2^30 tokens: 2^32 steps and more."""
    cfg = good_cfg(batch=128 // good_cfg().n_kv_heads, max_pages_per_seq=(1 << 30) // good_cfg().page_size,
                   max_sel_pages=(1 << 30) // good_cfg().page_size)
    full = dict(cfg=cfg, q=A[6], cache=cache(), out=A[9], lse=A[10], ws=A[12], nbytes=1 << 60, stream=None)
    assert status("ekv_decode8_full_softmax", *full.values()) == UNSUPPORTED
    lists = dict(cfg=cfg, q=A[6], cache=cache(), page_idx=A[7], n_sel=A[8], out=A[9], lse=A[10], ws=A[12], nbytes=1 << 60, stream=None)
    assert status("ekv_decode8_sparse_softmax", *lists.values()) == UNSUPPORTED


def test_the_binding_takes_rows_of_the_configs_type_and_heads_only(monkeypatch):
    """The library goes by the config's type and heads: rows of another are refused before it is called."""
    called = []

    class Library:
        def ekv_cache8_append(self, *args):
            called.append(args)
            return 0

    monkeypatch.setattr(ekv, "load_library", Library)
    monkeypatch.setattr(ekv, "_stream", lambda stream: None)
    cfg = good_cfg(n_kv_heads=4, n_q_heads=8, kv_dtype="bf16")
    rows = torch.zeros(5, 3, 4, 128, dtype=torch.bfloat16)
    k, v = rows[:, 1], rows[:, 2]
    ekv.ekv_cache8_append(cfg, cache(), None, tokens(max_tokens=5), k, v)
    assert len(called) == 1
    for bad in ((k.float(), v), (k, v.float()), (k.half(), v.half()), (k[:, :2], v), (k, v[:, 1:]), (k[:, :3], v[:, :3]),
                (k[..., :64], v[..., :64]), (torch.cat((k, k), 1), v)):
        with pytest.raises(AssertionError):
            ekv.ekv_cache8_append(cfg, cache(), None, tokens(max_tokens=5), *bad)
    with pytest.raises(AssertionError):                      # bfloat16 rows where the library reads float32
        ekv.ekv_cache8_append(good_cfg(n_kv_heads=4, n_q_heads=8, kv_dtype="f32"), cache(), None, tokens(max_tokens=5), k, v)
    assert len(called) == 1


def test_the_binding_takes_queries_of_the_configs_type_and_size_only(monkeypatch):
    called = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: called.append(name) or 0

    monkeypatch.setattr(ekv, "load_library", Library)
    monkeypatch.setattr(ekv, "_stream", lambda stream: None)
    cfg = good_cfg(batch=2, n_kv_heads=4, n_q_heads=8, kv_dtype="f32")
    q, x = torch.zeros(2, 8, 128), torch.zeros(4)
    for name, n_args in (("sparse", 6), ("sparse_group", 6), ("full", 4), ("sparse_softmax", 5), ("full_softmax", 3)):
        call = getattr(ekv, "ekv_decode8_" + name)
        call(cfg, q, cache(), *[x] * n_args)
        call(cfg, torch.zeros(3, 8, 128), cache(), *[x] * n_args)                # of a larger batch: its first rows
        for bad in (q.bfloat16(), q.double(), q[:1], q[:, :4].contiguous(), q[..., :64].contiguous()):
            with pytest.raises(AssertionError):
                call(cfg, bad, cache(), *[x] * n_args)
    assert len(called) == 10


def test_the_binding_takes_pools_and_scales_that_belong_together_only():
    k, v = (torch.zeros(6, 2, 16, 128, dtype=torch.uint8) for _ in range(2))
    ks, vs = (torch.ones(6, 2) for _ in range(2))
    table, lens = torch.zeros(1, 6, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    assert ekv.cache8_view(k, v, ks, vs, table, lens).n_phys_pages == 6
    assert ekv.cache8_view(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), ks, vs).n_phys_pages == 6
    for bad in ((k.bfloat16(), v, ks, vs), (k, v.bfloat16(), ks, vs), (k, v[:5], ks, vs), (k, v, ks.bfloat16(), vs), (k, v, ks, vs.double()),
                (k, v, ks[:5], vs), (k, v, ks, vs[:, :1].contiguous()), (k, v, ks, vs, table.long(), lens), (k, v, ks, vs, table, lens.long())):
        with pytest.raises(AssertionError):
            ekv.cache8_view(*bad)


@pytest.mark.parametrize("kind", ["entmax", "softmax"])
def test_the_limits_of_outputs_tell_right_from_wrong(kind):
    """Mistakes planted in the oracle -- the scale of one page of values, one page's values in another's place, a head's keys with
    its neighbour's values, one token left out -- change the output by more than the GPU tests allow, which is a small part of it."""
    from oracle import entmaxkv_oracle as orc
    from tests import cache8 as c8
    import numpy as np

    def attend(q, K, V):
        return orc.entmax_attention(q, K, V, 1.5, c.scale) if kind == "entmax" else orc.softmax_attention(q, K, V, c.scale)

    for n, page in ((4000, 12), (900, 16)):
        c = c8.Large(4, 2, page, [n], seed=n, flat=0.3, device="cpu")
        for h in range(4):
            q, (K, V) = c.query(0, h), c.keys_values(0, h // 2)
            ref = attend(q, K, V)
            limit = (c8.entmax_limits(ref, q, K, V, 1.5, c.scale) if kind == "entmax" else c8.softmax_limits(ref, q, K, V, c.scale))[1]
            assert np.linalg.norm(limit) <= 0.1 * np.linalg.norm(ref["o"])
            top = int(np.argmax(ref["p"]))
            at = slice(top // page * page, top // page * page + page)
            wrong = []
            for change in (lambda x: 2.0 * x, lambda x: 0.5 * x, lambda x: np.roll(V, page, 0)[at], lambda x: 0.0 * x):
                W = V.copy()
                W[at] = change(W[at])
                wrong.append(attend(q, K, W)["o"])
            wrong.append(attend(q, K, c.keys_values(0, 1 - h // 2)[1])["o"])
            rest = np.arange(n) != top
            wrong.append(attend(q, K[rest], V[rest])["o"])
            wrong.append(np.zeros(128))
            assert all(np.any(np.abs(o - ref["o"]) > limit) for o in wrong)
