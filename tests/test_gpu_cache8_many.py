"""Attention over the 8-bit cache where a wavefront has many items and a launch many units: outputs, value side included, of samples
against the oracle, with limits that are a small part of the outputs.  Statistics of large appends, and keys that are no number."""
import numpy as np
import pytest
import torch

from oracle import entmaxkv_oracle as orc
from paper_2605_21649_amd import binding as ekv
from tests import test_gpu_cache8_append as appends, test_gpu_cache8_decode as decodes
from tests.cache8 import D, VALUES, Cache8, Large, entmax_limits, softmax_limits

pytestmark = pytest.mark.gpu

CALLS = {"full": ekv.EKV_OP_DECODE_FULL, "sparse": ekv.EKV_OP_DECODE_SPARSE, "sparse_group": ekv.EKV_OP_DECODE_SPARSE,
         "full_softmax": ekv.EKV_OP_DECODE8_FULL_SOFTMAX, "sparse_softmax": ekv.EKV_OP_DECODE8_SPARSE_SOFTMAX}


def run(c, call, lists=()):
    c.out.fill_(float("nan"))
    c.tau.fill_(float("nan"))
    ws = c.workspace(CALLS[call])
    getattr(ekv, "ekv_decode8_" + call)(c.cfg, c.q, c.view(), *lists, c.out, c.tau, *(() if "softmax" in call else (c.supp,)), ws)
    torch.cuda.synchronize()


def check_sample(c, call, b, h, tok):
    """One row against the oracle on the tokens of its list (or all)."""
    out, first = c.out[b, h].cpu().numpy().astype(np.float64), float(c.tau[b, h])
    soft = "softmax" in call
    if len(tok) == 0:
        assert not out.any() and first == (-np.inf if soft else np.inf)
        return
    K, V = (x[tok] for x in c.keys_values(b, h // c.G))
    q = c.query(b, h)
    if soft:
        ref = orc.softmax_attention(q, K, V, c.scale)
        e, limit = softmax_limits(ref, q, K, V, c.scale)
    else:
        ref = orc.entmax_attention(q, K, V, c.alpha, c.scale)
        e, limit = entmax_limits(ref, q, K, V, c.alpha, c.scale)
    assert len(tok) < 2 or np.linalg.norm(limit) <= 0.2 * np.linalg.norm(ref["o"])     # wrong rows, scales or weights are beyond it
    assert abs(first - ref["lse" if soft else "tau"]) <= e, (b, h)
    assert np.all(np.abs(out - ref["o"]) <= limit), (b, h, (np.abs(out - ref["o"]) / limit).max())


def random_lists(c, n_lists, seed):
    """Ascending page lists of every length up to the capacity, with anything behind their ends."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    m = ((c.seq_lens + c.P - 1) // c.P)[:, None, None]
    score = torch.rand(c.B, n_lists, c.M, generator=g, device="cuda")
    score = torch.where(torch.arange(c.M, device="cuda") < m, score, -1.0)
    idx = score.topk(c.cap, dim=-1).indices
    most = m[..., 0].clamp(max=c.cap)
    n = (most - (torch.rand(c.B, n_lists, generator=g, device="cuda") * 0.4 * most).int()).to(torch.int32)
    taken = torch.arange(c.cap, device="cuda") < n[..., None]
    idx = torch.where(taken, idx, c.M + 1).sort(-1).values
    junk = torch.randint(-3, c.M + 3, idx.shape, generator=g, device="cuda")
    return torch.where(taken, idx, junk).to(torch.int32), n


def tokens_of(c, call, lists, b, h):
    if not lists:
        return np.arange(c.lens[b])
    i = h // c.G if call == "sparse_group" else h
    return c.tokens(b, lists[0][b, i, :int(lists[1][b, i])].cpu().numpy())


@pytest.mark.parametrize("page,heads,dtype", [
    (4, (16, 8), "bf16"), (12, (16, 8), "bf16"), (16, (16, 8), "bf16"), (20, (16, 8), "bf16"), (24, (16, 8), "bf16"), (44, (16, 8), "bf16"),
    (56, (16, 8), "bf16"), (64, (16, 8), "bf16"), (16, (8, 8), "bf16"), (12, (8, 8), "bf16"), (16, (16, 16), "bf16"), (12, (16, 16), "f32"), (40, (32, 8), "bf16"), (16, (32, 4), "bf16"),
    (12, (32, 4), "bf16"), (12, (16, 8), "f32"), (16, (16, 8), "f32"), (40, (8, 8), "f32")])
def test_outputs_where_wavefronts_have_many_items(page, heads, dtype):
    """24 uneven sequences of up to 12000 tokens: 18000 groups of tokens and more for 16384 wavefronts at most over all pages, three
    to six a wavefront over lists of about 4000 tokens, whose ends fall on any lane."""
    lens = [12000 - 487 * b for b in range(24)]
    c = Large(*heads, page, lens, cap=4000 // page, dtype=dtype, seed=page + heads[0], flat=0.3)
    rng = np.random.default_rng(page)
    for call in CALLS:
        lists = random_lists(c, c.Hkv if call == "sparse_group" else c.Hq, page) if "sparse" in call else ()
        run(c, call, lists)
        assert torch.isfinite(c.out).all() and torch.isfinite(c.tau).all()
        for b in (0, 7, 13, 23):
            for h in rng.permutation(c.Hq)[:2].tolist() + [c.Hq - 1]:
                check_sample(c, call, b, h, tokens_of(c, call, lists, b, h))


@pytest.mark.parametrize("page,heads,dtype", [(16, (8, 8), "bf16"), (12, (8, 8), "f32"), (16, (16, 8), "f32"), (12, (16, 8), "bf16")])
def test_more_units_than_a_workgroup_keeps_sums_of(page, heads, dtype):
    """1100 sequences, most of them empty, of 8 KV heads in a capacity beyond what one workgroup takes: the sums over the units before
    come from a launch of their own, for every kind of call."""
    lens = [0] * 1100
    for b, n in ((0, 5000), (1, 1), (2, 8320), (500, 33), (501, 2500), (777, 64), (1098, 1), (1099, 4111)):
        lens[b] = n
    c = Cache8(1100, *heads, page, lens, row_pages=8400 // page, cap=8400 // page, scale=0.3 / np.sqrt(D), dtype=dtype, seed=page)
    assert c.B * c.Hkv > 8192 and c.cap * page > 8192
    rng = np.random.default_rng(page)
    for call in CALLS:
        n_lists = c.Hkv if call == "sparse_group" else c.Hq
        idx, n = torch.zeros(c.B, n_lists, c.cap, dtype=torch.int32, device="cuda"), torch.zeros(c.B, n_lists, dtype=torch.int32, device="cuda")
        if "sparse" in call:
            for b, length in enumerate(lens):
                m = -(-length // page)
                for i in range(n_lists if m else 0):
                    k = int(rng.integers(max(1, m // 2), m + 1))
                    idx[b, i, :k] = torch.from_numpy(np.sort(rng.permutation(m)[:k]).astype(np.int32))
                    n[b, i] = k
            n[3], n[1000] = 5, c.cap                              # lists of sequences that have no token
        lists = (idx, n) if "sparse" in call else ()
        run(c, call, lists)
        assert torch.isfinite(c.out).all() and not c.out[c.seq_lens == 0].any()
        assert bool((c.tau[c.seq_lens == 0] == (-np.inf if "softmax" in call else np.inf)).all())
        for b in [b for b, length in enumerate(lens) if length]:
            for h in rng.permutation(c.Hq)[:3].tolist():
                check_sample(c, call, b, h, tokens_of(c, call, lists, b, h))


@pytest.mark.parametrize("heads,dtype", [((2, 2), "bf16"), ((4, 2), "f32"), ((8, 2), "bf16"), ((16, 2), "f32")])
@pytest.mark.parametrize("page", [24, 40, 56])
def test_pages_of_whole_octets_that_do_not_make_64(page, heads, dtype):
    for kind in ("entmax", "softmax"):
        decodes.test_every_page_of_ragged_sequences(page, heads, dtype, kind)
    for call in ("sparse", "group", "softmax"):
        decodes.test_page_lists(page, heads, dtype, call)
    if heads == (2, 2):
        decodes.test_steps_of_one_workgroup(page)
        decodes.test_the_longest_rows_of_one_workgroup(page, dtype)
        for call in ("sparse", "group", "softmax"):
            decodes.test_long_lists_of_grouped_heads(page, call)


@pytest.mark.parametrize("dtype,with8", [("bf16", False), ("bf16", True), ("f32", False)])
@pytest.mark.parametrize("page", [8, 20, 24, 28, 48, 60])
def test_statistics_of_small_steps(page, dtype, with8):
    appends.test_statistics_are_those_of_the_stored_keys(page, dtype, with8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [4, 16, 20, 28, 32, 48, 60, 64])
def test_statistics_of_large_appends(page, dtype):
    """Three steps of 20000 rows and more, of which a wavefront has up to 32 or 64 and with them several runs, beside partly filled pages
    and pages that are rounded again: all statistics equal ekv_stats_build's of a cache that holds the stored keys."""
    rng = np.random.default_rng(page)
    g = torch.Generator(device="cuda").manual_seed(page)
    B, H, M = 40, 8, 2400 // page + 1
    n_phys = B * M
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    cfg = ekv.make_config(B, H, H, D, page, dtype, 1.5, 1.0, M, M)
    i32 = dict(dtype=torch.int32, device="cuda")
    kp, vp = (torch.full((n_phys, H, page, D), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((n_phys, H), float("nan"), device="cuda") for _ in range(2))
    table, free = torch.zeros(B, M, **i32), torch.from_numpy(rng.permutation(n_phys).astype(np.int32)).cuda()
    lens, n_free = torch.zeros(B, **i32), torch.tensor([n_phys], **i32)
    box, gauss = (torch.zeros(B, H, M, 2, D, dtype=dt, device="cuda") for _ in range(2))
    box8 = torch.zeros(B, H, M, 16, 2, 8, dtype=torch.uint8, device="cuda") if dtype == "bf16" else None
    for step in range(3):
        counts = rng.integers(300, 800, B)
        counts[step], counts[step + 5] = 0, 1
        T = int(counts.sum())
        assert T * H * 2 > 8 * 4096                               # more rows to a wavefront than one
        slots, seq, pos, start, mapped = torch.zeros(T, dtype=torch.int64, device="cuda"), *(torch.zeros(k, **i32) for k in (T, T, B + 1, B))
        new_lens, left = torch.zeros(B, **i32), torch.zeros(1, **i32)
        tokens = ekv.token_map(slots, seq, pos, start, mapped)
        ekv.ekv_map_tokens(cfg, lens, torch.from_numpy(counts.astype(np.int32)).cuda(), table, free, n_free, tokens, new_lens, left)
        rows = torch.randn(T, 3, H, D, generator=g, device="cuda") * 2.0 ** torch.randint(-3, 6, (T, 1, 1, 1), generator=g, device="cuda")
        rows = rows.to(dt)
        ekv.ekv_cache8_append(cfg, ekv.cache8_view(kp, vp, ks, vs), ekv.stats_view(box, gauss, box8), tokens, rows[:, 1], rows[:, 2])
        lens, n_free = new_lens, left
        assert lens.tolist() == [int(x) for x in (counts if step == 0 else total + counts)]
        total = lens.cpu().numpy()
        value = torch.from_numpy(VALUES).float().cuda()
        stored = torch.nan_to_num(value[kp.int()] * ks[:, :, None, None]).to(dt)
        ref = [torch.zeros_like(box), torch.zeros_like(gauss)]
        ref8 = torch.zeros_like(box8) if box8 is not None else None
        ekv.ekv_stats_build(cfg, ekv.cache_view(stored, stored, table, lens), ekv.stats_view(*ref, ref8))
        torch.cuda.synchronize()
        has = torch.arange(M, device="cuda") < ((lens + page - 1) // page)[:, None]
        for got, want in ((box, ref[0]), (gauss, ref[1])) + (((box8, ref8),) if box8 is not None else ()):
            same = (got.view(torch.uint8) == want.view(torch.uint8)).flatten(3).all(-1)
            assert same.transpose(1, 2)[has].all(), step


def poisoned(c, rng, share):
    """NaN codes in a channel of some of each sequence's keys, a whole page's among them; which tokens stay."""
    stay = []
    for b in range(c.B):
        bad = rng.random(c.lens[b]) < share
        if c.lens[b] > 3 * c.P:
            bad[c.P:2 * c.P] = True
        at = torch.from_numpy(np.nonzero(bad)[0]).cuda()
        page = torch.as_tensor(np.asarray(c.table[b].cpu() if torch.is_tensor(c.table) else c.table[b]), device="cuda").long()[at // c.P]
        pool = c.k_pool if isinstance(c, Cache8) else c.pools[0]
        pool[page, :, at % c.P, int(rng.integers(0, D))] = 0x7F
        stay.append(np.nonzero(~bad)[0])
    return stay


@pytest.mark.parametrize("page,heads,dtype", [(16, (8, 2), "bf16"), (12, (8, 2), "bf16"), (16, (2, 2), "f32"), (44, (4, 2), "f32")])
def test_entmax_passes_keys_over_that_are_no_number(page, heads, dtype):
    """Short rows in one launch, longer ones in two, lists per query head and per KV head."""
    rng = np.random.default_rng(page)
    for lens in ([500, 77, 2], [3000, 4999, 900]):
        c = Cache8(3, *heads, page, lens, dtype=dtype, seed=page)
        stay = poisoned(c, rng, 0.1)
        for call in ("full", "sparse", "sparse_group"):
            n_lists = c.Hkv if call == "sparse_group" else c.Hq
            m = [-(-n // page) for n in lens]
            idx = torch.arange(c.M, dtype=torch.int32, device="cuda").expand(3, n_lists, c.M).contiguous()
            n = torch.tensor(m, dtype=torch.int32, device="cuda")[:, None].expand(3, n_lists).contiguous()
            run(c, call, (idx, n) if "sparse" in call else ())
            for b in range(3):
                for h in range(c.Hq):
                    decodes.check_entmax(c, b, h, stay[b], c.out[b, h].cpu().numpy().astype(np.float64), float(c.tau[b, h]), int(c.supp[b, h]))


@pytest.mark.parametrize("n", [300, 5000])
def test_a_key_that_is_no_number_is_in_the_log_sum_of_the_entmax_decode_alone(n):
    c = Cache8(1, 4, 2, 16, [n], seed=n)
    c.k_pool[c.table[0, 2], 0, 5, 3] = 0x7F                      # of the first KV head's queries
    lse = torch.zeros(1, 4, device="cuda")
    ekv.ekv_decode8_full(c.cfg, c.q, c.view(), c.out, c.tau, c.supp, c.workspace(ekv.EKV_OP_DECODE_FULL), extras=ekv.decode_extras(lse=lse))
    torch.cuda.synchronize()
    assert torch.isnan(lse[0, :2]).all() and torch.isfinite(lse[0, 2:]).all()
    assert torch.isfinite(c.out).all() and torch.isfinite(c.tau).all()


@pytest.mark.parametrize("page", [16, 12])
def test_entmax_passes_keys_over_that_are_no_number_in_large_calls(page):
    """Over 64 MiB of K, where pages of 16 put the stores of the scores off."""
    c = Large(16, 8, page, [40000 - 3001 * b for b in range(8)], seed=page, flat=0.3)
    keys = [[c.keys_values(b, h) for h in (0, 7)] for b in (0, 7)]
    stay = poisoned(c, np.random.default_rng(page), 0.1)
    run(c, "full")
    assert torch.isfinite(c.out).all()
    for i, b in enumerate((0, 7)):
        for j, h in enumerate((0, 15)):
            q, (K, V) = c.query(b, h), (x[stay[b]] for x in keys[i][j])
            ref = orc.entmax_attention(q, K, V, c.alpha, c.scale)
            e, limit = entmax_limits(ref, q, K, V, c.alpha, c.scale)
            assert abs(float(c.tau[b, h]) - ref["tau"]) <= e
            assert np.all(np.abs(c.out[b, h].cpu().numpy() - ref["o"]) <= limit)


@pytest.mark.parametrize("call", ["full", "full_softmax"])
def test_values_at_the_end_of_the_softmax_range(call):
    """Values of 448 * 2^81, just below 2^90, of both signs, in flat attention over 20011 tokens."""
    rng = np.random.default_rng(9)
    c = Cache8(1, 4, 1, 16, [20011], scale=0.01, seed=9)
    c.codes[1][:] = np.where(c.valid[:, None, :, None], np.where(rng.random(c.codes[1].shape) < 0.9, 0x7E, 0xFE), 0x7F)
    c.scales[1][c.valid.any(1)] = 2.0 ** 81
    c.v_pool.copy_(torch.from_numpy(c.codes[1]).cuda())
    c.v_scale.copy_(torch.from_numpy(c.scales[1].astype(np.float32)).cuda())
    run(c, call)
    for h in range(4):
        check_sample(c, call, 0, h, np.arange(20011))


@pytest.mark.parametrize("batch", [512, 513])
@pytest.mark.parametrize("heads", [(8, 8), (16, 8), (64, 8)])
def test_as_many_units_as_the_put_off_stores_take(batch, heads):
    """4096 units of 8 KV heads, the most that the pass takes which holds its stores back, with all of a compute unit's LDS; and more."""
    n = 512 if heads == (8, 8) else 256                           # 8 MiB of scores too
    lens = [n - 37 * b % (n + 1) for b in range(batch)]
    c = Large(*heads, 16, lens, row_pages=n // 16, seed=batch, flat=0.3)
    assert batch * 8 * n * D >= 64 << 20 and batch * c.Hq * n * 4 >= 8 << 20
    rng = np.random.default_rng(batch)
    run(c, "full")
    assert torch.isfinite(c.out).all()
    for b in rng.permutation(batch)[:30].tolist() + [0, 1, batch - 2, batch - 1]:
        check_sample(c, "full", b, int(rng.integers(0, c.Hq)), np.arange(lens[b]))


@pytest.mark.parametrize("page", [16, 32])
def test_how_far_a_stored_element_is_from_its_own(page):
    """Tokens one by one, each up to four times as large as those before, into a page whose scale grows with them.  An element is off by half
    a step when it is stored, 2^-4 of it or 2^-10 of the scale below the normal codes, and by at most 2^-10 of the scale again whenever
    that grows (a code moved by whole exponents is exact unless it falls below the normal ones): at least doubled each
    time, those sum to less than 2^-9 of the scale at the end."""
    rng = np.random.default_rng(page)
    H = 4
    kp, vp = (torch.full((1, H, page, D), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((1, H), float("nan"), device="cuda") for _ in range(2))
    cfg = ekv.make_config(1, H, H, D, page, "f32", 1.5, 1.0, 1, 1)
    x = rng.standard_normal((page, 2, H, D)) * 2.0 ** np.cumsum(rng.integers(-1, 3, page))[:, None, None, None]
    x = torch.from_numpy((x * 2.0 ** rng.integers(-12, 1, x.shape)).astype(np.float32))
    grown = 0
    for t in range(page):
        row, before = x[t:t + 1].cuda(), ks.clone()
        ekv.ekv_cache8_append(cfg, ekv.cache8_view(kp, vp, ks, vs), None, ekv.token_map(torch.tensor([t], device="cuda")), row[:, 0], row[:, 1])
        grown += int((ks > before).sum())
        for side, (pool, scale) in enumerate(((kp, ks), (vp, vs))):
            s = scale.cpu().numpy().astype(np.float64)[0, :, None, None]
            y = VALUES[pool.cpu().numpy()[0, :, :t + 1]] * s
            ref = x[:t + 1, side].double().numpy().transpose(1, 0, 2)
            assert np.all(np.abs(y - ref) <= np.maximum(2.0 ** -4 * np.abs(ref), 2.0 ** -10 * s) + 2.0 ** -9 * s)
            assert np.all(s < np.abs(ref).max((1, 2), keepdims=True) / 224)
    assert grown > 3 * H
