"""Attention of drafted rows against the definition in 64 bits: types, layouts, lists, masks, lengths."""
import math

import pytest
import torch

from paper_2605_21649_amd import binding as ekv
from tests.tree import D, Tree, check

pytestmark = pytest.mark.gpu

# lens, trees, heads, page, dtype, cache
SHAPES = [
    ([1], [1], (1, 1), 16, "bf16", "same"),
    ([5, 0, 17], [3, 2, 1], (4, 2), 16, "bf16", "same"),
    ([63, 64, 65, 128], [1, 16, 5, 0], (8, 2), 16, "bf16", "same"),
    ([700, 31, 0], [7, 64, 33], (4, 1), 32, "bf16", "same"),
    ([333], [64], (8, 1), 64, "bf16", "same"),
    ([130, 1], [17, 9], (6, 3), 12, "bf16", "same"),
    ([777, 100], [5, 12], (2, 2), 12, "f32", "same"),
    ([95, 0, 31], [32, 64, 2], (4, 2), 4, "f32", "same"),
    ([300, 77], [24, 40], (8, 1), 60, "f32", "same"),
    ([513, 40], [16, 3], (4, 2), 16, "bf16", "e4m3"),
    ([200, 0, 9], [40, 8, 64], (8, 2), 32, "bf16", "e4m3"),
    ([99, 450], [4, 21], (2, 1), 20, "f32", "e4m3"),
    ([64, 333], [50, 64], (4, 2), 48, "f32", "e4m3"),
    ([2900, 17], [4, 2], (4, 1), 8, "bf16", "e4m3"),
    ([260, 100], [32, 20], (4, 1), 16, "bf16", "same"),
    ([150, 300], [30, 26], (8, 2), 8, "bf16", "e4m3"),
]
IDS = ["x".join(map(str, s[0])) + "-" + "x".join(map(str, s[1])) + f"-{s[2][0]}.{s[2][1]}-p{s[3]}-{s[4]}-{s[5]}" for s in SHAPES]


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
@pytest.mark.parametrize("over", ["full", "heads"])
def test_softmax(shape, over):
    lens, trees, heads, page, dtype, cache = shape
    check("softmax", lens=lens, trees=trees, heads=heads, page=page, dtype=dtype, cache=cache, over=over)


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
@pytest.mark.parametrize("over", ["full", "heads", "group"])
def test_entmax(shape, over):
    lens, trees, heads, page, dtype, cache = shape
    alpha = (1.25, 1.5, 2.0, 1.7, 4 / 3)[SHAPES.index(shape) % 5]
    check("entmax", lens=lens, trees=trees, heads=heads, page=page, dtype=dtype, cache=cache, over=over, alpha=alpha)


@pytest.mark.parametrize("form", ["softmax", "entmax"])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_any_mask_is_good(form, cache, dtype):
    """Rows that see none of the drafted keys, not themselves, others behind them; bits beyond the tree; an empty cache with them."""
    check(form, lens=[0, 50, 200], trees=[13, 64, 30], heads=(4, 2), dtype=dtype, cache=cache, masks="any", seed=4)
    check(form, lens=[0, 50, 0], trees=[3, 2, 6], heads=(2, 2), dtype=dtype, cache=cache, masks="any", over="heads", seed=5)


@pytest.mark.parametrize("form", ["softmax", "entmax"])
@pytest.mark.parametrize("lens,trees,heads,page,dtype,cache,over", [
    ([20000], [2], (4, 1), 16, "bf16", "same", "full"), ([9000, 33000, 0, 100], [3, 1, 4, 2], (2, 1), 32, "bf16", "same", "full"),
    ([17000], [17], (4, 2), 16, "bf16", "e4m3", "full"), ([12000, 500], [3, 2], (2, 2), 12, "f32", "same", "full"),
    ([70000, 30000], [2, 1], (2, 1), 16, "bf16", "same", "heads"), ([15000], [34], (4, 1), 16, "bf16", "same", "full"),
    ([40000], [1], (1, 1), 8, "bf16", "e4m3", "heads"),
])
def test_long_contexts_shared_by_workgroups(form, lens, trees, heads, page, dtype, cache, over):
    check(form, lens=lens, trees=trees, heads=heads, page=page, dtype=dtype, cache=cache, over=over, seed=7)


@pytest.mark.parametrize("form", ["softmax", "entmax"])
def test_capacity_far_above_the_lengths(form):
    t = Tree([100, 3], [5, 6], extra_pages=9000, over="full")
    t.check(form, t.run(form))
    t = Tree([100, 3000], [5, 40], extra_pages=3000, over="heads", chosen=0.02)
    t.check(form, t.run(form))


@pytest.mark.parametrize("form", ["softmax", "entmax"])
@pytest.mark.parametrize("scale", [0.001, 3.0])
def test_flat_and_peaked_rows(form, scale):
    """Flat: every key has weight, more of them than LDS holds; peaked: one."""
    check(form, lens=[3000, 40], trees=[2, 3], heads=(2, 1), scale=scale, alpha=1.5, seed=8)
    check(form, lens=[2600], trees=[3], heads=(2, 1), scale=scale, alpha=1.25, cache="e4m3", seed=9)


@pytest.mark.parametrize("alpha", [1.1, 3.0])
def test_other_alphas(alpha):
    check("entmax", lens=[400, 20], trees=[9, 20], alpha=alpha, seed=3)


@pytest.mark.parametrize("form", ["softmax", "entmax"])
def test_rows_of_no_sequence_are_left_and_a_cut_tree_is_its_first_rows(form):
    check(form, lens=[90, 20], trees=[5, 9], extra_rows=4, max_tree=7, masks="chain")


@pytest.mark.parametrize("form", ["softmax", "entmax"])
def test_starts_that_are_no_prefix_sums_read_nothing_outside(form):
    t = Tree([90, 20, 50], [5, 9, 4])
    d = t.device(form)
    for start in ([0, 900, -3, 1 << 30], [-5, -5, 30, 2], [18, 18, 18, 18]):
        d["start"].copy_(torch.tensor(start, dtype=torch.int32))
        t.call(d, form)
        torch.cuda.synchronize()
    d["start"].copy_(t.start)
    t.call(d, form)
    torch.cuda.synchronize()
    t.check(form, (d["out"].cpu(), d["norm"].cpu(), d["supp"].cpu()))


@pytest.mark.parametrize("form", ["softmax", "entmax"])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_lists_and_tables_out_of_range_are_clamped(form, cache):
    t = Tree([90, 200], [5, 9], over="heads", cache=cache)
    d = t.device(form)
    d["page_idx"].fill_(-9), d["n_sel"].fill_(1 << 30), d["table"].fill_(1 << 29)
    t.call(d, form)
    torch.cuda.synchronize()


@pytest.mark.parametrize("form", ["softmax", "entmax"])
@pytest.mark.parametrize("dtype,trees", [("bf16", [6]), ("bf16", [60]), ("f32", [6]), ("f32", [40])])
def test_what_a_mask_hides_counts_for_nothing(form, dtype, trees):
    """Infinities and NaN in drafted keys and values: rows that do not see them are as without, rows that see a value have it."""
    t = Tree([100], trees, heads=(2, 1), dtype=dtype, masks="chain", scale=0.02, alpha=1.25)
    clean = t.run(form)
    t.check(form, clean)
    t.k_new, t.v_new = t.k_new.clone(), t.v_new.clone()
    t.k_new[3, :, 5], t.v_new[4, :, 7], t.v_new[4, :, 9], t.v_new[5, :, 1] = math.nan, math.inf, math.nan, -math.inf
    out, norm, supp = t.run(form)
    assert torch.equal(out[:3], clean[0][:3]) and torch.equal(norm[:3], clean[1][:3])
    if form == "softmax":
        assert out[3:].isnan().all() and norm[3:].isnan().all()
    else:                                                     # a key that is no number is passed over
        assert out[3].isfinite().all() and norm[3:].isfinite().all()
    t.k_new[3, :, 5] = 0.0
    t.visible[:] = torch.tensor([(1 << r) | (0x30 if r in (2, 5) else 0) for r in range(trees[0])])
    out, norm, supp = t.run(form)
    for r in (2, 5):                                          # flat: every key has weight
        assert (out[r, :, 7] == math.inf).all() and out[r, :, 9].isnan().all() and (out[r, :, 1] == -math.inf).all()
        assert out[r, :, 10:].isfinite().all() and norm[r].isfinite().all()
    assert (out[4, :, 7] == math.inf).all() and out[4, :, 1].isfinite().all()
    for r in (0, 1, 3):
        assert out[r].isfinite().all()


@pytest.mark.parametrize("form", ["softmax", "entmax"])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_what_lies_behind_the_last_token_counts_for_nothing(form, cache):
    t = Tree([37, 5], [4, 3], cache=cache)
    clean = t.run(form)
    for b, n in enumerate(t.lens):
        ph, tok = int(t.table[b, n // 16]), n % 16
        for pool in (t.k, t.v):
            pool[ph, :, tok:] = 0x7F if cache == "e4m3" else math.nan
    dirty = t.run(form)
    assert all(torch.equal(x, y) for x, y in zip(clean, dirty))


@pytest.mark.parametrize("over", ["full", "heads", "group"])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_one_row_that_sees_nothing_drafted_is_the_single_token_call(over, cache):
    t = Tree([400, 90, 0], [1, 1, 1], heads=(8, 2), cache=cache, over=over, masks="any")
    out, tau, supp = t.run("entmax")
    d = t.device("entmax")
    o, x, s = torch.empty(3, 8, D, device="cuda"), torch.empty(3, 8, device="cuda"), torch.empty(3, 8, dtype=torch.int32, device="cuda")
    op = ekv.EKV_OP_DECODE_FULL if over == "full" else ekv.EKV_OP_DECODE_SPARSE
    ws = torch.empty(max(16, ekv.ekv_workspace_bytes(t.cfg, op)), dtype=torch.uint8, device="cuda")
    name = ("ekv_decode8_" if cache == "e4m3" else "ekv_decode_") + {"full": "full", "heads": "sparse", "group": "sparse_group"}[over]
    getattr(ekv, name)(t.cfg, d["q"], d["cache"], *(() if over == "full" else (d["page_idx"], d["n_sel"])), o, x, s, ws)
    live = slice(0, 2)
    # both are within the limits of check(); their thresholds are roots of scores in two orders of summation
    assert torch.allclose(tau[live], x.cpu()[live], rtol=1e-5, atol=1e-5) and torch.allclose(out, o.cpu(), rtol=1e-4, atol=1e-4)
    assert tau[2].isinf().all() and (out[2] == 0).all()


@pytest.mark.parametrize("form", ["softmax", "entmax"])
def test_a_range_of_the_heads_of_larger_pools(form):
    check(form, lens=[100, 300], trees=[4, 20], heads=(4, 2), pool_heads=5, over="full")
    check(form, lens=[100, 300], trees=[4, 20], heads=(4, 2), pool_heads=3, over="heads", cache="e4m3")


@pytest.mark.parametrize("form", ["softmax", "entmax"])
def test_many_sequences(form):
    """More lists than one workgroup keeps the lengths of in LDS."""
    b = 2100
    t = Tree([i % 40 for i in range(b)], [1 if i % 7 else 2 for i in range(b)], heads=(4, 4), page=16, masks="chain")
    got = t.run(form)
    keep = [0, 1, 2, 39, 40, 1000, 2000, b - 1]
    sub = {i: t.trees[i] for i in keep}
    t.trees = [sub.get(i, 0) for i in range(b)]
    taken = torch.zeros(t.n, dtype=torch.bool)
    for i in keep:
        taken[int(t.start[i]):int(t.start[i]) + t.trees[i]] = True
    for x in got:
        x[~taken] = 77
    t.check(form, got)


@pytest.mark.parametrize("form", ["softmax", "entmax"])
@pytest.mark.parametrize("lens,trees", [([3000, 50], [6, 3]), ([300, 50], [64, 3])])
def test_graph_replays_and_another_stream(form, lens, trees):
    t = Tree(lens, trees, heads=(4, 1))
    d = t.device(form)
    t.call(d, form)
    torch.cuda.synchronize()
    first = [d[x].clone() for x in ("out", "norm", "supp")]
    s = torch.cuda.Stream()
    for x in ("out", "norm", "supp"):
        d[x].fill_(77)
    torch.cuda.synchronize()
    t.call(d, form, stream=s.cuda_stream)
    s.synchronize()
    assert all(torch.equal(d[x], y) for x, y in zip(("out", "norm", "supp"), first))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        t.call(d, form)
    for lens2 in ([lens[0] // 2, 11], [0, 1], lens):
        t.lens = lens2
        d["lens"].copy_(torch.tensor(lens2, dtype=torch.int32))
        for x in ("out", "norm", "supp"):
            d[x].fill_(77)
        g.replay()
        torch.cuda.synchronize()
        t.check(form, (d["out"].cpu(), d["norm"].cpu(), d["supp"].cpu()))
    assert all(torch.equal(d[x], y) for x, y in zip(("out", "norm", "supp"), first))


@pytest.mark.parametrize("form", ["softmax", "entmax"])
def test_nearly_as_many_lists_as_lds_holds_the_lengths_of(form):
    t = Tree([(7 * i) % 50 for i in range(2040)], [1] * 2040, heads=(4, 4), page=16)
    got = t.run(form)
    keep = [0, 1, 7, 50, 1999, 2039]
    t.trees = [1 if i in keep else 0 for i in range(2040)]
    for x in got:
        x[[i for i in range(2040) if i not in keep]] = 77
    t.check(form, got)


@pytest.mark.parametrize("form", ["softmax", "entmax"])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_pages_beyond_4_gb_of_a_pool(form, cache):
    """The same pages at the far end of large pools, bit for bit."""
    t = Tree([300, 77], [9, 3], heads=(4, 2), page=16, cache=cache)
    near = t.run(form)
    d = t.device(form)
    per = 2 * 16 * D * (1 if cache == "e4m3" else 2)
    n = (5 << 30) // per + 1
    move = n - t.n_phys
    big = [torch.zeros(n, *d["k"].shape[1:], dtype=d["k"].dtype, device="cuda") for _ in "kv"]
    big[0][move:], big[1][move:] = d["k"], d["v"]
    table = d["table"] + move
    if cache == "e4m3":
        scales = [torch.ones(n, 2, device="cuda") for _ in "kv"]
        scales[0][move:], scales[1][move:] = d["ks"], d["vs"]
        d["cache"] = ekv.cache8_view(*big, *scales, table, d["lens"])
    else:
        d["cache"] = ekv.cache_view(*big, table, d["lens"])
    t.call(d, form)
    torch.cuda.synchronize()
    assert torch.equal(d["out"].cpu(), near[0]) and torch.equal(d["norm"].cpu(), near[1])


def long_batch(rows, heads, alpha=1.5, rising=False):
    """64 sequences of 94 groups of 64 keys: a workgroup goes through a dozen and more of them, so that it bounds rows and leaves groups out."""
    t = Tree([6000 - 7 * i for i in range(64)], [rows] * 64, heads=heads, alpha=alpha, seed=12, scale=0.15)
    if rising:                                             # scores that rise along the sequence: every group has the largest so far
        lift = torch.zeros(t.n_phys)
        for row in t.table:
            pages = row[row >= 0].long()
            lift[pages] = torch.arange(len(pages)) / t.m
        t.k = (t.k.float() + 0.5 * lift[:, None, None, None] * t.q.float().mean((0, 1))).to(t.dt)
        t.values[0] = t.k.double()
    return t


def check_some(t, form, got, keep):
    """The sequences `keep` alone, the others' rows as if they were none's: the definition takes its time."""
    start = t.start.tolist()
    for b in range(t.b):
        if b not in keep:
            t.trees[b] = 0
            for x in got:
                x[start[b]:start[b + 1]] = 77
    t.check(form, got)


@pytest.mark.parametrize("form", ["softmax", "entmax"])
def test_the_same_bits_from_run_to_run(form):
    t = long_batch(40, (8, 2))
    first = t.run(form)
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(first, t.run(form)))


@pytest.mark.parametrize("rows,heads", [(17, (1, 1)), (30, (4, 1)), (40, (4, 1))])
@pytest.mark.parametrize("alpha", [1.25, 1.5, 2.0, 2.7])
def test_groups_that_are_not_stored(rows, heads, alpha):
    t = long_batch(rows, heads, alpha)
    check_some(t, "entmax", t.run("entmax"), (0, 63) if rows == 17 else (31,))


@pytest.mark.parametrize("alpha", [1.5, 2.0])
def test_scores_that_rise_along_the_sequence(alpha):
    t = long_batch(18, (1, 1), alpha, rising=True)
    check_some(t, "entmax", t.run("entmax"), (0, 30, 63))


@pytest.mark.parametrize("length,others", [(262144 + 70, 0), (262144 - 1, 0), (131072 + 70, 600), (32768, 0), (32768, 600)])
@pytest.mark.parametrize("alpha", [1.5, 2.0])
def test_more_maxima_than_registers(length, others, alpha):
    """Rows whose drafted key has the largest score: it counts once, however the maxima are folded; with few rows in the call and with many."""
    t = Tree([length], [4], heads=(1, 1), alpha=alpha, seed=13, extra_rows=others)
    t.check("entmax", t.run("entmax"))


@pytest.mark.parametrize("length,others", [(40000, 0), (40000, 600), (8000, 2100), (140000, 600)])
@pytest.mark.parametrize("alpha", [1.05, 1.1, 1.25])
def test_rows_with_thousands_of_candidates(length, others, alpha):
    """Flat rows: more candidates than a workgroup keeps at its first try, or at any; with few rows in the call, with many, with very many."""
    t = Tree([length], [3], heads=(1, 1), alpha=alpha, seed=14, extra_rows=others)
    t.check("entmax", t.run("entmax"))


@pytest.mark.parametrize("lens,heads,cache", [([19000], (8, 8), "same"), ([3000] * 70, (4, 1), "same"), ([5000, 0, 4100, 4999] * 9, (4, 1), "e4m3")])
def test_softmax_of_32_rows_by_two_wavefronts(lens, heads, cache):
    t = Tree(lens, [20 if heads[1] == 8 else 7] * len(lens), heads=heads, cache=cache, seed=15)
    check_some(t, "softmax", t.run("softmax"), (0, 1, 2, len(lens) - 1))


@pytest.mark.parametrize("form", ["softmax", "entmax"])
def test_two_graphs_that_share_a_workspace(form):
    a, b = Tree([700, 90], [9, 4], heads=(4, 2), seed=16), Tree([40, 2000], [3, 16], heads=(4, 2), seed=17)
    da, db = a.device(form), b.device(form)
    db["ws"] = da["ws"] = max(da["ws"], db["ws"], key=lambda w: w.numel())
    graphs = []
    for t, d in ((a, da), (b, db)):
        t.call(d, form)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            t.call(d, form)
    for _ in range(3):
        for t, d, g in ((a, da, graphs[0]), (b, db, graphs[1])):
            for x in ("out", "norm", "supp"):
                d[x].fill_(77)
            g.replay()
            torch.cuda.synchronize()
            t.check(form, (d["out"].cpu(), d["norm"].cpu(), d["supp"].cpu()))
