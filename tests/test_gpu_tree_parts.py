"""Calls for some of a batch's sequences: drafted rows in front of the first sequence's and behind the last one's are nobody's."""
import pytest
import torch

from paper_2605_21649_amd import binding as ekv
from tests.tree import D, Tree

pytestmark = pytest.mark.gpu


def call_part(t, d, form, b0, b1):
    """Sequences b0 .. b1 - 1 of the batch by slices of its tensors: the entry in front of their start is another sequence's."""
    cfg = ekv.make_config(b1 - b0, t.hq, t.hk, D, t.page, t.dtype, t.alpha, t.scale, t.m, t.cap, t.pool_heads)
    table, lens, start = d["table"][b0:b1], d["lens"][b0:b1], d["start"][b0:b1 + 1]
    if t.cache == "e4m3":
        cache = ekv.cache8_view(d["k"], d["v"], d["ks"], d["vs"], table, lens)
    else:
        cache = ekv.cache_view(d["k"], d["v"], table, lens)
    tree = ekv.tree_view(start, d["visible"], d["rows"][:, 1], d["rows"][:, 2], t.max_tree)
    lists = () if t.over == "full" else (d["page_idx"][b0:b1], d["n_sel"][b0:b1])
    outs = (d["out"], d["norm"]) + ((d["supp"],) if form == "entmax" else ())
    getattr(ekv, t.name(form))(cfg, d["q"], cache, tree, *lists, *outs, d["ws"])
    torch.cuda.synchronize()


# lens, drafted rows, sequences of the call
PARTS = {
    "3 from 1": ([40, 90, 20], [4, 3, 5], 1, 3),
    "3 from 2": ([40, 90, 20], [4, 3, 5], 2, 3),
    "4, the middle two": ([300, 0, 65, 17], [9, 2, 6, 1], 1, 3),
    "70 from 68": ([(5 * i) % 37 for i in range(70)], [1 + i % 2 for i in range(70)], 68, 70),
    "70 from 6": ([(5 * i) % 37 for i in range(70)], [1 + i % 2 for i in range(70)], 6, 70),
    "70 from 5": ([(5 * i) % 37 for i in range(70)], [1 + i % 2 for i in range(70)], 5, 70),
    "230 from 30": ([(11 * i) % 50 for i in range(230)], [1] * 230, 30, 230),
    "64 rows, 3 from 1": ([100, 50, 800], [64, 64, 33], 1, 3),
}


@pytest.mark.parametrize("part", PARTS, ids=[x.replace(" ", "-").replace(",", "") for x in PARTS])
@pytest.mark.parametrize("form,over", [("entmax", "full"), ("entmax", "heads"), ("entmax", "group"), ("softmax", "full"), ("softmax", "heads")])
def test_rows_of_other_sequences_are_left(form, over, part):
    lens, trees, b0, b1 = PARTS[part]
    t = Tree(lens, trees, heads=(2, 1), over=over, seed=21)
    d = t.device(form)
    call_part(t, d, form, b0, b1)
    got = [d[x].cpu() for x in ("out", "norm", "supp")]
    t.trees = [n if b0 <= b < b1 else 0 for b, n in enumerate(trees)]
    t.check(form, got)


@pytest.mark.parametrize("dtype,cache", [("f32", "same"), ("bf16", "e4m3"), ("f32", "e4m3")])
def test_other_types(dtype, cache):
    for over in ("full", "group"):
        lens, trees, b0, b1 = PARTS["70 from 5"]
        t = Tree(lens, trees, heads=(4, 2), over=over, dtype=dtype, cache=cache, seed=22)
        d = t.device("entmax")
        call_part(t, d, "entmax", b0, b1)
        got = [d[x].cpu() for x in ("out", "norm", "supp")]
        t.trees = [n if b0 <= b < b1 else 0 for b, n in enumerate(trees)]
        t.check("entmax", got)


@pytest.mark.parametrize("form", ["entmax", "softmax"])
@pytest.mark.parametrize("others", [0, 2100])
def test_no_row_is_anybodys(form, others):
    """Starts behind the last row, and starts that leave the first rows out; also with so many rows that one wavefront solves one."""
    t = Tree([90, 20, 50], [5, 9, 4], extra_rows=others)
    d = t.device(form)
    for start in ([18 + others] * 4, [1 << 30] * 4):
        d["start"].copy_(torch.tensor(start, dtype=torch.int32))
        t.call(d, form)
        torch.cuda.synchronize()
        assert all((d[x] == 77).all() for x in ("out", "norm", "supp")), start
    d["start"].copy_(torch.tensor([5, 5, 14, 18], dtype=torch.int32))
    t.call(d, form)
    torch.cuda.synchronize()
    t.trees[0] = 0                                           # the others' rows are where they were
    t.check(form, [d[x].cpu() for x in ("out", "norm", "supp")])
