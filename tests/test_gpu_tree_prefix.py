"""Softmax of drafted rows where workgroups share the lists' steps, with as many lists as LDS holds the lengths of and with more: the
steps before a list by a launch of their own, records and the join, and the lengths in LDS beside the largest tiles."""
import pytest
import torch

from tests.tree import Tree

pytestmark = pytest.mark.gpu
LISTS = 8192                                                 # what one workgroup keeps the lengths of


def batch_of(b, most, heads, cache="same", dtype="bf16", page=16):
    """b sequences of a row or two, a few with `most` rows; a capacity of more than 8192 tokens, whatever the lengths are: no block of rows is one
    workgroup's alone.  Lengths of a few steps and, of some, of many, whose rows several workgroups share."""
    big = {0, 5, b // 2, b - 1}
    lens = [3000 if i in (5, b // 2) else (7 * i) % 50 for i in range(b)]
    trees = [most if i in big else 0 if i % 9 == 3 else 1 for i in range(b)]
    return Tree(lens, trees, heads=heads, page=page, cache=cache, dtype=dtype, extra_pages=(8192 + page) // page, seed=31), sorted(big | {1, 2, 3, 50, b - 2})


def check_kept(t, got, keep):
    start = t.start.tolist()
    for i in range(t.b):
        if i not in keep:
            t.trees[i] = 0
            for x in got:
                x[start[i]:start[i + 1]] = 77
    t.check("softmax", got)


# a list for each of 4 KV heads: 2048 sequences have as many as LDS takes, 2049 more
@pytest.mark.parametrize("b", [LISTS // 4, LISTS // 4 + 1])
@pytest.mark.parametrize("most,heads", [(2, (4, 4)), (20, (4, 4)), (40, (4, 4)), (64, (4, 4)), (25, (16, 4)), (40, (16, 4))],
                         ids=["16-rows", "32-rows", "64-rows", "64-rows-full", "128-rows", "256-rows"])
def test_every_page(most, heads, b):
    t, keep = batch_of(b, most, heads)
    assert t.m * t.page > 8192
    check_kept(t, t.run("softmax"), keep)


@pytest.mark.parametrize("b", [LISTS // 4, LISTS // 4 + 1])
@pytest.mark.parametrize("most,heads,cache,dtype,page", [(3, (4, 4), "e4m3", "bf16", 16), (30, (16, 4), "e4m3", "bf16", 12), (3, (4, 4), "same", "f32", 16),
                                                         (20, (4, 4), "same", "f32", 16), (30, (4, 4), "e4m3", "f32", 32)])
def test_other_types(most, heads, cache, dtype, page, b):
    t, keep = batch_of(b, most, heads, cache, dtype, page)
    check_kept(t, t.run("softmax"), keep)


@pytest.mark.parametrize("b", [LISTS // 4 - 1, LISTS // 4 + 1])
@pytest.mark.parametrize("most", [2, 40])
def test_page_lists(most, b):
    """Lists whose room is above 8192 tokens, most of it not taken."""
    t = Tree([600 if i in (5, b - 1) else (7 * i) % 50 for i in range(b)], [most if i in (0, 5, b - 1) else 1 for i in range(b)], heads=(4, 4), over="heads",
             extra_pages=520, chosen=1.0, seed=32)
    assert t.cap * t.page > 8192
    check_kept(t, t.run("softmax"), [0, 1, 5, b - 2, b - 1])


@pytest.mark.parametrize("b", [LISTS // 4, LISTS // 4 + 1])
def test_the_same_bits_from_run_to_run(b):
    t, _ = batch_of(b, 40, (16, 4))
    d = t.device("softmax")
    first = None
    for _ in range(3):
        for x in ("out", "norm"):
            d[x].fill_(77)
        t.call(d, "softmax")
        torch.cuda.synchronize()
        got = [d[x].clone() for x in ("out", "norm")]
        first = first or got
        assert all(torch.equal(x, y) for x, y in zip(first, got))
