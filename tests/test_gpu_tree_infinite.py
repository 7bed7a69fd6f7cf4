"""Drafted rows that see infinities: scores of +inf and -inf, infinite values of the cache."""
import math

import pytest
import torch

from tests.tree import Tree

pytestmark = pytest.mark.gpu

# lens, trees, heads, sequences' rows that are compared: up to 16 rows, rows in blocks, more maxima than one wavefront has, and than all have
SHAPES = {"16": ([700, 40], [3, 2], (2, 1)), "64": ([3000, 40], [20, 2], (2, 1)), "256": ([2500], [64], (4, 1)), "long": ([40000], [2], (1, 1)),
          "longest": ([262144 + 70], [2], (1, 1))}


def with_key(t, drafted):
    """Channel 5 of one key that all rows of sequence 0 see is infinite; half the rows have a positive channel there, the others a negative one."""
    t.visible[:t.trees[0]] |= 1
    t.q, t.k_new, t.k = t.q.clone(), t.k_new.clone(), t.k.clone()
    t.q[..., 5] = 1.0
    t.q[1::2, :, 5] = -1.0
    if drafted:
        t.k_new[0, :, 5] = math.inf
    else:
        t.k[int(t.table[0, 20]), :, 7, 5] = math.inf
    t.values[0] = t.k.double()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("drafted", [False, True])
@pytest.mark.parametrize("alpha", [1.5, 2.0, 1.7])
def test_entmax_scores(shape, drafted, alpha):
    lens, trees, heads = SHAPES[shape]
    t = Tree(lens, trees, heads=heads, alpha=alpha, seed=41)
    with_key(t, drafted)
    out, tau, supp = t.run("entmax")
    up, down = slice(0, trees[0], 2), slice(1, trees[0], 2)
    assert (out[up] == 0).all() and (supp[up] == 0).all() and tau[up].isnan().all()
    assert out[down].isfinite().all() and tau[down].isfinite().all() and (supp[down] > 0).all()
    # without the key the rows that it has no weight in are the same row
    k = t.k_new[0, :, 5] if drafted else t.k[int(t.table[0, 20]), :, 7, 5]
    k.fill_(1e30)                                            # times -1: far below every threshold
    plain = t.run("entmax")
    assert all(torch.equal(x[down], y[down]) for x, y in zip((out, tau, supp), plain))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", ["16", "64", "256", "long"])
@pytest.mark.parametrize("drafted", [False, True])
def test_softmax_scores(shape, drafted, dtype):
    lens, trees, heads = SHAPES[shape]
    t = Tree(lens, trees, heads=heads, dtype=dtype, seed=42)
    with_key(t, drafted)
    out, lse, _ = t.run("softmax")
    up, down = slice(0, trees[0], 2), slice(1, trees[0], 2)
    assert out[up].isnan().all() and lse[up].isnan().all()
    assert out[down].isfinite().all() and lse[down].isfinite().all()
    k = t.k_new[0, :, 5] if drafted else t.k[int(t.table[0, 20]), :, 7, 5]
    k.fill_(1e30)
    plain = t.run("softmax")
    assert torch.equal(out[down], plain[0][down]) and torch.equal(lse[down], plain[1][down])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", ["softmax", "entmax"])
@pytest.mark.parametrize("shape", ["16", "64", "256"])
def test_infinite_values_of_the_cache_stay_in_their_channel(form, dtype, shape):
    lens, trees, heads = SHAPES[shape]
    t = Tree(lens, trees, heads=heads, dtype=dtype, scale=0.001, alpha=1.25, seed=43)      # flat: every key has weight
    t.v = t.v.clone()
    row = t.v[int(t.table[0, 20]), :, 7]
    clean = t.run(form)
    row[:, 3], row[:, 77] = math.inf, -math.inf
    got = t.run(form)
    n = trees[0]
    assert all(torch.equal(x[n:], y[n:]) for x, y in zip(clean, got)) and torch.equal(clean[1], got[1]) and torch.equal(clean[2], got[2])
    rest = [i for i in range(128) if i not in (3, 77)]
    assert torch.equal(clean[0][..., rest], got[0][..., rest])
    at3, at77 = got[0][:n, :, 3], got[0][:n, :, 77]
    if form == "entmax" or dtype == "f32":
        assert (at3 == math.inf).all() and (at77 == -math.inf).all()
    else:
        assert ((at3 == math.inf) | at3.isnan()).all() and ((at77 == -math.inf) | at77.isnan()).all()
