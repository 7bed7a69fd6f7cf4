"""What a view of drafted rows holds on to (no GPU is needed)."""
import gc
import weakref

import torch

from paper_2605_21649_amd import binding as ekv


def test_a_view_keeps_its_tensors_for_as_long_as_it_is_there():
    """Memory of tensors that nobody else has is given to the next allocation: outputs and workspaces of the very call."""
    rows = torch.zeros(5, 6, 128)
    made = [torch.tensor([0, 2, 5], dtype=torch.int32), torch.tensor([1, 3, 1, 3, 7]), rows[:, :2], rows[:, 2:4]]
    refs, pointers = [weakref.ref(t) for t in made], [t.data_ptr() for t in made]
    tree = ekv.tree_view(*made, 3)
    del made, rows
    gc.collect()
    assert all(r() is not None for r in refs)
    assert [tree.start, tree.visible, tree.k_new, tree.v_new] == pointers == [r().data_ptr() for r in refs]
    del tree
    gc.collect()
    assert all(r() is None for r in refs)
