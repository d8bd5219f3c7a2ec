"""Workspace queries of sizes that were asked before: what the library refuses is refused, and a size that changes in place is read anew."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2012_15198_amd import cxlm as lm

QUERIES = [("cx_embed_workspace", (2, 500, 70, 9)), ("cx_scan_workspace", (2, 500, 70)), ("cx_scores_workspace", (2, 500_000, 3)), ("cx_distill_workspace", (2, 500_000)),
           ("cx_norm_workspace", (2, 500, 70)), ("cx_conv_workspace", (1, 4, 500, 70, 3)), ("cx_select_workspace", (2, 500, 70, 5)),
           ("cx_select_grad_workspace", (2, 500, 70, 5))]


@pytest.mark.parametrize("name,sizes", QUERIES)
def test_a_fraction_is_no_size(name, sizes):
    query = getattr(lm, name)
    for _ in range(2):
        assert query(*sizes) >= 0
        for k in range(len(sizes)):
            with pytest.raises(ctypes.ArgumentError):
                query(*sizes[:k], float(sizes[k]), *sizes[k + 1:])


@pytest.mark.parametrize("name,sizes", QUERIES)
def test_sizes_of_other_types(name, sizes):
    """numpy's integers and tensors of one number, which may change between calls."""
    query = getattr(lm, name)
    first = query(*sizes)
    assert query(*map(np.int64, sizes)) == first
    held = [torch.tensor(n) for n in sizes]
    assert query(*held) == first
    held[1].fill_(3)
    assert query(*held) == query(sizes[0], 3, *sizes[2:])
