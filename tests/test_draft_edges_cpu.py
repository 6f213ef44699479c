"""Host checks of what the calls on drafted tokens and a bounded memory refuse at the edges of their arguments.  No device
calls: every refused call returns before its first one."""
import ctypes

import pytest
import torch

from paper_2607_14695_amd import reflex as R
from paper_2607_14695_amd.paged import PagedBatch

from .test_paged_cpu import A, batch_c, cache_c

B = ctypes.byref


def weighed_accept(cache=None, batch=None, path=A, most=4, counts=A, weights=A, lengths=A):
    return R.load_library().reflex_paged_weighed_accept(B(cache or cache_c()), B(batch or batch_c()), path, most, counts,
                                                        weights, lengths, None)


def test_weighed_acceptance_is_checked():
    assert weighed_accept(batch=batch_c(n_seqs=0), weights=None) == R.REFLEX_OK
    for bad in (dict(weights=None), dict(weights=A + 2), dict(path=None), dict(counts=None), dict(lengths=None),
                dict(most=-1), dict(cache=cache_c(k=None)), dict(batch=batch_c(cu_rows=None)),
                dict(batch=batch_c(n_seqs=(1 << 17) + 1))):
        assert weighed_accept(**bad) == R.REFLEX_EINVAL
    assert R.load_library().reflex_paged_weighed_accept(B(cache_c()), None, A, 4, A, A, A, None) == R.REFLEX_EINVAL



def test_a_tree_of_too_many_rows_says_what_to_do():
    """Rows of all sequences together may be more than one tree may have; only their number is known without max_rows."""
    b = PagedBatch.__new__(PagedBatch)
    b.device = torch.device("cuda:0")
    parents = torch.zeros(5000, dtype=torch.int32)
    with pytest.raises(ValueError, match="of 5000 rows in all, give max_rows"):
        b.tree(parents)
    with pytest.raises(ValueError, match="at most 4096 rows, not 4097"):
        b.tree(parents, max_rows=4097)
    with pytest.raises(ValueError, match="parents is on cpu"):
        b.tree(parents, max_rows=4096)
