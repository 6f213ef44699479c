"""Host checks of drafted trees, their acceptance, weighed attention and eviction: what they refuse, and their reference
definitions on cases worked out by hand.  No device calls: every refused call returns before its first one."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2607_14695_amd import reflex as R
from paper_2607_14695_amd.paged import PagedBatch, PagedCache, _mask

from . import draft_reference as ref
from .test_paged_cpu import A, batch_c, cache_c, rows_c

B = ctypes.byref


def tree(batch=None, parents=A, n=0, mask=A, words=1, pos=A):
    return R.load_library().reflex_paged_tree(B(batch or batch_c()), parents, n, mask, words, pos, None)


def attend(cache=None, batch=None, q=None, o=None, n=0, heads=4, dtype=R.DTYPE_BF16, scale=0.125, mask=A, words=1,
           ws=None, nb=0):
    return R.load_library().reflex_paged_tree_attention(
        B(cache or cache_c()), B(batch or batch_c()), B(q or rows_c()), B(o or rows_c()), n, heads, dtype, scale, mask,
        words, ws, nb, None)


def accept(cache=None, batch=None, path=A, most=4, counts=A, lengths=A):
    return R.load_library().reflex_paged_accept(B(cache or cache_c()), B(batch or batch_c()), path, most, counts, lengths,
                                                None)


def weigh_bytes(cache=None, batch=None, n=1, heads=4, dtype=R.DTYPE_BF16):
    need = ctypes.c_size_t(0)
    status = R.load_library().reflex_paged_weighed_attention_workspace(B(cache or cache_c()), B(batch or batch_c()), n,
                                                                       heads, dtype, B(need))
    assert status == R.REFLEX_OK
    return need.value


def weigh(cache=None, batch=None, q=None, o=None, n=0, heads=4, dtype=R.DTYPE_BF16, scale=0.125, window=0, weights=A,
          ws=A, nb=1 << 30):
    return R.load_library().reflex_paged_weighed_attention(
        B(cache or cache_c()), B(batch or batch_c()), B(q or rows_c()), B(o or rows_c()), n, heads, dtype, scale, 1, window,
        weights, ws, nb, None)


def evict(cache=None, batch=None, weights=A, keep=8, sinks=0, recent=0, kept=A, lengths=A, ws=A, nb=1 << 30):
    return R.load_library().reflex_paged_evict(B(cache or cache_c()), B(batch or batch_c()), weights, keep, sinks, recent,
                                               kept, lengths, ws, nb, None)


def test_empty_calls_are_done():
    assert tree() == attend() == weigh() == R.REFLEX_OK
    none = batch_c(n_seqs=0)
    assert tree(none, n=5) == attend(batch=none, n=5) == weigh(batch=none, n=5) == R.REFLEX_OK
    assert accept(batch=none) == evict(batch=none) == R.REFLEX_OK


@pytest.mark.parametrize("bad", [
    dict(k=None), dict(v=A + 2), dict(n_pages=0), dict(page_size=24), dict(n_kv_heads=0), dict(head_dim=96),
    dict(store=4), dict(store=R.STORE_FP8), dict(store=R.STORE_INT8, k_scale=A), dict(n_pages=1 << 26)])
def test_bad_caches(bad):
    c = cache_c(**bad)
    assert attend(c, n=1) == weigh(c, n=1) == accept(c) == evict(c) == R.REFLEX_EINVAL


@pytest.mark.parametrize("bad", [
    dict(cu_rows=None), dict(lengths=None), dict(page_table=None), dict(n_seqs=-1), dict(max_pages=-1),
    dict(max_length=-1), dict(max_pages=1 << 27)])
def test_bad_batches(bad):
    b = batch_c(**bad)
    assert attend(batch=b, n=1) == weigh(batch=b, n=1) == accept(batch=b) == evict(batch=b) == R.REFLEX_EINVAL
    if not {"page_table", "max_pages", "max_length"} & set(bad):
        assert tree(b, n=1) == R.REFLEX_EINVAL


@pytest.mark.parametrize("r", [rows_c(data=None), rows_c(data=A + 8), rows_c(rs=129), rows_c(hs=4)])
def test_bad_rows(r):
    assert attend(q=r, n=1) == attend(o=r, n=1) == weigh(q=r, n=1) == weigh(o=r, n=1) == R.REFLEX_EINVAL


def test_bad_scalars_and_pointers():
    for call in (attend, weigh):
        assert call(n=-1) == call(n=(1 << 27) + 1) == call(n=1, dtype=2) == R.REFLEX_EINVAL
        assert call(n=1, dtype=R.DTYPE_F32) == R.REFLEX_EDTYPE
        for heads in (0, -2, 3, 1 << 25):
            assert call(n=2, heads=heads) == R.REFLEX_EINVAL
        for scale in (float("nan"), float("inf"), 2.4e38):
            assert call(n=1, scale=scale) == R.REFLEX_EINVAL
    for words in (0, -1, 65):
        assert tree(n=1, words=words) == attend(n=1, words=words) == R.REFLEX_EINVAL
    assert tree(n=-1) == tree(n=(1 << 27) + 1) == R.REFLEX_EINVAL
    assert tree(n=1, parents=None) == tree(n=1, mask=None) == tree(n=1, mask=A + 4) == tree(n=1, pos=A + 4) == R.REFLEX_EINVAL
    assert attend(n=1, mask=None) == attend(n=1, mask=A + 4) == R.REFLEX_EINVAL
    assert weigh(n=1, weights=None) == weigh(n=1, weights=A + 2) == weigh(n=1, window=-1) == R.REFLEX_EINVAL
    assert accept(path=None) == accept(counts=None) == accept(lengths=None) == accept(most=-1) == R.REFLEX_EINVAL
    assert evict(weights=None) == evict(weights=A + 1) == evict(lengths=None) == R.REFLEX_EINVAL
    assert R.load_library().reflex_paged_tree(None, A, 1, A, 1, A, None) == R.REFLEX_EINVAL


@pytest.mark.parametrize("keep,sinks,recent", [(0, 0, 0), (-1, 0, 0), (8, -1, 0), (8, 0, -1), (8, 5, 4),
                                               (8, 2 ** 31 - 1, 2 ** 31 - 1), ((1 << 30) + 1, 0, 0)])
def test_bad_budgets(keep, sinks, recent):
    assert evict(keep=keep, sinks=sinks, recent=recent) == R.REFLEX_EINVAL


def test_workspaces_are_checked():
    c, q = cache_c(n_pages=4096), batch_c(max_pages=1024, n_seqs=1)
    need = weigh_bytes(c, q)
    assert need > 0
    for ws, nb in ((None, need), (A, need - 1), (A + 16, need)):
        assert weigh(c, q, n=1, ws=ws, nb=nb) == R.REFLEX_EINVAL
    lib, size = R.load_library(), ctypes.c_size_t(0)
    assert lib.reflex_paged_evict_workspace(B(c), B(q), 100, B(size)) == R.REFLEX_OK
    assert size.value >= 1 * 2 * 100 * 4  # one sequence, two heads
    for ws, nb in ((None, size.value), (A, size.value - 1), (A + 128, size.value)):
        assert evict(c, q, keep=100, ws=ws, nb=nb) == R.REFLEX_EINVAL
    assert lib.reflex_paged_evict_workspace(B(c), B(q), 100, None) == R.REFLEX_EINVAL


def test_too_many_sequences_are_refused():
    c, many = cache_c(), batch_c(n_seqs=(1 << 17) + 1)  # of two heads
    size = ctypes.c_size_t(0)
    lib = R.load_library()
    assert lib.reflex_paged_evict_workspace(B(c), B(many), 1, B(size)) == R.REFLEX_EINVAL
    assert lib.reflex_paged_weighed_attention_workspace(B(c), B(many), 1, 4, 1, B(size)) == R.REFLEX_EINVAL
    assert evict(batch=many) == accept(batch=many) == weigh(batch=many, n=1) == R.REFLEX_EINVAL
    assert tree(batch_c(n_seqs=(1 << 18) + 1), n=1) == R.REFLEX_EINVAL


def test_python_refusals():
    t32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    for bad in (torch.zeros(4, 1), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 0, dtype=torch.int64),
                torch.zeros(4, 65, dtype=torch.int64), torch.zeros(3, 1, dtype=torch.int64),
                torch.zeros(4, 2, dtype=torch.int64)[:, :1], torch.zeros(4, 1, dtype=torch.int64)):
        with pytest.raises(ValueError):  # (the last one: not on a GPU)
            _mask(bad, 4, torch.device("cuda:0"))
    b = PagedBatch.__new__(PagedBatch)
    b.device = torch.device("cuda:0")
    for parents in (t32(4), t32(4, 1), torch.zeros(4, dtype=torch.int64)):
        with pytest.raises(ValueError):
            b.tree(parents)
    c = PagedCache.__new__(PagedCache)
    c.device, c.k = torch.device("cuda:0"), torch.zeros(2, 1, 16, 64)
    for weights in (torch.zeros(2, 1, 16), torch.zeros(2, 1, 8), torch.zeros(2, 1, 16, dtype=torch.float64),
                    torch.zeros(2, 1, 16, requires_grad=True)):
        with pytest.raises(ValueError):
            c._weights(weights)
    for keep in (2 ** 32 + 8, -2 ** 40):
        with pytest.raises(ValueError, match="keep"):
            c.evict(b, torch.zeros(2, 1, 16), keep)


def test_reference_tree_by_hand():
    """Two roots; a chain 0 - 2 - 3; a parent that is no earlier row counts as none."""
    sees, pos = ref.tree([-1, -1, 0, 2, 1, 7, 6], [0, 7], [17], 1, 8)
    assert sees[:7] == [{0}, {1}, {0, 2}, {0, 2, 3}, {1, 4}, {5}, {6}] and sees[7] is None
    assert pos[:7] == [10, 10, 11, 12, 11, 10, 10]
    assert ref.words_of({0, 63, 64, 127}, 3) == [1 - 2 ** 63, 1 - 2 ** 63, 0]
    sees, pos = ref.tree([-1] + list(range(69)), [0, 70], [70], 1, 70)
    assert sees[63] == set(range(64)) and pos[63] == 63 and sees[64] == set() and pos[64] == 0


def test_reference_evict_by_hand():
    table = np.array([[1, 0]])
    w = np.array([[[5.0, 6.0]], [[1.0, np.nan]]], dtype=np.float32)  # tokens 0..3: 1, nan, 5, 6
    k = np.arange(4.0).reshape(2, 1, 2, 1)  # tokens 0..3: 2, 3, 0, 1
    kept, new = ref.evict([k], w, [4], table, 3, 0, 0)
    assert kept.tolist() == [[[0, 2, 3]]] and new == [3]
    assert k[:, 0, :, 0].tolist() == [[1, 1], [2, 0]] and w[:, 0].tolist() == [[6, 0], [1, 5]]
    kept, _ = ref.evict([np.zeros((2, 1, 2, 1))], np.zeros((2, 1, 2), np.float32), [4], table, 2, 0, 1)
    assert kept.tolist() == [[[0, 3]]]  # equal weights: the earlier token, and the last one


def test_reference_accept_by_hand():
    k = np.arange(8.0).reshape(4, 1, 2, 1)
    new = ref.accept([k], [0, 5], [7], np.array([[0, 1, 2, 3]]), np.array([[1, 3, 4, 9]]), [3])
    assert new == [5] and k.reshape(-1).tolist() == [0, 1, 3, 5, 6, 5, 6, 7]
