"""GPU checks of drafted tokens and a bounded memory where a call meets the edge of what its arguments allow: tables
without pages, lengths past the table, paths below the rows."""
import numpy as np
import pytest
import torch

from paper_2607_14695_amd.paged import PagedBatch

from . import draft_reference as ref
from .test_gpu_draft import raw, same_pages
from .test_gpu_paged import DEV, batch, draw, filled, pool

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------------------
# a page table of no pages: every token is absent
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("news,heads,dtype,store", [
    ([1], 4, "bf16", "bf16"), ([300, 0, 20], 8, "bf16", "bf16"), ([1200], 1, "bf16", "fp8"), ([700, 500], 4, "bf16", "int8"),
    ([40], 4, "f32", "f32")])
def test_a_table_of_no_pages(news, heads, dtype, store):
    """From single tokens to lists of more than 1,024 rows: zeros, no weight, no move."""
    gen = torch.Generator().manual_seed(sum(news))
    n = sum(news)
    cache, _, _ = filled(3, 1, 16, 128, store, gen)
    want, w = raw(cache), torch.rand(3, 1, 16, generator=gen).to(DEV)
    w0 = w.clone()
    lengths = i32([m + 100 for m in news])
    b = PagedBatch(i32([0] + list(np.cumsum(news))), lengths, torch.zeros(len(news), 0, dtype=torch.int32, device=DEV))
    q = draw(gen, (n, heads, 128), dtype).to(DEV)
    mask, _ = b.tree(torch.arange(-1, n - 1, dtype=torch.int32, device=DEV))
    for causal, window in ((True, 0), (False, 0), (True, 9)):
        assert not cache.attend(b, q, causal=causal, window=window).any()
        out = torch.full_like(q, 7.0)
        cache.attend(b, q, causal=causal, window=window, weights=w, out=out)
        assert not out.any() and torch.equal(w, w0)
    out = torch.full_like(q, 7.0)
    cache.attend_tree(b, q, mask, out=out)
    assert not out.any()
    counts = [min(m, 2) for m in news]
    cache.accept(b, i32([[0, 1]] * len(news)), i32(counts))
    assert lengths.tolist() == [100 + c for c in counts]
    assert (cache.evict(b, w, 5000) == -1).all()
    same_pages(cache, want)
    assert torch.equal(w, w0) and lengths.tolist() == [100 + c for c in counts]


# ---------------------------------------------------------------------------
# paths that begin with negative entries
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("store,hk,dh", [("bf16", 1, 256), ("f32", 1, 64), ("fp8", 3, 64), ("bf16", 8, 128), ("int8", 2, 256)])
@pytest.mark.parametrize("lead", [1, 5, 90])
def test_accept_a_path_that_begins_below_the_rows(store, hk, dh, lead):
    """Negative entries read as zeros, and the rows after them move up and then, past those left out, down: over many
    steps, equal to a copy taken before.  Rows past the last one end the path."""
    gen = torch.Generator().manual_seed(lead + dh)
    news = [900, 700, 40, lead]
    cu, lens, table, n_pages = pool(news, [n + 30 for n in news], 16, gen)
    table[0, 5] = -1
    cache, _, _ = filled(n_pages, hk, 16, dh, store, gen)
    path = torch.full((4, 900), 7, dtype=torch.int32)
    counts = []
    for s, n in enumerate(news):
        some = torch.randperm(n, generator=gen)[:n - lead // 2 if s == 1 else n // 2].sort().values.to(torch.int32)
        mine = torch.cat([torch.arange(-lead, 0, dtype=torch.int32), some[:n - lead] if n > lead else some[:0]])
        counts.append(min(n, len(mine)))
        path[s, :counts[-1]] = mine[:counts[-1]]
    path[2, counts[2] - 1] = 40
    want = raw(cache)
    new = ref.accept(want, cu.tolist(), lens.tolist(), table.numpy(), path.numpy(), counts)
    b = batch(cu, lens, table)
    cache.accept(b, path.to(DEV), i32(counts))
    same_pages(cache, want)
    assert b.tensors[1].tolist() == new
