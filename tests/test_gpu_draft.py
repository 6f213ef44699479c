"""GPU parity of drafted trees, their acceptance, weighed attention and eviction against their float64 definitions.

Tolerances.  Trees, acceptance and eviction move and choose: equal.  The attention of drafted tokens is held as the
attention of a run is.  Weights: a probability is off by its scores' error (twice (dh + 4) 2^-24 of `reach`, the row's
largest scale * sum |q||k|, as score and maximum are formed apart), by exp2's and its sum's (2^-21 and 64 steps, as for
the attention); the sum over n probabilities adds at most n 2^-24 of itself, and the addition to the weight half a step.
"""
import numpy as np
import pytest
import torch
from torch.autograd import forward_ad

from paper_2607_14695_amd import reflex as R
from paper_2607_14695_amd.paged import PagedBatch, PagedCache, Rotary

from . import draft_reference as ref
from . import paged_reference as pref
from .test_gpu_paged import DEV, DT, ROUND, batch, check_attention, draw, f64, filled, pool

pytestmark = pytest.mark.gpu


def random_parents(news, gen, back=6):
    """Every row follows one of the rows before it, mostly a near one, or the cached tokens."""
    out = []
    for n in news:
        for i in range(n):
            out.append(max(-1, i - 1 - int(torch.randint(0, back, (1,), generator=gen))))
    return torch.tensor(out, dtype=torch.int32)


def whole_words(mask):
    """[rows, words] int64 as one whole number a row."""
    return [sum((int(w) & (2 ** 64 - 1)) << (64 * i) for i, w in enumerate(r)) for r in mask.tolist()]


# ---------------------------------------------------------------------------
# trees
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("news,lengths,words", [
    ([1], [1], 1), ([16], [833], 1), ([64, 65, 63], [70, 65, 1000], 2), ([0, 5, 0, 200, 1], [3, 9, 0, 210, 2 ** 30], 4),
    ([130], [40], 2), ([150], [150], 1), ([3] * 70, list(range(70)), 3)])
def test_tree(news, lengths, words):
    """More rows than tokens, rows that the words cannot name, parents that are no earlier row, rows of no sequence."""
    gen = torch.Generator().manual_seed(sum(news))
    n = sum(news)
    parents = torch.cat([random_parents(news, gen), torch.zeros(3, dtype=torch.int32)])
    if n > 4:
        parents[n // 2], parents[n // 3] = 2 ** 31 - 1, -2 ** 31
    cu = torch.tensor([0] + news).cumsum(0).to(torch.int32)
    b = PagedBatch(cu.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV),
                   torch.zeros(len(news), 0, dtype=torch.int32, device=DEV))
    out = (torch.full((n + 3, words), 77, dtype=torch.int64, device=DEV), torch.full((n + 3,), 77, device=DEV))
    mask, pos = b.tree(parents.to(DEV), out=out)
    sees, want = ref.tree(parents.tolist(), cu.tolist(), lengths, words, n + 3)
    assert mask.tolist() == [[77] * words if s is None else ref.words_of(s, words) for s in sees]
    assert pos.tolist() == [77 if p is None else p for p in want]
    if words == -(-max(news) // 64):
        mask2, pos2 = b.tree(parents.to(DEV), max_rows=max(news))
        assert torch.equal(mask2[:n], mask[:n]) and torch.equal(pos2[:n], pos[:n])


def test_tree_of_one_long_chain():
    n = 4096
    b = batch(torch.tensor([0, n], dtype=torch.int32), torch.tensor([n + 7], dtype=torch.int32),
              torch.zeros(1, 1, dtype=torch.int32))
    mask, pos = b.tree(torch.arange(-1, n - 1, dtype=torch.int32, device=DEV))
    assert torch.equal(pos.cpu(), torch.arange(7, n + 7))
    bits = (mask.cpu()[:, :, None] >> torch.arange(64)) & 1
    assert torch.equal(bits.reshape(n, n), torch.ones(n, n, dtype=torch.int64).tril())


# ---------------------------------------------------------------------------
# attention of drafted tokens
# ---------------------------------------------------------------------------
def check_tree(q, cache, kv, cu, lens, table, mask, dtype, max_length=0, out=None, scale=None):
    dh = q.shape[-1]
    got = f64(cache.attend_tree(batch(cu, lens, table, max_length), q.to(DEV), mask.to(DEV), scale=scale, out=out))
    scale = dh ** -0.5 if scale is None else scale
    want, spread, reach, _, _ = ref.attend_seen(f64(q), *kv, cu.tolist(), lens.tolist(), table.numpy(),
                                                ref.in_tree(whole_words(mask), cu.tolist()), scale)
    rows = ~np.isnan(want[:, 0, 0])
    moved = 2 * (2 * (dh + 4) * 2.0 ** -24 * reach + 2.0 ** -21 + 64 * 2.0 ** -24) + (2.0 ** -8 if dtype == "bf16" else 0)
    under = 2.0 ** -126 * (1 + max(int(lens.max()), 0) * np.abs(kv[1]).max())
    off = np.abs(got - want)[rows] - (moved * spread + ROUND[dtype] * np.abs(want) + under)[rows]
    assert not np.isnan(off).any()
    assert off.max(initial=-1) <= 0, (off.max(), np.argwhere(off > 0)[:5])
    return got


TREES = {
    # (drafted, length) of each sequence, query heads, kv heads, head dim, page size, words
    "one_node": ([(1, 1)], 8, 1, 256, 16, 1),
    "one_node_long": ([(1, 817), (1, 300)], 8, 1, 256, 64, 1),
    "few_rows": ([(2, 70), (3, 3), (1, 129)], 4, 2, 64, 8, 1),
    "robot": ([(16, 833)], 8, 1, 256, 16, 1),
    "ragged": ([(5, 40), (0, 9), (33, 33), (64, 500), (1, 0), (17, 200)], 4, 2, 128, 16, 1),
    "wide_mask": ([(130, 391), (70, 70)], 8, 2, 64, 32, 3),
    "words_to_spare": ([(10, 100)], 4, 1, 128, 64, 5),
    "words_too_few": ([(100, 300)], 4, 1, 128, 64, 1),
    "before_start": ([(40, 25), (3, 1)], 8, 1, 64, 8, 1),
    "page_of_one": ([(9, 90)], 2, 1, 128, 1, 1),
    "odd_group": ([(21, 64), (50, 177)], 15, 3, 256, 128, 1),
}


@pytest.mark.parametrize("kind", ["tree", "random"])
@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "f32"), ("f32", "int8"),
                                         ("f32", "fp8")])
@pytest.mark.parametrize("name", sorted(TREES))
def test_attend_tree(name, dtype, store, kind):
    seqs, heads, hk, dh, ps, words = TREES[name]
    gen = torch.Generator().manual_seed(len(name) + dh + words)
    news, lengths = [s[0] for s in seqs], [s[1] for s in seqs]
    cu, lens, table, n_pages = pool(news, lengths, ps, gen, more_pages=2)
    n = sum(news)
    cache, kk, vv = filled(n_pages, hk, ps, dh, store, gen)
    q = draw(gen, (n, heads, dh), dtype)
    if kind == "tree":
        mask = batch(cu, lens, table).tree(random_parents(news, gen).to(DEV), out=(
            torch.zeros(n, words, dtype=torch.int64, device=DEV), torch.zeros(n, dtype=torch.int64, device=DEV)))[0].cpu()
    else:  # any rows, itself or not; some none
        mask = torch.randint(-2 ** 63, 2 ** 63 - 1, (n, words), generator=gen)
        mask[::3] = 0
    check_tree(q, cache, (kk, vv), cu, lens, table, mask, dtype)


@pytest.mark.parametrize("max_length", [0, 1, 2000])
@pytest.mark.parametrize("dtype,store,new", [("bf16", "bf16", 2), ("bf16", "fp8", 64), ("f32", "f32", 20)])
def test_attend_tree_over_splits(dtype, store, new, max_length):
    """Splits of the keys, one of which may hold drafted tokens alone, and a length that was expected otherwise."""
    gen = torch.Generator().manual_seed(new)
    cu, lens, table, n_pages = pool([new, new], [2000, 1100], 16, gen)
    cache, kk, vv = filled(n_pages, 1, 16, 128, store, gen)
    mask = batch(cu, lens, table).tree(random_parents([new, new], gen).to(DEV), max_rows=new)[0].cpu()
    check_tree(draw(gen, (2 * new, 4, 128), dtype), cache, (kk, vv), cu, lens, table, mask, dtype, max_length)


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "int8")])
def test_attend_tree_absent_pages_and_rows_of_no_sequence(dtype, store):
    gen = torch.Generator().manual_seed(3)
    news = [9, 30]
    cu, lens, table, n_pages = pool(news, [100, 64], 4, gen)
    table[0, 3], table[0, 23], table[1, 8], table[1, 15] = -1, n_pages, -7, -1
    cu += 2  # two rows before the first sequence
    cache, kk, vv = filled(n_pages, 2, 4, 64, store, gen)
    n = sum(news) + 5
    q = draw(gen, (n, 4, 64), dtype)
    mask = torch.randint(-2 ** 63, 2 ** 63 - 1, (n, 1), generator=gen)
    out = torch.full((n, 4, 64), 77.0, dtype=DT[dtype], device=DEV)
    got = check_tree(q, cache, (kk, vv), cu, lens, table, mask, dtype, out=out)
    assert np.all(got[:2] == 77) and np.all(got[-3:] == 77)
    # rows past the call's: cut off, with the tokens where they are
    m = 25
    cut = check_tree(q[:m], cache, (kk, vv), cu, lens, table, mask[:m], dtype)
    np.testing.assert_allclose(cut[2:], got[2:m], atol=0.05 if dtype == "bf16" else 1e-5)


@pytest.mark.parametrize("new,dtype,store", [(2, "bf16", "bf16"), (40, "bf16", "bf16"), (12, "f32", "f32"),
                                             (40, "bf16", "fp8")])
@pytest.mark.parametrize("value", ["nan", "inf"])
def test_what_a_drafted_row_does_not_see(new, dtype, store, value):
    """A drafted token with NaN or infinite K and V counts for itself and what follows it, and for no other row."""
    gen = torch.Generator().manual_seed(new)
    cu, lens, table, n_pages = pool([new], [new + 200], 16, gen)
    cache, kk, vv = filled(n_pages, 1, 16, 128, store, gen)
    parents = torch.tensor([-1] + [0] * (new - 1), dtype=torch.int32)  # all siblings below the first
    mask = batch(cu, lens, table).tree(parents.to(DEV))[0].cpu()
    q = draw(gen, (new, 4, 128), dtype)
    bad = new - 1
    page, slot = pref.place(table[0], n_pages, 16, 200 + bad)
    before = f64(cache.attend_tree(batch(cu, lens, table), q.to(DEV), mask.to(DEV)))
    if store == "fp8":
        cache.v_scale[page, 0, slot] = cache.k_scale[page, 0, slot] = float("nan")
    else:
        cache.k[page, 0, slot, 5] = cache.v[page, 0, slot, 7] = float(value)
    got = f64(cache.attend_tree(batch(cu, lens, table), q.to(DEV), mask.to(DEV)))
    assert not np.isfinite(got[bad]).all(-1).any()
    # (a row that is taken again key by key is rounded otherwise)
    moved = 2.0 ** -6 if dtype == "bf16" else 1e-5
    np.testing.assert_allclose(got[:bad], before[:bad], atol=moved, rtol=moved)


@pytest.mark.parametrize("new,dtype", [(2, "bf16"), (64, "bf16"), (12, "f32")])
@pytest.mark.parametrize("token", [3, 5000, 8190])
def test_an_infinite_value_over_many_splits(new, dtype, token):
    """An infinite element of a value that all rows see is theirs in that dim, in whichever of the splits it lies and
    whichever of them have no token; the other dims are as without it."""
    gen = torch.Generator().manual_seed(new)
    cu, lens, table, n_pages = pool([new], [new + 8191], 16, gen)
    table[0, 100:250] = -1  # (whole splits of absent tokens)
    cache, kk, vv = filled(n_pages, 1, 16, 128, dtype, gen)
    mask = batch(cu, lens, table).tree(random_parents([new], gen).to(DEV))[0].cpu()
    q = draw(gen, (new, 4, 128), dtype)
    before = check_tree(q, cache, (kk, vv), cu, lens, table, mask, dtype)
    page, slot = pref.place(table[0], n_pages, 16, token)
    cache.v[page, 0, slot, 7] = float("inf")
    got = f64(cache.attend_tree(batch(cu, lens, table), q.to(DEV), mask.to(DEV)))
    assert np.all(got[..., 7] == np.inf)
    # (a row that is taken again key by key is rounded otherwise)
    others = np.arange(128) != 7
    moved = 2.0 ** -6 if dtype == "bf16" else 1e-5
    np.testing.assert_allclose(got[..., others], before[..., others], atol=moved, rtol=moved)


@pytest.mark.parametrize("new,dtype", [(3, "bf16"), (100, "bf16"), (30, "f32")])
def test_tree_of_a_chain_is_causal_attention(new, dtype):
    """Each within its tolerance of its own definition, of which the two are one and the same here."""
    gen = torch.Generator().manual_seed(4)
    cu, lens, table, n_pages = pool([new], [new + 333], 16, gen)
    cache, kk, vv = filled(n_pages, 2, 16, 128, dtype, gen)
    q = draw(gen, (new, 4, 128), dtype)
    mask, pos = batch(cu, lens, table).tree(torch.arange(-1, new - 1, dtype=torch.int32, device=DEV))
    assert pos.tolist() == list(range(333, 333 + new))
    check_tree(q, cache, (kk, vv), cu, lens, table, mask.cpu(), dtype)
    check_attention(q, cache, (kk, vv), cu, lens, table, True, 0, dtype)
    seen = ref.in_tree(whole_words(mask), cu.tolist())
    assert all(list(seen(r, 0, 333 + r, 333 + new)) == list(range(334 + r)) for r in range(new))


def test_attend_tree_strides_and_scales():
    """Queries and results as slices of packed rows; other scales, a negative and a tiny one among them."""
    gen = torch.Generator().manual_seed(8)
    cu, lens, table, n_pages = pool([12, 5], [50, 90], 8, gen)
    cache, kk, vv = filled(n_pages, 1, 8, 64, "bf16", gen)
    packed = torch.randn(17, 12, 64, generator=gen).bfloat16().to(DEV)
    mask = torch.randint(-2 ** 63, 2 ** 63 - 1, (17, 1), generator=gen)
    b = batch(cu, lens, table)
    want = cache.attend_tree(b, packed[:, 4:8].contiguous(), mask.to(DEV))
    out = packed[:, 8:]
    assert cache.attend_tree(b, packed[:, 4:8], mask.to(DEV), out=out) is out and torch.equal(out, want)
    for scale in (-0.3, 1e-40, 0.0, 5.0):
        check_tree(packed[:, 4:8].cpu(), cache, (kk, vv), cu, lens, table, mask, "bf16", scale=scale)


# ---------------------------------------------------------------------------
# weighed attention
# ---------------------------------------------------------------------------
def check_weighed(q, cache, kv, cu, lens, table, causal, window, dtype, gen, max_length=0, scale=None, start=None):
    dh = q.shape[-1]
    w0 = torch.rand(cache.k.shape[:3], generator=gen) if start is None else start
    w = w0.to(DEV)
    b = batch(cu, lens, table, max_length)
    got = cache.attend(b, q.to(DEV), causal=causal, window=window, scale=scale, weights=w)
    plain = cache.attend(b, q.to(DEV), causal=causal, window=window, scale=scale)
    lo, hi = max(0, int(cu[0])), min(int(cu[-1]), q.shape[0])
    assert torch.equal(got[lo:hi].nan_to_num(7.0), plain[lo:hi].nan_to_num(7.0))
    scale = dh ** -0.5 if scale is None else scale
    _, _, _, want, (reach, parts, n) = ref.attend_seen(f64(q), *kv, cu.tolist(), lens.tolist(), table.numpy(),
                                                       ref.in_run(causal, window), scale, f64(w0))
    tol = (2 * (2 * (dh + 4) * 2.0 ** -24 * reach + (2.0 ** -21 + 64 * 2.0 ** -24) * parts) + n * 2.0 ** -24 * parts +
           2.0 ** -24 * np.abs(want) + n * 2.0 ** -126)
    off = np.abs(f64(w) - want) - tol
    assert not np.isnan(off).any()
    assert off.max() <= 0, (off.max(), np.argwhere(off > 0)[:5])
    assert np.array_equal(f64(w)[n == 0], f64(w0)[n == 0])  # keys that nothing sees
    return w


WEIGH = {
    # (new, length) of each sequence, query heads, kv heads, head dim, page size, causal, window
    "one_token": ([(1, 1)], 8, 1, 256, 16, True, 0),
    "tokens_ragged": ([(1, 817), (1, 1), (1, 64), (1, 65), (1, 0), (1, 300)], 8, 1, 256, 16, True, 0),
    "tokens_mha": ([(1, 129), (1, 31)], 3, 3, 64, 32, True, 0),
    "tokens_window": ([(1, 500)] * 3, 10, 2, 128, 64, True, 100),
    "wide_group": ([(1, 70), (2, 40)], 40, 1, 64, 8, True, 0),
    "page_of_one": ([(5, 90)], 2, 1, 128, 1, True, 0),
    "chunk": ([(51, 400)], 8, 1, 256, 64, False, 0),
    "chunk_causal": ([(130, 259), (33, 33)], 4, 2, 128, 16, True, 0),
    "window": ([(150, 200), (9, 60), (0, 5), (1, 1)], 4, 2, 64, 16, True, 33),
    "window_only": ([(70, 150)], 4, 1, 128, 8, False, 21),
    "before_start": ([(40, 25), (3, 1)], 8, 1, 64, 8, True, 0),
    "widest_window": ([(40, 60), (1, 33)], 4, 1, 64, 8, False, 2 ** 31 - 1),
    # rows of five and three heads, whose tokens end inside the stages, and rows that workgroups divide
    "heads_of_five": ([(130, 259), (33, 64)], 10, 2, 64, 16, True, 0),
    "heads_of_three": ([(70, 333), (1, 1)], 3, 1, 256, 32, True, 90),
    "divided_rows": ([(150, 400)], 8, 1, 128, 16, True, 0),
    "divided_window": ([(260, 300), (100, 100)], 5, 1, 64, 8, True, 70),
}


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "f32"), ("f32", "int8"),
                                         ("f32", "fp8")])
@pytest.mark.parametrize("name", sorted(WEIGH))
def test_weighed(name, dtype, store):
    seqs, heads, hk, dh, ps, causal, window = WEIGH[name]
    gen = torch.Generator().manual_seed(len(name) + dh)
    news, lengths = [s[0] for s in seqs], [s[1] for s in seqs]
    cu, lens, table, n_pages = pool(news, lengths, ps, gen, more_pages=2)
    cache, kk, vv = filled(n_pages, hk, ps, dh, store, gen)
    check_weighed(draw(gen, (sum(news) + 2, heads, dh), dtype), cache, (kk, vv), cu, lens, table, causal, window, dtype, gen)


def test_weighed_strides():
    """Queries as slices of packed rows, with heads in turn and rows backwards in memory; equal to packed ones."""
    gen = torch.Generator().manual_seed(31)
    for new, heads, dtype in ((130, 8, "bf16"), (70, 5, "bf16"), (3, 8, "bf16"), (40, 4, "f32")):
        cu, lens, table, n_pages = pool([new], [new + 200], 16, gen)
        cache, _, _ = filled(n_pages, 1, 16, 64, dtype, gen)
        b = batch(cu, lens, table)
        packed = torch.randn(new, 3 * heads, 64, generator=gen).to(DT[dtype]).to(DEV)
        heads_first = packed[:, heads:2 * heads].transpose(0, 1).contiguous().transpose(0, 1)
        want = cache.zero_weights()
        cache.attend(b, packed[:, heads:2 * heads].contiguous(), weights=want)
        for q in (packed[:, heads:2 * heads], heads_first):
            w = cache.zero_weights()
            cache.attend(b, q, weights=w)
            assert torch.equal(w, want)


@pytest.mark.parametrize("n_seqs", [70, 300])
@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("f32", "int8")])
def test_many_sequences(n_seqs, dtype, store):
    """More sequences than lanes, and more than CUs; empty ones among them."""
    gen = torch.Generator().manual_seed(n_seqs)
    news = [(b * 7) % 5 for b in range(n_seqs)]
    lengths = [n + (b * 37) % 90 for b, n in enumerate(news)]
    cu, lens, table, n_pages = pool(news, lengths, 8, gen)
    cache, kk, vv = filled(n_pages, 1, 8, 64, store, gen)
    q = draw(gen, (sum(news), 4, 64), dtype)
    parents = random_parents(news, gen)
    mask, pos = batch(cu, lens, table).tree(parents.to(DEV), max_rows=4)
    sees, at = ref.tree(parents.tolist(), cu.tolist(), lengths, 1, sum(news))
    assert mask[:, 0].tolist() == [ref.words_of(s, 1)[0] for s in sees] and pos.tolist() == at
    check_tree(q, cache, (kk, vv), cu, lens, table, mask.cpu(), dtype)
    check_weighed(q, cache, (kk, vv), cu, lens, table, True, 0, dtype, gen)


@pytest.mark.parametrize("max_length", [0, 1, 2000])
@pytest.mark.parametrize("dtype,store,new", [("bf16", "bf16", 1), ("bf16", "fp8", 64), ("f32", "f32", 3)])
def test_weighed_over_splits(dtype, store, new, max_length):
    """A length that was expected otherwise only sizes the launch."""
    gen = torch.Generator().manual_seed(new)
    cu, lens, table, n_pages = pool([new, new], [2000, 1100], 16, gen)
    cache, kk, vv = filled(n_pages, 1, 16, 128, store, gen)
    check_weighed(draw(gen, (2 * new, 4, 128), dtype), cache, (kk, vv), cu, lens, table, True, 0, dtype, gen, max_length)


@pytest.mark.parametrize("new", [1, 60])
@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("f32", "int8")])
def test_weighed_with_a_table_of_many_pages(dtype, store, new):
    """A table for a million tokens, of which the sequences have a few hundred: the scores of few rows over all that it
    could hold are not kept."""
    gen = torch.Generator().manual_seed(new)
    cu, lens, table, n_pages = pool([new] * 3, [300, 64, 129], 8, gen)
    table = torch.nn.functional.pad(table, (0, 2 ** 17 - table.shape[1]), value=-1)
    cache, kk, vv = filled(n_pages, 2, 8, 64, store, gen)
    check_weighed(draw(gen, (3 * new, 16, 64), dtype), cache, (kk, vv), cu, lens, table, True, 0, dtype, gen)


@pytest.mark.parametrize("new,dtype,store", [(1, "bf16", "bf16"), (40, "bf16", "fp8"), (12, "f32", "f32")])
def test_weighed_absent_pages_and_cut_rows(new, dtype, store):
    gen = torch.Generator().manual_seed(new)
    cu, lens, table, n_pages = pool([new, new], [100, 64], 4, gen)
    table[0, 3], table[1, 8], table[1, 15] = -1, n_pages, -1
    cu += 1
    cache, kk, vv = filled(n_pages, 2, 4, 64, store, gen)
    q = draw(gen, (2 * new + 3, 4, 64), dtype)
    for n in (2 * new + 3, new + 1 + new // 2):
        check_weighed(q[:n], cache, (kk, vv), cu, lens, table, True, 0, dtype, gen)


@pytest.mark.parametrize("new,dtype", [(1, "bf16"), (40, "bf16"), (12, "f32")])
def test_weighed_nan_and_infinities(new, dtype):
    """A NaN key makes the rows that see it NaN, and so the weights of all that they see; a key that no row of the
    sequence sees has no part; NaN values leave the weights as they are; a row without a sum adds nothing."""
    gen = torch.Generator().manual_seed(new)
    cu, lens, table, n_pages = pool([new, new], [150, 90], 8, gen)
    cache, kk, vv = filled(n_pages, 1, 8, 128, dtype, gen)
    q = draw(gen, (2 * new, 4, 128), dtype)
    b = batch(cu, lens, table)
    clean = cache.zero_weights()
    cache.attend(b, q.to(DEV), weights=clean)
    page, slot = pref.place(table[1], n_pages, 8, 89)  # the last token of the second: its last row alone sees it
    cache.v[page, 0, slot] = float("nan")
    w = cache.zero_weights()
    cache.attend(b, q.to(DEV), weights=w)
    # (the row's result is NaN and is formed again key by key, its maximum and sum with it: each time they are off by
    # the scores' (dh + 4) 2^-24 of reach, exp2's 2^-21 and a step for each of up to 150 keys added in turn)
    _, _, reach, _, _ = ref.attend_seen(f64(q), kk, vv, cu.tolist(), lens.tolist(), table.numpy(), ref.in_run(True, 0),
                                        128 ** -0.5)
    moved = 2 * (2 * (128 + 4) * 2.0 ** -24 * reach.max() + 2.0 ** -21 + 150 * 2.0 ** -24)
    assert bool(((w - clean).abs() <= moved * clean).all())
    cache.k[page, 0, slot, 3] = float("nan")
    w = cache.zero_weights()
    cache.attend(b, q.to(DEV), weights=w)
    mine = [pref.place(table[1], n_pages, 8, j) for j in range(90)]
    assert all(bool(w[p, 0, s].isnan()) for p, s in mine)
    assert int(w.isnan().sum()) == 90
    first = [pref.place(table[0], n_pages, 8, j) for j in range(150)]
    assert all(w[p, 0, s] == clean[p, 0, s] for p, s in first)
    # with a window of 1 the last row sees the NaN key alone
    w = cache.zero_weights()
    cache.attend(b, q.to(DEV), window=1, weights=w)
    assert bool(w[page, 0, slot].isnan()) and int(w.isnan().sum()) == 1
    # scores of -infinity for every key: zeros, and nothing added
    cache.k.fill_(-3e38)
    w = cache.zero_weights()
    out = cache.attend(b, torch.full_like(q, 3e38).to(DEV), weights=w)
    assert not out.any() and not w.any()


def test_weighed_refusals_and_no_gradient():
    gen = torch.Generator().manual_seed(1)
    cu, lens, table, n_pages = pool([2], [20], 8, gen)
    cache, _, _ = filled(n_pages, 2, 8, 64, "bf16", gen)
    b, q = batch(cu, lens, table), draw(gen, (2, 4, 64), "bf16").to(DEV)
    good = cache.zero_weights()
    mask = torch.ones(2, 1, dtype=torch.int64, device=DEV)
    for bad in (good.double(), good[:1], good.transpose(0, 1), good.clone().requires_grad_(), good.cpu()):
        with pytest.raises(ValueError):
            cache.attend(b, q, weights=bad)
        with pytest.raises(ValueError):
            cache.evict(b, bad, 4)
    for call in (lambda x: cache.attend_tree(b, x, mask), lambda x: cache.attend(b, x, weights=good)):
        with pytest.raises(ValueError, match="gradient"):
            call(q.clone().requires_grad_())
        with forward_ad.dual_level(), pytest.raises(ValueError, match="tangent"):
            call(forward_ad.make_dual(q, torch.ones_like(q)))
    for bad in (mask.int(), mask[:1], mask[:, 0], mask.cpu()):
        with pytest.raises(ValueError):
            cache.attend_tree(b, q, bad)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    for path, counts in ((i32(1, 2).long(), i32(1)), (i32(2, 2), i32(1)), (i32(1, 2), i32(2)), (i32(2), i32(1)),
                         (i32(1, 2).cpu(), i32(1))):
        with pytest.raises(ValueError):
            cache.accept(b, path, counts)
    for keep, sinks, recent in ((0, 0, 0), (4, 3, 2), (4, -1, 0)):
        with pytest.raises((R.ReflexError, ValueError)):
            cache.evict(b, good, keep, sinks, recent)
    with pytest.raises(ValueError):
        cache.evict(b, good, 4, kept=i32(1, 2, 5))
    with pytest.raises(ValueError):
        b.tree(i32(5000))
    assert not good.any()


# ---------------------------------------------------------------------------
# acceptance and eviction: what moves
# ---------------------------------------------------------------------------
def raw(cache):
    """Copies of the pages and scales as bytes or floats: [pages, heads, page size, ...]."""
    out = [t.cpu().view(torch.uint8).numpy().reshape(*t.shape[:3], -1).copy() for t in (cache.k, cache.v)]
    if cache.k_scale is not None:
        out += [t.cpu().view(torch.uint8).numpy().reshape(*t.shape, 4).copy() for t in (cache.k_scale, cache.v_scale)]
    return out


def same_pages(cache, want):
    for a, b in zip(raw(cache), want):
        np.testing.assert_array_equal(a, b)


STORES = [("bf16", 1, 256, 16), ("f32", 2, 64, 4), ("fp8", 3, 64, 1), ("int8", 8, 128, 64), ("bf16", 40, 64, 8)]


@pytest.mark.parametrize("store,hk,dh,ps", STORES)
def test_accept(store, hk, dh, ps):
    gen = torch.Generator().manual_seed(hk)
    news, lengths = [5, 1, 0, 40, 30, 7, 3], [100, 1, 33, 90, 30, 4, 50]  # (the sixth has rows before its start)
    cu, lens, table, n_pages = pool(news, lengths, ps, gen, more_pages=1)
    if ps < 64:
        table[3, 70 // ps] = -1  # absent pages among the drafted tokens
        table[4, 10 // ps] = n_pages
    cache, _, _ = filled(n_pages, hk, ps, dh, store, gen)
    most = 33
    path = torch.full((len(news), most), -5, dtype=torch.int32)
    counts = torch.tensor([3, 1, 4, 33, 30, 5, -2], dtype=torch.int32)
    for b, n in enumerate(news):
        c = min(max(int(counts[b]), 0), n, most)
        path[b, :c] = torch.randperm(n, generator=gen)[:c].sort().values
    path[0, 2] = 99  # no row of the sequence: zeros
    want = raw(cache)
    new = ref.accept(want, cu.tolist(), lengths, table.numpy(), path.numpy(), counts.tolist())
    b = batch(cu, lens, table)
    cache.accept(b, path.to(DEV), counts.to(DEV))
    same_pages(cache, want)
    assert b.tensors[1].tolist() == new


def test_accept_none_and_all():
    gen = torch.Generator().manual_seed(2)
    cu, lens, table, n_pages = pool([4, 6], [20, 9], 8, gen)
    cache, _, _ = filled(n_pages, 2, 8, 64, "bf16", gen)
    want = raw(cache)
    b = batch(cu, lens, table)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    cache.accept(b, i32([list(range(6))] * 2), i32([4, 6]))
    assert b.tensors[1].tolist() == [20, 9]
    cache.accept(b, torch.zeros(2, 0, dtype=torch.int32, device=DEV), i32([4, 6]))
    assert b.tensors[1].tolist() == [16, 3]
    same_pages(cache, want)


def long_accept(n, hk, dh, store, gen):
    cu, lens, table, n_pages = pool([n], [n + 50], 16, gen)
    cache, _, _ = filled(n_pages, hk, 16, dh, store, gen)
    path = torch.randperm(n, generator=gen)[:n * 2 // 3].sort().values.to(torch.int32)[None].contiguous()
    want = raw(cache)
    ref.accept(want, cu.tolist(), lens.tolist(), table.numpy(), path.numpy(), [path.shape[1]])
    cache.accept(batch(cu, lens, table), path.to(DEV), torch.tensor([path.shape[1]], dtype=torch.int32, device=DEV))
    same_pages(cache, want)


@pytest.mark.parametrize("n,hk,dh,store", [(700, 8, 128, "bf16"), (1500, 2, 256, "f32"), (3000, 3, 64, "int8")])
def test_accept_many_steps(n, hk, dh, store):
    """More than a workgroup moves in a step: every place is read before it is written."""
    long_accept(n, hk, dh, store, torch.Generator().manual_seed(n))


def check_evict(cache, w, lens, table, keep, sinks, recent, max_length=0):
    want, ww = raw(cache), w.cpu().numpy().copy()
    kept, new = ref.evict(want, ww, lens.tolist(), table.numpy(), keep, sinks, recent)
    b = batch(torch.zeros(len(lens) + 1, dtype=torch.int32), lens, table, max_length)
    got = cache.evict(b, w, keep, sinks=sinks, recent=recent)
    np.testing.assert_array_equal(got.cpu().numpy(), kept)
    assert b.tensors[1].tolist() == new
    same_pages(cache, want)
    np.testing.assert_array_equal(w.cpu().numpy().view(np.int32), ww.view(np.int32))


@pytest.mark.parametrize("store,hk,dh,ps", STORES)
@pytest.mark.parametrize("keep,sinks,recent", [(1, 0, 0), (1, 1, 0), (64, 4, 10), (63, 0, 63), (100, 0, 0), (131, 100, 31)])
def test_evict(store, hk, dh, ps, keep, sinks, recent):
    """Sequences shorter than, as long as and longer than the budget; ties; absent pages; more length than pages."""
    gen = torch.Generator().manual_seed(keep + hk)
    lengths = [200, 0, keep, keep + 1, 1, 333, 65]
    cu, lens, table, n_pages = pool([0] * 7, lengths, ps, gen)
    lens[5] += 1000  # its table ends before
    if ps < 64:
        table[0, 37 // ps], table[0, 150 // ps], table[5, 0] = -1, n_pages + 3, -1
    cache, _, _ = filled(n_pages, hk, ps, dh, store, gen)
    w = torch.exp(2 * torch.randn(n_pages, hk, ps, generator=gen))
    w = torch.where(torch.rand(w.shape, generator=gen) < 0.3, torch.round(w), w)  # many ties, zeros among them
    check_evict(cache, w.to(DEV), lens, table, keep, sinks, recent)


@pytest.mark.parametrize("values", ["equal", "two", "special", "negative", "bits"])
def test_evict_orders(values):
    gen = torch.Generator().manual_seed(7)
    lens, n = [500, 3000], 3500
    cu, lens, table, n_pages = pool([0, 0], lens, 8, gen)
    cache, _, _ = filled(n_pages, 2, 8, 64, "bf16", gen)
    shape = (n_pages, 2, 8)
    if values == "equal":
        w = torch.full(shape, 0.25)
    elif values == "two":
        w = (torch.rand(shape, generator=gen) < 0.05).float()
    elif values == "special":
        pick = torch.tensor([0.0, -0.0, float("nan"), float("inf"), -float("inf"), 1e-45, -1e-45, 3e38])
        w = pick[torch.randint(0, 8, shape, generator=gen)]
    elif values == "negative":
        w = -torch.exp(torch.randn(shape, generator=gen))
    else:
        w = torch.randint(-2 ** 31, 2 ** 31 - 1, shape, generator=gen).to(torch.int32).view(torch.float32)
    for keep, sinks, recent in ((300, 3, 50), (77, 0, 0)):
        check_evict(cache, w.to(DEV).clone(), lens.clone(), table, keep, sinks, recent)


@pytest.mark.parametrize("length", [3000, 4100, 17000])
def test_evict_longer_than_expected(length):
    """max_length only sizes the launch."""
    gen = torch.Generator().manual_seed(length)
    cu, lens, table, n_pages = pool([0, 0], [length, 77], 16, gen)
    cache, _, _ = filled(n_pages, 2, 16, 64, "int8", gen)
    w = torch.round(torch.rand(n_pages, 2, 16, generator=gen) * 999) / 999
    for keep, max_length in ((length - 5, 100), (1000, 4096)):
        check_evict(cache, w.to(DEV).clone(), lens.clone(), table, keep, 4, 50, max_length)


@pytest.mark.parametrize("length,keep", [(40000, 39000), (70001, 1234), (33000, 32900)])
def test_evict_long(length, keep):
    """Longer than the keys held on chip, and more steps of moves than one."""
    gen = torch.Generator().manual_seed(keep)
    cu, lens, table, n_pages = pool([0], [length], 128, gen)
    cache, _, _ = filled(n_pages, 1, 128, 64, "int8", gen)
    w = torch.rand(n_pages, 1, 128, generator=gen)
    w = torch.where(w < 0.4, torch.round(w * 16) / 16, w)
    check_evict(cache, w.to(DEV), lens, table, keep, 4, 500)


# ---------------------------------------------------------------------------
# graphs, streams, and all of it together
# ---------------------------------------------------------------------------
def test_graph_replays_follow_the_device_arrays():
    """Captured once, replayed with other trees, lengths and weights; each replay against the eager calls."""
    gen = torch.Generator().manual_seed(6)
    news, hk, dh, ps = [12, 30], 2, 64, 8
    cu, lens, table, n_pages = pool(news, [120, 200], ps, gen)
    n = sum(news)

    def make():
        c, _, _ = filled(n_pages, hk, ps, dh, "bf16", torch.Generator().manual_seed(9))
        return c

    eager, graphed = make(), make()
    b, bg = batch(cu, lens, table), batch(cu, lens, table)
    q = draw(gen, (n, 4, dh), "bf16").to(DEV)
    parents = random_parents(news, gen).to(DEV)
    path = torch.stack([torch.arange(0, 12, 3), torch.arange(1, 13, 3)]).to(torch.int32).to(DEV)
    counts = torch.tensor([3, 4], dtype=torch.int32, device=DEV)
    w, wg = eager.zero_weights(), graphed.zero_weights()

    def step(c, bb, ww):
        mask, pos = bb.tree(parents, max_rows=30)
        out = c.attend_tree(bb, q, mask)
        weighed = c.attend(bb, q, weights=ww)
        c.accept(bb, path, counts)
        kept = c.evict(bb, ww, 90, sinks=2, recent=10)
        return mask, pos, out, weighed, kept

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(graphed, bg, wg)
    torch.cuda.synchronize()
    saved = [t.clone() for t in (graphed.k, graphed.v, wg)]
    fresh = make()
    graphed.k.copy_(fresh.k)
    graphed.v.copy_(fresh.v)
    wg.zero_()
    bg.tensors[1].copy_(lens.to(DEV))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(graphed, bg, wg)
    for turn in range(4):
        parents.copy_(random_parents(news, gen).to(DEV))
        q.copy_(draw(gen, (n, 4, dh), "bf16"))
        # the tokens come back
        b.tensors[1].copy_((lens - 3 * turn).to(DEV))
        bg.tensors[1].copy_((lens - 3 * turn).to(DEV))
        want = step(eager, b, w)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y)
        assert torch.equal(wg, w) and torch.equal(graphed.k, eager.k) and torch.equal(graphed.v, eager.v)
        assert torch.equal(bg.tensors[1], b.tensors[1])
        if turn == 0:
            for x, y in zip((eager.k, eager.v, w), saved):
                assert x.shape == y.shape


def test_equal_calls_give_equal_bits():
    gen = torch.Generator().manual_seed(11)
    cu, lens, table, n_pages = pool([1, 40, 200], [900, 700, 1500], 16, gen)
    for dtype, store in (("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")):
        cache, _, _ = filled(n_pages, 2, 16, 128, store, gen)
        q = draw(gen, (241, 8, 128), dtype).to(DEV)
        b = batch(cu, lens, table)
        mask = torch.randint(-2 ** 63, 2 ** 63 - 1, (241, 4), generator=gen).to(DEV)
        outs = []
        for _ in range(3):
            w = cache.zero_weights()
            outs.append((cache.attend_tree(b, q, mask), cache.attend(b, q, weights=w), w))
        for x in outs[1:]:
            assert all(torch.equal(s, t) for s, t in zip(x, outs[0]))


def test_two_streams_at_once():
    gen = torch.Generator().manual_seed(12)
    cu, lens, table, n_pages = pool([20, 30], [900, 700], 16, gen)
    cache, _, _ = filled(n_pages, 1, 16, 256, "bf16", gen)
    q = draw(gen, (50, 8, 256), "bf16").to(DEV)
    b = batch(cu, lens, table)
    mask = torch.randint(-2 ** 63, 2 ** 63 - 1, (50, 1), generator=gen).to(DEV)
    w = cache.zero_weights()
    want = (cache.attend_tree(b, q, mask), cache.attend(b, q, weights=w), w)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        with torch.cuda.stream(s):
            ws = cache.zero_weights()
            got.append((cache.attend_tree(b, q, mask), cache.attend(b, q, weights=ws), ws))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(x, y) for x, y in zip(g, want))


def test_no_rows():
    gen = torch.Generator().manual_seed(13)
    cu, lens, table, n_pages = pool([0, 0], [9, 20], 8, gen)
    cache, _, _ = filled(n_pages, 1, 8, 64, "bf16", gen)
    b, w = batch(cu, lens, table), cache.zero_weights()
    q = torch.empty(0, 4, 64, dtype=torch.bfloat16, device=DEV)
    mask, pos = b.tree(torch.empty(0, dtype=torch.int32, device=DEV))
    assert mask.shape == (0, 1) and pos.shape == (0,)
    assert cache.attend_tree(b, q, mask).shape == q.shape and cache.attend(b, q, weights=w).shape == q.shape
    assert not w.any()


def test_drafting_over_a_bounded_memory():
    """As a program runs them: a prompt that weighs its tokens, a cut to a budget, then drafts that are checked and
    accepted, token by token against a cache of lists."""
    gen = torch.Generator().manual_seed(21)
    hk, heads, dh, ps, keep, theta = 2, 8, 64, 8, 60, 10000.0
    lengths, table = [90, 75], torch.randperm(40, generator=gen)[:32].view(2, 16).to(torch.int32)
    cache = PagedCache.zeros(40, ps, hk, dh, torch.float32)
    rope = Rotary(dh, theta=theta)
    w = cache.zero_weights()
    lens = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    # the model: per sequence and head lists of (rotated key, value, weight), in 64 bits
    model = [[[] for _ in range(hk)] for _ in lengths]

    def rotated(x, pos):
        return pref.rotate(f64(x), pref.rotary_angles(np.asarray(pos), (dh // 2,), theta, "shared", dh // 2))

    def attended(s, q, visible):  # visible(j) of one row, in tokens of the lists
        out = np.zeros((heads, dh))
        for h in range(heads):
            g = h // (heads // hk)
            seen = [t for j, t in enumerate(model[s][g]) if visible(j)]
            sc = np.array([t[0] @ q[h] for t in seen]) * dh ** -0.5
            p = np.exp(sc - sc.max())
            p /= p.sum()
            out[h] = sum(pi * t[1] for pi, t in zip(p, seen))
            for pi, t in zip(p, seen):
                t[3] += pi
        return out

    # the prompt
    rows = sum(lengths)
    cu = torch.tensor([0, lengths[0], rows], dtype=torch.int32, device=DEV)
    k, v, q = (torch.randn(rows, h, dh, generator=gen) for h in (hk, hk, heads))
    b = PagedBatch(cu, lens, table.to(DEV))
    pos = torch.cat([torch.arange(n) for n in lengths])
    cache.write(b, k.to(DEV), v.to(DEV), rotary=rope, positions=pos.to(DEV))
    got = f64(cache.attend(b, rope.apply(q.to(DEV), pos.to(DEV)), weights=w))
    rk, rq = rotated(k, pos), rotated(q, pos)
    for s, n in enumerate(lengths):
        for i in range(n):
            for g in range(hk):
                r = int(cu[s]) + i
                model[s][g].append([rk[r, g], f64(v)[r, g], i, 0.0])
    for s, n in enumerate(lengths):
        for i in range(n):
            r = int(cu[s]) + i
            np.testing.assert_allclose(got[r], attended(s, rq[r], lambda j: j <= i), atol=2e-5)
    # the cut: what the weights say, as far as they differ by more than their rounding
    kept = cache.evict(b, w, keep, sinks=4, recent=8).cpu().numpy()
    assert lens.tolist() == [keep, keep]
    for s, n in enumerate(lengths):
        for g in range(hk):
            weights = np.array([t[3] for t in model[s][g]])
            middle = np.array([j for j in kept[s, g] if 4 <= j < n - 8])
            others = np.array([j for j in range(4, n - 8) if j not in set(middle)])
            assert weights[middle].min() >= weights[others].max() - 1e-5
            assert list(kept[s, g][:4]) == [0, 1, 2, 3] and list(kept[s, g][-8:]) == list(range(n - 8, n))
            model[s][g] = [model[s][g][j] for j in kept[s, g]]
    # two rounds of drafts
    absolute = list(lengths)
    for turn in range(2):
        news = [9, 6]
        n = sum(news)
        lens += torch.tensor(news, dtype=torch.int32, device=DEV)
        cu = torch.tensor([0, 9, 15], dtype=torch.int32, device=DEV)
        b = PagedBatch(cu, lens, table.to(DEV))
        parents = random_parents(news, gen)
        mask, at = b.tree(parents.to(DEV), max_rows=9)
        sees, _ = ref.tree(parents.tolist(), [0, 9, 15], lens.tolist(), 1, n)
        depth = [len(x) - 1 for x in sees]
        # positions go on from the uncut sequence
        where = [absolute[0 if r < 9 else 1] + depth[r] for r in range(n)]
        first = [int(x) - m for x, m in zip(lens.tolist(), news)]
        assert at.tolist() == [first[0 if r < 9 else 1] + depth[r] for r in range(n)]
        shift = torch.tensor([absolute[0 if r < 9 else 1] - first[0 if r < 9 else 1] for r in range(n)], device=DEV)
        k, v, q = (torch.randn(n, h, dh, generator=gen) for h in (hk, hk, heads))
        cache.write(b, k.to(DEV), v.to(DEV), rotary=rope, positions=at + shift)
        got = f64(cache.attend_tree(b, rope.apply(q.to(DEV), at + shift), mask))
        rk, rq = rotated(k, where), rotated(q, where)
        for s in range(2):
            for g in range(hk):
                model[s][g] += [[rk[r, g], f64(v)[r, g], -1, 0.0] for r in range(9 * s, 9 * s + news[s])]
        for r in range(n):
            s = 0 if r < 9 else 1
            mine = {first[s] + j for j in sees[r]}
            np.testing.assert_allclose(got[r], attended(s, rq[r], lambda j: j < first[s] or j in mine), atol=2e-5)
        # the deepest row's way down is accepted
        path, counts = torch.zeros(2, 9, dtype=torch.int32), []
        for s in range(2):
            leaf = max(range(9 * s, 9 * s + news[s]), key=lambda r: depth[r])
            way = sorted(sees[leaf])
            path[s, :len(way)] = torch.tensor(way, dtype=torch.int32)
            counts.append(len(way))
            for g in range(hk):
                drafted = model[s][g][first[s]:]
                model[s][g] = model[s][g][:first[s]] + [drafted[j] for j in way]
            absolute[s] += len(way)
        cache.accept(b, path.to(DEV), torch.tensor(counts, dtype=torch.int32, device=DEV))
        assert lens.tolist() == [f + c for f, c in zip(first, counts)]
    # one more token over what is left
    lens += 1
    b = PagedBatch(torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV), lens, table.to(DEV))
    k, v, q = (torch.randn(2, h, dh, generator=gen) for h in (hk, hk, heads))
    at = torch.tensor(absolute, device=DEV)
    cache.write(b, k.to(DEV), v.to(DEV), rotary=rope, positions=at)
    got = f64(cache.attend(b, rope.apply(q.to(DEV), at)))
    rk, rq = rotated(k, absolute), rotated(q, absolute)
    for s in range(2):
        for g in range(hk):
            model[s][g].append([rk[s, g], f64(v)[s, g], -1, 0.0])
        np.testing.assert_allclose(got[s], attended(s, rq[s], lambda j: True), atol=2e-5)


def test_pages_past_4_gib():
    """The same sequences in the last pages of a cache of 4.6 GB a side: the same bits as in a small one."""
    gen = torch.Generator().manual_seed(17)
    news, lengths, ps, dh, far = [1, 12, 40], [300, 200, 333], 64, 256, 70000
    cu, lens, table, n_pages = pool(news, lengths, ps, gen)
    small, _, _ = filled(n_pages, 1, ps, dh, "f32", gen)
    big = PagedCache.zeros(far + n_pages, ps, 1, dh, torch.float32)
    big.k[far:], big.v[far:] = small.k, small.v
    assert big.k[far].data_ptr() - big.k.data_ptr() > 2 ** 32
    q = draw(gen, (sum(news), 4, dh), "f32").to(DEV)
    mask = torch.randint(-2 ** 63, 2 ** 63 - 1, (sum(news), 1), generator=gen).to(DEV)
    path, counts = torch.tensor([[0, 0], [3, 9], [0, 38]], dtype=torch.int32, device=DEV), torch.tensor(
        [1, 2, 2], dtype=torch.int32, device=DEV)
    got = []
    for cache, shift in ((small, 0), (big, far)):
        b = batch(cu, lens, torch.where(table >= 0, table + shift, table))
        w = cache.zero_weights()
        outs = [cache.attend_tree(b, q, mask), cache.attend(b, q, weights=w), w[shift:].clone()]
        cache.accept(b, path, counts)
        outs += [cache.evict(b, w, 150, sinks=3, recent=20), w[shift:], b.tensors[1], cache.k[shift:], cache.v[shift:]]
        assert not shift or not (w[:shift].any() or cache.k[:shift].any() or cache.v[:shift].any())
        got.append(outs)
    for x, y in zip(*got):
        assert torch.equal(x, y)


def test_c_entries_without_what_is_optional():
    """No positions, no list of kept tokens, lengths written to an array of their own."""
    import ctypes
    gen = torch.Generator().manual_seed(19)
    cu, lens, table, n_pages = pool([5, 9], [60, 90], 8, gen)
    lib, ref_ = R.load_library(), ctypes.byref
    one, two = (filled(n_pages, 2, 8, 64, "int8", torch.Generator().manual_seed(3))[0] for _ in range(2))
    b1, b2 = batch(cu, lens, table), batch(cu, lens, table)
    s = torch.cuda.current_stream().cuda_stream
    parents = random_parents([5, 9], gen).to(DEV)
    mask, _ = b1.tree(parents, max_rows=9)
    mask2 = torch.zeros_like(mask)
    assert lib.reflex_paged_tree(ref_(b2.c), parents.data_ptr(), 14, mask2.data_ptr(), 1, None, s) == R.REFLEX_OK
    assert torch.equal(mask, mask2)
    path = torch.tensor([[0, 2, 4], [1, 3, 8]], dtype=torch.int32, device=DEV)
    counts = torch.tensor([2, 3], dtype=torch.int32, device=DEV)
    one.accept(b1, path, counts)
    other = torch.zeros(2, dtype=torch.int32, device=DEV)
    assert lib.reflex_paged_accept(ref_(two.c), ref_(b2.c), path.data_ptr(), 3, counts.data_ptr(), other.data_ptr(),
                                   s) == R.REFLEX_OK
    assert b2.tensors[1].tolist() == [60, 90] and torch.equal(other, b1.tensors[1])
    same_pages(two, raw(one))
    b3 = batch(cu, other.cpu(), table)
    w1 = torch.rand(n_pages, 2, 8, generator=gen).to(DEV)
    w2 = w1.clone()
    one.evict(b1, w1, 33, sinks=1, recent=7)
    ws = torch.empty(2 * 2 * (8 + 33 * 4), dtype=torch.uint8, device=DEV)
    out = torch.zeros(2, dtype=torch.int32, device=DEV)
    assert lib.reflex_paged_evict(ref_(two.c), ref_(b3.c), w2.data_ptr(), 33, 1, 7, None, out.data_ptr(), ws.data_ptr(),
                                  ws.numel(), s) == R.REFLEX_OK
    assert torch.equal(w1, w2) and out.tolist() == b1.tensors[1].tolist() == [33, 33]
    assert b3.tensors[1].tolist() == other.tolist()
    same_pages(two, raw(one))
