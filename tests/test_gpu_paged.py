"""GPU parity of the backbone operators against their float64 definitions.

Tolerances.  One rounding to a type is off by at most half a step: 2^-8 of the value in bf16, 2^-24 in fp32.
* rotary: the result's rounding, and in fp32 the sine, the cosine and three operations on |a| + |b| (8 * 2^-24).
* pages of 8 bits hold the definition's codes and scales exactly; bf16 and fp32 pages are rotary results.
* attention: a score's fp32 products and sums move it by (dh + 4) 2^-24 of `reach` (the row's largest scale *
  sum |q||k|), so its probability by that share, and so does the maximum; exp2 and the probability's own sums add
  2^-21 and a step for each of the keys' partial sums, at most 2^-24 * 64 as they are taken in trees; in bf16 the
  probability is rounded once (2^-8).  All of it weighs on `spread` = sum p|v|, and the sum of the probabilities
  doubles it.  Then the result's own rounding.
"""
import ctypes

import numpy as np
import pytest
import torch
from torch.autograd import forward_ad

from paper_2607_14695_amd import reflex as R
from paper_2607_14695_amd import workloads as WL
from paper_2607_14695_amd.paged import PagedBatch, PagedCache, Rotary

from . import paged_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
CODE = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "int8": torch.int8}


def draw(gen, shape, dtype):
    return torch.randn(shape, generator=gen).to(DT[dtype])


def f64(t):
    return t.detach().float().cpu().double().numpy() if t.dtype != torch.float64 else t.cpu().numpy()


def pool(news, lengths, ps, gen, spare=3, more_pages=0):
    """(cu, lengths, table, pages): every sequence's pages drawn from one shuffled pool."""
    need = [-(-max(n, 0) // ps) for n in lengths]
    n_pages = sum(need) + spare
    order = torch.randperm(n_pages, generator=gen).to(torch.int32)
    table = torch.full((len(lengths), max(need + [1]) + more_pages), -1, dtype=torch.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    cu = torch.tensor([0] + list(news)).cumsum(0).to(torch.int32)
    return cu, torch.tensor(lengths, dtype=torch.int32), table, n_pages


def batch(cu, lengths, table, max_length=0):
    return PagedBatch(cu.to(DEV), lengths.to(DEV), table.to(DEV), max_length)


def filled(n_pages, hk, ps, dh, store, gen):
    """(cache, values of K, values of V): every slot filled, in 8 bits by the definition's encoder."""
    sides, values = [], []
    for strong in (True, False):
        x = torch.randn(n_pages, hk, ps, dh, generator=gen)
        if strong:
            x *= torch.exp(0.5 * torch.randn(hk, 1, dh, generator=gen))
        if store in ("f32", "bf16"):
            sides.append((x.to(CODE[store]).to(DEV), None))
            values.append(f64(x.to(CODE[store])))
            continue
        scale = torch.exp2(torch.randint(-6, 3, (n_pages, hk, ps), generator=gen).float()) * 1.25
        if store == "int8":
            code = torch.randint(-127, 128, x.shape, generator=gen).to(torch.int8)
            scale /= 64
        else:
            code = (x * 4).to(torch.float8_e4m3fn)
        sides.append((code.to(DEV), scale.to(DEV)))
        values.append(f64(code.float()) * f64(scale)[..., None])
    (k, ks), (v, vs) = sides
    return PagedCache(k, v, ks, vs), values[0], values[1]


# ---------------------------------------------------------------------------
# rotary
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,heads,dh,sections,ladder,far", [
    (1, 1, 64, (32,), "shared", 0), (3, 8, 256, (32, 48, 48), "shared", 10 ** 9), (257, 5, 80, (13, 27), "per_axis", 5000),
    (61, 2, 16, (8,), "shared", 100), (40, 33, 96, (0, 20, 20, 8), "per_axis", 10 ** 6), (5000, 3, 128, (16, 24, 24), "shared", 0)])
def test_rotary(n, heads, dh, sections, ladder, far, dtype):
    gen = torch.Generator().manual_seed(n * dh)
    x = draw(gen, (n, heads, dh), dtype)
    pos = torch.randint(-3, 4096, (len(sections), n), generator=gen) + far
    rot = Rotary(dh, sections, theta=10000.0, ladder=ladder)
    ang = ref.rotary_angles(pos.numpy(), sections, 10000.0, ladder, dh // 2)
    for inverse in (False, True):
        got = f64(rot.apply(x.to(DEV), pos.to(DEV), inverse=inverse))
        want = ref.rotate(f64(x), ang, inverse)
        half = dh // 2
        both = np.abs(f64(x)[..., :half]) + np.abs(f64(x)[..., half:])
        both = np.concatenate([both, both], -1)
        # the angle itself: 64-bit products of positions up to 10^9
        tol = ROUND[dtype] * np.abs(want) + both * (8 * 2.0 ** -24 + 4 * 2.0 ** -53 * (far + 5000))
        assert np.all(np.abs(got - want) <= tol)


def test_rotary_strides_in_place_and_gradient():
    """A slice of packed rows, written into another slice; in place; one set of positions for all axes; and the
    inverse as the gradient of the rotation, against differences."""
    gen = torch.Generator().manual_seed(5)
    n, heads, dh = 37, 4, 64
    packed = torch.randn(n, 3 * heads * dh, generator=gen)
    pos = torch.randint(0, 1000, (n,), generator=gen)
    rot = Rotary(dh, (12, 20))
    want = ref.rotate(f64(packed).reshape(n, 3 * heads, dh)[:, heads:2 * heads],
                      ref.rotary_angles(pos.numpy(), (12, 20), 10000.0, "shared", 32))
    dev = packed.to(DEV)
    x = dev.view(n, 3 * heads, dh)[:, heads:2 * heads]
    out = dev.view(n, 3 * heads, dh)[:, 2 * heads:]
    assert rot.apply(x, pos.to(DEV), out=out) is out
    np.testing.assert_allclose(f64(out), want, atol=4e-6)
    rot.apply(x, pos.to(DEV), out=x)
    np.testing.assert_allclose(f64(x), want, atol=4e-6)
    assert torch.equal(dev[:, :heads * dh].cpu(), packed[:, :heads * dh])
    # L = sum w . rotate(x); dL/dx = inverse rotation of w, and (L(x + e) - L(x - e)) / 2e along a direction
    w, d = torch.randn(n, heads, dh, generator=gen), torch.randn(n, heads, dh, generator=gen)
    x0 = torch.randn(n, heads, dh, generator=gen)
    grad = f64(rot.apply(w.to(DEV), pos.to(DEV), inverse=True))
    ang = ref.rotary_angles(pos.numpy(), (12, 20), 10000.0, "shared", 32)
    loss = lambda t: float((f64(w) * ref.rotate(t, ang)).sum())  # noqa: E731
    e = 1e-4
    diff = (loss(f64(x0) + e * f64(d)) - loss(f64(x0) - e * f64(d))) / (2 * e)
    assert abs(diff - float((grad * f64(d)).sum())) <= 1e-5 * float(np.abs(grad * f64(d)).sum())


# ---------------------------------------------------------------------------
# write and read
# ---------------------------------------------------------------------------
SEQS = {
    "one": ([1], [1]),
    "tokens": ([1] * 9, [1, 5, 16, 17, 40, 3, 8, 9, 33]),
    "ragged": ([0, 7, 33, 0, 0, 1, 130], [3, 7, 50, 0, 1, 20, 131]),
    "many_empty": ([0] * 70 + [3] + [0] * 130 + [2, 1], [4] * 203),
    "cut_off": ([5, 4], [3, 4]),  # more rows than tokens: the first two lie before the sequence's start
}


@pytest.mark.parametrize("seqs", sorted(SEQS))
@pytest.mark.parametrize("dtype,store,hk,dh,ps", [
    ("bf16", "bf16", 1, 256, 16), ("bf16", "fp8", 2, 128, 8), ("bf16", "int8", 3, 64, 1), ("f32", "f32", 2, 64, 128),
    ("f32", "fp8", 1, 64, 32), ("f32", "int8", 5, 256, 4)])
def test_write_then_read(seqs, dtype, store, hk, dh, ps):
    news, lengths = SEQS[seqs]
    gen = torch.Generator().manual_seed(dh + ps)
    cu, lens, table, n_pages = pool(news, lengths, ps, gen)
    n = int(cu[-1])
    k = draw(gen, (n + 2, hk, dh), dtype) * 3
    v = draw(gen, (n + 2, hk, dh), dtype)
    k[0, 0] = 0  # a row of zeros
    sections = (dh // 2 - 10, 10)
    rot = Rotary(dh, sections)
    pos = torch.randint(0, 5000, (2, n + 2), generator=gen)
    cache = PagedCache.zeros(n_pages, ps, hk, dh, CODE[store])
    for t in (cache.k, cache.v):
        t.view(torch.uint8).fill_(7)
    b = batch(cu, lens, table)
    cache.write(b, k.to(DEV), v.to(DEV), rotary=rot, positions=pos.to(DEV))

    rk = ref.rotate(f64(k), ref.rotary_angles(pos.numpy(), sections, 10000.0, "shared", dh // 2))
    got = {m: getattr(cache, m).cpu() for m in ("k", "v")}
    written = np.zeros((n_pages, ps), dtype=bool)
    want_read = {m: np.zeros((n + 2, hk, dh)) for m in ("k", "v")}
    for r, s, p in ref.rows_of(cu, lens):
        at = ref.place(table[s], n_pages, ps, p)
        if at is None:
            continue
        written[at] = True
        for m, x in (("k", rk), ("v", f64(v))):
            for h in range(hk):
                stored = got[m][at[0], h, at[1]].float().double().numpy()
                if store in ("fp8", "int8"):
                    code, scale = ref.encode_row(x[r, h], store)
                    np.testing.assert_array_equal(stored, code)
                    assert getattr(cache, m + "_scale").cpu()[at[0], h, at[1]].item() == scale
                    want_read[m][r, h] = code * scale
                else:
                    both = 2 * np.abs(f64(k)[r, h]).max()
                    tol = ROUND[dtype] * np.abs(x[r, h]) + (8 * 2.0 ** -24 * both if m == "k" else 0)
                    assert np.all(np.abs(stored - x[r, h]) <= tol)
                    want_read[m][r, h] = stored
    # nothing else was touched
    for m in ("k", "v"):
        raw = got[m].view(torch.uint8).numpy().reshape(n_pages, hk, ps, -1)
        assert np.all(raw.transpose(0, 2, 1, 3)[~written] == 7)

    out = [torch.full((n + 2, hk, dh), 77.0, dtype=DT[dtype], device=DEV) for _ in range(2)]
    cache.read(b, n + 2, out=(out[0], out[1]))
    for m, o in zip(("k", "v"), out):
        back = f64(o)
        assert np.all(back[n:] == 77)  # rows of no sequence
        exact = torch.from_numpy(want_read[m]).float().to(DT[dtype])  # code * scale in fp32, rounded once
        assert np.array_equal(back[:n], f64(exact)[:n])


@pytest.mark.parametrize("store", ["fp8", "int8"])
def test_quantiser_borders(store):
    """Values on and next to the borders between codes, powers of two, subnormal rows and every code itself."""
    gen = torch.Generator().manual_seed(11)
    dh, rows = 64, []
    grid = ref.E4M3 if store == "fp8" else np.arange(128.0)
    mids = (grid[1:] + grid[:-1]) / 2
    for scale in (1.0, 2.0 ** -20, 2.0 ** 30, 2.0 ** -126, 0.37, 1.0000001):
        vals = np.concatenate([grid, mids, np.nextafter(np.float32(mids), np.float32(0)), np.nextafter(np.float32(mids), np.float32(1e9))])
        vals = np.float32(vals) * np.float32(scale)
        top = np.float32(grid[-1]) * np.float32(scale)
        for at in range(0, len(vals), dh - 1):
            part = vals[at:at + dh - 1]
            rows.append(np.concatenate([[top], part, np.zeros(dh - 1 - len(part))]).astype(np.float32))
    for e in (-149, -140, -130, -127, -126, 0, 100, 126):
        rows.append((np.random.RandomState(e + 200).uniform(-1, 1, dh) * 2.0 ** e).astype(np.float32))
        rows.append(np.full(dh, np.float32(1.75 * 2.0 ** e if e > -126 else 2.0 ** e)))
    x = torch.from_numpy(np.stack(rows))[:, None].clone()
    x *= torch.where(torch.rand(x.shape, generator=gen) < 0.5, -1.0, 1.0)
    n = x.shape[0]
    cache = PagedCache.zeros(-(-n // 64), 64, 1, dh, CODE[store])
    b = batch(torch.tensor([0, n], dtype=torch.int32), torch.tensor([n], dtype=torch.int32),
              torch.arange(-(-n // 64), dtype=torch.int32)[None])
    cache.write(b, x.to(DEV), x.to(DEV))
    code = cache.v.cpu().float().reshape(-1, dh)[:n].double().numpy()
    scale = cache.v_scale.cpu().reshape(-1)[:n].double().numpy()
    for r in range(n):
        want, s = ref.encode_row(f64(x)[r, 0], store)
        assert scale[r] == s
        np.testing.assert_array_equal(code[r], want)
    assert torch.equal(cache.k.view(torch.uint8), cache.v.view(torch.uint8))


@pytest.mark.parametrize("store", ["fp8", "int8"])
def test_rows_that_are_not_finite_read_as_nan(store):
    dh = 128
    x = torch.randn(4, 2, dh, generator=torch.Generator().manual_seed(3))
    x[0, 1, 5], x[2, 0, 127], x[3, 1, 64] = float("nan"), float("inf"), -float("inf")
    cache = PagedCache.zeros(1, 4, 2, dh, CODE[store])
    b = batch(*[torch.tensor(t, dtype=torch.int32) for t in ([0, 4], [4], [[0]])])
    cache.write(b, x.to(DEV), x.to(DEV), rotary=Rotary(dh))
    k, v = cache.read(b, 4, dtype=torch.float32)
    bad = torch.zeros(4, 2, dtype=torch.bool)
    bad[0, 1] = bad[2, 0] = bad[3, 1] = True
    for t in (k, v):
        assert torch.equal(t.isnan().all(-1).cpu(), bad) and torch.equal(t.isnan().any(-1).cpu(), bad)


def test_default_positions_are_the_tokens_indices():
    gen = torch.Generator().manual_seed(8)
    cu, lens, table, n_pages = pool([3, 5], [10, 900], 16, gen)
    k = draw(gen, (8, 2, 64), "f32").to(DEV)
    rot, b = Rotary(64, (16, 16)), batch(cu, lens, table)
    one, two = (PagedCache.zeros(n_pages, 16, 2, 64, torch.float32) for _ in range(2))
    one.write(b, k, k, rotary=rot)
    two.write(b, k, k, rotary=rot, positions=torch.tensor([7, 8, 9, 895, 896, 897, 898, 899], device=DEV))
    assert torch.equal(one.k, two.k) and torch.equal(one.v, two.v) and bool(one.k.any())


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def check_attention(q, cache, kv, cu, lens, table, causal, window, dtype, max_length=0, out=None, scale=None):
    dh = q.shape[-1]
    got = f64(cache.attend(batch(cu, lens, table, max_length), q.to(DEV), causal=causal, window=window, scale=scale,
                           out=out))
    scale = dh ** -0.5 if scale is None else scale
    want, spread, reach = ref.attend(f64(q), *kv, cu.numpy(), lens.numpy(), table.numpy(), causal, window, scale)
    rows = ~np.isnan(want[:, 0, 0])
    moved = 2 * (2 * (dh + 4) * 2.0 ** -24 * reach + 2.0 ** -21 + 64 * 2.0 ** -24) + (2.0 ** -8 if dtype == "bf16" else 0)
    # what lies under the smallest normal number (2^-126) may be taken as 0: a probability, which then misses that
    # share of its |v|, and the result
    under = 2.0 ** -126 * (1 + max(int(lens.max()), 0) * np.abs(kv[1]).max())
    tol = moved * spread + ROUND[dtype] * np.abs(want) + under
    off = np.abs(got - want)[rows] - tol[rows]
    assert not np.isnan(off).any()
    assert off.max(initial=-1) <= 0, (off.max(), np.argwhere(off > 0)[:5])
    return got


ATTEND = {
    # (new, length) of each sequence, query heads, kv heads, head dim, page size, causal, window
    "one_token": ([(1, 1)], 8, 1, 256, 16, True, 0),
    "tokens_ragged": ([(1, 817), (1, 1), (1, 64), (1, 65), (1, 0), (1, 300)], 8, 1, 256, 16, True, 0),
    "tokens_mha": ([(1, 129), (1, 31)], 3, 3, 64, 32, True, 0),
    "tokens_gqa5": ([(1, 500)] * 3, 10, 2, 128, 64, True, 0),
    "wide_group": ([(1, 70), (2, 40)], 40, 1, 64, 8, True, 0),
    "page_of_one": ([(5, 90)], 2, 1, 128, 1, True, 0),
    "chunk": ([(51, 400)], 8, 1, 256, 64, False, 0),
    "chunk_causal": ([(130, 259), (33, 33)], 4, 2, 128, 16, True, 0),
    "prefill": ([(300, 300)], 2, 1, 64, 128, True, 0),
    "window": ([(100, 300), (1, 300), (40, 40)], 4, 2, 64, 16, True, 37),
    "window_of_one": ([(20, 33)], 2, 2, 128, 8, True, 1),
    "window_full": ([(20, 200)], 4, 1, 128, 32, False, 50),
    "rows_without_keys": ([(9, 4), (3, 0), (0, 7), (2, 5)], 6, 2, 64, 4, True, 0),
    "mixed": ([(1, 650), (70, 210), (0, 9), (1, 3), (200, 330), (17, 1000)], 4, 1, 128, 64, True, 0),
    "large_page": ([(3, 1500)], 2, 1, 256, 1024, True, 0),
    "many_sequences": ([(i % 3, 5 + i % 40) for i in range(150)], 2, 1, 64, 8, True, 0),
    "many_sequences_of_chunks": ([(0, 3)] * 64 + [(40, 60)] * 3 + [(0, 9)] * 70 + [(50, 50)] * 2, 4, 2, 128, 16, True, 0),
}


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "f32"),
                                         ("f32", "fp8"), ("f32", "int8")])
@pytest.mark.parametrize("case", sorted(ATTEND))
def test_attention(case, dtype, store):
    seqs, hq, hk, dh, ps, causal, window = ATTEND[case]
    gen = torch.Generator().manual_seed(sum(map(ord, case)))
    cu, lens, table, n_pages = pool([s[0] for s in seqs], [s[1] for s in seqs], ps, gen)
    cache, k, v = filled(n_pages, hk, ps, dh, store, gen)
    q = draw(gen, (int(cu[-1]), hq, dh), dtype)
    check_attention(q, cache, (k, v), cu, lens, table, causal, window, dtype)


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
@pytest.mark.parametrize("window,max_length", [(600, 0), (129, 300), (2900, 0)])
def test_splits_of_a_window(dtype, store, window, max_length):
    """Single tokens whose windows are split, at any place of the sequence and beyond the expected length."""
    gen = torch.Generator().manual_seed(window)
    cu, lens, table, n_pages = pool([1, 1, 2, 1, 1], [5000, 3, 700, 1281, 0], 16, gen)
    cache, k, v = filled(n_pages, 2, 16, 128, store, gen)
    q = draw(gen, (6, 4, 128), dtype)
    check_attention(q, cache, (k, v), cu, lens, table, True, window, dtype, max_length=max_length)


@pytest.mark.parametrize("store", ["bf16", "int8"])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 150)])
def test_wide_heads_of_ragged_chunks(store, causal, window):
    """256-wide heads with many rows, fewer tiles than the launch has room for, some in splits."""
    gen = torch.Generator().manual_seed(37)
    cu, lens, table, n_pages = pool([0, 70, 0, 200, 1, 129, 0], [5, 210, 9, 900, 300, 129, 40], 16, gen)
    cache, k, v = filled(n_pages, 2, 16, 256, store, gen)
    q = draw(gen, (int(cu[-1]), 4, 256), "bf16")
    check_attention(q, cache, (k, v), cu, lens, table, causal, window, "bf16")


@pytest.mark.parametrize("store", ["f32", "fp8", "int8"])
@pytest.mark.parametrize("dh,window", [(64, 0), (128, 21), (256, 0)])
def test_fp32_tiles_of_many_chunks(store, dh, window):
    """Enough short chunks for the wider fp32 tiles, two of them to a chunk in one sequence."""
    gen = torch.Generator().manual_seed(dh + window)
    seqs = [(9, 9 + 7 * i % 70) for i in range(270)] + [(20, 75), (0, 4), (1, 1)]
    cu, lens, table, n_pages = pool([s[0] for s in seqs], [s[1] for s in seqs], 8, gen)
    cache, k, v = filled(n_pages, 2, 8, dh, store, gen)
    q = draw(gen, (int(cu[-1]), 4, dh), "f32")
    check_attention(q, cache, (k, v), cu, lens, table, True, window, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128, 256])
def test_attention_strided_rows_and_rows_of_no_sequence(dtype, dh):
    """Queries as a slice of packed projections, the result into a slice; rows before the first and behind the last
    sequence stay as they were."""
    gen = torch.Generator().manual_seed(dh)
    hq, hk, ps = 4, 2, 16
    cu, lens, table, n_pages = pool([3, 40], [100, 61], ps, gen)
    cu = cu + 2
    n = int(cu[-1]) + 3
    cache, k, v = filled(n_pages, hk, ps, dh, dtype, gen)
    packed = draw(gen, (n, hq + 2 * hk, dh), dtype)
    q = packed.to(DEV)[:, 1:1 + hq]
    wide = torch.full((n, 2 * hq, dh), 77.0, dtype=DT[dtype], device=DEV)
    out = wide[:, hq:]
    check_attention(q, cache, (k, v), cu, lens, table, True, 0, dtype, out=out)
    assert bool((wide[:, :hq] == 77).all() and (wide[:2] == 77).all() and (wide[n - 3:] == 77).all())


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32"), ("f32", "int8")])
@pytest.mark.parametrize("new", [1, 40])
def test_absent_pages_are_not_seen(dtype, store, new):
    """Table entries outside the pool, and tokens beyond the table."""
    gen = torch.Generator().manual_seed(4)
    ps, dh = 16, 128
    cu, lens, table, n_pages = pool([new, new], [400, 300], ps, gen)
    table[0, 3], table[0, 7:10], table[1, 0], table[1, 5] = -1, n_pages, 2 ** 31 - 1, -2 ** 31
    lens[1] = 40 * ps  # the table holds 25 pages
    cache, k, v = filled(n_pages, 2, ps, dh, store, gen)
    q = draw(gen, (2 * new, 4, dh), dtype)
    check_attention(q, cache, (k, v), cu, lens, table, True, 0, dtype)
    table[:] = -1
    got = cache.attend(batch(cu, lens, table), q.to(DEV))
    assert not bool(got.any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 256])
@pytest.mark.parametrize("new,length,window", [(1, 40, 0), (70, 170, 0), (200, 700, 64), (16, 4000, 1000)])
def test_what_is_not_seen_does_not_matter(dtype, dh, new, length, window):
    """NaN and infinities in every slot that no row sees, and in the last tokens' K/V, which only they see."""
    gen = torch.Generator().manual_seed(9)
    ps, hk = 32, 1
    cu, lens, table, n_pages = pool([new], [length], ps, gen)
    cache, k, v = filled(n_pages, hk, ps, dh, dtype, gen)
    seen = np.zeros((n_pages, ps), dtype=bool)
    first = max(0, length - new - window + 1) if window else 0
    for j in range(first, length):
        seen[ref.place(table[0], n_pages, ps, j)] = True
    hide = torch.from_numpy(~seen)
    q = draw(gen, (new, 2, dh), dtype)
    for junk in (float("nan"), float("inf")):
        for t in (cache.k, cache.v):
            t.permute(0, 2, 1, 3)[hide.to(DEV)] = junk
        check_attention(q, cache, (k, v), cu, lens, table, True, window, dtype)
    if new > 1:
        at = ref.place(table[0], n_pages, ps, length - 1)
        cache.v[at[0], :, at[1], 3] = float("inf")
        cache.v[at[0], :, at[1], 4] = float("nan")
        got = cache.attend(batch(cu, lens, table), q.to(DEV), window=window)
        want = check_attention(q[:-1], cache, (k, v), cu - torch.tensor([0, 1], dtype=torch.int32),
                               lens - 1, table, True, window, dtype)
        assert bool(got[:-1].isfinite().all())
        np.testing.assert_allclose(f64(got[:-1]), want, atol=0.05 if dtype == "bf16" else 1e-4)
        assert bool(torch.isposinf(got[-1, :, 3]).all() and got[-1, :, 4].isnan().all() and got[-1, :, 5:].isfinite().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 256])
@pytest.mark.parametrize("new,length", [(1, 900), (6, 40), (70, 600)])
def test_what_is_seen_and_not_finite_matters(dtype, dh, new, length):
    """An infinity and a NaN among the values of a key that every row sees stay in their dimensions; a key that is not
    finite makes all of the rows that see it NaN."""
    gen = torch.Generator().manual_seed(29)
    cu, lens, table, n_pages = pool([new], [length], 16, gen)
    cache, k, v = filled(n_pages, 1, 16, dh, dtype, gen)
    q = draw(gen, (new, 4, dh), dtype)
    clean = check_attention(q, cache, (k, v), cu, lens, table, True, 0, dtype)
    at = ref.place(table[0], n_pages, 16, 5)
    cache.v[at[0], 0, at[1], 3] = float("-inf")
    cache.v[at[0], 0, at[1], 4] = float("nan")
    got = f64(cache.attend(batch(cu, lens, table), q.to(DEV)))
    assert np.isneginf(got[..., 3]).all() and np.isnan(got[..., 4]).all()
    # the same sums, at most in another order: each side is within check_attention's tolerance of the formula
    np.testing.assert_allclose(np.delete(got, [3, 4], -1), np.delete(clean, [3, 4], -1),
                               atol=0.05 if dtype == "bf16" else 1e-4)
    cache.k[at[0], 0, at[1], 9] = float("nan")
    assert bool(cache.attend(batch(cu, lens, table), q.to(DEV)).isnan().all())


@pytest.mark.parametrize("new", [7, 90])
def test_widest_window(new):
    """The largest window masks nothing, also for rows before a sequence's start."""
    gen = torch.Generator().manual_seed(31)
    cu, lens, table, n_pages = pool([new, 3], [4, 60], 8, gen)
    cache, k, v = filled(n_pages, 1, 8, 64, "f32", gen)
    q = draw(gen, (new + 3, 2, 64), "f32")
    got = check_attention(q, cache, (k, v), cu, lens, table, False, 2 ** 31 - 1, "f32")
    assert np.abs(got[0]).max() > 0


def test_no_pages_and_no_sequences():
    """A table without columns holds no tokens; a batch without sequences touches nothing."""
    cache = PagedCache.zeros(2, 8, 1, 64, torch.float32, DEV)
    cache.k.fill_(3.0)
    x = torch.ones(5, 1, 64, device=DEV)
    none = batch(torch.tensor([0, 5], dtype=torch.int32), torch.tensor([5], dtype=torch.int32),
                 torch.empty(1, 0, dtype=torch.int32))
    out = torch.full((5, 2, 64), 7.0, device=DEV)
    cache.write(none, x, x)
    k, v = cache.read(none, 5, torch.float32)
    cache.attend(none, x.expand(5, 2, 64).contiguous(), out=out)
    assert bool((cache.k == 3.0).all()) and not bool(k.any() or v.any() or out.any())
    empty = batch(torch.zeros(1, dtype=torch.int32), torch.empty(0, dtype=torch.int32),
                  torch.empty(0, 4, dtype=torch.int32))
    out.fill_(7.0)
    cache.write(empty, x, x)
    cache.attend(empty, x.expand(5, 2, 64).contiguous(), out=out)
    assert bool((cache.k == 3.0).all() and (out == 7.0).all())


@pytest.mark.parametrize("dtype,store", [("bf16", "fp8"), ("bf16", "int8"), ("f32", "fp8")])
@pytest.mark.parametrize("dh", [64, 128, 256])
@pytest.mark.parametrize("new,length,window", [(1, 40, 0), (70, 400, 0), (200, 700, 64)])
def test_scales_that_are_not_seen_do_not_matter(dtype, store, dh, new, length, window):
    """NaN scales in every slot that no row sees, and for the last token, which only its own row does."""
    gen = torch.Generator().manual_seed(19)
    cu, lens, table, n_pages = pool([new], [length], 16, gen)
    cache, k, v = filled(n_pages, 1, 16, dh, store, gen)
    hide = torch.ones(n_pages, 16, dtype=torch.bool)
    for j in range(max(0, length - new - window + 1) if window else 0, length):
        hide[ref.place(table[0], n_pages, 16, j)] = False
    q = draw(gen, (new, 2, dh), dtype)
    for t in (cache.k_scale, cache.v_scale):
        t[:, 0][hide.to(DEV)] = float("nan")
    clean = check_attention(q, cache, (k, v), cu, lens, table, True, window, dtype)
    if new > 1:
        at = ref.place(table[0], n_pages, 16, length - 1)
        for t in (cache.k_scale, cache.v_scale):
            t[at[0], 0, at[1]] = float("nan")
            got = f64(cache.attend(batch(cu, lens, table), q.to(DEV), window=window))
            assert np.isnan(got[-1]).all()
            np.testing.assert_array_equal(got[:-1], clean[:-1])


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("bf16", "int8"), ("f32", "f32")])
def test_large_scores_and_queries_that_are_not_finite(dtype, store):
    """Scores far apart (one key takes all) and running maxima that move; a NaN query keeps to its row."""
    gen = torch.Generator().manual_seed(21)
    cu, lens, table, n_pages = pool([50], [900], 16, gen)
    cache, k, v = filled(n_pages, 1, 16, 128, store, gen)
    q = draw(gen, (50, 4, 128), dtype) * torch.exp(torch.linspace(-3, 4, 50))[:, None, None].to(DT[dtype])
    check_attention(q, cache, (k, v), cu, lens, table, True, 0, dtype)
    clean = cache.attend(batch(cu, lens, table), q.to(DEV))
    q[17, 2, 5] = float("nan")
    got = cache.attend(batch(cu, lens, table), q.to(DEV))
    assert bool(got[17, 2].isnan().all())
    got[17, 2] = clean[17, 2]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
@pytest.mark.parametrize("new", [1, 3, 100])
def test_max_length_only_sizes_the_launch(dtype, store, new):
    """A hint that is too short, and results that are the same bit for bit from call to call."""
    gen = torch.Generator().manual_seed(2)
    cu, lens, table, n_pages = pool([new, new], [5000, 70 + new], 64, gen, more_pages=3)
    cache, k, v = filled(n_pages, 1, 64, 128, store, gen)
    q = draw(gen, (2 * new, 8, 128), dtype)
    for hint in (0, 64, 100000):
        check_attention(q, cache, (k, v), cu, lens, table, True, 0, dtype, max_length=hint)
    b = batch(cu, lens, table)
    assert torch.equal(cache.attend(b, q.to(DEV)), cache.attend(b, q.to(DEV)))


@pytest.mark.parametrize("store", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("dh,ps,causal,window", [(64, 8, True, 0), (128, 8, False, 0), (128, 64, True, 700),
                                                 (256, 16, True, 0), (256, 4, False, 900)])
def test_long_loops(store, dh, ps, causal, window):
    """Many tiles in one workgroup (the hint keeps the keys together): every turn of the rings, pages smaller than a
    copy, and more table entries than are held at once."""
    gen = torch.Generator().manual_seed(dh + ps)
    cu, lens, table, n_pages = pool([40, 33], [5200 if ps == 4 else 1500, 771], ps, gen)
    cache, k, v = filled(n_pages, 1, ps, dh, store, gen)
    q = draw(gen, (73, 4, dh), "bf16")
    check_attention(q, cache, (k, v), cu, lens, table, causal, window, "bf16", max_length=64)
    one = torch.tensor([0, 1, 2], dtype=torch.int32)
    check_attention(q[:2], cache, (k, v), one, lens, table, causal, window, "bf16", max_length=64)


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("bf16", "int8"), ("f32", "f32")])
@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.0, 1e-30])
def test_scales(dtype, store, new, scale):
    gen = torch.Generator().manual_seed(31)
    cu, lens, table, n_pages = pool([new, new], [200, 90], 16, gen)
    cache, k, v = filled(n_pages, 1, 16, 64, store, gen)
    q = draw(gen, (2 * new, 2, 64), dtype)
    check_attention(q, cache, (k, v), cu, lens, table, True, 0, dtype, scale=scale)


def test_scale_of_zero_and_sharing_pages():
    """scale 0 gives the mean of the visible values; sequences that share their prefix's pages."""
    gen = torch.Generator().manual_seed(6)
    cu, lens, table, n_pages = pool([2, 1, 3], [40, 40, 37], 8, gen)
    table[1, :4] = table[0, :4]
    table[2, :2] = table[0, :2]
    cache, k, v = filled(n_pages, 1, 8, 64, "f32", gen)
    q = draw(gen, (6, 2, 64), "f32")
    check_attention(q, cache, (k, v), cu, lens, table, True, 0, "f32")
    got = f64(cache.attend(batch(cu, lens, table), q.to(DEV), causal=False, scale=0.0))
    mean = np.mean([v[p][0, s] for p, s in (ref.place(table[0], n_pages, 8, j) for j in range(40))], 0)
    np.testing.assert_allclose(got[0, 0], mean, atol=1e-5)


def test_offsets_past_32_bits():
    """A pool whose pages begin past 2^32 bytes of codes, written, read and attended at its end."""
    dh, ps, hk = 256, 1024, 8
    n_pages = 2 ** 32 // (dh * ps * hk) + 2
    gen = torch.Generator().manual_seed(1)
    cache = PagedCache.zeros(n_pages, ps, hk, dh, torch.int8)
    n = 40
    table = torch.tensor([[n_pages - 1, 0]], dtype=torch.int32)
    cu, lens = torch.tensor([0, n], dtype=torch.int32), torch.tensor([n], dtype=torch.int32)
    b = batch(cu, lens, table)
    k, v = draw(gen, (n, hk, dh), "bf16"), draw(gen, (n, hk, dh), "bf16")
    cache.write(b, k.to(DEV), v.to(DEV))
    assert not bool(cache.k[:-1].any())
    rk, rv = cache.read(b, n)
    for x, y in ((k, rk), (v, rv)):
        assert float((y.cpu().float() - x.float()).abs().max()) <= float(x.float().abs().max()) * (0.5 / 127 + 2.0 ** -8)
    q = draw(gen, (n, hk, dh), "bf16")
    kv = [f64(t.cpu()).transpose(1, 0, 2)[None] for t in cache.read(b, n, dtype=torch.float32)]
    want, spread, _ = ref.attend(f64(q), *kv, cu.numpy(), lens.numpy(), np.zeros((1, 1), dtype=int), True, 0, dh ** -0.5)
    got = f64(cache.attend(b, q.to(DEV)))
    assert np.all(np.abs(got - want) <= 2.0 ** -7 * spread + 2.0 ** -8 * np.abs(want))


# ---------------------------------------------------------------------------
# streams, graphs, the engine
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("new", [1, 24])
def test_captured_graph_follows_the_lengths(new):
    """Write and attend captured once, replayed while the sequences grow in device memory; two graphs captured one
    after the other and replayed in turn; every replay against the eager result."""
    gen = torch.Generator().manual_seed(13)
    ps, dh, hk, hq = 16, 128, 2, 8
    cu, lens, table, n_pages = pool([new, new], [2000, 1500], ps, gen)
    b = batch(cu, lens.clone(), table, 2000)
    cache = PagedCache.zeros(n_pages, ps, hk, dh, torch.float8_e4m3fn)
    rot = Rotary(dh)
    k, v, q = (draw(gen, (2 * new, h, dh), "bf16").to(DEV) for h in (hk, hk, hq))
    dlens = b.tensors[1]

    def step():
        cache.write(b, k, v, rotary=rot)
        return cache.attend(b, q)

    dlens.copy_(torch.tensor([new, new], dtype=torch.int32))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step())
        graphs.append(g)
    for i, n in enumerate((new, 100, 777, 1500)):
        dlens.fill_(n)
        k.copy_(draw(gen, k.shape, "bf16"))
        q.copy_(draw(gen, q.shape, "bf16"))
        graphs[i % 2].replay()
        got = outs[i % 2].clone()
        torch.cuda.synchronize()
        assert torch.equal(got, step())


def test_streams():
    """Two calls at once on two streams, each with its own workspace, against the calls one by one."""
    gen = torch.Generator().manual_seed(17)
    cu, lens, table, n_pages = pool([1] * 4, [3000] * 4, 64, gen)
    cache, _, _ = filled(n_pages, 1, 64, 256, "bf16", gen)
    b = batch(cu, lens, table)
    qs = [draw(gen, (4, 8, 256), "bf16").to(DEV) for _ in range(2)]
    want = [cache.attend(b, q) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(cache.attend(b, qs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


def test_prefix_of_the_engine_through_the_paged_cache():
    """As a backbone uses them: each layer's prefix rotated into its pages in two chunks and attended, then read back,
    turned back and given to the engine, whose own cache rows and actions are those of the original prefix."""
    cfg = WL.CONFIGS["tiny_fp32"].replace(frame_dim=0, static_len=64)
    L, S, dh = cfg.n_layers, cfg.static_len, cfg.head_dim
    w = WL.make_weights(cfg)
    sk, sv = WL.make_static_kv(cfg)  # [1, L, S, dh], before RoPE
    k, v = (torch.from_numpy(np.ascontiguousarray(t[0])).to(DEV) for t in (sk, sv))
    gen = torch.Generator().manual_seed(3)
    rot = Rotary(dh, theta=cfg.rope_theta)
    _, _, table, n_pages = pool([S] * L, [S] * L, 16, gen)
    cache = PagedCache.zeros(n_pages, 16, 1, dh, torch.float32)
    q = torch.randn(L, S, cfg.n_q_heads, dh, generator=gen).to(DEV)
    outs, done = [], 0
    for n in (48, 16):
        rows = slice(done, done + n)
        done += n
        b = batch(torch.arange(0, L * n + 1, n, dtype=torch.int32), torch.full((L,), done, dtype=torch.int32), table)
        cache.write(b, k[:, rows].reshape(L * n, 1, dh), v[:, rows].reshape(L * n, 1, dh), rotary=rot)
        pos = torch.arange(rows.start, rows.stop, device=DEV).repeat(L)
        qr = rot.apply(q[:, rows].reshape(L * n, cfg.n_q_heads, dh), pos)
        outs.append(cache.attend(b, qr).view(L, n, cfg.n_q_heads, dh))
    out = f64(torch.cat(outs, 1))
    ang = ref.rotary_angles(np.arange(S), (dh // 2,), cfg.rope_theta, "shared", dh // 2)
    for layer in range(L):  # plain attention over the rotated prefix; N(0, 1) values: 1e-5 is 80 steps of fp32
        kr, qr = ref.rotate(f64(k[layer])[:, None], ang)[:, 0], ref.rotate(f64(q[layer]), ang)
        s = np.einsum("ihd,jd->ihj", qr, kr) * dh ** -0.5
        s[np.broadcast_to(np.arange(S)[None, None] > np.arange(S)[:, None, None], s.shape)] = -np.inf
        p = np.exp(s - s.max(-1, keepdims=True))
        want = np.einsum("ihj,jd->ihd", p / p.sum(-1, keepdims=True), f64(v[layer]))
        np.testing.assert_allclose(out[layer], want, atol=1e-5)

    whole = batch(torch.arange(0, L * S + 1, S, dtype=torch.int32), torch.full((L,), S, dtype=torch.int32), table)
    rk, rv = cache.read(whole, L * S, dtype=torch.float32)
    back = rot.apply(rk, torch.arange(S, device=DEV).repeat(L), inverse=True)
    engines = [R.ReflexEngine(cfg, w, a, b) for a, b in (
        (sk, sv), (back.view(1, L, S, dh), rv.view(1, L, S, dh)))]
    rows = [e.cache_views()[0][0, :, :S].clone() for e in engines]
    # two more rotations of values up to 5: 16 roundings of fp32
    np.testing.assert_allclose(f64(rows[0]), f64(rk.view(L, S, dh)), atol=5e-6)
    np.testing.assert_allclose(f64(rows[1]), f64(rows[0]), atol=5e-6)
    state, noise = WL.make_state(cfg, 0), WL.make_noise(cfg, 0)
    acts = [e.denoise(state, noise).clone() for e in engines]
    np.testing.assert_allclose(f64(acts[1]), f64(acts[0]), atol=1e-4)  # the bar of the engine's own fp32 parity
    for e in engines:
        e.close()


def test_python_refusals_on_the_gpu():
    gen = torch.Generator().manual_seed(1)
    cu, lens, table, n_pages = pool([2], [20], 16, gen)
    cache, b = PagedCache.zeros(n_pages, 16, 2, 64), batch(cu, lens, table)
    ok = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device=DEV)
    for bad in (ok.cpu(), ok[:, :1], ok.half(), ok.clone().requires_grad_(), ok.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError):
            cache.write(b, bad, bad)
    with pytest.raises(R.ReflexError):
        cache.write(b, ok.float(), ok.float())  # bf16 pages
    with pytest.raises(R.ReflexError):
        cache.attend(b, torch.zeros(2, 3, 64, dtype=torch.bfloat16, device=DEV))  # 3 heads on 2
    odd = torch.zeros(2 * 2 * 64 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(2, 2, 64)
    with pytest.raises(R.ReflexError):
        cache.attend(b, odd)  # not on a 16-byte boundary
    with pytest.raises(ValueError):
        cache.write(b, ok, ok, positions=torch.zeros(2, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        cache.write(b, ok, ok, rotary=Rotary(64), positions=torch.zeros(3, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        cache.write(b, ok, ok, rotary=Rotary(64), positions=torch.zeros(2, dtype=torch.int32, device=DEV))


# ---------------------------------------------------------------------------
# codes and scales that are not numbers
# ---------------------------------------------------------------------------
def attend_ref(q, k, v, cu, lens, table, window, dtype, scale=None, prob=None):
    """(result, tolerance) of causal attention: the bound of check_attention; `prob`: what a probability's own
    rounding may be off by, where it is less than a step of dtype."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    want, spread, reach = ref.attend(f64(q), k, v, cu.numpy(), lens.numpy(), table.numpy(), True, window, scale)
    prob = (2.0 ** -8 if dtype == "bf16" else 0) if prob is None else prob
    moved = 2 * (2 * (q.shape[-1] + 4) * 2.0 ** -24 * reach + 2.0 ** -21 + 64 * 2.0 ** -24) + prob
    under = 2.0 ** -126 * (1 + max(int(lens.max()), 0) * np.abs(v).max())
    return want, moved * spread + ROUND[dtype] * np.abs(want) + under


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128, 256])
@pytest.mark.parametrize("new,length,window", [(1, 40, 0), (6, 40, 0), (70, 170, 0), (200, 700, 64), (16, 4000, 1000)])
def test_nan_codes_keep_to_the_rows_that_see_them(dtype, dh, new, length, window):
    """e4m3 codes that are NaN: in every slot that no row sees, and in V or K of a token that the last rows see, or
    the first ones."""
    gen = torch.Generator().manual_seed(dh + new)
    cu, lens, table, n_pages = pool([new], [length], 16, gen)
    cache, k, v = filled(n_pages, 1, 16, dh, "fp8", gen)
    first = max(0, length - new - window + 1) if window else 0
    hide = torch.ones(n_pages, 16, dtype=torch.bool)
    for j in range(first, length):
        hide[ref.place(table[0], n_pages, 16, j)] = False
    for t in (cache.k, cache.v):
        t.view(torch.uint8)[:, 0][hide.to(DEV)] = 0x7F
    q = draw(gen, (new, 2, dh), dtype)
    b, pos = batch(cu, lens, table), np.arange(length - new, length)
    want, tol = attend_ref(q, k, v, cu, lens, table, window, dtype)
    assert np.all(np.abs(f64(cache.attend(b, q.to(DEV), window=window)) - want) <= tol)
    for key in (max(length - 3, length - new), first):
        see = (pos >= key) & ((pos < key + window) if window else True)
        page, slot = ref.place(table[0], n_pages, 16, key)
        kept = [t.view(torch.uint8)[page, 0, slot].clone() for t in (cache.k, cache.v)]
        codes = cache.v.view(torch.uint8)[page, 0, slot]
        codes[3], codes[dh - 2] = 0x7F, 0xFF
        got = f64(cache.attend(b, q.to(DEV), window=window))
        bad = np.zeros(got.shape, dtype=bool)
        bad[see, :, 3] = bad[see, :, dh - 2] = True
        np.testing.assert_array_equal(np.isnan(got), bad)
        assert np.all((np.abs(got - want) <= tol)[~bad])
        cache.k.view(torch.uint8)[page, 0, slot, 7] = 0xFF
        got = f64(cache.attend(b, q.to(DEV), window=window))
        assert np.isnan(got[see]).all() and np.all((np.abs(got - want) <= tol)[~see])
        for t, old in zip((cache.k, cache.v), kept):
            t.view(torch.uint8)[page, 0, slot] = old


@pytest.mark.parametrize("dtype,store", [("bf16", "fp8"), ("bf16", "int8"), ("f32", "fp8"), ("f32", "int8")])
@pytest.mark.parametrize("dh", [64, 128, 256])
@pytest.mark.parametrize("new,length", [(1, 130), (6, 43), (70, 200), (70, 1100)])
def test_nan_scale_of_a_value_that_hardly_counts(dtype, store, dh, new, length):
    """A value whose scale is NaN makes the rows that see it NaN, also where its probability is 0 in fp32, in a tile
    that all rows see whole and in one that is masked or cut off."""
    gen = torch.Generator().manual_seed(dh + length)
    cu, lens, table, n_pages = pool([new], [length], 16, gen)
    cache, _, _ = filled(n_pages, 1, 16, dh, store, gen)
    q = torch.full((new, 2, dh), 4.0, dtype=DT[dtype], device=DEV)
    b, pos = batch(cu, lens, table), np.arange(length - new, length)
    for key in (5, length - 1, max(length - 4, length - new)):
        page, slot = ref.place(table[0], n_pages, 16, key)
        # q . k = -4 dh 127 * 8 or less, scaled by dh ** -0.5: under -30,000, where the other keys' are above -1,000
        cache.k.view(torch.uint8)[page, 0, slot] = 0x81 if store == "int8" else 0xFE
        cache.k_scale[page, 0, slot] = 8.0
        clean = f64(cache.attend(b, q))
        assert np.isfinite(clean).all()
        old = cache.v_scale[page, 0, slot].clone()
        cache.v_scale[page, 0, slot] = float("nan")
        got = f64(cache.attend(b, q))
        cache.v_scale[page, 0, slot] = old
        assert np.isnan(got[pos >= key]).all()
        np.testing.assert_array_equal(got[pos < key], clean[pos < key])


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "int8")])
@pytest.mark.parametrize("new,length", [(1, 3), (3, 12), (70, 90)])
@pytest.mark.parametrize("scale", [0.0, 4e-39, -4e-39, 1e-42])
def test_scales_under_the_normal_numbers(dtype, store, new, length, scale):
    """Scales next to zero against products of up to 2^127: their share of the scores, and no more."""
    gen = torch.Generator().manual_seed(41)
    cu, lens, table, n_pages = pool([new], [length], 16, gen)
    cache, k, v = filled(n_pages, 1, 16, 64, store, gen)
    up = 2.0 ** 60
    if store == "int8":
        cache.k_scale *= up
    else:
        cache.k.mul_(up)
    q = (draw(gen, (new, 2, 64), "bf16").float() * 2.0 ** 58).to(DT[dtype])
    got = f64(cache.attend(batch(cu, lens, table), q.to(DEV), scale=scale))
    # (the scale as the call takes it, rounded to fp32)
    want, tol = attend_ref(q, k * up, v, cu, lens, table, 0, dtype, scale=float(np.float32(scale)))
    assert np.all(np.abs(got - want) <= tol)


def test_gradients_that_would_be_dropped_are_refused():
    """Pages that need a gradient, whatever mode the cache is made in, and tangents of forward-mode differentiation on
    pages or rows."""
    gen = torch.Generator().manual_seed(1)
    cu, lens, table, n_pages = pool([2], [20], 16, gen)
    b = batch(cu, lens, table)
    x = torch.zeros(2, 2, 64, device=DEV)
    for name, dtype in (("k", torch.float32), ("v", torch.float32), ("k_scale", torch.int8), ("v_scale", torch.int8)):
        cache = PagedCache.zeros(n_pages, 16, 2, 64, dtype)
        held = {m: getattr(cache, m) for m in ("k", "v", "k_scale", "v_scale")}
        with torch.no_grad(), pytest.raises(ValueError, match=f"{name} needs a gradient"):
            PagedCache(**{**held, name: held[name].clone().requires_grad_()})
        PagedCache(**held)
        with forward_ad.dual_level(), pytest.raises(ValueError, match=f"{name} carries a tangent"):
            PagedCache(**{**held, name: forward_ad.make_dual(held[name], torch.ones_like(held[name]))})
    cache = PagedCache.zeros(n_pages, 16, 2, 64, torch.float32)
    with forward_ad.dual_level():
        d = forward_ad.make_dual(x, torch.ones_like(x))
        for call in (lambda: cache.write(b, d, x), lambda: cache.write(b, x, d), lambda: cache.attend(b, d),
                     lambda: cache.attend(b, x, out=d), lambda: cache.read(b, 2, out=(x, d))):
            with pytest.raises(ValueError, match="tangent"):
                call()
        cache.attend(b, x)


def test_windows_that_do_not_fit_are_refused():
    gen = torch.Generator().manual_seed(1)
    cu, lens, table, n_pages = pool([2], [20], 16, gen)
    cache, b = PagedCache.zeros(n_pages, 16, 2, 64, torch.float32), batch(cu, lens, table)
    x = torch.zeros(2, 2, 64, device=DEV)
    for window in (2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 31 - 1):
        with pytest.raises(ValueError, match="window"):
            cache.attend(b, x, window=window)


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "int8")])
def test_rows_for_the_same_slot(dtype, store):
    """Sequences that share their prefix's pages and write them in one call: equal rows leave what one of them would;
    rows that differ leave every other slot as it should be."""
    gen = torch.Generator().manual_seed(43)
    n, ps, dh = 40, 8, 128
    cu, lens, table, n_pages = pool([n, n, n], [n, n, n], ps, gen)
    shared = 16
    table[1:, :shared // ps] = table[0, :shared // ps]
    k, v = (draw(gen, (3, n, 2, dh), dtype) for _ in range(2))
    k[1:, :shared], v[1:, :shared] = k[0, :shared], v[0, :shared]
    rot = Rotary(dh)
    one, two = (PagedCache.zeros(n_pages, ps, 2, dh, CODE[store]) for _ in range(2))
    b = batch(cu, lens, table)
    one.write(b, k.view(-1, 2, dh).to(DEV), v.view(-1, 2, dh).to(DEV), rotary=rot)
    for s in range(3):  # the same one sequence at a time
        two.write(batch(cu[:2], lens[:1], table[s:s + 1]), k[s].to(DEV), v[s].to(DEV), rotary=rot)
    names = ("k", "v", "k_scale", "v_scale") if one.k_scale is not None else ("k", "v")
    for m in names:
        assert torch.equal(getattr(one, m).view(torch.uint8), getattr(two, m).view(torch.uint8))
    k[1, :shared] += 1
    one.write(b, k.view(-1, 2, dh).to(DEV), v.view(-1, 2, dh).to(DEV), rotary=rot)
    kept = torch.ones(n_pages, dtype=torch.bool)
    kept[table[0, :shared // ps].long()] = False
    for m in names:
        assert torch.equal(getattr(one, m).cpu()[kept].view(torch.uint8), getattr(two, m).cpu()[kept].view(torch.uint8))


@pytest.mark.parametrize("store", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("dh", [64, 128, 256])
def test_probabilities_of_few_rows_keep_sixteen_bits(store, dh):
    """With few rows the probabilities enter the second product as two bf16 halves, 2^-16 of each.  Here the value of
    the largest one cancels the others', so that the result's own rounding hides nothing."""
    gen = torch.Generator().manual_seed(dh)
    seqs = [2, 5, 33, 64, 200]
    cu, lens, table, n_pages = pool([1] * len(seqs), seqs, 16, gen)
    cache, k, v = filled(n_pages, 1, 16, dh, store, gen)
    q = draw(gen, (len(seqs), 1, dh), "bf16") * 0.25
    for b, n in enumerate(seqs):
        pg, sl = np.array([ref.place(table[b], n_pages, 16, j) for j in range(n)]).T
        p = np.exp(dh ** -0.5 * (k[pg, 0, sl] @ f64(q)[b, 0]))
        top = int(np.argmax(p))
        rest = -(np.delete(p, top) @ np.delete(v[pg, 0, sl], top, 0)) / p[top]
        at = pg[top], 0, sl[top]
        if store == "bf16":
            cache.v[at] = torch.from_numpy(rest).to(torch.bfloat16).to(DEV)
            v[at] = f64(cache.v[at])
        else:
            code, scale = ref.encode_row(np.float64(np.float32(rest)), store)
            cache.v[at] = torch.from_numpy(code).float().to(CODE[store]).to(DEV)
            cache.v_scale[at] = float(scale)
            v[at] = code * scale
    got = f64(cache.attend(batch(cu, lens, table), q.to(DEV)))
    want, tol = attend_ref(q, k, v, cu, lens, table, 0, "bf16", prob=2.0 ** -16)
    assert np.all(np.abs(got - want) <= tol)


@pytest.mark.parametrize("dtype,store,dh", [("bf16", "bf16", 128), ("bf16", "int8", 256), ("f32", "f32", 64)])
@pytest.mark.parametrize("new", [1, 60])
def test_workspace_holds_every_window(dtype, store, dh, new):
    """The workspace query knows no window: a call with any uses no more than it reports, and asks for no less."""
    gen = torch.Generator().manual_seed(23)
    cu, lens, table, n_pages = pool([new, new], [3000, 700], 16, gen)
    cache, k, v = filled(n_pages, 1, 16, dh, store, gen)
    q = draw(gen, (2 * new, 2, dh), dtype).to(DEV)
    b = batch(cu, lens, table)
    lib, need = R.load_library(), ctypes.c_size_t(0)
    code = R.DTYPE_BF16 if dtype == "bf16" else R.DTYPE_F32
    assert lib.reflex_paged_attention_workspace(cache._ref, b._ref, 2 * new, 2, code, ctypes.byref(need)) == R.REFLEX_OK
    assert need.value > 0
    ws = torch.empty(need.value + 4096, dtype=torch.uint8, device=DEV)
    assert ws.data_ptr() % 256 == 0
    qr = R.RowsC(q.data_ptr(), 2 * dh, dh)
    for window in (0, 1, 63, 128, 129, 500, 1025, 2999, 2 ** 31 - 1):
        ws.fill_(0xA5)
        out = torch.empty_like(q)
        yr = R.RowsC(out.data_ptr(), 2 * dh, dh)
        call = lambda nb: lib.reflex_paged_attention(  # noqa: E731
            cache._ref, b._ref, ctypes.byref(qr), ctypes.byref(yr), 2 * new, 2, code, dh ** -0.5, 1, window,
            ws.data_ptr(), nb, torch.cuda.current_stream().cuda_stream)
        assert call(need.value - 1) == R.REFLEX_EINVAL
        assert call(need.value) == R.REFLEX_OK
        torch.cuda.synchronize()
        assert bool((ws[need.value:] == 0xA5).all())
        assert torch.equal(out, cache.attend(b, q, window=window))


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("f32", "int8")])
@pytest.mark.parametrize("cu,n", [([0, 5, 12], 8), ([3, 100, 300], 160), ([0, 1, 2], 1), ([9, 9, 12], 7)])
def test_rows_past_the_call_are_cut_off(dtype, store, cu, n):
    """Row offsets that run past the call's rows: the rows that it has keep their tokens, in all three calls."""
    gen = torch.Generator().manual_seed(n)
    hk, ps, dh = 2, 16, 64
    _, lens, table, n_pages = pool([0, 0], [130, 260], ps, gen)
    cu = torch.tensor(cu, dtype=torch.int32)
    cache, k, v = filled(n_pages, hk, ps, dh, store, gen)
    q = draw(gen, (n, 4, dh), dtype)
    out = torch.full((n, 4, dh), 77.0, dtype=DT[dtype], device=DEV)
    check_attention(q, cache, (k, v), cu, lens, table, True, 0, dtype, out=out)
    own = torch.arange(n) >= int(cu[0])
    assert bool((out.cpu()[~own] == 77).all())
    b = batch(cu, lens, table)
    rk, rv = (torch.full((n, hk, dh), 77.0, dtype=DT[dtype], device=DEV) for _ in range(2))
    cache.read(b, n, out=(rk, rv))
    want = np.full((n, hk, dh), 77.0)
    new = torch.randn(n, hk, dh, generator=gen).to(DT[dtype]).to(DEV)
    old = cache.k.view(torch.uint8).cpu().clone()
    cache.write(b, new, new)
    changed = (cache.k.view(torch.uint8).cpu() != old).any(-1).any(1).numpy()
    rows = np.zeros((n_pages, ps), dtype=bool)
    for r, s, p in ref.rows_of(cu, lens):
        if r < n:
            at = ref.place(table[s], n_pages, ps, p)
            want[r] = k[at[0], :, at[1]]
            rows[at] = True
    assert np.array_equal(f64(rk), f64(torch.from_numpy(want).float().to(DT[dtype])))
    np.testing.assert_array_equal(changed, rows)


@pytest.mark.parametrize("through", ["apply", "write"])
def test_small_sines_of_fp32(through):
    """Next to whole and half turns the sine is small and keeps its bits.  With x = 0 in the first half a result is one
    product: the sine's or the cosine's rounding and its own, 2^-23 of it; the angle's 64 bits leave 2^-52 of it, the
    series 2^-49 of the sine's quarter turn."""
    pos = torch.tensor([0, 1, 3, 22, 355, 710, 103993, 104348, 833719, 10 ** 6], dtype=torch.int64)
    n, dh = len(pos), 64
    x = torch.zeros(n, 1, dh)
    x[..., dh // 2:] = 1.0 + torch.rand(n, 1, dh // 2, generator=torch.Generator().manual_seed(3))
    rot = Rotary(dh)
    ang = ref.rotary_angles(pos.numpy(), (dh // 2,), 10000.0, "shared", dh // 2)
    want = ref.rotate(f64(x), ang)
    if through == "apply":
        got = f64(rot.apply(x.to(DEV), pos.to(DEV)))
    else:
        cache = PagedCache.zeros(1, 16, 1, dh, torch.float32)
        b = batch(*[torch.tensor(t, dtype=torch.int32) for t in ([0, n], [n], [[0]])])
        cache.write(b, x.to(DEV), x.to(DEV), rotary=rot, positions=pos.to(DEV))
        got = f64(cache.read(b, n, torch.float32)[0])
    # (the angle in turns has steps of 2^-53 of the angle, which is up to 10^6)
    tol = 2.0 ** -23 * np.abs(want) + 2 * (2.0 ** -49 + 4 * 2.0 ** -53 * np.concatenate([ang, ang], 1)[:, None])
    assert np.all(np.abs(got - want) <= tol)
