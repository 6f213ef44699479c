"""Float64 definitions of drafted trees, their acceptance, weighed attention and eviction, on the CPU, token by token as
the header states them."""
import numpy as np

from .paged_reference import place, rows_of


def tree(parents, cu, lengths, words, n_rows):
    """(sets of rows that each row sees, positions); None for rows of no sequence."""
    sees, positions = [None] * n_rows, [None] * n_rows
    for r, b, pos in rows_of(cu, lengths):
        if r >= n_rows:
            continue
        i, first = r - int(cu[b]), int(lengths[b]) - int(cu[b + 1]) + int(cu[b])
        chain, j = [], i
        while j >= 0 and i < 64 * words:
            chain.append(j)
            p = int(parents[int(cu[b]) + j])
            j = p if 0 <= p < j else -1
        sees[r], positions[r] = set(chain), first + max(0, len(chain) - 1)
    return sees, positions


def words_of(sees, words):
    """int64 words of a set of rows."""
    x = sum(1 << j for j in sees)
    out = [x >> (64 * w) & (2 ** 64 - 1) for w in range(words)]
    return [w - 2 ** 64 if w >= 2 ** 63 else w for w in out]


def attend_seen(q, kpages, vpages, cu, lengths, table, seen_by, scale, weights=None):
    """(out, spread, reach, weights, weights' spread): attention of every row over the tokens that seen_by(r, b, pos,
    length) names.  The spread of a weight is the sum of its parts times (reach + 1), and their number."""
    n, heads, dh = q.shape
    n_pages, hk, ps, _ = kpages.shape
    out, spread, reach = np.full(q.shape, np.nan), np.zeros(q.shape), np.zeros((n, heads, 1))
    w = None if weights is None else weights.astype(np.float64).copy()
    w_reach, w_sum, w_n = (np.zeros((n_pages, hk, ps)) for _ in range(3))
    for r, b, pos in rows_of(cu, lengths):
        if r >= n:
            continue
        out[r] = 0.0
        seen = [p for p in (place(table[b], n_pages, ps, j) for j in seen_by(r, b, pos, int(lengths[b]))) if p is not None]
        if not seen:
            continue
        pg, sl = np.array([s[0] for s in seen]), np.array([s[1] for s in seen])
        for h in range(heads):
            g = h // (heads // hk)
            k, v = kpages[pg, g, sl], vpages[pg, g, sl]
            s = scale * (k @ q[r, h])
            p = np.exp(s - s.max())
            p /= p.sum()
            out[r, h], spread[r, h] = p @ v, p @ np.abs(v)
            reach[r, h] = abs(scale) * np.max(np.abs(k) @ np.abs(q[r, h]))
            if w is not None:
                np.add.at(w, (pg, g, sl), p)
                np.add.at(w_sum, (pg, g, sl), p)
                np.add.at(w_reach, (pg, g, sl), p * reach[r, h])
                np.add.at(w_n, (pg, g, sl), 1)
    return out, spread, reach, w, (w_reach, w_sum, w_n)


def in_tree(bits, cu):
    """seen_by of a tree: bits[r] is row r's words as one whole number."""
    def seen(r, b, pos, length):
        first = length - int(cu[b + 1]) + int(cu[b])
        return list(range(0, max(0, first))) + [first + j for j in range(int(cu[b + 1]) - int(cu[b])) if bits[r] >> j & 1]
    return seen


def in_run(causal, window):
    def seen(r, b, pos, length):
        hi = min(pos + 1, length) if causal else length
        return range(max(0, pos - window + 1) if window else 0, hi)
    return seen


def accept(arrays, cu, lengths, table, path, counts):
    """arrays: [pages, kv heads, page size, ...] each, changed in place; returns the new lengths."""
    n_pages, _, ps = arrays[0].shape[:3]
    new = []
    for b in range(len(lengths)):
        n = int(cu[b + 1]) - int(cu[b])
        first, c = int(lengths[b]) - n, min(max(int(counts[b]), 0), n, path.shape[1])
        old = [a.copy() for a in arrays]
        for i in range(c):
            p = int(path[b, i])
            dst = place(table[b], n_pages, ps, first + i)
            src = place(table[b], n_pages, ps, first + p) if 0 <= p < n else None
            for a, o in zip(arrays, old):
                if dst is not None:
                    a[dst[0], :, dst[1]] = o[src[0], :, src[1]] if src is not None else 0
        new.append(max(0, first + c))
    return new


def evict(arrays, weights, lengths, table, keep, sinks, recent):
    """arrays and weights changed in place; returns (kept, new lengths)."""
    n_pages, hk, ps = weights.shape
    kept, new = np.full((len(lengths), hk, keep), -1, dtype=np.int32), []
    for b in range(len(lengths)):
        length = min(max(int(lengths[b]), 0), table.shape[1] * ps)
        new.append(keep if length > keep else int(lengths[b]))
        if length <= keep:
            kept[b, :, :length] = np.arange(length)
            continue
        at = [place(table[b], n_pages, ps, j) for j in range(length)]
        for g in range(hk):
            def rank(j):
                if at[j] is None:
                    return (1, 0.0, j)
                w = float(weights[at[j][0], g, at[j][1]])
                return (0, np.inf if np.isnan(w) else -w, j)
            middle = sorted(range(sinks, length - recent), key=rank)[:keep - sinks - recent]
            chosen = list(range(sinks)) + sorted(middle) + list(range(length - recent, length))
            kept[b, g] = chosen
            old = [a.copy() for a in (*arrays, weights)]
            for i, j in enumerate(chosen):
                for a, o in zip((*arrays, weights), old):
                    if at[i] is not None:
                        a[at[i][0], g, at[i][1]] = o[at[j][0], g, at[j][1]] if at[j] is not None else 0
            for j in range(keep, length):
                if at[j] is not None:
                    weights[at[j][0], g, at[j][1]] = 0
    return kept, new
