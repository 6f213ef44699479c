"""Float64 definitions of the backbone operators (rotary positions, the paged cache, its attention), on the CPU,
row by row as the header states them."""
import numpy as np
import torch

# values of the e4m3 codes 0 .. 126 (0 .. 448), increasing
E4M3 = torch.arange(0x7F, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()


def rotary_angles(positions, sections, theta, ladder, half):
    """[n, half] angles; positions [n] or [axes, n]."""
    pos = np.broadcast_to(np.asarray(positions, dtype=np.float64), (len(sections), np.shape(positions)[-1]))
    cols, i = [], 0
    for a, m in enumerate(sections):
        for j in range(m):
            e = i / half if ladder == "shared" else j / m
            cols.append(pos[a] * theta ** -e)
            i += 1
    return np.stack(cols, 1)


def rotate(x, angles, inverse=False):
    """x [n, heads, dh] float64."""
    half = x.shape[-1] // 2
    c, s = np.cos(angles)[:, None], np.sin(angles)[:, None] * (-1 if inverse else 1)
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def encode_row(x, store):
    """(values of the codes, scale) of one row."""
    if not np.all(np.isfinite(x)):
        return np.zeros_like(x), np.float64("nan")
    most = np.float32(np.max(np.abs(x)))
    if store == "int8":
        scale = max(most * (np.float32(1) / np.float32(127)), np.float32(2.0 ** -126))
        return np.clip(np.rint(x / np.float64(scale)), -127, 127), np.float64(scale)
    k = -126
    while float(most) > 448.0 * 2.0 ** k:
        k += 1
    y = np.abs(x) / 2.0 ** k
    hi = np.minimum(np.searchsorted(E4M3, y), len(E4M3) - 1)
    lo = np.maximum(hi - 1, 0)
    below, above = y - E4M3[lo], E4M3[hi] - y
    at = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return np.sign(x) * E4M3[at], 2.0 ** k


def place(table_row, n_pages, page_size, pos):
    """(page, slot) of a token, or None where it is absent."""
    if pos < 0 or pos // page_size >= len(table_row):
        return None
    page = int(table_row[pos // page_size])
    return (page, pos % page_size) if 0 <= page < n_pages else None


def rows_of(cu, lengths):
    """(row, sequence, token) of every row of the batch."""
    for b in range(len(lengths)):
        for r in range(int(cu[b]), int(cu[b + 1])):
            yield r, b, int(lengths[b]) - int(cu[b + 1]) + r


def attend(q, kpages, vpages, cu, lengths, table, causal, window, scale):
    """(out, spread, reach): out [n, heads, dh]; spread = sum p |v| / sum p; reach = the largest scale * sum |q||k|
    of a row, which bounds how far rounding moves its scores.  Rows of no sequence are NaN.  kpages, vpages:
    [pages, kv heads, page size, dh] float64."""
    n, heads, dh = q.shape
    n_pages, hk, ps, _ = kpages.shape
    out, spread, reach = np.full(q.shape, np.nan), np.zeros(q.shape), np.zeros((n, heads, 1))
    for r, b, pos in rows_of(cu, lengths):
        if r >= n:
            continue
        hi = min(pos + 1, int(lengths[b])) if causal else int(lengths[b])
        lo = max(0, pos - window + 1) if window else 0
        seen = [p for p in (place(table[b], n_pages, ps, j) for j in range(lo, hi)) if p is not None]
        out[r] = 0.0
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
    return out, spread, reach
