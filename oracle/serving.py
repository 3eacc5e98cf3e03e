"""A decode step over a paged key/value cache, and products with 4-bit weights (oracle; test only).

Not part of the paper; written out from the definitions that include/ringattn.h states, one
request, token, head and element at a time where that matters, in float64:

  plan       the pages, cache slots and positions of a step's new tokens, handed out as an
             allocator would, token after token.
  rope       the rotary embedding of oracle.llama at given positions.
  e4m3       what an 8-bit cache row stands for: nearest e4m3 value (ties to even) under the
             smallest power-of-two scale that brings every finite element to at most 448.
  attention  softmax attention of each new token over its request's pages.
  mx4        4-bit weights: the values a packed block stands for, and the packing.
"""
import math

import numpy as np

FLAG_PAGES, FLAG_CAPACITY, FLAG_ROWS, FLAG_BAD = 1, 2, 4, 8


def plan(lens, n_new, free, head, table, page, n_pages, T):
    """table, cu, new_lens, slots, positions, counts as paged_plan leaves them (int64 arrays)."""
    table = np.array(table, dtype=np.int64)
    R, max_pages = table.shape
    flags = 0
    if head < 0:
        head, flags = 0, FLAG_BAD
    head0 = head = min(head, len(free))
    cu, new_lens, slots, positions = [0], [], [], []

    def valid(i):
        return i if 0 <= i < n_pages else -1

    for r in range(R):
        n, m = int(lens[r]), int(n_new[r])
        if n < 0 or m < 0:
            flags |= FLAG_BAD
            n, m = max(n, 0), max(m, 0)
        if len(slots) + m > T:
            flags |= FLAG_ROWS
            m = T - len(slots)
        held = min(-(-n // page), max_pages)
        if n + m > max_pages * page:
            flags |= FLAG_CAPACITY
        for j in range(held, min(-(-(n + m) // page), max_pages)):
            if head < len(free):
                table[r, j] = valid(int(free[head]))
                head += 1
            else:
                table[r, j] = -1
                flags |= FLAG_PAGES
        for p in range(n, n + m):
            j = p // page
            i = valid(int(table[r, j])) if j < max_pages else -1
            slots.append(i * page + p % page if i >= 0 else -1)
            positions.append(min(p, 2 ** 31 - 1))
        cu.append(len(slots))
        new_lens.append(min(n + m, 2 ** 31 - 1))
    counts = [len(slots), head - head0, head, flags]
    rest = [-1] * (T - len(slots))
    return tuple(np.array(x, dtype=np.int64) for x in (table, cu, new_lens, slots + rest, positions + rest, counts))


def rope(x, positions):
    """x [T, H, D] rotated: pair (2i, 2i + 1) by positions * 10000^(-2i/D)."""
    D = x.shape[-1]
    ang = np.asarray(positions, dtype=np.float64)[:, None] * 10000.0 ** (-2.0 * np.arange(D // 2) / D)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    out = np.empty(x.shape)
    out[..., 0::2] = x[..., 0::2] * c - x[..., 1::2] * s
    out[..., 1::2] = x[..., 0::2] * s + x[..., 1::2] * c
    return out


def _pow2_scale(top, most):
    """Exponent of the smallest power of two with top <= most * 2^e, at least -126; 0 for top = 0."""
    if top == 0:
        return 0
    e = math.ceil(math.log2(top / most)) - 2
    while top > most * 2.0 ** e:
        e += 1
    return max(e, -126)


def _e4m3_grid():
    vals = [m * 2.0 ** -9 for m in range(8)]
    vals += [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)]
    return np.array([v for v in vals if v <= 448])


def _nearest(x, grid):
    """Nearest of an ascending grid, ties to the even index; x >= 0."""
    hi = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    lo = hi - 1
    up, down = grid[hi] - x, x - grid[lo]
    take_hi = (up < down) | ((up == down) & (hi % 2 == 0))
    return np.where(take_hi, hi, lo)


def e4m3(row):
    """(values [D], scale exponent) of one token's head; infinities and NaN become NaN."""
    row = np.asarray(row, dtype=np.float64)
    fin = np.isfinite(row)
    e = _pow2_scale(float(np.max(np.abs(row[fin]), initial=0.0)), 448.0)
    grid = _e4m3_grid()
    out = np.full(row.shape, np.nan)
    out[fin] = np.sign(row[fin]) * grid[_nearest(np.abs(row[fin]) * 2.0 ** -e, grid)] * 2.0 ** e
    return out, e


def cached(pages, scales=None):
    """float64 pages [n_pages, page, Hkv, D] times 2^(scale - 127)."""
    pages = np.asarray(pages, dtype=np.float64)
    return pages if scales is None else pages * 2.0 ** (np.asarray(scales, dtype=np.float64)[..., None] - 127)


def attention(q, k_pages, v_pages, table, lens, cu, max_new=32):
    """o [T, Hq, D], lse [T, Hq] and the weighted mean of |v| (for error bounds); rows of no
    request are NaN.  k_pages, v_pages as ``cached`` gives them."""
    T, Hq, D = q.shape
    n_pages, page, Hkv, _ = k_pages.shape
    G = Hq // Hkv
    o, mag, lse = np.full(q.shape, np.nan), np.full(q.shape, np.nan), np.full((T, Hq), np.nan)
    for r in range(len(lens)):
        n = cu[r + 1] - cu[r]
        for t in range(min(n, max_new)):
            i = cu[r] + t
            keys = []  # (page, row) of every key the row sees
            for p in range(min(lens[r] - n + t + 1, lens[r], table.shape[1] * page)):
                j = table[r, p // page]
                if 0 <= j < n_pages:
                    keys.append((j, p % page))
            if not keys:
                o[i], mag[i], lse[i] = 0, 0, -np.inf
                continue
            a, b = np.array(keys).T
            for h in range(Hkv):
                k, v = k_pages[a, b, h], v_pages[a, b, h]
                hs = slice(h * G, (h + 1) * G)
                x = q[i, hs] @ k.T / math.sqrt(D)
                m = np.max(x, axis=1, keepdims=True)
                with np.errstate(invalid="ignore"):
                    w = np.exp(x - np.where(np.isneginf(m), 0, m))
                    l = np.sum(w, axis=1, keepdims=True)
                    dead = l[:, 0] == 0  # every score -inf
                    l[dead] = 1
                    o[i, hs] = w @ v / l
                    mag[i, hs] = w @ np.abs(v) / l
                    lse[i, hs] = np.where(dead, -np.inf, (m + np.log(l))[:, 0])
    return o, lse, mag


E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def mx4_values(w4, scales, K, N):
    """The weights [K, N] that packed blocks stand for."""
    w4, scales = np.asarray(w4), np.asarray(scales)
    out = np.zeros((K, N))
    n = np.arange(N)
    for k in range(K):
        byte = w4[n // 16, k // 128, (k // 8 % 4) * 16 + n % 16, 4 * (k // 32 % 4) + k % 8 // 2]
        code = (byte >> 4 if k % 2 else byte & 15).astype(np.int64)
        s = scales[n // 16, k // 128, n % 16, k // 32 % 4].astype(np.float64)
        out[k] = np.where(code >= 8, -1, 1) * E2M1[code % 8] * np.where(s == 255, np.nan, 2.0 ** (s - 127))
    return out


def mx4_pack(w):
    """(w4, scales) of weights [K, N]."""
    K, N = w.shape
    nb, kb = -(-N // 16), -(-K // 128)
    w4 = np.zeros((nb, kb, 64, 16), dtype=np.uint8)
    scales = np.full((nb, kb, 16, 4), 127, dtype=np.uint8)
    for n in range(N):
        for k0 in range(0, K, 32):
            x = w[k0:k0 + 32, n]
            b, s = k0 // 128, k0 // 32 % 4
            if not np.isfinite(x).all():
                scales[n // 16, b, n % 16, s] = 255
                continue
            e = _pow2_scale(float(np.max(np.abs(x))), 6.0)
            scales[n // 16, b, n % 16, s] = e + 127
            code = _nearest(np.abs(x) * 2.0 ** -e, E2M1)
            code = code + np.where((x < 0) & (code > 0), 8, 0)
            for j in range(32):
                w4[n // 16, b, (j // 8) * 16 + n % 16, 4 * s + j % 8 // 2] |= int(code[j]) << (4 * (j % 2))
    return w4, scales
