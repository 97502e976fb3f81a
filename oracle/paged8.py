"""The 8-bit paged cache in plain numpy, in 64 bits: codes and scales, writes, rows,
attention, token weights and eviction, and norms with rotation (include/fastcoder.h,
"8-bit paged cache").  Where results are computed numbers, also what the kernels'
roundings may move them by."""
from __future__ import annotations

import numpy as np

from . import rope

PAGE, BLOCK, DIM, PAGE_BYTES = 64, 32, 128, 16512
V0, SCALES = PAGE * DIM, 2 * PAGE * DIM
LOG2E = np.log2(np.e)


def _values() -> np.ndarray:
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7.0))
    v[(b & 127) == 127] = np.nan
    return np.where(b >= 128, -v, v)


VALUES = _values()


def exponent(top) -> np.ndarray:
    """The least e in [-117, 119] with top <= 448 * 2^e, or 119."""
    e = np.full(np.shape(top), -117)
    for k in range(-117, 119):
        e = np.where(np.asarray(top) > 448 * 2.0 ** k, k + 1, e)
    return e


def codes(x, e) -> np.ndarray:
    """The nearest codes of x at the scales 2^e, ties to the even one; NaN for what is not finite."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0) / 2.0 ** np.asarray(e, np.float64)
    a = np.minimum(a, 448.0)
    at = np.searchsorted(VALUES[:127], a)             # the first value not below
    lo = np.maximum(at - 1, 0)
    up, down = VALUES[at] - a, a - VALUES[lo]
    c = np.where(up < down, at, np.where(down < up, lo, np.where(at % 2 == 0, at, lo)))
    return np.where(np.isfinite(x), c + 128 * np.signbit(x), 127).astype(np.uint8)


def largest(x, axis) -> np.ndarray:
    return np.where(np.isfinite(x), np.abs(np.where(np.isfinite(x), x, 0)), 0).max(axis, initial=0.0)


def key_codes(page: np.ndarray) -> np.ndarray:
    """[64][128], in place."""
    return page[:V0].reshape(PAGE, DIM)


def value_codes(page: np.ndarray) -> np.ndarray:
    """[64][128], a copy."""
    return page[V0:SCALES].reshape(4, DIM, 16).transpose(0, 2, 1).reshape(PAGE, DIM)


def put_values(page: np.ndarray, c: np.ndarray) -> None:
    page[V0:SCALES] = c.reshape(4, 16, DIM).transpose(0, 2, 1).reshape(-1)


def held(page: np.ndarray):
    """Keys and values [64][128] that a page stands for."""
    out = []
    for i, c in enumerate((key_codes(page), value_codes(page))):
        s = 2.0 ** (page[SCALES + 2 * i:SCALES + 2 * i + 2].astype(np.float64) - 127)
        out.append(VALUES[c] * np.repeat(s, BLOCK)[:, None])
    return out


def _put(page, part, rows, x, e) -> None:
    """Codes of rows x at 2^e into a page's keys (0) or values (1)."""
    c = key_codes(page) if part == 0 else value_codes(page)
    c[rows] = codes(x, e)
    if part:
        put_values(page, c)


def write(pool: np.ndarray, k, v, slot, src=None) -> np.ndarray:
    """The pool after rows of k and v [n_src][Hkv][128] are placed, a run of entries of one block at a
    time; entries that are skipped end none."""
    pool = pool.copy()
    n_pages, Hkv = pool.shape[:2]
    slot = np.asarray(slot).astype(np.int64)
    src = np.arange(len(slot)) if src is None else np.asarray(src).astype(np.int64)
    placed = (slot >= 0) & (slot < PAGE * n_pages) & (src >= 0) & (src < len(k))
    slot, src = slot[placed], src[placed]
    i = 0
    while i < len(slot):
        block, j = slot[i] // BLOCK, i
        while j < len(slot) and slot[j] // BLOCK == block:
            j += 1
        rows = [(int(slot[x]) % BLOCK, int(src[x])) for x in range(i, j)]
        i = j
        at, half = np.array([t for t, _ in rows]), int(block % 2)
        from_ = [r for _, r in rows]
        for h in range(Hkv):
            page = pool[block // 2, h]
            for part, x in enumerate((k, v)):
                x = np.asarray(x, np.float64)[from_, h]
                byte = SCALES + 2 * part + half
                e, was = int(exponent(largest(x, None))), int(np.clip(int(page[byte]) - 127, -117, 119))
                all_ = slice(BLOCK * half, BLOCK * half + BLOCK)
                if 0 in at:
                    c = key_codes(page) if part == 0 else value_codes(page)
                    c[all_] = 0
                    if part:
                        put_values(page, c)
                else:
                    e = max(e, was)
                    if e > was:
                        c = key_codes(page) if part == 0 else value_codes(page)
                        old = VALUES[c[all_]]
                        c[all_] = np.where(np.isnan(old), c[all_], codes(old, e - was))
                        if part:
                            put_values(page, c)
                _put(page, part, BLOCK * half + at, x, e)
                page[byte] = e + 127
    return pool


def rows(pool: np.ndarray, table, n: int):
    """Keys and values (float64 [n][Hkv][128]) of the first n tokens of a table row, and which are there."""
    n_pages, Hkv = pool.shape[:2]
    k, v, there = np.zeros((n, Hkv, DIM)), np.zeros((n, Hkv, DIM)), np.zeros(n, bool)
    for p in range(-(-n // PAGE)):
        a, b = PAGE * p, min(PAGE * p + PAGE, n)
        if not 0 <= table[p] < n_pages:
            continue
        there[a:b] = True
        for h in range(Hkv):
            x, y = held(pool[table[p], h])
            k[a:b, h], v[a:b, h] = x[:b - a], y[:b - a]
    return k, v, there


# fp32 sums of 128 products: 2^-23 each of the sum of magnitudes, and a few roundings
# of what is done to the sum
SUM = 136 * 2.0 ** -23


def attention(q, k_tree, v_tree, pool, table, prefix_len, num_nodes=None, mask=None, max_len=None):
    """The result, each row's logarithm of its sum, and what either may be off by.

    A score, as a power of two's exponent, is off by d = SUM of the sum of its
    products' magnitudes, 2^-22 of itself and of the row's largest (scaling, the
    maximum taken off), and 2^-22 (the power).  A weight moves by t = 2^d (1 + 2^-8)
    - 1 of itself (it is rounded to bf16), so the result by sum p t |v - o| / (1 -
    sum p t); sums are fp32, the result is bf16.  The logarithm takes the weights
    before they are rounded."""
    q, k_tree, v_tree = (np.asarray(x, np.float64) for x in (q, k_tree, v_tree))
    B, R, H, _ = q.shape
    Hkv = k_tree.shape[2]
    out, most = np.zeros((B, R, H, DIM)), np.zeros((B, R, H, DIM))
    lse, lse_most = np.full((B, R, H), -np.inf), np.zeros((B, R, H))
    c = LOG2E / np.sqrt(DIM)
    for b in range(B):
        P = min(max(int(prefix_len[b]), 0), PAGE * np.shape(table)[1] if max_len is None else max_len)
        n = R if num_nodes is None else min(max(int(num_nodes[b]), 0), R)
        kc, vc, there = rows(pool, table[b], P)
        see = np.tril(np.ones((R, R), bool)) if mask is None else np.asarray(mask[b]) == 1
        see = see & (np.arange(R) < n)
        for h in range(H):
            g = h // (H // Hkv)
            keys, vals = np.concatenate([kc[there, g], k_tree[b, :, g]]), np.concatenate([vc[there, g], v_tree[b, :, g]])
            cached = np.ones(there.sum(), bool)
            for i in range(n):
                on = np.concatenate([cached, see[i]])
                if not on.any():
                    continue
                with np.errstate(all="ignore"):
                    s = keys[on] @ q[b, i, h] * c
                    top = s.max()
                    p = 2.0 ** (s - top)
                    total = p.sum()
                    p = p / total
                    o = p @ vals[on]
                    d = SUM * c * (np.abs(keys[on]) @ np.abs(q[b, i, h])) + 2.0 ** -22 * (np.abs(s) + np.abs(top) + 1)
                    t = 2.0 ** d * (1 + 2.0 ** -8) - 1
                    off = (p * t) @ np.abs(vals[on] - o) / (1 - min((p * t).sum(), 0.5))
                    sums = (on.sum() + 300) * 2.0 ** -23
                    out[b, i, h] = o
                    most[b, i, h] = (off + sums * (p @ np.abs(vals[on]) + np.abs(o))) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(o) + 1e-38
                    lse[b, i, h] = (top + np.log2(total)) / LOG2E
                    lse_most[b, i, h] = d.max() / LOG2E + sums + 2.0 ** -21 * (1 + np.abs(lse[b, i, h]) + np.abs(top))
    return out, lse, most, lse_most


def weights(w, q, lse, pool, table, length, new_length, cu, src=None, max_len=None):
    """Token weights after a step's rows, and what each may be off by: as a score above,
    with the logarithm's own scaling; fp32 sums over the rows."""
    w = np.asarray(w, np.float64).copy()
    most = np.zeros_like(w)
    q, lse = np.asarray(q, np.float64), np.asarray(lse, np.float64)
    n_rows, H, _ = q.shape
    n_pages, Hkv = pool.shape[:2]
    n = n_rows if src is None else len(src)
    c = LOG2E / np.sqrt(DIM)
    cap = PAGE * np.shape(table)[1] if max_len is None else max_len
    for b in range(len(length)):
        P, E = (min(max(int(x[b]), 0), cap) for x in (length, new_length))
        if E <= P:
            continue
        kc, _, there = rows(pool, table[b], E)
        got, off = np.zeros((E, Hkv)), np.zeros((E, Hkv))
        for t in range(E - P):
            at = int(cu[b]) + t
            r = -1 if not 0 <= at < n else at if src is None else int(src[at])
            if not 0 <= r < n_rows:
                continue
            for h in range(H):
                if lse[r, h] == -np.inf:
                    continue
                g = h // (H // Hkv)
                seen = kc[:P + t + 1, g]
                with np.errstate(all="ignore"):
                    s = seen @ q[r, h] * c
                    p = 2.0 ** (s - lse[r, h] * LOG2E)
                    d = SUM * c * (np.abs(seen) @ np.abs(q[r, h])) + 2.0 ** -22 * (np.abs(s) + np.abs(lse[r, h]) * LOG2E + 1)
                    e = p * (2.0 ** d - 1)
                got[:P + t + 1, g] += p
                # 2^(s - inf) is 0 whatever the rounding of a finite s: nothing is off
                off[:P + t + 1, g] += 0.0 if lse[r, h] == np.inf else e
        sums = (E - P) * (H // Hkv) * 2.0 ** -23
        for j in np.flatnonzero(there):
            at = (table[b][j // PAGE], slice(None), j % PAGE)
            old = w[at] if j < P else 0.0
            w[at] = old + got[j]
            most[at] = off[j] + (sums + 2.0 ** -22) * (np.abs(got[j]) + np.abs(old)) + 1e-38
    return w, most


def evict(pool, w, table, length, budget, first=0, recent=0, max_len=None):
    """pool, token weights and add after sequences are cut to their budgets."""
    pool, w = pool.copy(), w.copy()
    n_pages, Hkv = pool.shape[:2]
    add = np.zeros(len(length), np.int32)
    cap = PAGE * np.shape(table)[1] if max_len is None else max_len
    for b in range(len(length)):
        n = min(max(int(length[b]), 0), cap)
        keep = min(max(int(budget[b]), 0), n)
        add[b] = keep - n
        if keep == n or keep == 0:
            continue
        tok = np.arange(n)
        page = np.asarray(table[b])[tok // PAGE]
        there = (page >= 0) & (page < n_pages)
        late = n - min(recent, keep)
        new_k, new_v, new_w = [], [], []
        for h in range(Hkv):
            x = [np.zeros((n, DIM)) for _ in "kv"]
            for p in range(-(-n // PAGE)):
                if there[p * PAGE]:
                    for part, y in enumerate(held(pool[table[b][p], h])):
                        x[part][p * PAGE:p * PAGE + PAGE] = y[:n - p * PAGE]
            wt = np.where(there, w[np.where(there, page, 0), h, tok % PAGE], 0).astype(np.float64)
            rank = np.where(wt > 0, wt, 0)
            # last ones, first ones, others; the heaviest of each, of equal ones the earlier
            group = np.where(tok >= late, 0, np.where(tok < first, 1, 2))
            stay = np.sort(np.lexsort((tok, -rank, group))[:keep])
            new_k.append(x[0][stay])
            new_v.append(x[1][stay])
            new_w.append(wt[stay])
        for h in range(Hkv):
            for a in range(0, keep, BLOCK):
                p = table[b][a // PAGE]
                if not 0 <= p < n_pages:
                    continue
                half, page_ = a // BLOCK % 2, pool[p, h]
                m = min(BLOCK, keep - a)
                for part, x in enumerate((new_k[h], new_v[h])):
                    y = np.zeros((BLOCK, DIM))
                    y[:m] = x[a:a + m]
                    e = int(exponent(largest(y, None)))
                    _put(page_, part, slice(BLOCK * half, BLOCK * half + BLOCK), y, e)
                    page_[SCALES + 2 * part + half] = e + 127
                w[p, h, a % PAGE:a % PAGE + m] = new_w[h][a:a + m]
    return pool, w, add


def norm_rotate(x, weight=None, pos=None, eps=1e-6, rope_base=10000.0):
    """Rows [n][heads][128] normed and rotated, and what each value may be off by: fp32
    sums of 128 squares and a handful of roundings (2^-16 of a value together), the
    hardware's sine and cosine (2^-18 of a pair's magnitudes), the result in bf16."""
    x = np.asarray(x, np.float64)
    with np.errstate(all="ignore"):
        y = x if weight is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    pair = np.abs(y)
    if rope_base:
        half = np.abs(y[..., :DIM // 2]) + np.abs(y[..., DIM // 2:])
        pair = np.concatenate([half, half], -1)
        y = np.stack([rope(row, np.full(len(row), p), rope_base) for row, p in zip(y, np.asarray(pos))]) if len(y) else y
    return y, 2.0 ** -8 * np.abs(y) + (1 + 2.0 ** -8) * (2.0 ** -16 + 2.0 ** -18) * pair + 1e-38
