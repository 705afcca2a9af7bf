"""Generation from a paged cache on the CPU, in 64 bits and one request at a time: the page plan, the append with page bounds, the
selection of pages and the attention of one new token, from their definitions.  Shares no code with the library."""
import math

import numpy as np


def pages_of(tokens, page):
    return -(-int(tokens) // page)


def page_plan(lens, grow, page, table, ring, head, tail, space):
    """All outputs of a step; `table` and `ring` are copied."""
    table, ring = table.copy(), ring.copy()
    before = ring.copy()
    cap, width = ring.size, table.shape[1]
    new_lens, starts = [], [0]
    slots, positions, requests = (np.full(space, -1, np.int64) for _ in range(3))
    asked, used, back = 0, 0, 0
    for b, (n, g) in enumerate(zip(map(int, lens), map(int, grow))):
        held, at = pages_of(n, page), starts[-1]
        if g < 0:
            for j in range(held):
                ring[(tail + back) % cap] = table[b, j]
                back += 1
            new_lens.append(0)
            starts.append(at)
            continue
        starts.append(at + g)
        for t in range(at, min(space, at + g)):
            requests[t] = b
        want = pages_of(n + g, page) - held
        if held + want > width or at + g > space:
            new_lens.append(n)
            continue
        asked += want
        if want and asked > tail - head:
            new_lens.append(n)
            continue
        for j in range(want):
            table[b, held + j] = before[(head + used) % cap]
            used += 1
        for i in range(g):
            positions[at + i] = n + i
            slots[at + i] = table[b, (n + i) // page] * page + (n + i) % page
        new_lens.append(n + g)
    return {"table": table, "ring": ring, "lens": np.array(new_lens), "state": np.array([head + used, tail + back]),
            "starts": np.array(starts), "slots": slots, "positions": positions, "requests": requests}


def append(k_new, slots, page, pool, low=None, high=None):
    """pool [P,H,page,d] with the rows of k_new [T,H,d] at their slots; low, high [P,H,d]: bounds of the pages."""
    pool = pool.copy()
    low, high = (None, None) if low is None else (low.copy(), high.copy())
    for t, s in enumerate(map(int, slots)):
        if not 0 <= s < pool.shape[0] * page:
            continue
        p, r = divmod(s, page)
        pool[p, :, r] = k_new[t]
        if low is not None:
            if r == 0:
                low[p], high[p] = math.inf, -math.inf
            low[p], high[p] = np.minimum(low[p], k_new[t]), np.maximum(high[p], k_new[t])
    return pool, low, high


def budget_pages(budget, n, least=1, first=0, last=0):
    if n == 0:
        return 0
    share = (int(np.float32(budget).astype(np.float64) * (1 << 20)) * n + (1 << 20) - 1) >> 20
    return min(n, max(share, 1, least, first + last))


def page_scores(q, low, high):
    """M [G, n]: sum_c max(q_c low_c, q_c high_c) in float32, by the tree of the definition; of two products of which one is no number (zero times
    infinity) the other.  q [G,d], low and high [n,d] float32."""
    q, low, high = (np.asarray(x, np.float32) for x in (q, low, high))
    with np.errstate(invalid="ignore"):
        x = np.fmax(q[:, None] * low[None], q[:, None] * high[None]).reshape(q.shape[0], low.shape[0], -1, 8)
    while x.shape[3] > 1:
        half = x.shape[3] // 2
        x = x[..., :half] + x[..., half:]
    x = x[..., 0]
    while x.shape[2] > 1:
        half = x.shape[2] // 2
        x = x[..., :half] + x[..., half:]
    return x[..., 0]


def select(q, low, high, budget, least=1, first=0, last=0):
    """Ascending list of the pages kept, of n; q [G,d].  A page that holds a head's maximum ranks 0 for it, whatever that maximum is; a score that is no
    number counts for nothing."""
    n = low.shape[0]
    if n == 0:
        return np.zeros(0, np.int64)
    m = page_scores(q, low, high)
    m = np.where(np.isnan(m), np.float32(-math.inf), m)
    top = m.max(axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        r = np.where((m == top) & (m > -math.inf), np.float32(0), np.where(m == -math.inf, m, m - top)).max(axis=0).astype(np.float64)
    r[:first] = math.inf
    r[n - min(n, last):] = math.inf
    order = sorted(range(n), key=lambda j: (-r[j], j))
    return np.array(sorted(order[:budget_pages(budget, n, least, first, last)]), np.int64)


def attention(q, k, v, scale):
    """q [G,d], k, v [T,d] -> out [G,d], lse [G], and the largest sum of |q_c k_c| scale of a logit (for error bounds)."""
    if k.shape[0] == 0:
        return np.zeros_like(q), np.full(q.shape[0], -math.inf), 0.0
    x = q @ k.T * scale
    top = x.max(axis=1, keepdims=True)
    ref = np.where(np.isneginf(top), 0.0, top)
    p = np.exp(x - ref)
    total = p.sum(axis=1, keepdims=True)
    out = np.where(total > 0, (p @ v) / np.where(total > 0, total, 1.0), 0.0)
    with np.errstate(divide="ignore"):
        lse = np.log(total[:, 0]) + ref[:, 0]
    return out, lse, float((np.abs(q) @ np.abs(k).T).max() * scale)


def kept_tokens(length, page, pages=None, window=0):
    """Positions a new token attends to: all of [0, length), those in listed pages, those in the window."""
    n = pages_of(length, page)
    if pages is None:
        t = np.arange(length)
    else:
        ids = np.array([j for j in pages if 0 <= j < n], np.int64)
        t = (ids[:, None] * page + np.arange(page)).reshape(-1)
        t = t[t < length]
    return t[t >= length - window] if window else t
