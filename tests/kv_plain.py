"""The 4-bit key/value cache in plain numpy: the layout, the quantizer in the fp32 steps that define it, attention in 64 bits, the
page books one row after the other.  Test infrastructure, written from the definitions in quantpipe.h."""
import numpy as np

HEADER = 16


def slab_bytes(dim, page):
    return page * (dim + 16)


def new_pages(layers, n_pages, heads, dim, page, rng=None):
    """Pages with anything in them (rng), NaN grids among it, or zeros."""
    shape = (layers, n_pages, heads, slab_bytes(dim, page))
    if rng is None:
        return np.zeros(shape, np.uint8)
    p = rng.integers(0, 256, shape, dtype=np.uint8)
    k, v, gk, gv = pieces(p, dim, page)
    gk[..., ::3, :] = np.nan
    gv[..., ::2, 1] = np.inf
    return p


def pieces(pages, dim, page):
    """Views: key codes [.., page, dim / 8] and value codes [.., page / 8, dim] as uint32, key and value grids [.., page, 2]."""
    lead, half = pages.shape[:-1], page * dim // 2
    w, f = pages.view(np.uint32), pages.view(np.float32)
    k = w[..., :half // 4].reshape(*lead, page, dim // 8)
    v = w[..., half // 4:half // 2].reshape(*lead, page // 8, dim)
    g = f[..., half // 2:].reshape(*lead, 2, page, 2)
    for x in (k, v, g):
        assert np.shares_memory(x, pages)
    return k, v, g[..., 0, :, :], g[..., 1, :, :]


def grid(x):
    """(lo, scale, inv) of x [dim] in fp32."""
    x = np.asarray(x, np.float32)
    fine = x[np.isfinite(x)]
    if fine.size == 0:
        return np.float32(0), np.float32(0), np.float32(0)
    big = np.float32(2.0 ** 126)
    lo, hi = np.clip(fine.min(), -big, big), np.clip(fine.max(), -big, big)
    scale = np.float32(np.float32(hi - lo) / np.float32(15))
    if not scale >= np.float32(2.0 ** -120):
        scale = np.float32(0)
    return lo, scale, np.float32(1) / scale if scale > 0 else np.float32(0)


def codes(x, lo, inv):
    with np.errstate(all="ignore"):
        c = np.rint((np.asarray(x, np.float32) - lo) * inv)
    return np.clip(np.where(np.isnan(c), 0, c), 0, 15).astype(np.uint32)


def put(pages, dim, page, p, slot, head, k, v):
    """One token's key and value of one head into pages [n_pages, heads, slab]."""
    kc, vc, gk, gv = pieces(pages, dim, page)
    lo, scale, inv = grid(k)
    c = codes(k, lo, inv).reshape(-1, 8)
    kc[p, head, slot] = (c << (4 * np.arange(8, dtype=np.uint32))).sum(1)
    gk[p, head, slot] = lo, scale
    lo, scale, inv = grid(v)
    c = codes(v, lo, inv)
    sh = np.uint32(4 * (slot % 8))
    vc[p, head, slot // 8] = (vc[p, head, slot // 8] & ~np.uint32(15 << int(sh))) | (c << sh)
    gv[p, head, slot] = lo, scale


def get(pages, dim, page, p, slot, head):
    """(codes, lo, scale) of keys and of values, in 64 bits; p and slot may be arrays of places [n]: codes [n, dim], grids [n, 1]."""
    kc, vc, gk, gv = pieces(pages, dim, page)
    p, slot = np.asarray(p), np.asarray(slot)
    w = kc[p, head, slot]
    ck = ((w[..., None] >> (4 * np.arange(8, dtype=np.uint32))) & 15).reshape(*w.shape[:-1], dim)
    cv = (vc[p, head, slot // 8] >> (4 * (slot % 8)).astype(np.uint32)[..., None]) & 15
    gk, gv = gk[p, head, slot].astype(np.float64), gv[p, head, slot].astype(np.float64)
    return (ck.astype(np.float64), gk[..., :1], gk[..., 1:]), (cv.astype(np.float64), gv[..., :1], gv[..., 1:])


def place(table, r, t, page, n_pages):
    """(page, slot) of token t of row r, or None."""
    if t < 0 or t // page >= table.shape[1]:
        return None
    p = int(table[r, t // page])
    return (p, t % page) if 0 <= p < n_pages else None


def ranges(begin, tokens):
    """(first token, count) of every row of a call."""
    b = np.clip(np.asarray(begin, np.int64), 0, tokens)
    return [(int(b[r]), int(max(0, b[r + 1] - b[r]))) for r in range(len(b) - 1)]


def capped(lengths, table, page):
    return np.clip(np.asarray(lengths, np.int64), 0, table.shape[1] * page)


def append(pages, dim, page, table, lengths, begin, k, v):
    n_pages = pages.shape[0]
    L = capped(lengths, table, page)
    for r, (b, m) in enumerate(ranges(begin, k.shape[0])):
        for i in range(m):
            at = place(table, r, int(L[r]) - m + i, page, n_pages)
            if at:
                for h in range(pages.shape[1]):
                    put(pages, dim, page, *at, h, k[b + i, h], v[b + i, h])


def read(pages, dim, page, table, lengths, begin, first, k, v):
    """Into k, v [tokens, heads, dim], float64: value = fma(c, scale, lo), not rounded."""
    L = capped(lengths, table, page)
    for r, (b, m) in enumerate(ranges(begin, k.shape[0])):
        for i in range(m):
            t = (0 if first is None else int(first[r])) + i
            at = place(table, r, t, page, pages.shape[0]) if t < L[r] else None
            for h in range(pages.shape[1]):
                if at is None:
                    k[b + i, h] = v[b + i, h] = 0
                    continue
                (ck, lk, sk), (cv, lv, sv) = get(pages, dim, page, *at, h)
                k[b + i, h], v[b + i, h] = lk + ck * sk, lv + cv * sv


def attention(pages, dim, page, table, lengths, begin, q, scale, causal, window, u_out, split):
    """(out, tolerance) [tokens, q_heads, dim] in 64 bits; NaN where a token is no row's.

    The tolerance adds up what the fp32 evaluation on codes may lose (u = 2^-24, half a step of fp32; 2^-11 of fp16):
      scores     a dot product of dim terms, the grid's two terms and the exponent's argument: (dim + 16) roundings of
                 B = scale sum |q_d| (|c_d - 8| s + |lo + 8 s|), and the query's own: 2^-22 of it if split in two halves, else
                 2^-24 (exact but for elements 2^-30 below the largest); then exp2's own error, 2 u: a relative error e of each p,
                 which moves the answer by at most 2 e V, V = max (8 s + |lo + 8 s|) over the tokens seen
      sums       n + 64 additions in whatever order: (n + 64) 2 u V for numerator and denominator together
      p s        rounded to fp16, or split: 2^-11 or 2^-22, of at most 8 s
      out        u_out of itself
    """
    tokens, q_heads, _ = q.shape
    n_pages, heads = pages.shape[:2]
    group = q_heads // heads
    u = 2.0 ** -24
    out, tol = np.full(q.shape, np.nan), np.zeros(q.shape)
    L = capped(lengths, table, page)
    for r, (b, m) in enumerate(ranges(begin, tokens)):
        if m == 0:
            continue
        seen_at = [(t, place(table, r, t, page, n_pages)) for t in range(int(L[r]))]
        seen_at = [(t, a) for t, a in seen_at if a]
        ts = np.array([t for t, _ in seen_at], np.int64)
        for h in range(heads):
            (ck, lk, sk), (cv, lv, sv) = get(pages, dim, page, np.array([a[0] for _, a in seen_at], int), np.array([a[1] for _, a in seen_at], int), h)
            K, V = lk + ck * sk, lv + cv * sv
            Kb, Vb, Sb = np.abs(ck - 8) * sk + np.abs(lk + 8 * sk), (8 * sv + np.abs(lv + 8 * sv))[:, 0], 8 * sv[:, 0]
            for i in range(m):
                pos = int(L[r]) - m + i
                see = ts <= pos if causal else np.ones(len(ts), bool)
                if window:
                    see &= ts > pos - window
                x = q[b + i, h * group:(h + 1) * group].astype(np.float64)        # [group, dim]
                fine = np.isfinite(x).all(1)
                to = np.arange(h * group, (h + 1) * group)[fine]                  # the others stay NaN
                if not see.any():
                    out[b + i, to] = 0
                    continue
                x = x[fine]
                z = scale * (x @ K[see].T)
                p = np.exp(z - z.max(1, keepdims=True))
                o = (p @ V[see]) / p.sum(1, keepdims=True)
                B = scale * (np.abs(x) @ Kb[see].T).max(1)
                e = (dim + 16) * u * B + (2.0 ** -22 if split else 2.0 ** -24) * B + 3 * u * (1 + np.abs(z).max(1) + np.abs(z - z.max(1, keepdims=True)).max(1)) + 2 * u
                top = Vb[see].max()
                out[b + i, to] = o
                tol[b + i, to] = (2 * e * top + (see.sum() + 64) * 2 * u * top + (2.0 ** -22 if split else 2.0 ** -11) * Sb[see].max())[:, None] + u_out * np.abs(o)
    return out, tol


# ---- the books ---------------------------------------------------------------------------------------------------------

def pages_of(tokens, page):
    return -(-int(tokens) // page)


def reserve(table, lengths, refs, want, page):
    """Changes table, lengths, refs; returns (short, outgrown, moves) with moves a list of (from, to)."""
    t, L, R = table.copy(), lengths.copy(), refs.copy()
    cap = table.shape[1] * page
    outgrown = sum(int(want[r]) > 0 and min(max(int(L[r]), 0), cap) + int(want[r]) > cap for r in range(len(L)))
    if outgrown:
        return 0, outgrown, []
    moves, short = [], 0

    def take():
        nonlocal short
        free = np.nonzero(R == 0)[0]
        if free.size == 0:
            short += 1
            return -2
        R[free[0]] = 1
        return int(free[0])

    for r in range(len(L)):
        n, w = max(int(L[r]), 0), int(want[r])
        if w <= 0:
            continue
        if n % page:
            p = int(t[r, n // page])
            if 0 <= p < len(R) and R[p] > 1:
                new = take()
                R[p] -= 1
                moves.append((p, new))
                t[r, n // page] = new
        for s in range(pages_of(n, page), pages_of(n + w, page)):
            t[r, s] = take()
        L[r] = n + w
    if short:
        return short, 0, []
    table[:], lengths[:], refs[:] = t, L, R
    return 0, 0, moves


def fork(table, lengths, refs, parent, page):
    refused = 0
    was = lengths.copy()
    for r in range(len(lengths)):
        p = int(parent[r])
        if p < 0:
            continue
        if p >= len(lengths) or p == r or parent[p] >= 0 or was[r] > 0:
            refused += 1
            continue
        n = min(max(int(was[p]), 0), table.shape[1] * page)
        for s in range(pages_of(n, page)):
            table[r, s] = table[p, s]
            if 0 <= table[p, s] < len(refs):
                refs[table[p, s]] += 1
        lengths[r] = n
    return refused


def free(table, lengths, refs, keep, page):
    for r in range(len(lengths)):
        n = min(max(int(lengths[r]), 0), table.shape[1] * page)
        k = int(keep[r])
        if k < 0 or k >= n:
            continue
        for s in range(pages_of(k, page), pages_of(n, page)):
            if 0 <= table[r, s] < len(refs):
                refs[table[r, s]] -= 1
            table[r, s] = -1
        lengths[r] = k


def compact(table, lengths, refs, page):
    live = int((refs > 0).sum())
    moves = list(zip([int(i) for i in np.nonzero(refs > 0)[0] if i >= live], [int(i) for i in np.nonzero(refs <= 0)[0] if i < live]))
    went = dict(moves)
    for a, b in moves:
        refs[b], refs[a] = refs[a], 0
    for r in range(len(lengths)):
        n = min(max(int(lengths[r]), 0), table.shape[1] * page)
        for s in range(pages_of(n, page)):
            table[r, s] = went.get(int(table[r, s]), table[r, s])
    return live, moves
