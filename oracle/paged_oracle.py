"""Plain fp64 implementation of the calls on a paged cache, written from their definitions: append, attention with its
score forms, the account of attention weight, eviction.  Test infrastructure only; shares no code with the HIP path.

A cache is a pair of pools, keys [n_pages][Hk][128][D] and values [n_pages][Hk][D][128], as float64 arrays; a sequence's
tokens lie in the pages of its row of `pages`, 128 to a page.
"""
from __future__ import annotations

import numpy as np

BS = 128


def rows_of(row_start, n_rows, s):
    r0 = min(max(int(row_start[s]), 0), n_rows)
    return r0, min(max(int(row_start[s + 1]), r0), n_rows)


def token_slots(pages, n_pages, s, n):
    """(page, slot) of the tokens 0 .. n - 1 of sequence s; page -1 where there is none."""
    at = np.arange(n)
    page = np.asarray(pages)[s][at // BS] if n else np.zeros(0, int)
    return np.where((page >= 0) & (page < n_pages), page, -1), at % BS


def append(k_new, v_new, row_start, n_ctx, pages, k_pages, v_pages):
    """Returns the two pools after the call."""
    k, v = k_pages.copy(), v_pages.copy()
    for s in range(len(n_ctx)):
        r0, r1 = rows_of(row_start, len(k_new), s)
        n = min(max(int(n_ctx[s]), 0), pages.shape[1] * BS)
        page, slot = token_slots(pages, len(k), s, n)
        for r in range(r0, r1):
            p = n - (r1 - r0) + (r - r0)
            if p >= 0 and page[p] >= 0:
                k[page[p], :, slot[p]] = k_new[r]
                v[page[p], :, :, slot[p]] = v_new[r]
    return k, v


def attention(q, row_start, n_ctx, pages, k_pages, v_pages, scale, softcap=0.0, window=0, slopes=None, row_first=None,
              row_end=None, weight_rows=0, weights=None):
    """Returns out, lse, weights (None without), and what error bounds need: mass [rows][H][D] = sum p |v|,
    size [rows][H] = the largest |q| |k| product sum and bias that enters a score, votes = the sum added to the weights and
    votes_size = the sum of weight times size.  Rows that belong to no sequence are NaN."""
    n_rows, n_heads, d = q.shape
    hk_n = k_pages.shape[1]
    group = n_heads // hk_n
    out, lse = np.full((n_rows, n_heads, d), np.nan), np.full((n_rows, n_heads), np.nan)
    mass, size = np.zeros((n_rows, n_heads, d)), np.zeros((n_rows, n_heads))
    w_out = None if weights is None else weights.copy()
    votes = None if weights is None else np.zeros_like(weights)
    votes_size = None if weights is None else np.zeros_like(weights)
    for s in range(len(n_ctx)):
        r0, r1 = rows_of(row_start, n_rows, s)
        n = min(max(int(n_ctx[s]), 0), pages.shape[1] * BS)
        page, slot = token_slots(pages, len(k_pages), s, n)
        there = page >= 0
        for r in range(r0, r1):
            p = n - (r1 - r0) + (r - r0)
            j = np.arange(n)
            end = p + 1 if row_end is None else min(int(row_end[r]), n)
            first = 0 if row_first is None else max(0, int(row_first[r]))
            if window > 0:
                first = max(first, p - window + 1)
            see = np.nonzero((j >= first) & (j < end) & there & (p >= 0))[0]
            for h in range(n_heads):
                kh = h // group
                if len(see) == 0:
                    out[r, h], lse[r, h] = 0.0, -np.inf
                    continue
                k, v = k_pages[page[see], kh, slot[see]], v_pages[page[see], kh, :, slot[see]]
                z = scale * (k @ q[r, h])
                big = scale * (np.abs(k) @ np.abs(q[r, h]))
                if softcap > 0:
                    z = softcap * np.tanh(z / softcap)
                if slopes is not None:
                    z = z - slopes[h] * np.abs(p - see)
                    big = big + slopes[h] * np.abs(p - see)
                top = z.max()
                e = np.exp(z - top)
                lse[r, h] = top + np.log(e.sum())
                prob = e / e.sum()
                out[r, h], mass[r, h] = prob @ v, prob @ np.abs(v)
                size[r, h] = (big * (prob > 1e-12)).max()
                if weights is not None and r >= r1 - weight_rows:
                    votes[s, kh, see] += prob
                    votes_size[s, kh, see] += prob * (size[r, h] + big)
    if weights is not None:
        w_out += votes
    return dict(out=out, lse=lse, weights=w_out, mass=mass, size=size, votes=votes, votes_size=votes_size)


def keep(weights, n, keep_first, keep_last, budget):
    """Positions that one KV head keeps of n tokens, ascending."""
    if n <= budget:
        return list(range(n))
    middle = range(keep_first, n - keep_last)
    rank = lambda x: (-np.inf if np.isnan(weights[x]) else weights[x])
    best = sorted(middle, key=lambda x: (np.isnan(weights[x]), -rank(x), x))[: budget - keep_first - keep_last]
    return sorted([*range(keep_first), *best, *range(n - keep_last, n)])


def evict(n_ctx, pages, k_pages, v_pages, weights, keep_first, keep_last, budget, to_pages, to_weights):
    """Returns kept, n_kept, the two pools and to_weights after the call (pools are read as they were before it)."""
    k, v, w = k_pages.copy(), v_pages.copy(), to_weights.copy()
    batch, heads = weights.shape[:2]
    in_place = to_pages is pages
    kept = np.full((batch, heads, budget), -1)
    n_kept = np.zeros(batch, int)
    for s in range(batch):
        n = min(max(int(n_ctx[s]), 0), pages.shape[1] * BS)
        n_kept[s] = min(n, budget)
        page, slot = token_slots(pages, len(k), s, n)
        to_page, to_slot = token_slots(to_pages, len(k), s, n_kept[s])
        w[s, :, : to_pages.shape[1] * BS] = 0.0
        for h in range(heads):
            old = keep(weights[s, h], n, keep_first, keep_last, budget)
            kept[s, h, : len(old)] = old
            w[s, h, : len(old)] = weights[s, h, old]
            for t, o in enumerate(old):
                if to_page[t] >= 0 and not (in_place and n <= budget):
                    there = page[o] >= 0
                    k[to_page[t], h, to_slot[t]] = k_pages[page[o], h, slot[o]] if there else 0.0
                    v[to_page[t], h, :, to_slot[t]] = v_pages[page[o], h, :, slot[o]] if there else 0.0
    return kept, n_kept, k, v, w


# ---------------------------------------------------------------- rotation
def rotate(x, table, places, interleaved):
    """x [rows][heads][D] with its first R channels turned by rows `places` (clamped) of table [n][2][R / 2]; and what an error
    bound needs: the sum of the absolute values of the two products of every channel."""
    at = np.clip(np.asarray(places), 0, len(table) - 1)
    cos, sin = table[at, 0][:, None], table[at, 1][:, None]
    half = table.shape[2]
    a = np.arange(half) * 2 if interleaved else np.arange(half)
    b = a + 1 if interleaved else a + half
    y, size = x.copy(), np.abs(x)
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    size[..., a] = np.abs(x[..., a] * cos) + np.abs(x[..., b] * sin)
    size[..., b] = np.abs(x[..., b] * cos) + np.abs(x[..., a] * sin)
    return y, size


# ---------------------------------------------------------------- pages in 8 bits
def round_e4m3(x):
    """The nearest e4m3 value of |x| <= 448, ties to the even code; not a number where x is none or infinite."""
    x = np.asarray(x, np.float64)
    _, p = np.frexp(np.where(np.isfinite(x), x, 0.0))
    unit = np.exp2(np.maximum(p - 1, -6) - 3.0)
    return np.where(np.isfinite(x), np.rint(x / unit) * unit, np.nan)


def scale_exponent(x):
    """The least e >= -100 for which the largest finite |x| is at most 448 2^e."""
    finite = np.abs(x[np.isfinite(x)])
    top = finite.max() if finite.size else 0.0
    e = -100
    while top > 448.0 * 2.0 ** e:
        e += 1
    return e


def quantised_append(k_new, v_new, row_start, n_ctx, pages, k_codes, v_codes, k_scales, v_scales):
    """The pools of code values and the scales after the call; k_new and v_new are what is to be held (rotated, and fp32 values)."""
    kc, vc, ks, vs = k_codes.copy(), v_codes.copy(), k_scales.copy(), v_scales.copy()
    for s in range(len(n_ctx)):
        r0, r1 = rows_of(row_start, len(k_new), s)
        n = min(max(int(n_ctx[s]), 0), pages.shape[1] * BS)
        pos0 = n - (r1 - r0)
        for i in range(max(pos0, 0) // BS, -(-n // BS)):
            lo, hi, page = max(pos0, i * BS, 0), min(n, (i + 1) * BS), int(pages[s][i])
            if r1 == r0 or hi <= lo or not 0 <= page < len(kc):
                continue
            had, new = lo - i * BS, slice(r0 + lo - pos0, r0 + hi - pos0)
            for codes, scales, x in ((kc, ks, k_new), (vc.swapaxes(2, 3), vs, v_new)):
                for h in range(codes.shape[1]):
                    e = scale_exponent(x[new, h])
                    if had:
                        old = int(np.log2(scales[page, h]))
                        e = max(e, old)
                        codes[page, h, :had] = round_e4m3(codes[page, h, :had] * 2.0 ** (old - e))
                    codes[page, h, had: had + hi - lo] = round_e4m3(x[new, h] * 2.0 ** -e)
                    scales[page, h] = 2.0 ** e
    return kc, vc, ks, vs


# ---------------------------------------------------------------- selected pages
def key_bounds(n_ctx, pages, k_pages, bounds, news=None):
    """bounds [n_pages][Hk][2][D] after the call: of all pages, or of those with the last news[s] tokens of a sequence."""
    b = bounds.copy()
    for s in range(len(n_ctx)):
        n = min(max(int(n_ctx[s]), 0), pages.shape[1] * BS)
        first = 0 if news is None else max(n - news[s], 0) // BS
        for i in range(first, -(-n // BS)):
            page = int(pages[s][i])
            if 0 <= page < len(k_pages) and (news is None or news[s] > 0):
                k = k_pages[page, :, : min(n - i * BS, BS)]
                b[page, :, 0], b[page, :, 1] = k.min(1), k.max(1)
    return b


def page_scores(q, bounds, page):
    """Score of a page for one row: q [H][D]; [Hk], rounded to fp32."""
    hk = bounds.shape[1]
    x = q.reshape(hk, -1, q.shape[-1])
    return np.maximum(x * bounds[page, :, :1], x * bounds[page, :, 1:]).sum(-1).max(1).astype(np.float32)


def select_pages(q, row_start, n_ctx, pages, bounds, k_sel, keep_first, keep_last):
    """scores [rows][Hk][max_pages], and the selected pages as lists [row][Hk] (None for rows of no sequence)."""
    hk, max_pages = bounds.shape[1], pages.shape[1]
    scores = np.full((len(q), hk, max_pages), -np.inf, np.float32)
    chosen = [None] * len(q)
    for s in range(len(n_ctx)):
        r0, r1 = rows_of(row_start, len(q), s)
        n = min(max(int(n_ctx[s]), 0), max_pages * BS)
        for r in range(r0, r1):
            p = n - (r1 - r0) + (r - r0)
            last = p // BS if p >= 0 else -1
            seen = [b for b in range(last + 1) if 0 <= pages[s][b] < len(bounds)]
            for b in seen:
                scores[r, :, b] = page_scores(q[r], bounds, int(pages[s][b]))
            chosen[r] = []
            for h in range(hk):
                always = [b for b in seen if b < keep_first or b > last - keep_last]
                others = sorted(set(seen) - set(always), key=lambda b: (-scores[r, h, b], b))
                chosen[r].append(sorted((always + others)[:k_sel]))
    return scores, chosen


def attention_selected(q, row_start, n_ctx, pages, k_pages, v_pages, chosen, scale, **form):
    """attention, where row r and KV head h see the positions of the pages chosen[r][h] alone (a page listed twice counts twice)."""
    hk_n, group = k_pages.shape[1], q.shape[1] // k_pages.shape[1]
    got = dict(out=np.full(q.shape, np.nan), lse=np.full(q.shape[:2], np.nan), mass=np.zeros(q.shape), size=np.zeros(q.shape[:2]))
    slopes, first, end = (form.pop(x, None) for x in ("slopes", "row_first", "row_end"))
    softcap, window = form.pop("softcap", 0.0), form.pop("window", 0)
    assert not form
    for s in range(len(n_ctx)):
        r0, r1 = rows_of(row_start, len(q), s)
        n = min(max(int(n_ctx[s]), 0), pages.shape[1] * BS)
        for r in range(r0, r1):
            p = n - (r1 - r0) + (r - r0)
            hi = p + 1 if end is None else min(int(end[r]), n)
            lo = 0 if first is None else max(0, int(first[r]))
            if window > 0:
                lo = max(lo, p - window + 1)
            for h in range(hk_n):
                j = np.array([b * BS + t for b in chosen[r][h] if 0 <= b < pages.shape[1] for t in range(BS)], int)
                j = j[(j >= lo) & (j < hi)] if p >= 0 else j[:0]
                page = pages[s][j // BS]
                there = (page >= 0) & (page < len(k_pages))
                j, page = j[there], page[there]
                k, v = k_pages[page, h, j % BS], v_pages[page, h, :, j % BS]
                for x in range(h * group, (h + 1) * group):
                    if len(j) == 0:
                        got["out"][r, x], got["lse"][r, x] = 0.0, -np.inf
                        continue
                    z, big = scale * (k @ q[r, x]), scale * (np.abs(k) @ np.abs(q[r, x]))
                    if softcap > 0:
                        z = softcap * np.tanh(z / softcap)
                    if slopes is not None:
                        z, big = z - slopes[x] * np.abs(p - j), big + slopes[x] * np.abs(p - j)
                    e = np.exp(z - z.max())
                    prob = e / e.sum()
                    got["lse"][r, x] = z.max() + np.log(e.sum())
                    got["out"][r, x], got["mass"][r, x] = prob @ v, prob @ np.abs(v)
                    got["size"][r, x] = (big * (prob > 1e-12)).max()
    return got
