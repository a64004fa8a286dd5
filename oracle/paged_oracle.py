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
