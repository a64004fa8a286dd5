"""Inputs of the paged-cache tests: pools, tables and ragged batches, on the host and on the device."""
from __future__ import annotations

import numpy as np
import torch

from paper_2502_13542_amd import harness as H
from paper_2502_13542_amd.synth import LayerShape

BS = 128


def shape_of(hq, hkv, d, dtype):
    return LayerShape(hq, hkv, d, BS, 4, 128, 512, dtype)


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


class Batch:
    """A ragged batch over a pool: seqs is a list of (new rows, tokens in all); a few rows before and behind the sequences'
    belong to nobody, and a few pages to no sequence."""

    def __init__(self, shape, seqs, seed, extra_rows=(0, 0), spare_pages=2, extra_entries=1, garbage=float("nan"), scale=1.0):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.shape, self.seqs, self.batch = shape, seqs, len(seqs)
        td = shape.torch_dtype
        hq, hk, d = shape.n_q_heads, shape.n_kv_heads, shape.head_dim
        counts = [-(-n // BS) for _, n in seqs]
        self.max_pages = max(max(counts), 1) + extra_entries
        self.n_pages = max(sum(counts) + spare_pages, 1)
        order = rng.permutation(self.n_pages).tolist()
        self.pages = np.full((self.batch, self.max_pages), -1, np.int64)
        for s, c in enumerate(counts):
            for i in range(c):
                self.pages[s, i] = order.pop()
        self.free = order
        self.row_start = np.cumsum([extra_rows[0]] + [m for m, _ in seqs])
        self.n_rows = int(self.row_start[-1]) + extra_rows[1]
        self.max_new = max(1, max(m for m, _ in seqs))
        self.n_ctx = np.array([n for _, n in seqs])
        self.k_new, self.v_new = (torch.randn(self.n_rows, hk, d, generator=g).to(td) for _ in range(2))
        self.q = (torch.randn(self.n_rows, hq, d, generator=g) * scale).to(td)
        self.k_pages = torch.randn(self.n_pages, hk, BS, d, generator=g).to(td)
        self.v_pages = torch.randn(self.n_pages, hk, d, BS, generator=g).to(td)
        if garbage is not None:                   # behind the last token, and in pages of nobody
            for p in self.free:
                self.k_pages[p], self.v_pages[p] = garbage, garbage
            for s, (_, n) in enumerate(seqs):
                if n % BS:
                    p = self.pages[s, n // BS]
                    self.k_pages[p, :, n % BS:] = garbage
                    self.v_pages[p, :, :, n % BS:] = garbage

    def positions(self):
        """Position of every row (-1: of nobody)."""
        pos = np.full(self.n_rows, -1)
        for s, (m, n) in enumerate(self.seqs):
            pos[self.row_start[s]: self.row_start[s + 1]] = np.arange(n - m, n)
        return pos

    def dev(self, dev="cuda"):
        i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=dev)
        return dict(row_start=i32(self.row_start), n_ctx=i32(self.n_ctx), pages=i32(self.pages),
                    k_pages=self.k_pages.to(dev), v_pages=self.v_pages.to(dev))

    def runner(self, dev="cuda"):
        return H.PagedRunner(self.shape, self.batch, max(self.n_rows, 1), self.max_new, self.max_pages, dev)

    def pools64(self):
        """The pools with finite numbers where nobody may look."""
        return np.nan_to_num(f64(self.k_pages), nan=0, posinf=0, neginf=0), np.nan_to_num(f64(self.v_pages), nan=0, posinf=0, neginf=0)
