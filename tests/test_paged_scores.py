"""The selection's two ways to its scores, row by row and by the matrix instruction, against each other."""
import numpy as np
import pytest
import torch

from paper_2502_13542_amd import binding as B
from paper_2502_13542_amd import harness as H

from paged_utils import Batch, shape_of
from test_paged import SHAPES
from test_paged_selected import by_scores

DEV = "cuda"


@pytest.mark.gpu
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("values", ["exact", "any"])
def test_rows_are_scored_alike_by_both_ways(shape, values):
    """The same rows in chunks, scored by the matrix instruction, and each as a sequence of its own, scored row by row.  Of values whose products and sums 64
    bits hold (multiples of 2^-6 up to 4: of 2^-12 up to 2^11) the scores and the selection are equal; of others each sum of 128 exact products is
    off by at most 2^-46 of the size S of its terms and then rounded to fp32, so that two differ by a unit of the last place and 2^-45 S at most, and the
    selections are those of the scores."""
    sh, k_sel, first, last = shape_of(*SHAPES[shape]), 7, 1, 2
    seqs = [(400, 9000), (170, 3000), (33, 33), (1, 700)]
    more = 0 if sh.n_q_heads * sh.head_dim > 2000 else 1500
    b = Batch(sh, seqs, 61, extra_entries=more, garbage=None)
    g = torch.Generator().manual_seed(62)
    grid = (lambda *n: torch.randint(-256, 257, n, generator=g) / 64.0) if values == "exact" else (lambda *n: torch.randn(n, generator=g))
    q = grid(b.n_rows, sh.n_q_heads, sh.head_dim).to(sh.torch_dtype)
    if values == "exact" and sh.dtype == "bf16":
        assert torch.equal(q.float() * 64, (q.float() * 64).round())
    bounds = grid(b.n_pages, sh.n_kv_heads, 2, sh.head_dim).sort(2).values.to(sh.torch_dtype).to(DEV)
    b.pages[0, 5] = b.n_pages
    places = b.positions()
    seq_of = np.repeat(np.arange(b.batch), [m for m, _ in seqs])
    t = b.dev()
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)
    ways = [(t["row_start"], t["n_ctx"], t["pages"], b.batch, b.max_new),
            (i32(np.arange(b.n_rows + 1)), i32(places + 1), t["pages"][torch.tensor(seq_of, device=DEV)].contiguous(), b.n_rows, 1)]
    got = []
    for i, (start, n_ctx, pages, batch, max_new) in enumerate(ways):
        assert B.paged_cut(B.c_shape(sh), "select_pages", batch, b.n_rows, max_new, b.max_pages)[0] == (16 if i == 0 else 1)
        scores = torch.full((b.n_rows, sh.n_kv_heads, b.max_pages), 7.0, device=DEV)
        idx, n_sel = torch.full((b.n_rows, sh.n_kv_heads, k_sel), -7, dtype=torch.int32, device=DEV), torch.full((b.n_rows, sh.n_kv_heads), -7, dtype=torch.int32, device=DEV)
        H.PagedRunner(sh, batch, b.n_rows, max_new, b.max_pages).select_pages(q.to(DEV), start, n_ctx, pages, bounds, first, last, scores, idx, n_sel)
        torch.cuda.synchronize()
        got.append((scores.cpu(), idx.cpu(), n_sel.cpu()))
        chosen = by_scores(b, got[-1][0].numpy(), k_sel, first, last)
        for r in range(0, b.n_rows, 7):
            for h in range(sh.n_kv_heads):
                assert idx[r, h].tolist() == chosen[r][h] + [-1] * (k_sel - len(chosen[r][h])) and n_sel[r, h] == len(chosen[r][h])
    if values == "exact":
        assert all(torch.equal(x, y) for x, y in zip(*got))
    else:
        x, y = (s[0].numpy() for s in got)
        there = ~np.isneginf(x)
        size = (q.abs().double().sum(-1).reshape(b.n_rows, sh.n_kv_heads, -1).amax(-1) * bounds.abs().max().item()).numpy()[..., None]
        assert np.array_equal(there, ~np.isneginf(y))
        bound = np.spacing(np.maximum(np.abs(np.where(there, x, 1)), np.abs(np.where(there, y, 1)))) + 2.0 ** -45 * size
        assert (np.abs(x[there].astype(np.float64) - y[there]) <= bound[there]).all()
