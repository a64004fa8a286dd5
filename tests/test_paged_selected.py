"""Bounds of pages, the selection by them and attention over selected pages against the plain fp64 implementation, on the GPU.

Bounds are keys and the selection is exact: scores are sums in 64 bits rounded to fp32, the same whatever their order (products of fp32
numbers are exact, and a sum of 128 of them is off by 2^-46 of their size: next to a border of fp32 once in some 10^6 scores, so that
scores may differ by a unit of the last place, and then the selection is compared by the scores that the call itself gave).  Attention has the
bounds of attention over all pages (test_paged.py)."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2502_13542_amd import harness as H

from paged_utils import BS, Batch, f64, shape_of
from test_paged import BATCHES, FORMS, SHAPES, check_out, clamped_batch, form_of, on_device

pytestmark = pytest.mark.gpu
DEV = "cuda"


def bounds_of(b, news=None, start=5.0):
    """(on the device, by definition)"""
    t = b.dev()
    sh = b.shape
    bounds = torch.full((b.n_pages, sh.n_kv_heads, 2, sh.head_dim), start, dtype=sh.torch_dtype, device=DEV)
    want = po.key_bounds(b.n_ctx, b.pages, f64(b.k_pages), f64(bounds), news)
    kw = {} if news is None else dict(row_start=t["row_start"], n_rows=b.n_rows)
    b.runner().key_bounds(t["n_ctx"], t["pages"], t["k_pages"], bounds, **kw)
    torch.cuda.synchronize()
    assert np.array_equal(f64(bounds), want)
    return bounds


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("batch", list(BATCHES))
def test_bounds(shape, batch):
    b = Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 3, extra_rows=(1, 2))
    bounds_of(b)
    bounds_of(b, [m for m, _ in b.seqs])


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_bounds_without_pages_and_at_clamped_lengths(shape):
    b = Batch(shape_of(*SHAPES[shape]), BATCHES["chunks"], 5)
    b.pages[0, 1], b.pages[4, 2] = b.n_pages, -1
    bounds_of(b)
    c = clamped_batch(shape)
    bounds_of(c)
    bounds_of(c, [m for m, _ in c.seqs])


def run_select(b, k_sel, first, last, bounds=None, runner=None, more=3, stream=None, **kw):
    t, sh, q = b.dev(), b.shape, b.q.to(DEV)
    bounds = bounds_of(b) if bounds is None else bounds
    shape = (b.n_rows, sh.n_kv_heads)
    scores = torch.full((*shape, b.max_pages + more), 7.0, device=DEV)
    idx, n_sel = torch.full((*shape, k_sel), -7, dtype=torch.int32, device=DEV), torch.full(shape, -7, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    (runner or b.runner()).select_pages(q, t["row_start"], t["n_ctx"], t["pages"], bounds, first, last, scores, idx, n_sel, stream=stream, **kw)
    torch.cuda.synchronize()
    want, chosen = po.select_pages(f64(b.q), b.row_start, b.n_ctx, b.pages, f64(bounds), k_sel, first, last)
    got = scores.cpu().numpy()
    rows = np.arange(b.row_start[0], b.row_start[-1])
    nobody = np.setdiff1d(np.arange(b.n_rows), rows)
    assert (got[nobody] == 7.0).all() and (idx.cpu()[nobody] == -7).all() and (n_sel.cpu()[nobody] == -7).all()
    assert (got[rows][..., b.max_pages:] == 7.0).all()
    got = got[..., : b.max_pages]
    assert np.array_equal(np.isneginf(got[rows]), np.isneginf(want[rows]))
    there = ~np.isneginf(want[rows])
    x, y = got[rows][there], want[rows][there]
    assert (np.abs(x - y) <= np.spacing(np.abs(y))).all(), "a score is off by more than a unit of the last place"
    if not np.array_equal(got[rows], want[rows]):
        chosen = by_scores(b, got, k_sel, first, last)
    for r in rows:
        for h in range(sh.n_kv_heads):
            c = chosen[r][h]
            assert n_sel[r, h] == len(c) and idx[r, h].tolist() == c + [-1] * (k_sel - len(c)), (r, h)
    return idx, n_sel, chosen


def by_scores(b, scores, k_sel, first, last):
    """The selection from given scores."""
    chosen = [None] * b.n_rows
    for r, p in enumerate(b.positions()):
        if b.row_start[0] <= r < b.row_start[-1]:
            end = p // BS if p >= 0 else -1
            chosen[r] = []
            for h in range(scores.shape[1]):
                seen = [i for i in range(end + 1) if not np.isneginf(scores[r, h, i])]
                always = [i for i in seen if i < first or i > end - last]
                chosen[r].append(sorted((always + sorted(set(seen) - set(always), key=lambda i: (-scores[r, h, i], i)))[:k_sel]))
    return chosen


LONG = {"steps": [(1, 2900), (1, 128), (1, 129), (0, 300), (1, 1), (1, 1700)], "drafts": [(4, 2000), (3, 131), (1, 900)],
        "chunk": [(140, 1500), (1, 700), (20, 20)]}


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("batch", list(LONG))
@pytest.mark.parametrize("k_sel,first,last", [(1, 0, 0), (5, 1, 2), (8, 0, 1), (40, 3, 3), (2, 1, 1)])
def test_select(shape, batch, k_sel, first, last):
    run_select(Batch(shape_of(*SHAPES[shape]), LONG[batch], 7, extra_rows=(1, 2)), k_sel, first, last)


@pytest.mark.parametrize("shape", ["llama", "fp32_64", "mha64"])
@pytest.mark.parametrize("kind", ["equal", "zeros", "few"])
def test_select_of_equal_scores(shape, kind):
    """Pages with the same bounds, rows of zeros (every score is 0, of either sign), few different values: the lower page."""
    b = Batch(shape_of(*SHAPES[shape]), LONG["drafts"], 9, garbage=None)
    sh = b.shape
    bounds = torch.randn(b.n_pages, sh.n_kv_heads, 2, sh.head_dim).sort(2).values.to(sh.torch_dtype)
    if kind == "equal":
        bounds[:] = bounds[:1]
    if kind == "zeros":
        b.q[::2] = 0
        b.q[1::2] = -0.0
    if kind == "few":
        bounds = bounds[torch.arange(b.n_pages) % 3].contiguous()
    run_select(b, 6, 1, 1, bounds.to(DEV))


def beyond_fp32(b, seed):
    """Queries and bounds whose products, of up to 9 x 2^127, cancel in pairs, and two channels of small ones left: exact in 64 bits in any order."""
    d, g = b.shape.head_dim, torch.Generator().manual_seed(seed)
    ints = lambda *n: torch.randint(-3, 4, n, generator=g).double()
    q, k = ints(*b.q.shape[:2], d // 2) * 2.0**64, ints(b.n_pages, b.shape.n_kv_heads, 1, d // 2) * 2.0**63
    q, k = torch.cat([q, -q], -1), torch.cat([k, k], -1)
    for c in (0, d // 2):
        q[..., c] = ints(*b.q.shape[:2]) * 2.0**40
    b.q = q.to(b.q.dtype)
    return k.expand(-1, -1, 2, -1).to(b.q.dtype).contiguous().to(DEV)


@pytest.mark.parametrize("shape", ["llama", "fp32_64", "mha64"])
def test_select_by_products_beyond_fp32(shape):
    b = Batch(shape_of(*SHAPES[shape]), LONG["drafts"], 19, garbage=None)
    run_select(b, 5, 1, 1, beyond_fp32(b, 19))


WIDE = 3000                # entries of a table whose calls by many rows take the matrix instruction


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("kind", ["random", "beyond", "few", "zeros", "none"])
def test_select_of_many_rows(shape, kind):
    seqs = LONG["chunk"] + [(0, 300), (33, 33), (16, 2100)]
    b = Batch(shape_of(*SHAPES[shape]), seqs, 41, extra_rows=(1, 2), extra_entries=WIDE, **({} if kind in ("random", "none") else dict(garbage=None)))
    sh, bounds = b.shape, None
    if kind == "beyond":
        bounds = beyond_fp32(b, 23)
    elif kind in ("few", "zeros"):
        bounds = torch.randn(b.n_pages, sh.n_kv_heads, 2, sh.head_dim, generator=torch.Generator().manual_seed(3)).sort(2).values.to(sh.torch_dtype)
        bounds = bounds[torch.arange(b.n_pages) % 3].contiguous().to(DEV)
    if kind == "zeros":
        b.q[::2] = 0
        b.q[1::2] = -0.0
    if kind == "none":
        b.pages[0, [0, 3, 11]], b.pages[1, 5], b.pages[5, 15] = -1, b.n_pages, -7
    run_select(b, 6, 1, 1, bounds)


def test_select_of_many_rows_at_clamped_lengths():
    """Some rows at negative positions, lengths beyond the table."""
    b = Batch(shape_of(*SHAPES["llama"]), [(140, 300), (120, 140), (64, 64)], 43, extra_entries=WIDE, garbage=None)
    raw = torch.tensor([100, (b.max_pages + 5) * BS, 64], dtype=torch.int32, device=DEV)
    b.n_ctx = np.array([100, b.max_pages * BS, 64])
    b.seqs = [(m, n) for (m, _), n in zip(b.seqs, b.n_ctx)]
    b.dev = lambda dev=DEV: dict(Batch.dev(b, dev), n_ctx=raw.clone())
    run_select(b, 4, 1, 1)


def test_select_without_pages_and_at_clamped_lengths():
    b = Batch(shape_of(*SHAPES["llama"]), LONG["chunk"], 11)
    b.pages[0, [0, 3, 11]], b.pages[1, 5] = -1, b.n_pages
    run_select(b, 6, 1, 2)
    run_select(clamped_batch("llama"), 2, 0, 1)


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_select_from_many_pages(shape):
    """More pages than a workgroup has threads, and a table far wider than the sequence."""
    sh = shape_of(*((4, 1, 128, "bf16") if shape == "llama" else (4, 1, 64, "fp32")))
    run_select(Batch(sh, [(2, 90000), (1, 40000)], 13, extra_entries=0, garbage=None), 64, 1, 4)
    run_select(Batch(sh, [(2, 1000), (1, 33000)], 15, extra_entries=3000, garbage=None), 300, 0, 0)


@pytest.mark.parametrize("layer", [(4, 1, 64, "bf16"), (2, 2, 64, "fp32")])
@pytest.mark.parametrize("k_sel,first,last", [(64, 1, 4), (1500, 0, 0), (7, 0, 0)])
@pytest.mark.parametrize("kind", ["random", "equal"])
def test_select_from_more_pages_than_threads_hold_keys(layer, k_sel, first, last, kind):
    """More than 1024 visible pages: the scores are read again in each round."""
    b = Batch(shape_of(*layer), [(2, 150000), (1, 131073), (1, 131072)], 16, extra_entries=1, garbage=None)
    bounds = torch.randn(b.n_pages, layer[1], 2, layer[2], generator=torch.Generator().manual_seed(1)).sort(2).values.to(b.shape.torch_dtype)
    if kind == "equal":
        bounds = bounds[torch.arange(b.n_pages) % 3].contiguous()
    run_select(b, k_sel, first, last, bounds.to(DEV))


@pytest.mark.parametrize("layer", [(8, 1, 128, "bf16"), (7, 1, 64, "fp32"), (48, 6, 64, "bf16"), (5, 1, 128, "fp32")])
def test_other_groups(layer):
    b = Batch(shape_of(*layer), LONG["drafts"], 18, extra_rows=(1, 1))
    run_select(b, 5, 1, 1)
    run_selected(b, some_pages(b, 6, 4), 6, "all", 5)


def test_bounds_of_more_pages_than_a_launch_has_workgroups_for():
    sh = shape_of(1, 1, 64, "bf16")
    max_pages = 33000
    k = torch.randn(max_pages, 1, BS, 64, dtype=torch.bfloat16, device=DEV)
    bounds = torch.zeros(max_pages, 1, 2, 64, dtype=torch.bfloat16, device=DEV)
    pages = torch.randperm(max_pages, device=DEV).int()[None].contiguous()
    n = torch.tensor([max_pages * BS - 5], dtype=torch.int32, device=DEV)
    H.PagedRunner(sh, 1, 1, 1, max_pages).key_bounds(n, pages, k, bounds)
    torch.cuda.synchronize()
    k[pages[0, -1].long(), :, -5:] = k[pages[0, -1].long(), :, :1]
    assert torch.equal(bounds[:, :, 0], k.amin(2)) and torch.equal(bounds[:, :, 1], k.amax(2))


def run_selected(b, chosen, k_sel, kind="plain", seed=0, runner=None, garbage=True, **kw):
    """Attention over given lists; what is behind n_sel in a list is anything."""
    f = form_of(b, kind, seed)
    t, sh, q = b.dev(), b.shape, b.q.to(DEV)
    rng = np.random.default_rng(seed)
    idx = rng.integers(-3, b.max_pages + 3, (b.n_rows, sh.n_kv_heads, k_sel)) if garbage else np.full((b.n_rows, sh.n_kv_heads, k_sel), -1)
    n_sel = np.zeros((b.n_rows, sh.n_kv_heads), int)
    for r, of_row in enumerate(chosen):
        for h, c in enumerate(of_row or []):
            idx[r, h, : len(c)], n_sel[r, h] = c, len(c)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((b.n_rows, sh.n_q_heads), 7.0, device=DEV)
    (runner or b.runner()).attend_selected(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], i32(idx), i32(n_sel), out,
                                           lse, **on_device(f), **kw)
    torch.cuda.synchronize()
    k, v = b.pools64()
    want = po.attention_selected(f64(b.q), b.row_start, b.n_ctx, b.pages, k, v, chosen, sh.head_dim ** -0.5, **f)
    rows = np.arange(b.row_start[0], b.row_start[-1])
    check_out(b, want, out, lse, rows)
    nobody = np.setdiff1d(np.arange(b.n_rows), rows)
    assert (f64(out)[nobody] == 7.0).all() and (f64(lse)[nobody] == 7.0).all(), "rows of nobody were written"
    return out, lse, want


def some_pages(b, k_sel, seed):
    """For every row and KV head some of the pages that the row sees, of some none."""
    rng = np.random.default_rng(seed)
    chosen = [None] * b.n_rows
    for s, (m, n) in enumerate(b.seqs):
        for i in range(m):
            last = max(n - m + i, 0) // BS
            chosen[b.row_start[s] + i] = [sorted(rng.permutation(last + 1)[: rng.integers(0, min(k_sel, last + 1) + 1)].tolist())
                                          for _ in range(b.shape.n_kv_heads)]
    return chosen


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("batch", list(LONG))
def test_selected(shape, batch):
    b = Batch(shape_of(*SHAPES[shape]), LONG[batch], 17, extra_rows=(2, 1))
    run_selected(b, some_pages(b, 9, 1), 9)


@pytest.mark.parametrize("kind", [k for k in FORMS if k != "plain"])
@pytest.mark.parametrize("shape", ["llama", "fp32_64", "g5_64", "fp32_g3"])
def test_selected_forms(shape, kind):
    b = Batch(shape_of(*SHAPES[shape]), LONG["drafts"], 19, garbage=float("inf"), scale=2.0)
    run_selected(b, some_pages(b, 16, 2), 16, kind, 3)


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_selected_without_pages_and_at_clamped_lengths(shape):
    b = Batch(shape_of(*SHAPES[shape]), LONG["drafts"], 21)
    b.pages[0, [0, 3, 11]], b.pages[1, 0] = -1, b.n_pages
    chosen = some_pages(b, 6, 3)
    chosen[0][0], chosen[1][0], chosen[2][0] = [2, 5], [0, 3], []
    chosen[3][0] = [-5, -1, 4, 2 ** 30, 2 ** 31 - 1]
    run_selected(b, chosen, 6)
    c = clamped_batch(shape)
    c.positions = lambda: Batch.positions(c)
    run_selected(c, [[[0, 1]] * c.shape.n_kv_heads if c.row_start[0] <= r < c.row_start[-1] else None for r in range(c.n_rows)], 2)


# Calls that the chunks' kernels take, in every cut of theirs (128 pages a row: reading every list takes far longer); tables wider than the sequences
CHUNKS = [("llama", [(300, 2600), (64, 700), (1, 300), (0, 5), (130, 130)], 0, 128), ("g7", [(100, 5000), (70, 900)], 3, 128), ("mha64", [(500, 4000), (300, 300)], 0, 128),
          ("g8_64", [(260, 6000)], 30, 128), ("fp32_64", [(300, 2600), (64, 700), (1, 300)], 0, 128), ("fp32_g3", [(200, 3000), (3, 500)], 0, 128),
          ("fp32_g8", [(130, 3300)], 9, 128), ("g5_64", [(128, 9000), (40, 4200)], 0, 128)]


@pytest.mark.parametrize("case", range(len(CHUNKS)))
@pytest.mark.parametrize("kind", ["plain", "cap", "slopes", "all", "first", "window"])
def test_selected_of_chunks(case, kind):
    shape, seqs, more, k_sel = CHUNKS[case]
    b = Batch(shape_of(*SHAPES[shape]), seqs, 31 + case, extra_rows=(2, 1), extra_entries=more)
    if kind == "plain":
        b.pages[0, 3], b.pages[0, 1] = -1, b.n_pages
    chosen = some_pages(b, min(k_sel, 9), 8)
    for r in range(0, b.n_rows, 5):
        if chosen[r] is not None:
            chosen[r][0] = list(range(max(b.positions()[r], 0) // BS + 1))       # all that the row sees
    run_selected(b, chosen, k_sel, kind, 9)


def test_selected_of_chunks_takes_the_kernels_of_chunks():
    """The same call with rows few enough for lists, and with many: within the same bounds (as above), and the second one far less than its lists."""
    sh = shape_of(*SHAPES["llama"])
    b = Batch(sh, [(256, 8000)], 33, garbage=None)
    every = [[list(range(p // BS + 1))] * sh.n_kv_heads for p in b.positions()]
    t, q, r = b.dev(), b.q.to(DEV), b.runner()
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    idx = i32([[h + [-1] * (b.max_pages - len(h)) for h in row] for row in every])
    n_sel = (idx >= 0).sum(-1).int()
    outs = [torch.zeros_like(q) for _ in range(2)]
    r.attend_selected(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], idx, n_sel, outs[0])
    r.attend(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], outs[1])
    torch.cuda.synchronize()
    assert torch.equal(*outs)                     # (all pages selected: the chunks' attention, bit for bit)


@pytest.mark.parametrize("shape", ["llama", "fp32_g3", "g7"])
def test_all_pages_selected_is_attention(shape):
    b = Batch(shape_of(*SHAPES[shape]), [(1, 5003), (2, 2000), (1, 77)], 23)
    every = [[list(range(p // BS + 1))] * b.shape.n_kv_heads for p in b.positions()]
    out, lse, _ = run_selected(b, every, b.max_pages)
    t, q = b.dev(), b.q.to(DEV)
    dense, dense_lse = torch.zeros_like(q), torch.zeros_like(lse)
    b.runner().attend(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], dense, dense_lse)
    torch.cuda.synchronize()
    assert (f64(lse) - f64(dense_lse)).__abs__().max() < 1e-5


@pytest.mark.parametrize("shape,n", [("g7", 44), ("llama", 40), ("mha64", 90), ("fp32_64", 130), ("fp32_g3", 200)])
@pytest.mark.parametrize("kind,k_sel", [("plain", 3), ("cap", 6), ("slopes", 3), ("all", 12)])
def test_selected_of_many_short_sequences(shape, n, kind, k_sel):
    """More (row, KV head) pairs than compute units, of few pages: smaller workgroups."""
    b = Batch(shape_of(*SHAPES[shape]), [(1 + (i % 5 == 2), 2 + 97 * i % 724) for i in range(n)], 29, garbage=float("inf"))
    run_selected(b, some_pages(b, k_sel, 7), k_sel, kind, 5)


def test_more_rows_than_counters():
    """More (row, KV head) pairs than the workspace has counters: a workgroup each."""
    b = Batch(shape_of(16, 8, 64, "bf16"), [(1, 300)] * 60 + [(90, 400)], 25, extra_entries=0)
    run_selected(b, some_pages(b, 3, 5), 3)


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_a_sparse_step_as_it_is_used(shape):
    """Append with rotation, bounds of the pages with new tokens, selection, attention: a prompt, then steps and drafts; in a graph too."""
    sh = shape_of(*SHAPES[shape])
    g = torch.Generator().manual_seed(27)
    from test_paged_rotated import bound_of, table_of
    batch, max_pages, n_pages, k_sel = 3, 9, 30, 4
    pages = np.random.default_rng(3).permutation(n_pages)[: batch * max_pages].reshape(batch, max_pages)
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)
    r = H.PagedRunner(sh, batch, 1500, 900, max_pages)
    kp = torch.full((n_pages, sh.n_kv_heads, BS, sh.head_dim), float("nan"), dtype=sh.torch_dtype, device=DEV)
    vp = torch.full((n_pages, sh.n_kv_heads, sh.head_dim, BS), float("nan"), dtype=sh.torch_dtype, device=DEV)
    bounds = torch.full((n_pages, sh.n_kv_heads, 2, sh.head_dim), float("nan"), dtype=sh.torch_dtype, device=DEV)
    table, pages_d = table_of(64, 1200).to(DEV), i32(pages)
    n_ctx = np.zeros(batch, int)
    graph = None
    for news in [(900, 130, 5), (1, 1, 1), (1, 4, 2), (2, 2, 2), (2, 2, 2), (2, 2, 2)]:
        n_rows, start = sum(news), np.cumsum([0, *news])
        n_ctx = n_ctx + np.array(news)
        k_new, v_new = (torch.randn(n_rows, sh.n_kv_heads, sh.head_dim, generator=g).to(sh.torch_dtype) for _ in range(2))
        q = torch.randn(n_rows, sh.n_q_heads, sh.head_dim, generator=g).to(sh.torch_dtype)
        shape2 = (n_rows, sh.n_kv_heads)
        if news != (2, 2, 2) or graph is None:
            x = dict(k=k_new.to(DEV), v=v_new.to(DEV), q=q.to(DEV), start=i32(start), n=i32(n_ctx), scores=torch.zeros(*shape2, max_pages, device=DEV),
                     idx=torch.zeros(*shape2, k_sel, dtype=torch.int32, device=DEV), n_sel=torch.zeros(shape2, dtype=torch.int32, device=DEV))
            x["out"], x["lse"] = torch.zeros_like(x["q"]), torch.zeros(n_rows, sh.n_q_heads, device=DEV)
        else:
            for name, y in (("k", k_new), ("v", v_new), ("q", q), ("n", i32(n_ctx))):
                x[name].copy_(y)

        def step():
            call = (x["start"], x["n"], pages_d)
            r.append_rotated(x["k"], x["v"], *call, kp, vp, table, q=x["q"], q_out=x["q"], max_new=max(news))
            r.key_bounds(x["n"], pages_d, kp, bounds, row_start=x["start"], n_rows=n_rows, max_new=max(news))
            r.select_pages(x["q"], *call, bounds, 1, 1, x["scores"], x["idx"], x["n_sel"], max_new=max(news))
            r.attend_selected(x["q"], *call, kp, vp, x["idx"], x["n_sel"], x["out"], x["lse"], max_new=max(news))

        if graph is not None:
            graph.replay()
        else:
            step()
            torch.cuda.synchronize()
            if news == (2, 2, 2):                 # (captured once it has run; captured, it does nothing)
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    step()
        torch.cuda.synchronize()
        # what the cache holds, and what follows from it
        k64, v64 = (np.nan_to_num(f64(y), nan=0.0) for y in (kp, vp))
        q_now = f64(x["q"])
        places = np.concatenate([np.arange(n - m, n) for n, m in zip(n_ctx, news)])
        turned, size = po.rotate(f64(k_new), f64(table), places, False)
        for s in range(batch):
            for i in range(news[s]):
                p = n_ctx[s] - news[s] + i
                off = np.abs(k64[pages[s, p // BS], :, p % BS] - turned[start[s] + i])
                assert (off <= bound_of(sh.dtype, turned[start[s] + i], size[start[s] + i])).all()
                assert np.array_equal(v64[pages[s, p // BS], :, :, p % BS], f64(v_new)[start[s] + i])
        want_bounds = po.key_bounds(n_ctx, pages, f64(kp), np.full(bounds.shape, np.nan))
        assert np.array_equal(f64(bounds), want_bounds, equal_nan=True)
        b = type("B", (), dict(shape=sh, n_ctx=n_ctx, n_rows=n_rows, row_start=start, positions=lambda: places))
        chosen = by_scores(b, x["scores"].cpu().numpy(), k_sel, 1, 1)
        scores, _ = po.select_pages(q_now, start, n_ctx, pages, np.nan_to_num(want_bounds), k_sel, 1, 1)
        got = x["scores"].cpu().numpy()
        assert np.allclose(np.nan_to_num(got, neginf=-9), np.nan_to_num(scores, neginf=-9), rtol=2.0 ** -22, atol=0)
        assert [[x["idx"][i, h, : x["n_sel"][i, h]].tolist() for h in range(sh.n_kv_heads)] for i in range(n_rows)] == chosen
        want = po.attention_selected(q_now, start, n_ctx, pages, k64, v64, chosen, sh.head_dim ** -0.5)
        check_out(b, want, x["out"], x["lse"], np.arange(n_rows))


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_selected_twice_the_same_bits_two_streams_and_a_larger_runner(shape):
    b = Batch(shape_of(*SHAPES[shape]), [(1, 5000), (2, 3000)], 29)
    chosen = some_pages(b, 30, 7)
    made_for = H.PagedRunner(b.shape, 4, 300, 200, b.max_pages + 5)
    out, lse, _ = run_selected(b, chosen, 30, seed=1)
    for kw in (dict(runner=made_for), dict(runner=made_for, stream=torch.cuda.Stream(), max_new=2), {}):
        torch.cuda.synchronize()
        again = run_selected(b, chosen, 30, seed=1, **kw)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    run_select(b, 7, 1, 1, runner=made_for, stream=torch.cuda.Stream())


@pytest.mark.parametrize("shape", ["llama", "fp32_g3"])
def test_pages_past_32_bits(shape):
    sh = shape_of(*SHAPES[shape])
    b = Batch(sh, [(1, 300), (2, 140)], 97, garbage=None)
    r, t = b.runner(), b.dev()
    page = sh.n_kv_heads * BS * sh.head_dim
    n_far = 2 ** 31 // page + 40
    move = torch.tensor([n_far - 1 - 7 * i for i in range(b.n_pages)], device=DEV)
    far = dict(t, pages=torch.where(t["pages"] >= 0, move[t["pages"].clamp(min=0).long()].int(), -1).contiguous())
    for name in ("k_pages", "v_pages"):
        pool = torch.empty(n_far, *t[name].shape[1:], dtype=t[name].dtype, device=DEV)
        pool[move] = t[name]
        far[name] = pool
    got, q = [], b.q.to(DEV)
    from test_paged_rotated import table_of
    table = table_of(64, 400).to(DEV)
    for x in (t, far):
        call = (x["row_start"], x["n_ctx"], x["pages"])
        bounds = torch.zeros(len(x["k_pages"]), sh.n_kv_heads, 2, sh.head_dim, dtype=sh.torch_dtype, device=DEV)
        scores, idx = torch.zeros(b.n_rows, sh.n_kv_heads, b.max_pages, device=DEV), torch.zeros(b.n_rows, sh.n_kv_heads, 2, dtype=torch.int32, device=DEV)
        n_sel, out, lse = torch.zeros(b.n_rows, sh.n_kv_heads, dtype=torch.int32, device=DEV), torch.zeros_like(q), torch.zeros(b.n_rows, sh.n_q_heads, device=DEV)
        r.append_rotated(b.k_new.to(DEV), b.v_new.to(DEV), *call, x["k_pages"], x["v_pages"], table)
        r.key_bounds(x["n_ctx"], x["pages"], x["k_pages"], bounds)
        r.select_pages(q, *call, bounds, 0, 1, scores, idx, n_sel)
        r.attend_selected(q, *call, x["k_pages"], x["v_pages"], idx, n_sel, out, lse)
        torch.cuda.synchronize()
        at = slice(None) if x is t else move
        got.append((out, lse, idx, n_sel, scores, bounds[at], x["k_pages"][at], x["v_pages"][at]))
    assert all(torch.equal(x, y) for x, y in zip(*got))
