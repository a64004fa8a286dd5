"""Every way in which attention of chunks over pages in 8 bits and over selected pages is cut up: the cut of each case is asserted on the host (so that
figures which change it are noticed here), and the case runs in it on the GPU, against the plain fp64 implementation."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2502_13542_amd import binding as B

from paged_utils import BS, Batch, f64, shape_of
from test_paged import FORMS, SHAPES, check_out, form_of, on_device

DEV = "cuda"
KINDS = ["plain", "cap", "slopes", "cap_slopes_end"]
LISTS = 128                                        # entries of a row's list of pages (most are behind its last)


def ragged(batch, m, n):
    """Sequences of which the first has the full sizes, and a step at the end."""
    return [(m - 3 * s, n - 70 * s) for s in range(batch)] + [(1, n // 2)]


def sizes_of(seqs, more):
    return len(seqs), sum(m for m, _ in seqs), max(m for m, _ in seqs), max(-(-n // BS) for _, n in seqs) + more


# layer, sequences, entries of the table behind the longest, (wavefronts that share a page, pieces) over 8 bits and over selected pages.  At
# least four pages in a piece, of the last two more than 64.
CASES = [((64, 32, 64), (5, 90, 900), 5, (1, 1), (1, 1)),
         ((64, 32, 64), (2, 130, 900), 60, (1, 2), (1, 2)),
         ((64, 32, 64), (5, 40, 900), 20, (2, 1), (2, 1)),
         ((64, 32, 64), (3, 40, 900), 60, (2, 2), (2, 2)),
         ((3, 3, 64), (1, 600, 700), 0, (4, 1), (4, 1)),
         ((3, 3, 64), (8, 40, 4000), 0, (4, 8), (4, 8)),
         ((128, 32, 128), (5, 40, 900), 60, (1, 1), (4, 1)),
         ((128, 32, 128), (5, 40, 900), 0, (1, 1), (1, 1)),
         ((64, 32, 128), (3, 90, 900), 150, (1, 2), (1, 2)),
         ((128, 32, 128), (3, 40, 700), 0, (2, 1), (2, 1)),
         ((128, 32, 128), (1, 60, 900), 20, (2, 2), (2, 2)),
         ((64, 32, 128), (1, 40, 700), 0, (4, 1), (4, 1)),
         ((64, 32, 128), (1, 60, 900), 5, (4, 2), (4, 2)),
         ((64, 32, 64), (3, 200, 9000), 0, (1, 1), (1, 1)),
         ((64, 16, 128), (3, 200, 9000), 0, (1, 1), (1, 1))]


def cut_of(call, layer, seqs, more, kind="plain", dtype="bf16", **kw):
    f = FORMS[kind]
    return B.paged_cut(B.c_shape(shape_of(*layer, dtype)), call, *sizes_of(seqs, more), softcap=f.get("softcap", 0.0), window=f.get("window", 0),
                       documents=f.get("first", False), **kw)


@pytest.mark.parametrize("call", ["attention_quantised", "attention_selected"])
def test_the_cases_are_all_cuts_of_chunks(call):
    found = set()
    for layer, seqs, more, quantised, selected in CASES:
        want = quantised if call == "attention_quantised" else selected
        for kind in KINDS:
            got = cut_of(call, layer, ragged(*seqs), more, kind, k_sel=LISTS)
            assert got == (256 // want[0], *want), (layer, seqs, kind)
        found.add((layer[2], want[0], want[1] > 1))
    assert found == {(d, ks, cut) for d in (64, 128) for ks in (1, 2, 4) for cut in (False, True)}


@pytest.mark.parametrize("bad,code", [(dict(call=-1), -1), (dict(call=6), -1), (dict(batch=0), -1), (dict(max_new=0), -1), (dict(max_new=10), -1),
                                      (dict(max_pages=0), -1), (dict(call=2, k_sel=0), -1), (dict(n_rows=2 ** 22 + 1), -2), (dict(cut=None), -1)])
def test_cuts_refused(bad, code):
    cut = (ctypes.c_int32 * 3)(7, 7, 7)
    a = dict(call=0, batch=2, n_rows=9, max_new=5, max_pages=4, k_sel=4, queries=0, softcap=0.0, window=0, documents=0, cut=cut)
    a.update(bad)
    cs = B.c_shape(shape_of(32, 8, 128, "bf16"))
    assert B.load_library().actqkv_paged_cut(ctypes.byref(cs), *a.values()) == code
    assert list(cut) == [7, 7, 7]


def test_cuts_of_few_rows_and_of_lists():
    """Steps take the kernels of few rows, rows of short lists read those; fp32 has one kind of workgroup; a window and documents shorten what is cut."""
    assert cut_of("attention", (32, 8, 128), [(4, 900)] * 3, 0) == (0, 0, 0) == cut_of("attention_quantised", (8, 2, 64), [(1, 900)], 0, dtype="fp32")
    assert cut_of("attention_selected", (32, 8, 128), [(5, 900)], 0, k_sel=1) == (0, 0, 0)
    assert cut_of("attention_quantised", (8, 2, 64), [(300, 4000)], 0, dtype="fp32")[:2] == (128, 1)
    whole, window = (cut_of("attention", (32, 8, 128), [(300, 9000)], 0, kind)[2] for kind in ("plain", "window"))
    assert whole > window >= 1


def reference(b, k, v, form, chosen=None):
    """What po.attention and po.attention_selected give, by products in 64 bits on the pools' device; chosen: of a row and KV head the pages (bool)."""
    sh, dev = b.shape, k.device
    group, scale = sh.group, sh.head_dim ** -0.5
    q = b.q.to(dev).double()
    got = dict(out=torch.zeros_like(q), lse=torch.full(q.shape[:2], -torch.inf, dtype=q.dtype, device=dev), mass=torch.zeros_like(q),
               size=torch.zeros(q.shape[:2], dtype=q.dtype, device=dev))
    slopes, first, end = (form.get(x) for x in ("slopes", "row_first", "row_end"))
    assert set(form) <= {"slopes", "row_first", "row_end", "softcap", "window"}
    for s, (m, n) in enumerate(b.seqs):
        rows = slice(int(b.row_start[s]), int(b.row_start[s]) + m)
        if m == 0 or n == 0:
            continue
        page = torch.tensor(b.pages[s], device=dev)
        j, p = torch.arange(n, device=dev), torch.arange(n - m, n, device=dev)
        lo = torch.zeros_like(p) if first is None else torch.tensor(first[rows], device=dev)
        hi = p + 1 if end is None else torch.tensor(end[rows], device=dev).clamp(max=n)
        if form.get("window"):
            lo = torch.maximum(lo, p - form["window"] + 1)
        seen = (j >= lo[:, None]) & (j < hi[:, None]) & ((page >= 0) & (page < len(k)))[j // BS]
        at, slot = page[j // BS].clamp(0, len(k) - 1), j % BS
        far = (p[:, None] - j).abs().double()
        for h in range(sh.n_kv_heads):
            here = seen if chosen is None else seen & chosen[rows, h][:, j // BS]
            kh, vh = k[at, h, slot], v[at, h, :, slot]
            for x in range(h * group, (h + 1) * group):
                z, big = scale * (q[rows, x] @ kh.t()), scale * (q[rows, x].abs() @ kh.abs().t())
                if form.get("softcap", 0.0) > 0:
                    z = form["softcap"] * torch.tanh(z / form["softcap"])
                if slopes is not None:
                    z, big = z - float(slopes[x]) * far, big + float(slopes[x]) * far
                z = z.masked_fill(~here, -torch.inf)
                norm = torch.logsumexp(z, 1)
                prob = torch.exp(z - torch.where(norm.isinf(), 0.0, norm)[:, None])
                got["out"][rows, x], got["mass"][rows, x], got["lse"][rows, x] = prob @ vh, prob @ vh.abs(), norm
                got["size"][rows, x] = (big * (prob > 1e-12)).amax(1)
    return {name: x.cpu().numpy() for name, x in got.items()}


def some_pages(b, seed):
    """Of every row and KV head the pages that it looks at, as lists and as truth values: of most rows a few, of some none, of some all that they see."""
    g = torch.Generator().manual_seed(seed)
    hk = b.shape.n_kv_heads
    last = torch.tensor(np.maximum(b.positions(), -1)) // BS
    seen = torch.arange(b.max_pages) <= last[:, None]
    share = torch.rand(b.n_rows, hk, 1, generator=g)
    share = torch.where(share < 0.15, 0.0, torch.where(share > 0.85, 1.0, 0.4))
    chosen = (torch.rand(b.n_rows, hk, b.max_pages, generator=g) < share) & seen[:, None]
    place = chosen.int().cumsum(-1) - 1
    idx = torch.randint(-3, b.max_pages + 3, (b.n_rows, hk, LISTS), generator=g).int()       # behind n_sel: anything
    r, h, i = chosen.nonzero(as_tuple=True)
    idx[r, h, place[r, h, i].long()] = i.int()
    return idx, chosen.sum(-1).int(), chosen


def test_the_reference_is_the_oracle():
    for kind in ("plain", "all"):
        b = Batch(shape_of(4, 2, 64, "fp32"), [(30, 700), (1, 129), (0, 10), (5, 5)], 3)
        b.pages[0, 1] = b.n_pages
        k, v = b.pools64()
        f = form_of(b, kind, 3)
        idx, n_sel, chosen = some_pages(b, 5)
        lists = [[idx[r, h, : n_sel[r, h]].tolist() for h in range(2)] for r in range(b.n_rows)]
        for want, got in ((po.attention(f64(b.q), b.row_start, b.n_ctx, b.pages, k, v, 64 ** -0.5, **f), reference(b, torch.tensor(k), torch.tensor(v), f)),
                          (po.attention_selected(f64(b.q), b.row_start, b.n_ctx, b.pages, k, v, lists, 64 ** -0.5, **f),
                           reference(b, torch.tensor(k), torch.tensor(v), f, chosen))):
            assert all(np.allclose(got[x], want[x], rtol=1e-11, atol=1e-13) for x in ("out", "lse", "mass", "size"))


def finite(x):
    return torch.nan_to_num(x.double(), nan=0.0, posinf=0.0, neginf=0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("kind", KINDS)
def test_attention_over_8_bits_in_every_cut(case, kind):
    from test_paged_quantised import pools8, quantise
    layer, seqs, more, _, _ = CASES[case]
    b = quantise(Batch(shape_of(*layer, "bf16"), ragged(*seqs), 131 + case, extra_entries=more, garbage=None), 3)
    if more:
        b.pages[0, 2] = -1                         # (a page of nobody on the way)
    f, t, q, pools = form_of(b, kind, 7), b.dev(), b.q.to(DEV), pools8(b)
    out, lse = torch.full_like(q, 7.0), torch.full((b.n_rows, layer[0]), 7.0, device=DEV)
    b.runner().attend_quantised(q, t["row_start"], t["n_ctx"], t["pages"], *pools, out, lse, **on_device(f))
    torch.cuda.synchronize()
    k, v = (finite(x.float()) * finite(s)[..., None, None] for x, s in ((pools[0], pools[2]), (pools[1], pools[3])))
    check_out(b, reference(b, k, v, f), out, lse, np.arange(b.n_rows))


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("kind", KINDS + ["all"])
def test_attention_over_selected_pages_in_every_cut(case, kind):
    layer, seqs, more, _, _ = CASES[case]
    b = Batch(shape_of(*layer, "bf16"), ragged(*seqs), 151 + case, extra_entries=more)
    if more:
        b.pages[0, 2] = b.n_pages
    f, t, q = form_of(b, kind, 7), b.dev(), b.q.to(DEV)
    idx, n_sel, chosen = some_pages(b, case)
    out, lse = torch.full_like(q, 7.0), torch.full((b.n_rows, layer[0]), 7.0, device=DEV)
    b.runner().attend_selected(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], idx.to(DEV), n_sel.to(DEV), out, lse, **on_device(f))
    torch.cuda.synchronize()
    check_out(b, reference(b, finite(t["k_pages"]), finite(t["v_pages"]), f, chosen.to(DEV)), out, lse, np.arange(b.n_rows))
