"""The calls on a paged cache against a plain fp64 implementation (oracle/paged_oracle.py), on the GPU.

Tolerances are bounds by arithmetic.  e(t) = half a step of type t relative to the value: fp32 2^-24, bf16 2^-8.
A score is a sum of D products in fp32, each factor exact: off by at most (D + 8) e(fp32) sum |q k| scale, the 8 for the
scaling, cap, bias and the change to units of log2.  With S the largest such sum of a row (plus the bias, rounded once), a
probability is off by at most the factor 1 + delta, delta = 2 (D + 16) e(fp32) S + (n + 16) e(fp32) (the sum over n keys, the
exponential).  So with M = sum p |v|:
  out   fp32: 2 delta M + 2 e |out|;  bf16: the probabilities enter the product rounded to bf16, e(bf16) M more, and the result is
        rounded once, e(bf16) |out|.
  lse   delta + 4 e(fp32) |lse|
  weights  the sum over the rows of p (delta_row + ...) as above, + 2 e(fp32) per addition of what is there."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2502_13542_amd import binding as B

from paged_utils import BS, Batch, f64, shape_of

pytestmark = pytest.mark.gpu
DEV = "cuda"
E32, E16 = 2.0 ** -24, 2.0 ** -8

SHAPES = {"llama": (32, 8, 128, "bf16"), "g7": (28, 4, 128, "bf16"), "mha64": (3, 3, 64, "bf16"), "g8_64": (8, 1, 64, "bf16"),
          "fp32_64": (8, 2, 64, "fp32"), "fp32_g3": (6, 2, 128, "fp32"), "g5_64": (10, 2, 64, "bf16"), "fp32_g8": (8, 1, 128, "fp32")}
BATCHES = {
    "one": [(1, 1)],
    "steps": [(1, 127), (1, 128), (1, 129), (1, 1), (0, 5), (1, 700)],
    "few": [(3, 3), (2, 260), (4, 4), (0, 0), (1, 64)],
    "chunks": [(130, 130), (1, 300), (64, 321), (0, 10), (200, 513), (1, 1)],
    "prompt": [(513, 513)],
    "long_step": [(1, 5003), (1, 2000)],
    "long_tail": [(17, 3001)],
}
FORMS = {
    "plain": {},
    "cap": dict(softcap=20.0),
    "slopes": dict(slopes=True),
    "cap_slopes": dict(softcap=5.0, slopes=True),
    "window": dict(window=100),
    "window1": dict(window=1),
    "first": dict(first=True),
    "end": dict(end=True),
    "cap_slopes_end": dict(softcap=8.0, slopes=True, end=True),
    "all": dict(softcap=30.0, slopes=True, window=300, first=True, end=True),
}


def form_of(b, kind, seed):
    """The form's arguments on the host."""
    f = dict(kind if isinstance(kind, dict) else FORMS[kind])
    rng = np.random.default_rng(seed + 77)
    pos = b.positions()
    if f.pop("slopes", False):
        f["slopes"] = (2.0 ** -(1.0 + np.arange(b.shape.n_q_heads) % 8)).astype(np.float32)
    if f.pop("first", False):            # documents, rows that see nothing, and values that have to be clamped
        first = np.maximum(pos - rng.integers(0, 200, b.n_rows), 0)
        first[rng.random(b.n_rows) < 0.1] = 2 ** 31 - 1
        first[rng.random(b.n_rows) < 0.1] = -(2 ** 31)
        f["row_first"] = first
    if f.pop("end", False):
        end = np.maximum(pos + 1, rng.integers(0, 400, b.n_rows))
        end[rng.random(b.n_rows) < 0.1] = 2 ** 31 - 1
        end[rng.random(b.n_rows) < 0.05] = -5
        f["row_end"] = end
    return f


def on_device(f):
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    g = dict(f)
    for k in ("row_first", "row_end"):
        if k in g:
            g[k] = i32(g[k])
    if "slopes" in g:
        g["slopes"] = torch.tensor(g["slopes"], device=DEV)
    return g


def deltas(b, want):
    d = b.shape.head_dim
    n = max(b.n_ctx.max(), 1)
    return (2 * (d + 16) * want["size"] + n + 16) * E32


def check_out(b, want, out, lse, rows):
    delta = deltas(b, want)[rows]
    got, ref, mass = f64(out)[rows], want["out"][rows], want["mass"][rows]
    assert np.isfinite(got).all()
    bound = 2 * delta[..., None] * mass + 2 * E32 * np.abs(ref)
    if b.shape.dtype == "bf16":
        bound += E16 * mass + E16 * (np.abs(ref) + 2 * delta[..., None] * mass + E16 * mass)
    off = np.abs(got - ref) - bound
    assert (off <= 0).all(), f"out off by {off.max():.3e} more than its bound at {np.unravel_index(off.argmax(), off.shape)}"
    if lse is not None:
        got, ref = f64(lse)[rows], want["lse"][rows]
        none = np.isneginf(ref)
        assert (np.isneginf(got) == none).all()
        off = np.abs(got[~none] - ref[~none]) - (delta[~none] + 4 * E32 * np.abs(ref[~none]))
        assert off.size == 0 or (off <= 0).all(), f"lse off by {off.max():.3e} more than its bound"


def run_attention(b, kind="plain", seed=0, weight_rows=0, runner=None):
    f = form_of(b, kind, seed)
    r = runner or b.runner()
    t = b.dev()
    q = b.q.to(DEV)
    out = torch.full_like(q, 7.0)
    lse = torch.full((b.n_rows, b.shape.n_q_heads), 7.0, device=DEV)
    w = w_out = None
    if weight_rows:
        g = torch.Generator().manual_seed(seed + 5)
        w = torch.rand(b.batch, b.shape.n_kv_heads, b.max_pages * BS, generator=g)
        w_out = torch.full_like(w, -3.0).to(DEV)
        r.attend_weigh(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], out, lse, weight_rows, w.to(DEV),
                       w_out, **on_device(f))
    else:
        r.attend(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], out, lse, **on_device(f))
    torch.cuda.synchronize()
    k64, v64 = b.pools64()
    want = po.attention(f64(b.q), b.row_start, b.n_ctx, b.pages, k64, v64, b.shape.head_dim ** -0.5, weight_rows=weight_rows,
                        weights=None if w is None else w.double().numpy(), **f)
    rows = np.arange(b.row_start[0], b.row_start[-1])
    check_out(b, want, out, lse, rows)
    nobody = np.setdiff1d(np.arange(b.n_rows), rows)
    assert (f64(out)[nobody] == 7.0).all() and (f64(lse)[nobody] == 7.0).all(), "rows of nobody were written"
    if weight_rows:
        d, n, group = b.shape.head_dim, b.n_ctx.max(), b.shape.group
        adds = b.max_new * group + 2
        bound = 2 * (d + 16) * E32 * want["votes_size"] + (n + 32 + 2 * adds) * E32 * want["votes"] + 2 * E32 * np.abs(want["weights"])
        off = np.abs(f64(w_out) - want["weights"]) - bound
        assert (off <= 0).all(), f"weights off by {off.max():.3e} more than their bound"
    return out, lse, w_out, want


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("batch", list(BATCHES))
def test_attention(shape, batch):
    b = Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 11, extra_rows=(2, 3))
    run_attention(b)


@pytest.mark.parametrize("kind", [k for k in FORMS if k != "plain"])
@pytest.mark.parametrize("shape,batch", [("g7", "chunks"), ("g8_64", "chunks"), ("fp32_64", "chunks"), ("llama", "steps"),
                                         ("fp32_g3", "few"), ("mha64", "few"), ("llama", "long_tail"), ("fp32_g3", "long_tail")])
def test_attention_forms(shape, batch, kind):
    b = Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 13, extra_rows=(0, 1), garbage=float("inf"), scale=2.0)
    run_attention(b, kind, 3)


@pytest.mark.parametrize("shape", ["llama", "g7", "g5_64", "mha64", "fp32_64", "fp32_g3"])
@pytest.mark.parametrize("batch,rows,kind", [("steps", 1, "plain"), ("few", 2, "cap"), ("chunks", 32, "plain"),
                                             ("chunks", 1000, "all"), ("prompt", 513, "slopes"), ("long_step", 1, "window"),
                                             ("long_tail", 5, "first"), ("prompt", 64, "end")])
def test_attention_weights(shape, batch, rows, kind):
    b = Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 17, extra_rows=(1, 1))
    run_attention(b, kind, 5, weight_rows=rows)


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
@pytest.mark.parametrize("batch", ["steps", "chunks", "long_tail"])
def test_weights_in_place_and_twice_the_same_bits(shape, batch):
    b = Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 19)
    r, t, q = b.runner(), b.dev(), b.q.to(DEV)
    args = (q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"])
    got = []
    for _ in range(3):
        out, lse = torch.zeros_like(q), torch.zeros(b.n_rows, b.shape.n_q_heads, device=DEV)
        w = torch.ones(b.batch, b.shape.n_kv_heads, b.max_pages * BS, device=DEV)
        r.attend_weigh(*args, out, lse, 40, w)
        w2 = torch.empty_like(w)
        r.attend_weigh(*args, out, lse, 40, torch.ones_like(w), w2)
        torch.cuda.synchronize()
        assert torch.equal(w, w2)
        got.append((out, lse, w))
    for x in got[1:]:
        assert all(torch.equal(a, c) for a, c in zip(got[0], x))
    plain = torch.zeros_like(q)
    r.attend(*args, plain, None)
    torch.cuda.synchronize()
    assert torch.equal(plain, got[0][0]), "the attention of the two calls differs"


@pytest.mark.parametrize("shape", ["g7", "fp32_64"])
def test_pages_of_nobody_inside_a_sequence(shape):
    """Entries outside the pool are tokens that nobody sees; a page may serve two sequences."""
    b = Batch(shape_of(*SHAPES[shape]), [(3, 700), (150, 700), (1, 300), (1, 260)], 23)
    b.pages[0, 1], b.pages[1, 0], b.pages[1, 3], b.pages[2, 0] = -1, b.n_pages, 2 ** 31 - 1, -(2 ** 31)
    b.pages[3, :2] = b.pages[0, [0, 2]]
    out, lse, w, want = run_attention(b, weight_rows=2)
    b.pages[2, :] = -1                            # a whole sequence without pages: its row sees nothing
    out, lse, w, want = run_attention(b, weight_rows=2)
    assert np.isneginf(want["lse"][b.row_start[2]]).all()


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_lengths_that_have_to_be_clamped(shape):
    b = Batch(shape_of(*SHAPES[shape]), [(5, 200), (3, 130), (40, 256), (2, 256)], 29, garbage=None, extra_entries=0)
    b.n_ctx = np.array([2 ** 31 - 1, -(2 ** 31), 17, 256])      # more than the pages hold; none; 40 rows of 17 tokens
    b.pages = np.where(b.pages < 0, 0, b.pages)
    run_attention(b, weight_rows=3)
    r, t = b.runner(), b.dev()
    k0, v0 = b.pools64()
    r.append(b.k_new.to(DEV), b.v_new.to(DEV), t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"])
    b.pages[0] = b.pages[3] = [0, 1]
    torch.cuda.synchronize()
    # row_start out of order and out of range: nothing is read or written outside the arrays
    t["row_start"].copy_(torch.tensor([-(2 ** 31), 2 ** 31 - 1, 3, 1, 2 ** 31 - 1], dtype=torch.int32))
    guard = torch.full((b.n_rows + 2, b.shape.n_q_heads, b.shape.head_dim), 7.0, dtype=b.q.dtype, device=DEV)
    r.attend(b.q.to(DEV), t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], guard[1:-1], None)
    torch.cuda.synchronize()
    assert (guard[0] == 7.0).all() and (guard[-1] == 7.0).all()


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("batch", list(BATCHES))
def test_append(shape, batch):
    b = Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 31, extra_rows=(1, 2), garbage=None)
    if batch == "chunks":
        b.pages[0, 1] = -1                        # no page: its tokens go nowhere
    r, t = b.runner(), b.dev()
    r.append(b.k_new.to(DEV), b.v_new.to(DEV), t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"])
    torch.cuda.synchronize()
    # (rows of nobody lie outside row_start)
    k, v = po.append(f64(b.k_new), f64(b.v_new), b.row_start, b.n_ctx, b.pages, f64(b.k_pages), f64(b.v_pages))
    assert np.array_equal(f64(t["k_pages"]), k) and np.array_equal(f64(t["v_pages"]), v)


EVICT = [  # sequences, keep_first, keep_last, budget
    ([(0, 1000)], 4, 100, 300),
    ([(0, 300), (0, 299), (0, 301), (0, 0), (0, 1), (0, 900)], 0, 0, 300),
    ([(0, 5000), (0, 140)], 128, 12, 140),        # nothing to choose
    ([(0, 2500), (0, 700)], 1, 1, 3),
    ([(0, 300)], 0, 0, 1),
    ([(0, 4200), (0, 1030)], 7, 33, 1029),
]


@pytest.mark.parametrize("shape", ["llama", "fp32_64", "mha64", "fp32_g3"])
@pytest.mark.parametrize("case", range(len(EVICT)))
@pytest.mark.parametrize("kind", ["random", "ties", "flat", "odd"])
@pytest.mark.parametrize("in_place", [True, False])
def test_evict(shape, case, kind, in_place):
    seqs, first, last, budget = EVICT[case]
    sh = shape_of(*SHAPES[shape])
    to_max = -(-budget // BS)
    b = Batch(sh, seqs, 37 + case, spare_pages=2 + len(seqs) * to_max, garbage=None)
    g = torch.Generator().manual_seed(case)
    w = torch.rand(b.batch, sh.n_kv_heads, b.max_pages * BS, generator=g)
    if kind == "ties":
        w = (w * 5).floor()
    if kind == "flat":
        w = torch.full_like(w, 0.25)
    if kind == "odd":                             # every special value, small ones and negative ones
        pick = torch.randint(0, 10, w.shape, generator=g)
        values = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-42, -1e-42, -1.0, 3.4e38, 1.0])
        w = values[pick]
    r, t = b.runner(), b.dev()
    kept = torch.full((b.batch, sh.n_kv_heads, budget), -7, dtype=torch.int32, device=DEV)
    n_kept = torch.full((b.batch,), -7, dtype=torch.int32, device=DEV)
    wd = w.to(DEV)
    if in_place:
        to, to_w = b.pages, wd
        r.evict(t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], wd, first, last, budget, kept, n_kept)
    else:
        to = np.array([[b.free.pop() for _ in range(to_max)] for _ in seqs])
        to_w = torch.full((b.batch, sh.n_kv_heads, to_max * BS + 4), 9.0, device=DEV)
        r.evict(t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], wd, first, last, budget, kept, n_kept,
                to_pages=torch.tensor(to, dtype=torch.int32, device=DEV), to_weights=to_w)
    torch.cuda.synchronize()
    start_w = w.numpy() if in_place else np.full(to_w.shape, 9.0, np.float32)
    k2, n2, k, v, ww = po.evict(b.n_ctx, b.pages, f64(b.k_pages), f64(b.v_pages), w.numpy(), first, last, budget, to, start_w)
    assert np.array_equal(n_kept.cpu().numpy(), n2)
    assert np.array_equal(kept.cpu().numpy(), k2)
    assert np.array_equal(to_w.cpu().numpy(), ww, equal_nan=True)
    assert np.array_equal(f64(t["k_pages"]), k) and np.array_equal(f64(t["v_pages"]), v)


@pytest.mark.parametrize("shape", ["g7", "fp32_64"])
def test_a_cache_in_use(shape):
    """Prompts in chunks, steps, an eviction, more steps: every call's attention over a dense copy of what the cache holds."""
    sh = shape_of(*SHAPES[shape])
    hk, d, hq = sh.n_kv_heads, sh.head_dim, sh.n_q_heads
    g = torch.Generator().manual_seed(41)
    td = sh.torch_dtype
    batch, max_pages, n_pages, budget = 3, 6, 20, 200
    pages = np.random.default_rng(3).permutation(n_pages)[: batch * max_pages].reshape(batch, max_pages)
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)
    from paper_2502_13542_amd import harness as H
    r = H.PagedRunner(sh, batch, 700, 300, max_pages)
    kp = torch.full((n_pages, hk, BS, d), float("nan"), dtype=td, device=DEV)      # memory as it comes
    vp = torch.full((n_pages, hk, d, BS), float("nan"), dtype=td, device=DEV)
    weights = torch.zeros(batch, hk, max_pages * BS, device=DEV)
    held = [[[] for _ in range(hk)] for _ in range(batch)]         # what each head's slots hold: (k, v) rows
    account = np.zeros((batch, hk, max_pages * BS))
    n_ctx = np.zeros(batch, int)
    pages_d = i32(pages)
    for step, news in enumerate([(150, 1, 0), (300, 200, 129), (1, 1, 1), (7, 1, 90), "evict", (1, 1, 1), (130, 1, 3), "evict", (1, 1, 1)]):
        if news == "evict":
            kept = torch.zeros(batch, hk, budget, dtype=torch.int32, device=DEV)
            n_kept = torch.zeros(batch, dtype=torch.int32, device=DEV)
            chosen_by = weights.cpu().numpy()
            r.evict(i32(n_ctx), pages_d, kp, vp, weights, 4, 50, budget, kept, n_kept)
            torch.cuda.synchronize()
            for s in range(batch):
                for h in range(hk):
                    old = po.keep(chosen_by[s, h], n_ctx[s], 4, 50, budget)
                    assert kept[s, h, : len(old)].cpu().tolist() == old
                    held[s][h] = [held[s][h][o] for o in old]
                    account[s, h] = np.concatenate([account[s, h, old], np.zeros(max_pages * BS - len(old))])
            n_ctx = np.minimum(n_ctx, budget)
            assert n_kept.cpu().tolist() == n_ctx.tolist()
            continue
        n_rows = sum(news)
        k_new, v_new = (torch.randn(n_rows, hk, d, generator=g).to(td) for _ in range(2))
        q = torch.randn(n_rows, hq, d, generator=g).to(td)
        start = np.cumsum([0, *news])
        n_ctx = n_ctx + np.array(news)
        out, lse = torch.zeros_like(q, device=DEV), torch.zeros(n_rows, hq, device=DEV)
        table = (i32(start), i32(n_ctx), pages_d, kp, vp)
        r.append(k_new.to(DEV), v_new.to(DEV), *table)
        r.attend_weigh(q.to(DEV), *table, out, lse, 16, weights, softcap=25.0)
        torch.cuda.synchronize()
        k64, v64 = np.zeros(kp.shape), np.zeros(vp.shape)
        for s in range(batch):
            for h in range(hk):
                for i in range(start[s], start[s + 1]):
                    held[s][h].append((f64(k_new[i, h]), f64(v_new[i, h])))
                for j, (kk, vv) in enumerate(held[s][h]):
                    k64[pages[s, j // BS], h, j % BS], v64[pages[s, j // BS], h, :, j % BS] = kk, vv
        want = po.attention(f64(q), start, n_ctx, pages, k64, v64, d ** -0.5, softcap=25.0, weight_rows=16, weights=account)
        b = type("B", (), dict(shape=sh, n_ctx=n_ctx))
        check_out(b, want, out, lse, np.arange(n_rows))
        account = want["weights"]
        assert np.abs(f64(weights) - account).max() < 1e-4, step


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_replayed_graph(shape):
    """Append, attention with weights and eviction in one graph, replayed with other lengths and inputs between eager calls."""
    sh = shape_of(*SHAPES[shape])
    b = Batch(sh, [(1, 600), (4, 300), (90, 90)], 43, garbage=None)
    r, t = b.runner(), b.dev()
    hk = sh.n_kv_heads
    q, kn, vn = b.q.to(DEV), b.k_new.to(DEV), b.v_new.to(DEV)
    budget = 128
    kept = torch.zeros(3, hk, budget, dtype=torch.int32, device=DEV)
    n_kept = torch.zeros(3, dtype=torch.int32, device=DEV)
    to = torch.tensor(b.free[:2] + b.pages[2, :1].tolist(), dtype=torch.int32, device=DEV).reshape(3, 1)
    spare = torch.zeros_like(t["k_pages"][:3]), torch.zeros_like(t["v_pages"][:3])
    kp, vp = torch.cat([t["k_pages"], spare[0]]), torch.cat([t["v_pages"], spare[1]])
    to = torch.arange(b.n_pages, b.n_pages + 3, dtype=torch.int32, device=DEV).reshape(3, 1)
    out, lse = torch.zeros_like(q), torch.zeros(b.n_rows, sh.n_q_heads, device=DEV)
    w_in = torch.rand(3, hk, b.max_pages * BS, device=DEV)
    w_out, to_w = torch.zeros_like(w_in), torch.zeros(3, hk, BS, device=DEV)

    def step():
        table = (t["row_start"], t["n_ctx"], t["pages"], kp, vp)
        r.append(kn, vn, *table)
        r.attend_weigh(q, *table, out, lse, 3, w_in, w_out)
        r.evict(t["n_ctx"], t["pages"], kp, vp, w_out, 2, 30, budget, kept, n_kept, to_pages=to, to_weights=to_w)

    def state():
        torch.cuda.synchronize()
        return [x.clone() for x in (out, lse, w_out, kept, n_kept, kp, vp, to_w)]

    step()
    state()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n_ctx in ([600, 300, 90], [130, 299, 90], [5, 4, 90], [600, 17, 95]):
        t["n_ctx"].copy_(torch.tensor(n_ctx, dtype=torch.int32))
        q.copy_(torch.randn(q.shape).to(q.dtype))
        step()
        want = state()
        for x in (out, lse, w_out, kept, n_kept, to_w):
            x.zero_()
        graph.replay()
        for a, c in zip(state(), want):
            assert torch.equal(a, c)


def test_one_workspace_for_smaller_calls_and_a_side_stream():
    sh = shape_of(*SHAPES["llama"])
    big = Batch(sh, [(200, 900), (1, 2000), (17, 64), (3, 3)], 47)
    r = big.runner()
    for seqs in ([(1, 1)], [(200, 900), (1, 2000)], [(1, 2100)], [(16, 2000)], [(1, 5)] * 4, [(40, 40), (0, 3), (180, 1000)]):
        run_attention(Batch(sh, seqs, 53, extra_entries=0), runner=r)
    side = torch.cuda.Stream()
    b = Batch(sh, [(1, 700), (30, 300)], 59)
    t, q = b.dev(), b.q.to(DEV)
    out, want = torch.zeros_like(q), torch.zeros_like(q)
    r.attend(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], want)
    torch.cuda.synchronize()
    r.attend(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("shape", ["fp32_64", "fp32_g3"])
@pytest.mark.parametrize("batch", ["chunks", "steps"])
def test_fp32_values_near_the_largest(shape, batch):
    """Values above the largest bf16 in fp32 storage, and keys and queries whose product alone is ordinary."""
    b = Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 61, garbage=float("nan"))
    big = 3.4e38
    g = torch.Generator().manual_seed(9)
    hk, d = b.shape.n_kv_heads, b.shape.head_dim
    for s, (_, n) in enumerate(b.seqs):
        # one per sequence and channel: output sums are taken before they are divided by that of the probabilities, so two of
        # them, each with a probability above a half of the largest, would not be representable
        if n:
            slot = torch.randint(0, min(n, BS), (hk, d, 1), generator=g)
            b.v_pages[b.pages[s, 0]].scatter_(2, slot, big)
    b.k_pages *= 2.0 ** -3
    b.q[::7] = 0
    b.q[::7, :, 5] = big                                            # one huge channel, against keys that are tiny there
    b.k_pages[:, :, :, 5] *= 1e-38
    run_attention(b, "cap" if batch == "chunks" else "plain")


@pytest.mark.parametrize("shape", ["llama", "fp32_64", "mha64"])
@pytest.mark.parametrize("batch", ["few", "chunks"])
@pytest.mark.parametrize("softcap", [1e-6, 1e-3, 3e4, 1e6])
def test_smallest_and_largest_caps(shape, batch, softcap):
    """Caps under which every score is the cap, or none is changed, with queries of zeros among the others."""
    b = Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 67)
    b.q[::3] = 0
    run_attention(b, dict(softcap=softcap), weight_rows=2)


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
@pytest.mark.parametrize("in_place", [True, False])
def test_evict_with_pages_of_nobody(shape, in_place):
    """Kept tokens without a page move as zeros, never as what their new slots held; nothing is written where there is no
    page to move to."""
    sh = shape_of(*SHAPES[shape])
    b = Batch(sh, [(0, 900), (0, 700), (0, 100), (0, 513)], 71, spare_pages=10, garbage=None)
    b.pages[0, [0, 3]], b.pages[1, 1], b.pages[2, 0], b.pages[3, 4] = -1, b.n_pages, -(2 ** 31), 2 ** 31 - 1
    budget = 290
    w = torch.rand(4, sh.n_kv_heads, b.max_pages * BS, generator=torch.Generator().manual_seed(1))
    r, t, wd = b.runner(), b.dev(), w.to(DEV)
    kept = torch.zeros(4, sh.n_kv_heads, budget, dtype=torch.int32, device=DEV)
    n_kept = torch.zeros(4, dtype=torch.int32, device=DEV)
    args = (t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], wd, 3, 40, budget, kept, n_kept)
    to, to_w = b.pages, wd
    if in_place:
        r.evict(*args)
    else:
        to = np.array([[b.free.pop(), b.free.pop(), b.free.pop()], [b.free.pop(), -1, b.free.pop()], [b.free.pop(), b.n_pages, -1],
                       [-1, b.free.pop(), b.free.pop()]])
        to_w = torch.full((4, sh.n_kv_heads, 3 * BS), 9.0, device=DEV)
        r.evict(*args, to_pages=torch.tensor(to, dtype=torch.int32, device=DEV), to_weights=to_w)
    torch.cuda.synchronize()
    start = w.numpy() if in_place else np.full(to_w.shape, 9.0, np.float32)
    k2, n2, k, v, ww = po.evict(b.n_ctx, b.pages, f64(b.k_pages), f64(b.v_pages), w.numpy(), 3, 40, budget, to, start)
    assert np.array_equal(n_kept.cpu().numpy(), n2) and np.array_equal(kept.cpu().numpy(), k2)
    assert np.array_equal(to_w.cpu().numpy(), ww)
    assert np.array_equal(f64(t["k_pages"]), k) and np.array_equal(f64(t["v_pages"]), v)


@pytest.mark.parametrize("n,keep", [(9000, 700), (33000, 1500), (40000, 39000)])
@pytest.mark.parametrize("kind", ["random", "ties", "flat"])
def test_evict_from_long_sequences(n, keep, kind):
    """More candidates than a workgroup's registers hold at 8 and at 32 a thread."""
    sh = shape_of(2, 1, 64, "bf16")
    b = Batch(sh, [(0, n), (0, keep + 1)], 73, garbage=None)
    w = torch.rand(2, 1, b.max_pages * BS, generator=torch.Generator().manual_seed(n))
    w = {"random": w, "ties": (w * 20).floor(), "flat": torch.zeros_like(w)}[kind]
    r, t, wd = b.runner(), b.dev(), w.to(DEV)
    kept = torch.zeros(2, 1, keep, dtype=torch.int32, device=DEV)
    n_kept = torch.zeros(2, dtype=torch.int32, device=DEV)
    r.evict(t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], wd, 5, 60, keep, kept, n_kept)
    torch.cuda.synchronize()
    k2, n2, k, v, ww = po.evict(b.n_ctx, b.pages, f64(b.k_pages), f64(b.v_pages), w.numpy(), 5, 60, keep, b.pages, w.numpy())
    assert np.array_equal(kept.cpu().numpy(), k2) and np.array_equal(n_kept.cpu().numpy(), n2)
    assert np.array_equal(wd.cpu().numpy(), ww)
    assert np.array_equal(f64(t["k_pages"]), k) and np.array_equal(f64(t["v_pages"]), v)


# Calls that chunks in bf16 are cut up for in other ways: query heads, KV heads, head size, rows and tokens of the sequences, entries
# of the table behind the longest one's (the cut goes by the table's width)
CUTS = [(64, 32, 64, [(100, 120), (99, 99), (1, 3), (100, 130), (70, 70), (100, 100)], 0),      # 256 rows a workgroup
        (64, 32, 128, [(100, 120), (99, 99), (1, 3), (100, 130), (70, 70), (100, 100)], 0),
        (64, 8, 64, [(200, 300), (180, 181), (200, 200)], 0),                                   # 128 rows
        (64, 8, 128, [(200, 300), (180, 181), (200, 200)], 0),
        (16, 2, 128, [(690, 800)], 22),                                                         # 256 rows, pages in pieces
        (32, 8, 64, [(166, 500)], 32),
        (16, 4, 128, [(338, 700)], 5),                                                          # 128 rows, pages in pieces
        (32, 8, 64, [(81, 400), (80, 160)], 8)]


@pytest.mark.parametrize("case", range(len(CUTS)))
@pytest.mark.parametrize("kind", ["plain", "cap", "cap_slopes_end"])
def test_attention_in_every_cut(case, kind):
    hq, hkv, d, seqs, more = CUTS[case]
    run_attention(Batch(shape_of(hq, hkv, d, "bf16"), seqs, 79, extra_entries=more), kind, 7, weight_rows=50)


@pytest.mark.parametrize("shape", ["llama", "g8_64", "fp32_64"])
@pytest.mark.parametrize("kind", ["plain", "all"])
def test_steps_and_chunks_of_a_wide_table(shape, kind):
    """So many pages for sequences of few rows that those take a launch of their own, beside the chunks'."""
    b = Batch(shape_of(*SHAPES[shape]), [(1, 300), (60, 200), (2, 2), (0, 70), (1, 129), (16, 16), (1, 1), (2, 500)], 83,
              extra_rows=(1, 2), extra_entries=60 if shape == "llama" else 450)
    run_attention(b, kind, 9, weight_rows=4)


@pytest.mark.parametrize("shape", ["mha64", "fp32_64"])
def test_more_sequences_than_lanes(shape):
    rng = np.random.default_rng(5)
    seqs = [(int(min(m, n)), int(n)) for m, n in zip(rng.integers(0, 30, 150), rng.integers(0, 140, 150))]
    b = Batch(shape_of(*SHAPES[shape]), seqs, 89, extra_entries=0)
    run_attention(b, weight_rows=3)
    r, t = b.runner(), b.dev()
    r.append(b.k_new.to(DEV), b.v_new.to(DEV), t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"])
    torch.cuda.synchronize()
    k, v = po.append(f64(b.k_new), f64(b.v_new), b.row_start, b.n_ctx, b.pages, *(np.nan_to_num(f64(x)) for x in (b.k_pages, b.v_pages)))
    assert np.array_equal(np.nan_to_num(f64(t["k_pages"])), k) and np.array_equal(np.nan_to_num(f64(t["v_pages"])), v)


@pytest.mark.parametrize("shape", ["llama", "fp32_g3"])
@pytest.mark.parametrize("seqs", [[(1, 300), (2, 140)], [(150, 300), (3, 140)]])
def test_pages_past_32_bits(shape, seqs):
    """A pool of more than 2^32 bytes, and of more than 2^31 elements: the same bits as from a small one."""
    sh = shape_of(*SHAPES[shape])
    b = Batch(sh, seqs, 97, garbage=None)
    r, t = b.runner(), b.dev()
    page = sh.n_kv_heads * BS * sh.head_dim
    n_far = 2 ** 31 // page + 40
    move = torch.tensor([n_far - 1 - 7 * i for i in range(b.n_pages)], device=DEV)     # the last pages of the pool
    far = dict(t, pages=torch.where(t["pages"] >= 0, move[t["pages"].clamp(min=0).long()].int(), -1).contiguous())
    for name in ("k_pages", "v_pages"):
        pool = torch.empty(n_far, *t[name].shape[1:], dtype=t[name].dtype, device=DEV)
        pool[move] = t[name]
        far[name] = pool
    kn, vn, q = b.k_new.to(DEV), b.v_new.to(DEV), b.q.to(DEV)
    got = []
    for x in (t, far):
        table = (x["row_start"], x["n_ctx"], x["pages"], x["k_pages"], x["v_pages"])
        out, lse = torch.zeros_like(q), torch.zeros(b.n_rows, sh.n_q_heads, device=DEV)
        w = torch.zeros(b.batch, sh.n_kv_heads, b.max_pages * BS, device=DEV)
        kept, n_kept = torch.zeros(b.batch, sh.n_kv_heads, 130, dtype=torch.int32, device=DEV), torch.zeros(b.batch, dtype=torch.int32, device=DEV)
        r.append(kn, vn, *table)
        r.attend_weigh(q, *table, out, lse, 2, w)
        r.evict(*table[1:], w, 1, 20, 130, kept, n_kept)
        torch.cuda.synchronize()
        got.append((out, lse, w, kept, *((x["k_pages"], x["v_pages"]) if x is t else (x["k_pages"][move], x["v_pages"][move]))))
    assert all(torch.equal(a, c) for a, c in zip(*got))


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_two_calls_at_once(shape):
    """Two runners on two streams over one cache: neither disturbs the other."""
    sh = shape_of(*SHAPES[shape])
    calls = [Batch(sh, [(1, 900), (1, 40)], 101), Batch(sh, [(120, 900), (1, 40)], 103)]
    streams = [torch.cuda.Stream() for _ in calls]
    prepared = []
    for b in calls:
        t, q = b.dev(), b.q.to(DEV)
        args = (q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"])
        outs = [torch.zeros_like(q) for _ in range(9)]
        r = b.runner()
        r.attend(*args, outs[0])
        prepared.append((r, args, outs))
    torch.cuda.synchronize()
    for i in range(1, 9):
        for (r, args, outs), stream in zip(prepared, streams):
            r.attend(*args, outs[i], stream=stream)
    torch.cuda.synchronize()
    for _, _, outs in prepared:
        assert all(torch.equal(o, outs[0]) for o in outs[1:])


def test_a_call_that_says_how_many_rows_it_brings():
    """Decode steps through a runner made for prompts: the kernels for few rows, their results within the same bounds."""
    sh = shape_of(*SHAPES["llama"])
    b = Batch(sh, [(1, 300), (1, 129), (1, 1)], 107)
    from paper_2502_13542_amd import harness as H
    made_for = H.PagedRunner(sh, 3, 500, 400, b.max_pages)
    t, q = b.dev(), b.q.to(DEV)
    args = (q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"])
    got = []
    for r, kw in ((b.runner(), {}), (made_for, dict(max_new=1))):
        out, lse = torch.zeros_like(q), torch.zeros(3, sh.n_q_heads, device=DEV)
        w = torch.zeros(3, sh.n_kv_heads, b.max_pages * BS, device=DEV)
        r.attend_weigh(*args, out, lse, 1, w, **kw)
        torch.cuda.synchronize()
        got.append((out, lse, w))
    assert all(torch.equal(a, c) for a, c in zip(*got))
    run_attention(b, runner=made_for)


@pytest.mark.parametrize("shape,rows", [("llama", 64), ("g8_64", 64), ("fp32_64", 64), ("fp32_g8", 16)])
@pytest.mark.parametrize("more", [0, 1])
@pytest.mark.parametrize("kind", ["plain", "all", "cap_slopes_end"])
def test_weights_of_as_many_rows_as_stay_staged(shape, rows, more, kind):
    """At and above the number of voting rows up to which they are staged once."""
    r = rows + more
    b = Batch(shape_of(*SHAPES[shape]), [(r + 5, 400), (1, 200), (0, 3), (r, r), (2, 131)], 109, extra_rows=(1, 0))
    run_attention(b, kind, 11, weight_rows=r)


def test_weights_of_a_long_sequence_among_many():
    """One wavefront's keys of more than 64 steps: 64 short sequences of 16 KV heads leave few workgroups for the long one."""
    b = Batch(shape_of(16, 16, 64, "bf16"), [(1, 3)] * 40 + [(20, 17000)] + [(2, 5)] * 23, 113, extra_entries=0)
    run_attention(b, weight_rows=3)


@pytest.mark.parametrize("shape", ["llama", "g8_64", "fp32_64", "fp32_g3"])
@pytest.mark.parametrize("batch", ["few", "steps", "chunks", "long_tail"])
@pytest.mark.parametrize("start", ["first", "window", "both"])
def test_rows_that_end_at_the_least_number(shape, batch, start):
    """row_end of -2^31 and its neighbours beside a first position above 0: the row sees nothing, whatever the rows beside it see."""
    b = Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 127, extra_rows=(1, 1))
    pos = b.positions()
    f = dict(row_end=pos + 1)
    f["row_end"][::2] = np.resize([-(2 ** 31), -(2 ** 31) + 1, -(2 ** 31) + 40, -1, 0], len(pos[::2]))
    if start != "window":
        f["row_first"] = np.maximum(pos - 50, 0)
        f["row_first"][::4] = np.resize([2 ** 31 - 1, 1, 60, 2 ** 30], len(pos[::4]))
    if start != "first":
        f["window"] = 30
    run_attention(b, f, weight_rows=40)


CLAMPED = [2 ** 31 - 1, -(2 ** 31), 17, 256]     # more tokens than the pages hold; none; fewer than rows; all that the pages hold


def clamped_batch(shape):
    """Sequences with such lengths on the device, and on the host what they are taken as; no page is two sequences'."""
    b = Batch(shape_of(*SHAPES[shape]), [(5, 200), (3, 130), (40, 256), (2, 256)], 131, extra_rows=(1, 2), extra_entries=0, garbage=None)
    b.n_ctx = np.clip(CLAMPED, 0, b.max_pages * BS)
    b.seqs = [(m, n) for (m, _), n in zip(b.seqs, b.n_ctx)]
    raw = torch.tensor(CLAMPED, dtype=torch.int32, device=DEV)
    b.dev = lambda dev=DEV: dict(Batch.dev(b, dev), n_ctx=raw.clone())
    return b


@pytest.mark.parametrize("shape", ["llama", "g8_64", "fp32_64", "fp32_g3"])
@pytest.mark.parametrize("kind", ["plain", "all"])
def test_clamped_lengths_give_what_the_lengths_they_stand_for_give(shape, kind):
    """The bounds are those of the lengths after clamping: zeros in the place of the results are far outside."""
    b = clamped_batch(shape)
    out, lse, w_out, want = run_attention(b, kind, 13, weight_rows=3)
    rows = np.arange(b.row_start[0], b.row_start[-1])
    assert b.n_ctx.tolist() == [256, 0, 17, 256]
    with pytest.raises(AssertionError, match="out off"):
        check_out(b, want, torch.zeros_like(out), lse, rows)
    with pytest.raises(AssertionError):
        check_out(b, want, out, torch.where(torch.isinf(lse), lse, 0.0), rows)
    if kind == "plain":                           # of 40 rows of 17 tokens the last 17 see some, of the sequence of none no row
        assert (~np.isneginf(want["lse"][rows]).all(1)).sum() == 5 + 17 + 2
    few = Batch(b.shape, [(2, 200), (1, 130), (2, 256), (2, 256)], 137, extra_entries=0, garbage=None)      # the kernels for few rows
    few.seqs = [(m, n) for (m, _), n in zip(few.seqs, b.n_ctx)]
    few.n_ctx, few.dev = b.n_ctx, lambda dev=DEV: dict(Batch.dev(few, dev), n_ctx=b.dev()["n_ctx"])
    run_attention(few, kind, 13, weight_rows=3)


@pytest.mark.parametrize("shape", list(SHAPES))
def test_append_at_clamped_lengths(shape):
    b = clamped_batch(shape)
    t = b.dev()
    b.runner().append(b.k_new.to(DEV), b.v_new.to(DEV), t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"])
    torch.cuda.synchronize()
    k, v = po.append(f64(b.k_new), f64(b.v_new), b.row_start, b.n_ctx, b.pages, f64(b.k_pages), f64(b.v_pages))
    assert (k != f64(b.k_pages)).any((1, 3)).sum() == 5 + 17 + 2           # tokens that have new keys
    assert np.array_equal(f64(t["k_pages"]), k) and np.array_equal(f64(t["v_pages"]), v)


@pytest.mark.parametrize("shape", ["llama", "g8_64", "fp32_64"])
@pytest.mark.parametrize("in_place", [True, False])
def test_replayed_graph_from_pools_as_they_were(shape, in_place):
    """Every replay starts from the pools and weights that the eager calls started from, with new keys, values and queries, so that
    a graph without the append, the weights or the move, or with old inputs, ends with other pools."""
    sh = shape_of(*SHAPES[shape])
    hk, budget = sh.n_kv_heads, 140
    b = Batch(sh, [(1, 600), (4, 300), (90, 90), (2, 131)], 139, spare_pages=10, garbage=None)
    r, t = b.runner(), b.dev()
    to = torch.tensor([[b.free.pop(), b.free.pop()] for _ in b.seqs], dtype=torch.int32, device=DEV)
    given = [t["k_pages"], t["v_pages"], torch.rand(b.batch, hk, b.max_pages * BS, device=DEV)]
    kp, vp, w = (x.clone() for x in given)
    q, kn, vn = b.q.to(DEV), b.k_new.to(DEV), b.v_new.to(DEV)
    out, lse = torch.zeros_like(q), torch.zeros(b.n_rows, sh.n_q_heads, device=DEV)
    to_w = torch.zeros(b.batch, hk, 2 * BS, device=DEV)
    kept, n_kept = torch.zeros(b.batch, hk, budget, dtype=torch.int32, device=DEV), torch.zeros(b.batch, dtype=torch.int32, device=DEV)
    results = (out, lse, to_w, kept, n_kept)

    def step():
        table = (t["row_start"], t["n_ctx"], t["pages"], kp, vp)
        r.append(kn, vn, *table)
        r.attend_weigh(q, *table, out, lse, 3, w)
        r.evict(*table[1:], w, 2, 30, budget, kept, n_kept, **({} if in_place else dict(to_pages=to, to_weights=to_w)))

    def start():
        for x, x0 in zip((kp, vp, w), given):
            x.copy_(x0)
        for x in results:
            x.zero_()

    def state():
        torch.cuda.synchronize()
        return [x.clone() for x in (kp, vp, w, *results)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    last = None
    for n_ctx in ([600, 300, 90, 131], [130, 299, 90, 140], [5, 141, 90, 142], [600, 17, 95, 256]):
        t["n_ctx"].copy_(torch.tensor(n_ctx, dtype=torch.int32))
        for x in (q, kn, vn):
            x.copy_(torch.randn(x.shape).to(x.dtype))
        start()
        step()
        want = state()
        for a, x0 in zip(want, given):
            assert not torch.equal(a, x0)
        assert last is None or not any(torch.equal(a, c) for a, c in zip(want[:4], last))
        last = want
        for _ in range(2):
            start()
            graph.replay()
            assert all(torch.equal(a, c) for a, c in zip(state(), want))
        # what the pools hold by the definitions: the new tokens, then the move
        k, v = po.append(f64(kn), f64(vn), b.row_start, n_ctx, b.pages, f64(given[0]), f64(given[1]))
        k_end, v_end, kept_end = f64(want[0]), f64(want[1]), want[6].cpu().numpy()
        cut = np.asarray(n_ctx) > budget
        for s in range(b.batch):
            for h in range(hk):
                old = kept_end[s, h][kept_end[s, h] >= 0]
                assert len(old) == min(n_ctx[s], budget) and cut[s] == (old[-1] >= budget)
                dst = b.pages[s] if in_place else to[s].cpu().numpy()
                new = np.arange(len(old))
                src = b.pages[s][old // BS]
                assert np.array_equal(k_end[dst[new // BS], h, new % BS], k[src, h, old % BS])
                assert np.array_equal(v_end[dst[new // BS], h, :, new % BS], v[src, h, :, old % BS])


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_evict_in_place_by_the_table_itself(shape):
    """to_pages as `pages`: keys, values and weights move as with None, and the next eviction goes by weights that have moved."""
    sh = shape_of(*SHAPES[shape])
    b = Batch(sh, [(0, 900), (0, 140), (0, 513)], 149, garbage=None)
    r, t = b.runner(), b.dev()
    w = torch.rand(b.batch, sh.n_kv_heads, b.max_pages * BS, generator=torch.Generator().manual_seed(2))
    wd, n_ctx = w.to(DEV), t["n_ctx"]
    n, k, v, want_w = b.n_ctx, f64(b.k_pages), f64(b.v_pages), w.numpy()
    for budget in (400, 150):
        kept = torch.zeros(b.batch, sh.n_kv_heads, budget, dtype=torch.int32, device=DEV)
        n_kept = torch.zeros(b.batch, dtype=torch.int32, device=DEV)
        r.evict(n_ctx, t["pages"], t["k_pages"], t["v_pages"], wd, 3, 20, budget, kept, n_kept, to_pages=t["pages"])
        torch.cuda.synchronize()
        want_kept, n, k, v, want_w = po.evict(n, b.pages, k, v, want_w, 3, 20, budget, b.pages, want_w)
        n_ctx = n_kept
        assert np.array_equal(kept.cpu().numpy(), want_kept) and np.array_equal(n_kept.cpu().numpy(), n)
        assert np.array_equal(wd.cpu().numpy(), want_w)
        assert np.array_equal(f64(t["k_pages"]), k) and np.array_equal(f64(t["v_pages"]), v)
