"""The paged cache without a GPU: the oracle on cases worked by hand, and everything the calls refuse."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2502_13542_amd import binding as B
from paper_2502_13542_amd import harness as H

from paged_utils import BS, Batch, f64, shape_of

A16 = 0x10000  # fake, aligned, never dereferenced: every check below fails before a launch
LLAMA = shape_of(32, 8, 128, "bf16")


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


# ---------------------------------------------------------------- the oracle
def test_oracle_attention_by_hand():
    """Two keys with scores ln 3 and 0, values 1 and 5: out = 0.75 * 1 + 0.25 * 5 = 2, lse = ln 4."""
    k, v = np.zeros((2, 1, BS, 2)), np.zeros((2, 1, 2, BS))
    k[1, 0, 0] = [math.log(3), 0]
    v[1, 0, :, 0], v[1, 0, :, 1] = 1.0, 5.0
    q = np.array([[[1.0, 0.0]]])
    got = po.attention(q, [0, 1], [2], np.array([[1]]), k, v, 1.0, weight_rows=1, weights=np.ones((1, 1, BS)))
    assert np.allclose(got["out"], 2.0) and np.allclose(got["lse"], math.log(4))
    assert np.allclose(got["weights"][0, 0, :3], [1.75, 1.25, 1.0])
    # capped: 1 tanh(ln 3) = 0.8; biased: the row is at position 1, the first key one away
    got = po.attention(q, [0, 1], [2], np.array([[1]]), k, v, 1.0, softcap=1.0, slopes=np.array([0.3]))
    assert np.allclose(got["lse"], math.log(math.exp(0.8 - 0.3) + 1))
    for f in (dict(window=1), dict(row_first=np.array([1]))):      # only itself
        assert np.allclose(po.attention(q, [0, 1], [2], np.array([[1]]), k, v, 1.0, **f)["out"], 5.0)
    assert np.allclose(po.attention(q, [0, 1], [2], np.array([[1]]), k, v, 1.0, row_end=np.array([1]))["out"], 1.0)
    for f in (dict(row_first=np.array([2])), dict(row_end=np.array([0]))):
        got = po.attention(q, [0, 1], [2], np.array([[1]]), k, v, 1.0, **f)
        assert (got["out"] == 0).all() and np.isneginf(got["lse"]).all()


def test_oracle_attention_is_dense_attention():
    b = Batch(shape_of(4, 2, 64, "fp32"), [(70, 70), (3, 200)], 1)
    k64, v64 = b.pools64()
    got = po.attention(f64(b.q), b.row_start, b.n_ctx, b.pages, k64, v64, 0.125)
    for s, (m, n) in enumerate(b.seqs):
        page = b.pages[s, np.arange(n) // BS]
        k, v = (torch.tensor(x) for x in (k64[page, :, np.arange(n) % BS], v64[page, :, :, np.arange(n) % BS]))
        q = torch.tensor(f64(b.q))[b.row_start[s]: b.row_start[s + 1]]
        z = torch.einsum("mhd,nhd->hmn", q, k.repeat_interleave(2, 1)) * 0.125
        z = z.masked_fill(torch.ones(m, n).triu(n - m + 1).bool(), -math.inf)
        want = torch.einsum("hmn,nhd->mhd", z.softmax(-1), v.repeat_interleave(2, 1)).numpy()
        assert np.abs(got["out"][b.row_start[s]: b.row_start[s + 1]] - want).max() < 1e-12


def test_oracle_eviction_by_hand():
    w = np.array([5.0, 1, 3, np.nan, 3, -0.0, 0.0, 2, 9, 9])
    assert po.keep(w, 10, 1, 2, 10) == list(range(10))
    assert po.keep(w, 10, 1, 2, 5) == [0, 2, 4, 8, 9]
    assert po.keep(w, 10, 1, 2, 4) == [0, 2, 8, 9]                 # equal weights: the lower position
    assert po.keep(w, 10, 0, 0, 8) == [0, 1, 2, 4, 5, 7, 8, 9]     # -0 is 0, NaN below everything
    assert po.keep(w, 10, 0, 0, 9) == [0, 1, 2, 4, 5, 6, 7, 8, 9]


def test_oracle_append_and_evict_move_what_they_say():
    b = Batch(shape_of(2, 1, 64, "fp32"), [(0, 200), (140, 300)], 2, garbage=None, spare_pages=4)
    k, v = po.append(f64(b.k_new), f64(b.v_new), b.row_start, b.n_ctx, b.pages, f64(b.k_pages), f64(b.v_pages))
    p = b.pages[1]
    assert np.array_equal(k[p[1], 0, 32], f64(b.k_new)[0, 0]) and np.array_equal(v[p[2], 0, :, 43], f64(b.v_new)[139, 0])
    assert (k != f64(b.k_pages)).any(-1).sum() == 140
    w = np.random.default_rng(0).random((2, 1, b.max_pages * BS))
    to = np.array([b.free[:1], b.free[1:2]])
    kept, n_kept, k2, v2, w2 = po.evict(b.n_ctx, b.pages, k, v, w, 0, 0, 100, to, np.ones((2, 1, BS)))
    assert n_kept.tolist() == [100, 100]
    o = kept[1, 0, 50]
    assert np.array_equal(k2[to[1, 0], 0, 50], k[p[o // BS], 0, o % BS]) and w2[1, 0, 50] == w[1, 0, o] and (w2[:, :, 100:] == 0).all()
    assert (np.sort(w[1, 0, :300])[-100:] == np.sort(w2[1, 0, :100])).all()


# ---------------------------------------------------------------- refusals
def _append(lib, cs, **kw):
    a = dict(batch=2, n_rows=9, max_new=5, k=A16, v=A16, rs=A16, n=A16, pages=A16, max_pages=4, kp=A16, vp=A16, n_pages=9)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.actqkv_paged_append(ctypes.byref(cs), *a.values(), None)


def _attend(lib, cs, **kw):
    a = dict(batch=2, n_rows=9, max_new=5, q=A16, rs=A16, n=A16, pages=A16, max_pages=4, kp=A16, vp=A16, n_pages=9, softcap=0.0,
             window=0, slopes=None, first=None, end=None, out=A16, lse=None, ws=A16, wsb=1 << 40)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.actqkv_paged_attention(ctypes.byref(cs), *a.values(), None)


def _weigh(lib, cs, **kw):
    a = dict(batch=2, n_rows=9, max_new=5, q=A16, rs=A16, n=A16, pages=A16, max_pages=4, kp=A16, vp=A16, n_pages=9, softcap=0.0,
             window=0, slopes=None, first=None, end=None, out=A16, lse=A16, rows=1, w_in=A16, w_out=A16, stride=512, ws=A16,
             wsb=1 << 40)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.actqkv_paged_attention_weights(ctypes.byref(cs), *a.values(), None)


def _evict(lib, cs, **kw):
    a = dict(batch=2, n=A16, pages=A16, max_pages=4, kp=A16, vp=A16, n_pages=9, w=A16, stride=512, first=1, last=2, budget=100,
             to=2 * A16, to_max=1, to_w=3 * A16, to_stride=128, kept=A16, n_kept=4 * A16)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.actqkv_paged_evict(ctypes.byref(cs), *a.values(), None)


TABLE = [(dict(batch=0), -1), (dict(batch=1025), -2), (dict(max_pages=0), -1), (dict(max_pages=(1 << 23) + 1), -2),
         (dict(n_pages=0), -1), (dict(n_pages=(1 << 23) + 1), -2), (dict(n=None), -1), (dict(n=A16 + 2), -3), (dict(pages=None), -1),
         (dict(pages=A16 + 1), -3), (dict(kp=None), -1), (dict(kp=A16 + 8), -3), (dict(vp=None), -1), (dict(vp=A16 + 4), -3)]
ROWS = [(dict(n_rows=0), -1), (dict(n_rows=-3), -1), (dict(max_new=0), -1), (dict(max_new=10), -1),
        (dict(n_rows=(1 << 22) + 1), -2), (dict(rs=None), -1), (dict(rs=A16 + 3), -3)]
FORM = [(dict(softcap=-1.0), -1), (dict(softcap=math.inf), -1), (dict(softcap=math.nan), -1), (dict(window=-1), -1),
        (dict(slopes=A16 + 2), -3), (dict(first=A16 + 2), -3), (dict(end=A16 + 1), -3), (dict(lse=A16 + 2), -3), (dict(q=None), -1),
        (dict(q=A16 + 8), -3), (dict(out=None), -1), (dict(out=A16 + 8), -3), (dict(ws=None), -4), (dict(ws=A16 + 8), -4),
        (dict(wsb=64), -4)]


@pytest.mark.parametrize("bad,code", TABLE + ROWS + [(dict(k=None), -1), (dict(v=A16 + 8), -3)])
def test_append_refusals(lib, bad, code):
    assert _append(lib, B.c_shape(LLAMA), **bad) == code
    assert B.last_error()


@pytest.mark.parametrize("bad,code", TABLE + ROWS + FORM)
def test_attention_refusals(lib, bad, code):
    assert _attend(lib, B.c_shape(LLAMA), **bad) == code
    assert _weigh(lib, B.c_shape(LLAMA), **bad) == code


@pytest.mark.parametrize("bad,code", [(dict(lse=None), -1), (dict(rows=0), -1), (dict(w_in=None), -1), (dict(w_out=A16 + 4), -3),
                                      (dict(stride=508), -1), (dict(stride=513), -3)])
def test_weights_refusals(lib, bad, code):
    assert _weigh(lib, B.c_shape(LLAMA), **bad) == code


@pytest.mark.parametrize("bad,code", TABLE + [
    (dict(w=None), -1), (dict(stride=511), -1), (dict(first=-1), -1), (dict(last=-1), -1), (dict(budget=0), -1),
    (dict(first=60, last=41), -1), (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), -1), (dict(budget=129), -1), (dict(to=A16 + 2), -3),
    (dict(to_max=0), -1), (dict(to_max=(1 << 23) + 1, to_stride=1 << 40), -2), (dict(to_stride=127), -1), (dict(to_w=A16 + 1), -3),
    (dict(kept=None), -1), (dict(n_kept=None), -1), (dict(n_kept=A16), -1), (dict(to=A16), -1), (dict(to_w=A16), -1),
    (dict(to=None, budget=513), -1)])
def test_evict_refusals(lib, bad, code):
    assert _evict(lib, B.c_shape(LLAMA), **bad) == code


@pytest.mark.parametrize("shape,code", [((32, 8, 96, "bf16"), -2), ((9, 2, 64, "bf16"), -2), ((18, 2, 64, "fp32"), -2)])
def test_shapes_refused(lib, shape, code):
    cs = B.c_shape(shape_of(*shape))
    for call in (_append, _attend, _weigh, _evict):
        assert call(lib, cs) == code
    assert lib.actqkv_paged_workspace_bytes(ctypes.byref(cs), 1, 1, 1, 1) == 0


def test_workspace_serves_smaller_calls(lib):
    rng = np.random.default_rng(0)
    for shape in ((32, 8, 128, "bf16"), (28, 4, 128, "bf16"), (8, 2, 64, "fp32"), (8, 8, 64, "bf16"), (16, 2, 128, "fp32")):
        cs = B.c_shape(shape_of(*shape))
        for _ in range(300):
            batch, max_new, max_pages = (int(2 ** rng.uniform(0, t)) for t in (8, 12, 11))
            n_rows = int(rng.integers(max_new, batch * max_new + 1))
            big = B.paged_workspace_bytes(cs, batch, n_rows, max_new, max_pages)
            for _ in range(4):
                small = [int(rng.integers(1, x + 1)) for x in (batch, n_rows, max_new, max_pages)]
                small[2] = min(small[1], small[2])
                assert B.paged_workspace_bytes(cs, *small) <= big, (shape, batch, n_rows, max_new, max_pages, small)
        for bad in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 2, 1), (1, 1, 1, 0), (1, 1, 1, 1 << 24)):
            with pytest.raises(B.ActQKVError):
                B.paged_workspace_bytes(cs, *bad)


def test_the_runner_checks_sizes():
    b = Batch(shape_of(4, 2, 64, "fp32"), [(2, 40), (3, 200)], 3)
    r, t = b.runner("cpu"), b.dev("cpu")
    table = dict(t)
    rows = dict(k_new=b.k_new, v_new=b.v_new)
    out, lse = torch.zeros_like(b.q), torch.zeros(5, 4)
    w = torch.zeros(2, 2, b.max_pages * BS)
    kept, n_kept = torch.zeros(2, 2, 50, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    ev = dict(n_ctx=t["n_ctx"], pages=t["pages"], k_pages=t["k_pages"], v_pages=t["v_pages"], weights=w, keep_first=1, keep_last=1,
              budget=50, kept=kept, n_kept=n_kept)
    calls = [
        (r.append, {**rows, **table}, ["k_new", "v_new", "row_start", "n_ctx", "k_pages", "v_pages"]),
        (r.attend, dict(q=b.q, **table, out=out, lse=lse, slopes=torch.ones(4), row_first=torch.zeros(5, dtype=torch.int32),
                        row_end=torch.zeros(5, dtype=torch.int32)),
         ["out", "row_start", "n_ctx", "lse", "slopes", "row_first", "row_end", "k_pages"]),
        (r.attend_weigh, dict(q=b.q, **table, out=out, lse=lse, weight_rows=1, weights=w, weights_out=w.clone()),
         ["out", "lse", "weights", "weights_out"]),
        (r.evict, ev, ["n_ctx", "k_pages", "kept", "n_kept"]),
    ]
    for call, good, names in calls:
        with pytest.raises(B.ActQKVError, match="not on the GPU"):     # sizes are right: the next check is the device
            call(**good)
        for name in names:
            bad = dict(good)
            bad[name] = good[name].reshape(-1)[:-1] if good[name].dim() == 1 else good[name][..., :-1].contiguous()
            with pytest.raises(B.ActQKVError) as e:
                call(**bad)
            assert "not on the GPU" not in str(e.value), name
    small = H.PagedRunner(b.shape, 1, 5, 3, b.max_pages, "cpu")
    with pytest.raises(B.ActQKVError, match="made for"):
        small.append(**rows, **table)
    with pytest.raises(B.ActQKVError, match="made for"):
        H.PagedRunner(b.shape, 2, 4, 3, b.max_pages, "cpu").append(**rows, **table)
    r.append(b.k_new[:0], b.v_new[:0], t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"])   # no rows: nothing to do


@pytest.mark.parametrize("softcap", [1e-45, 1e-30, 9e-7, 1.1e6, 3e38])
def test_caps_out_of_range_are_refused(lib, softcap):
    """A cap whose reciprocal overflows, or that is so large that a capped score may be below a hidden one's mark."""
    assert _attend(lib, B.c_shape(LLAMA), softcap=softcap) == -1 and "softcap" in B.last_error()
    assert _weigh(lib, B.c_shape(LLAMA), softcap=softcap) == -1


def test_calls_of_more_threads_than_a_launch_has_are_refused(lib):
    wide = B.c_shape(shape_of(256, 256, 64, "bf16"))
    big = dict(n_rows=(1 << 20) + 1, max_new=1, wsb=1 << 60)
    assert _attend(lib, wide, **big) == -2 and "2^28" in B.last_error()
    assert _weigh(lib, wide, **big) == -2
    assert _weigh(lib, B.c_shape(LLAMA), max_pages=(1 << 19) + 1, stride=1 << 40, wsb=1 << 60) == -2 and "2^22" in B.last_error()


@pytest.mark.parametrize("max_new", [0, -1, 4])
def test_the_runner_checks_the_rows_a_call_says_it_brings(max_new):
    b = Batch(shape_of(4, 2, 64, "fp32"), [(2, 40), (3, 200)], 3)
    r, t = b.runner("cpu"), b.dev("cpu")
    out, lse, w = torch.zeros_like(b.q), torch.zeros(5, 4), torch.zeros(2, 2, b.max_pages * BS)
    with pytest.raises(B.ActQKVError, match="max_new"):
        r.append(b.k_new, b.v_new, **t, max_new=max_new)
    with pytest.raises(B.ActQKVError, match="max_new"):
        r.attend(b.q, **t, out=out, max_new=max_new)
    with pytest.raises(B.ActQKVError, match="max_new"):
        r.attend_weigh(b.q, **t, out=out, lse=lse, weight_rows=1, weights=w, max_new=max_new)


def test_workspace_of_steps_holds_no_pieces_of_chunks():
    """64 steps of 32 heads at 8192 tokens: kept scores (32 x 8192 x 4 bytes each) and at most 2048 parts of 16 rows."""
    cs = B.c_shape(LLAMA)
    assert B.paged_workspace_bytes(cs, 64, 64, 1, 64) <= 64 * 32 * 8192 * 4 + 2048 * 16 * 130 * 4 + 65536
    assert B.paged_workspace_bytes(cs, 64, 64 * 5, 5, 64) >= B.paged_workspace_bytes(cs, 64, 64 * 4, 4, 64)


def test_in_place_eviction_takes_the_weights_along(monkeypatch):
    """Both ways to say in place, None and the table itself (or a view of it), move the account with the tokens."""
    b = Batch(shape_of(4, 2, 64, "fp32"), [(0, 400), (0, 200)], 3)
    r, t = b.runner("cpu"), b.dev("cpu")
    w, other = torch.zeros(2, 2, b.max_pages * BS), torch.zeros(2, 2, b.max_pages * BS)
    kept, n_kept = torch.zeros(2, 2, 50, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    calls = []
    monkeypatch.setattr(B, "paged_evict", lambda *a: calls.append(dict(to_pages=a[13], to_weights=a[15], stride=a[16])))
    pages = t["pages"]
    for to_pages in (None, pages, pages.view(-1).view(pages.shape)):
        for to_weights, gets in ((None, w), (other, other)):
            r.evict(t["n_ctx"], pages, t["k_pages"], t["v_pages"], w, 1, 1, 50, kept, n_kept, to_pages=to_pages, to_weights=to_weights)
            c = calls.pop()
            assert c["to_pages"].data_ptr() == pages.data_ptr() and c["to_weights"] is gets and c["stride"] == b.max_pages * BS
    r.evict(t["n_ctx"], pages, t["k_pages"], t["v_pages"], w, 1, 1, 50, kept, n_kept, to_pages=pages.clone())
    assert calls.pop()["to_weights"] is None      # other pages: nothing is written unless it is said where
