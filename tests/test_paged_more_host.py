"""Rotation, pages in 8 bits and selected pages without a GPU: the oracle on cases worked by hand, and everything the calls refuse."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2502_13542_amd import binding as B
from paper_2502_13542_amd import harness as H

from paged_utils import BS, Batch, f64, shape_of
from test_paged_host import A16, FORM, LLAMA, ROWS, TABLE

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


# ---------------------------------------------------------------- the oracle
def test_oracle_rotation_by_hand():
    table = np.array([[[1.0] * 8, [0.0] * 8], [[0.0] * 8, [1.0] * 8]])        # not at all; a quarter turn
    x = np.arange(40.0).reshape(2, 1, 20)
    y, size = po.rotate(x, table, [-3, 99], False)                            # (clamped to 0 and 1)
    assert np.array_equal(y[0], x[0])
    assert np.array_equal(y[1, 0, :8], -x[1, 0, 8:16]) and np.array_equal(y[1, 0, 8:16], x[1, 0, :8])
    assert np.array_equal(y[1, 0, 16:], x[1, 0, 16:]) and (size >= np.abs(y)).all()
    y, _ = po.rotate(x, table, [0, 1], True)
    assert np.array_equal(y[1, 0, :16:2], -x[1, 0, 1:16:2]) and np.array_equal(y[1, 0, 1:16:2], x[1, 0, :16:2])
    # a turn keeps the length of a pair, and two turns add up
    a = np.array([0.3, 1.9])
    t = np.stack([np.cos(a)[:, None] * np.ones(8), np.sin(a)[:, None] * np.ones(8)], 1)
    both = np.stack([np.cos(a.sum()) * np.ones((1, 8)), np.sin(a.sum()) * np.ones((1, 8))], 1)
    z = po.rotate(po.rotate(x, t, [0, 0], False)[0], t, [1, 1], False)[0]
    assert np.allclose(z, po.rotate(x, both, [0, 0], False)[0])


def test_oracle_codes_are_those_of_the_type():
    """All values between neighbouring codes, their middles and just beside them, against torch's type."""
    codes = torch.arange(0, 127, dtype=torch.uint8).view(E4M3).double().numpy()
    middle = (codes[1:] + codes[:-1]) / 2
    x = np.concatenate([codes, middle, np.nextafter(middle, 0), np.nextafter(middle, 999)])
    x = np.concatenate([x, -x])
    # the nearest of the type's values, of two the one with the even code (torch's own conversion goes through fp32 first)
    far = np.abs(np.abs(x)[:, None] - codes)
    best = far.argmin(1)
    best += (best + 1 < len(codes)) & (far[np.arange(len(x)), np.minimum(best + 1, len(codes) - 1)] == far.min(1)) & (best % 2 == 1)
    assert np.array_equal(po.round_e4m3(x), np.sign(x) * codes[best])
    assert np.array_equal(po.round_e4m3(np.float32(x)), torch.tensor(np.float32(x)).to(E4M3).double().numpy())
    assert np.isnan(po.round_e4m3([np.nan, np.inf])).all()


def test_oracle_scales_by_hand():
    for x, e in ((448.0, 0), (448.0001, 1), (1.0, -8), (1.75, -8), (1.7500001, -7), (0.0, -100), (2.0 ** -110, -100), (np.inf, -100), (2.0 ** 126, 118)):
        assert po.scale_exponent(np.array([0.0, -x, np.nan])) == e, x


def test_oracle_quantised_append_by_hand():
    """A page with two tokens of scale 2^-8 gets one that needs 2^-4: the old codes lose up to four bits at the bottom."""
    k0, v0 = np.zeros((1, 1, BS, 2)), np.zeros((1, 1, 2, BS))
    k0[0, 0, 0], k0[0, 0, 1] = [16.0, 0.046875], [-448.0, 2.0 ** -9]
    s = np.full((1, 1), 2.0 ** -8)
    k, v, ks, vs = po.quantised_append(np.array([[[20.0, 0.3]]]), np.array([[[0.5, -1.5]]]), [0, 1], [3], np.array([[0]]), k0, v0, s, s)
    assert ks[0, 0] == 2.0 ** -4 and vs[0, 0] == 2.0 ** -8
    assert k[0, 0, :3].tolist() == [[1.0, 0.00390625], [-28.0, 0.0], [320.0, 4.5 + 0.5]]
    assert v[0, 0, :, 2].tolist() == [128.0, -384.0] and (v[0, 0, :, :2] == 0).all()
    k, _, ks, _ = po.quantised_append(np.array([[[20.0, 0.3]]]), np.array([[[0.5, -1.5]]]), [0, 1], [1], np.array([[0]]), k0, v0, s * 2.0 ** 90, s)
    assert ks[0, 0] == 2.0 ** -4 and k[0, 0, 1].tolist() == k0[0, 0, 1].tolist()     # its first slot is new: anew; the others are left alone


def test_oracle_selection_by_hand():
    bounds = np.zeros((5, 1, 2, 2))
    bounds[:, 0, 0], bounds[:, 0, 1] = -1.0, [[1, 1], [2, 1], [3, 0], [0, 0], [2, 1]]
    q = np.array([[[1.0, -2.0], [0.5, 0.5]]])                                 # largest of two heads: x + 2 and (x + y) / 2
    pages = np.array([[4, 0, 1, 2, 3, -1]])
    scores, chosen = po.select_pages(q, [0, 1], [5 * BS], pages, bounds, 3, 1, 1)
    assert scores[0, 0, :5].tolist() == [4.0, 3.0, 4.0, 5.0, 2.0] and np.isneginf(scores[0, 0, 5])
    assert chosen[0] == [[0, 3, 4]]                                           # the first, the last, the best
    assert po.select_pages(q, [0, 1], [5 * BS], pages, bounds, 2, 0, 0)[1][0] == [[0, 3]]      # of equals the lower page
    assert po.select_pages(q, [0, 1], [2 * BS], pages, bounds, 3, 0, 0)[1][0] == [[0, 1]]
    pages[0, 0] = -1
    assert po.select_pages(q, [0, 1], [5 * BS], pages, bounds, 3, 1, 1)[1][0] == [[2, 3, 4]]   # a page of nobody is no candidate


def test_a_page_score_bounds_every_product_in_the_page():
    b = Batch(shape_of(4, 2, 64, "fp32"), [(3, 900)], 5, garbage=None)
    bounds = po.key_bounds(b.n_ctx, b.pages, f64(b.k_pages), np.zeros((b.n_pages, 2, 2, 64)))
    scores, _ = po.select_pages(f64(b.q), b.row_start, b.n_ctx, b.pages, bounds, 2, 0, 0)
    for i in range(7):
        k = f64(b.k_pages)[b.pages[0, i], :, : min(900 - i * BS, BS)]
        most = np.einsum("rhgd,htd->rhgt", f64(b.q).reshape(3, 2, 2, 64), k).max((2, 3))
        assert (scores[:, :, i] >= most).all()


def test_selected_attention_of_all_pages_is_attention():
    b = Batch(shape_of(4, 2, 64, "fp32"), [(3, 300), (2, 129)], 7)
    k, v = b.pools64()
    every = [[list(range(b.max_pages))] * 2 for _ in range(b.n_rows)]
    f = dict(softcap=3.0, window=200, slopes=np.array([0.1, 0.2, 0.3, 0.4]))
    want = po.attention(f64(b.q), b.row_start, b.n_ctx, b.pages, k, v, 0.1, **f)
    got = po.attention_selected(f64(b.q), b.row_start, b.n_ctx, b.pages, k, v, every, 0.1, **f)
    for x in ("out", "lse", "mass", "size"):
        assert np.allclose(got[x], want[x], rtol=1e-12)


# ---------------------------------------------------------------- refusals
def call(lib, name, order, defaults, cs, kw):
    assert set(kw) <= set(defaults)
    a = {**defaults, **kw}
    return getattr(lib, "actqkv_paged_" + name)(ctypes.byref(cs), *(a[x] for x in order.split()), None)


T = dict(batch=2, n_rows=9, max_new=5, rs=A16, n=A16, pages=A16, max_pages=4, kp=A16, vp=A16, n_pages=9)
TURN = dict(rotation=A16, n_positions=100, rotary=64, pairs=0, row_pos=None, q=A16, q_out=A16)
F = dict(softcap=0.0, window=0, slopes=None, first=None, end=None, out=A16, lse=None, ws=A16, wsb=1 << 40)


def rotated(lib, cs, **kw):
    return call(lib, "append_rotated", "batch n_rows max_new q k v rs n pages max_pages kp vp n_pages rotation n_positions rotary pairs row_pos q_out",
                dict(T, **TURN, k=A16, v=A16), cs, kw)


def append8(lib, cs, **kw):
    return call(lib, "append_quantised", "batch n_rows max_new q k v rs n pages max_pages kp vp n_pages ks vs rotation n_positions rotary pairs row_pos q_out",
                dict(T, **TURN, k=A16, v=A16, ks=A16, vs=2 * A16), cs, kw)


def attend8(lib, cs, **kw):
    return call(lib, "attention_quantised", "batch n_rows max_new q rs n pages max_pages kp vp n_pages ks vs softcap window slopes first end out lse ws wsb",
                dict(T, **F, q=A16, ks=A16, vs=A16), cs, kw)


def bounds(lib, cs, **kw):
    return call(lib, "key_bounds", "batch n_rows max_new rs n pages max_pages kp n_pages bounds", dict(T, bounds=2 * A16), cs, kw)


def select(lib, cs, **kw):
    return call(lib, "select_pages", "batch n_rows max_new q rs n pages max_pages bounds n_pages k_sel keep_first keep_last scores stride idx n_sel ws wsb",
                dict(T, q=A16, bounds=A16, k_sel=4, keep_first=1, keep_last=1, scores=A16, stride=4, idx=A16, n_sel=A16, ws=A16, wsb=1 << 40), cs, kw)


def selected(lib, cs, **kw):
    return call(lib, "attention_selected", "batch n_rows max_new q rs n pages max_pages kp vp n_pages idx n_sel k_sel softcap window slopes first end out lse ws wsb",
                dict(T, **F, q=A16, idx=A16, n_sel=A16, k_sel=4), cs, kw)


TURNS = [(dict(rotation=A16 + 4), -3), (dict(n_positions=0), -1), (dict(rotary=0), -2), (dict(rotary=8), -2), (dict(rotary=24), -2),
         (dict(rotary=144), -2), (dict(rotary=-16), -2), (dict(pairs=2), -1), (dict(pairs=-1), -1), (dict(row_pos=A16 + 2), -3), (dict(q=None), -1),
         (dict(q_out=None), -1), (dict(q=A16 + 8), -3), (dict(q_out=A16 + 4), -3)]
NEW = [(dict(k=None), -1), (dict(v=None), -1), (dict(k=A16 + 4), -3), (dict(v=A16 + 8), -3)]


@pytest.mark.parametrize("bad,code", TABLE + ROWS + TURNS + NEW)
def test_append_refusals(lib, bad, code):
    for f in (rotated, append8):
        assert f(lib, B.c_shape(LLAMA), **bad) == code
        assert B.last_error()


NONE = dict(rotation=None, n_positions=0, rotary=0, q=None, q_out=None)


@pytest.mark.parametrize("bad,code", [(dict(ks=None), -1), (dict(vs=None), -1), (dict(ks=A16 + 2), -3), (dict(vs=A16 + 1), -3), (dict(vs=A16), -1),
                                      (dict(NONE, q=A16, q_out=A16), -1), (dict(NONE, row_pos=A16), -1), (dict(NONE, rotary=64), -1)])
def test_append8_refusals(lib, bad, code):
    assert append8(lib, B.c_shape(LLAMA), **bad) == code
    assert B.last_error()


def test_rotation_is_required_where_it_is_what_the_call_does(lib):
    assert rotated(lib, B.c_shape(LLAMA), **NONE) == -1


@pytest.mark.parametrize("bad,code", TABLE + ROWS + FORM)
def test_attention_refusals(lib, bad, code):
    assert attend8(lib, B.c_shape(LLAMA), **bad) == code
    assert selected(lib, B.c_shape(LLAMA), **bad) == code


@pytest.mark.parametrize("bad,code", [(dict(ks=None), -1), (dict(vs=None), -1), (dict(ks=A16 + 2), -3), (dict(vs=A16 + 1), -3), (dict(softcap=1e-30), -1)])
def test_attention8_refusals(lib, bad, code):
    assert attend8(lib, B.c_shape(LLAMA), **bad) == code


LISTS = [(dict(k_sel=0), -1), (dict(k_sel=-1), -1), (dict(k_sel=(1 << 23) + 1), -2), (dict(idx=None), -1), (dict(idx=A16 + 2), -3), (dict(n_sel=None), -1),
         (dict(n_sel=A16 + 1), -3), (dict(n_rows=(1 << 19) + 1, max_new=1), -2)]


@pytest.mark.parametrize("bad,code", LISTS)
def test_selected_refusals(lib, bad, code):
    assert selected(lib, B.c_shape(LLAMA), **bad) == code
    assert select(lib, B.c_shape(LLAMA), **bad) == code


@pytest.mark.parametrize("bad,code", [x for x in TABLE if "kp" not in x[0] and "vp" not in x[0]] + ROWS + [
    (dict(bounds=None), -1), (dict(bounds=A16 + 8), -3), (dict(q=None), -1), (dict(q=A16 + 8), -3), (dict(keep_first=-1), -1), (dict(keep_last=-1), -1),
    (dict(keep_first=3, keep_last=2), -1), (dict(keep_first=2 ** 31 - 1, keep_last=2 ** 31 - 1), -1), (dict(scores=None), -1), (dict(scores=A16 + 2), -3),
    (dict(stride=3), -1), (dict(ws=None), -4), (dict(ws=A16 + 8), -4), (dict(wsb=64), -4)])
def test_select_refusals(lib, bad, code):
    assert select(lib, B.c_shape(LLAMA), **bad) == code


@pytest.mark.parametrize("bad,code", [x for x in TABLE if "vp" not in x[0]] + [(dict(bounds=None), -1), (dict(bounds=A16 + 4), -3), (dict(bounds=A16), -1),
                                      (dict(rs=A16 + 2), -3), (dict(n_rows=0), -1), (dict(max_new=10), -1)])
def test_bounds_refusals(lib, bad, code):
    assert bounds(lib, B.c_shape(LLAMA), **bad) == code


@pytest.mark.parametrize("shape,code", [((32, 8, 96, "bf16"), -2), ((9, 2, 64, "bf16"), -2), ((18, 2, 64, "fp32"), -2)])
def test_shapes_refused(lib, shape, code):
    for f in (rotated, append8, attend8, bounds, select, selected):
        assert f(lib, B.c_shape(shape_of(*shape))) == code


def test_the_runner_checks_sizes():
    b = Batch(shape_of(4, 2, 64, "fp32"), [(2, 40), (3, 200)], 3)
    r, t = b.runner("cpu"), b.dev("cpu")
    call = dict(row_start=t["row_start"], n_ctx=t["n_ctx"], pages=t["pages"])
    table = dict(t)
    table8 = dict(call, k_pages=t["k_pages"].to(E4M3), v_pages=t["v_pages"].to(E4M3), k_scales=torch.ones(b.n_pages, 2), v_scales=torch.ones(b.n_pages, 2))
    rows = dict(k_new=b.k_new, v_new=b.v_new)
    turn = dict(rotation=torch.zeros(300, 2, 16), q=b.q, q_out=torch.zeros_like(b.q), row_pos=torch.zeros(5, dtype=torch.int32))
    out, lse = torch.zeros_like(b.q), torch.zeros(5, 4)
    bounds = torch.zeros(b.n_pages, 2, 2, 64)
    lists = dict(idx=torch.zeros(5, 2, 3, dtype=torch.int32), n_sel=torch.zeros(5, 2, dtype=torch.int32))
    form = dict(out=out, lse=lse, slopes=torch.ones(4), row_first=torch.zeros(5, dtype=torch.int32), row_end=torch.zeros(5, dtype=torch.int32))
    calls = [
        (r.append_rotated, {**rows, **table, **turn}, ["k_new", "v_new", "row_start", "n_ctx", "k_pages", "q", "q_out", "row_pos"]),
        (r.append_quantised, {**rows, **table8, **turn}, ["k_new", "v_new", "row_start", "n_ctx", "k_pages", "v_pages", "k_scales", "v_scales", "q", "q_out", "row_pos"]),
        (r.attend_quantised, dict(q=b.q, **table8, **form), ["out", "lse", "row_start", "n_ctx", "k_scales", "v_scales", "slopes", "row_first", "row_end"]),
        (r.key_bounds, dict(n_ctx=t["n_ctx"], pages=t["pages"], k_pages=t["k_pages"], bounds=bounds), ["n_ctx", "k_pages", "bounds"]),
        (r.key_bounds, dict(call, k_pages=t["k_pages"], bounds=bounds, n_rows=5), ["n_ctx", "k_pages", "bounds", "row_start"]),
        (r.select_pages, dict(q=b.q, **call, bounds=bounds, keep_first=0, keep_last=1, scores=torch.zeros(5, 2, b.max_pages), **lists),
         ["row_start", "n_ctx", "bounds", "n_sel"]),
        (r.attend_selected, dict(q=b.q, **table, **lists, **form), ["out", "lse", "row_start", "n_ctx", "n_sel", "slopes", "row_first", "row_end"]),
    ]
    for f, good, names in calls:
        with pytest.raises(B.ActQKVError, match="not on the GPU"):     # sizes are right: the next check is the device
            f(**good)
        for name in names:
            bad = dict(good)
            bad[name] = good[name].reshape(-1)[:-1] if good[name].dim() == 1 else good[name][..., :-1].contiguous()
            with pytest.raises(B.ActQKVError) as e:
                f(**bad)
            assert "not on the GPU" not in str(e.value), name
        if "max_new" in f.__code__.co_varnames and (f != r.key_bounds or "row_start" in good):
            for max_new in (0, 4, -1):
                with pytest.raises(B.ActQKVError, match="max_new"):
                    f(**good, max_new=max_new)
    short = {**lists, "idx": lists["idx"][:4]}
    with pytest.raises(B.ActQKVError):
        r.select_pages(b.q, **call, bounds=bounds, keep_first=0, keep_last=1, scores=torch.zeros(5, 2, b.max_pages), **short)
    with pytest.raises(B.ActQKVError):
        r.attend_selected(b.q, **table, **short, **form)
    with pytest.raises(B.ActQKVError):
        r.select_pages(b.q, **call, bounds=bounds, keep_first=0, keep_last=1, scores=torch.zeros(4, 2, b.max_pages), **lists)
    with pytest.raises(B.ActQKVError, match="rotary_dim"):
        r.append_rotated(**rows, **table, rotation=torch.zeros(300, 16))
    with pytest.raises(B.ActQKVError, match="made for"):
        r.key_bounds(**call, k_pages=t["k_pages"], bounds=bounds, n_rows=6)
    small = H.PagedRunner(b.shape, 1, 5, 3, b.max_pages, "cpu")
    for f, good, _ in calls:
        with pytest.raises(B.ActQKVError, match="made for"):
            getattr(small, f.__name__)(**good)
    none = dict(k_new=b.k_new[:0], v_new=b.v_new[:0])                 # no rows: nothing to do
    r.append_rotated(**none, **table, rotation=turn["rotation"])
    r.append_quantised(**none, **table8)
    r.key_bounds(**call, k_pages=t["k_pages"], bounds=bounds, n_rows=0)


def test_the_calls_want_their_types():
    """Codes as float8, scales, tables and scores as fp32: another type is refused before anything is launched."""
    b = Batch(shape_of(4, 2, 64, "fp32"), [(2, 40), (3, 200)], 3)
    r, t = b.runner("cpu"), b.dev("cpu")
    assert {"paged_append_quantised", "paged_attention_quantised"} <= set(dir(B._calls()))
    with pytest.raises(B.ActQKVError):
        r.append_quantised(b.k_new, b.v_new, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], torch.ones(b.n_pages, 2), torch.ones(b.n_pages, 2))


def test_workspace_holds_the_parts_of_selected_rows(lib):
    cs = B.c_shape(LLAMA)
    assert B.paged_workspace_bytes(cs, 1, 200, 200, 64) >= 8192 + 16 * 130 * 4 * (1024 + 1024)
    rng = np.random.default_rng(0)
    for _ in range(200):
        batch, max_new, max_pages = (int(2 ** rng.uniform(0, t)) for t in (8, 12, 11))
        n_rows = int(rng.integers(max_new, batch * max_new + 1))
        big = B.paged_workspace_bytes(cs, batch, n_rows, max_new, max_pages)
        small = [int(rng.integers(1, x + 1)) for x in (batch, n_rows, max_new, max_pages)]
        small[2] = min(small[1], small[2])
        assert B.paged_workspace_bytes(cs, *small) <= big
