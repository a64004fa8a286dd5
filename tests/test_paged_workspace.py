"""What the calls on pages need of a workspace: each what it needs itself, and attention no more for the calls that were added beside it."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2502_13542_amd import binding as B
from paper_2502_13542_amd import harness as H

from paged_utils import Batch, shape_of
from test_paged_host import LLAMA, _attend, _weigh
from test_paged_more_host import attend8, select, selected

MIB = 1 << 20
# shape, (batch, n_rows, max_new, max_pages), bytes of the attention's pieces of chunks and counters: 512 pieces of 256 rows (fp32: 128), each 4 bytes
# a channel and 8 a row and lane half, or as many as there can be
PIECE16, PIECE32 = 8 * (16 * 64 + 32) * 16, 4 * (16 * 64 + 32) * 16
SIZES = [(LLAMA, (2, 4096, 2048, 128), 512 * PIECE16),
         (shape_of(32, 8, 128, "fp32"), (2, 4096, 2048, 128), 512 * PIECE32)]


@pytest.mark.parametrize("case", range(len(SIZES)))
def test_attention_needs_no_more_for_the_other_calls(case):
    """Pieces of chunks (or the kept scores of few rows, if those are more), and the counters."""
    shape, sizes, pieces = SIZES[case]
    cs = B.c_shape(shape)
    batch, _, _, max_pages = sizes
    pairs, cols = batch * shape.n_kv_heads, 16 // shape.group * shape.group
    steps = (min(pairs, 1024) + 1024) * 16 * (shape.head_dim + 2) * 4 + pairs * cols * max_pages * 128 * 4
    assert B.paged_attention_workspace_bytes(cs, *sizes) <= 8192 + max(pieces, steps) + 512
    assert B.paged_workspace_bytes(cs, *sizes) >= 2 * pieces                   # (pages in 8 bits are cut into twice as many)


@pytest.mark.parametrize("sizes", [(1, 1, 1, 1), (64, 64, 1, 64), (2, 4096, 2048, 128), (1, 200, 200, 64), (16, 512, 64, 3000)])
@pytest.mark.parametrize("shape", [LLAMA, shape_of(8, 2, 64, "fp32"), shape_of(28, 4, 128, "bf16")])
def test_a_call_is_refused_for_less_than_it_needs_and_told_how_much(sizes, shape):
    """(refused before anything is launched: the pointers are not looked at)"""
    cs, lib = B.c_shape(shape), B.load_library()
    batch, n_rows, max_new, max_pages = sizes
    kw = dict(batch=batch, n_rows=n_rows, max_new=max_new, max_pages=max_pages)
    needs = {}
    for name, call, more in (("attention", _attend, {}), ("attention_weights", _weigh, dict(stride=max_pages * 128)), ("attention_quantised", attend8, {}),
                             ("select_pages", select, dict(stride=max_pages)), ("attention_selected", selected, {})):
        assert call(lib, cs, **kw, **more, wsb=1) == -4
        text = B.last_error()
        assert f"paged_{name} needs" in text
        needs[name] = int(text.split()[-1])
        assert call(lib, cs, **kw, **more, wsb=needs[name] - 1) == -4
    assert needs["attention"] == needs["attention_weights"] == B.paged_attention_workspace_bytes(cs, *sizes)
    assert max(needs.values()) == B.paged_workspace_bytes(cs, *sizes)


def test_workspace_of_attention_serves_smaller_calls():
    rng = np.random.default_rng(1)
    for shape in (LLAMA, shape_of(8, 2, 64, "fp32"), shape_of(16, 2, 128, "fp32"), shape_of(8, 8, 64, "bf16")):
        cs = B.c_shape(shape)
        for _ in range(100):
            batch, max_new, max_pages = (int(2 ** rng.uniform(0, t)) for t in (8, 12, 11))
            n_rows = int(rng.integers(max_new, batch * max_new + 1))
            big = B.paged_attention_workspace_bytes(cs, batch, n_rows, max_new, max_pages)
            assert big <= B.paged_workspace_bytes(cs, batch, n_rows, max_new, max_pages)
            for _ in range(4):
                small = [int(rng.integers(1, x + 1)) for x in (batch, n_rows, max_new, max_pages)]
                small[2] = min(small[1], small[2])
                assert B.paged_attention_workspace_bytes(cs, *small) <= big
    lib = B.load_library()
    for bad in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 2, 1), (1, 1, 1, 0), (1, 1, 1, 1 << 24)):
        assert lib.actqkv_paged_attention_workspace_bytes(ctypes.byref(B.c_shape(LLAMA)), *bad) == 0
        with pytest.raises(B.ActQKVError):
            B.paged_attention_workspace_bytes(B.c_shape(LLAMA), *bad)


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [(32, 8, 128, "bf16"), (8, 2, 64, "fp32")])
def test_calls_in_a_workspace_of_exactly_what_they_need(layer):
    """With a guard behind it, attention and the account in the smaller one: the results of a large one."""
    shape = shape_of(*layer)
    b = Batch(shape, [(300, 2100), (1, 900), (40, 700)], 5, garbage=None, extra_entries=30)
    t, q = b.dev(), b.q.to("cuda")
    got = []
    for kind in ("exact", "large"):
        r = H.PagedRunner(shape, b.batch, b.n_rows, b.max_new, b.max_pages, attention_only=kind == "exact")
        if kind == "exact":
            assert r.workspace.numel() < H.PagedRunner(shape, b.batch, b.n_rows, b.max_new, b.max_pages).workspace.numel()
            size, guard = r.workspace.numel(), torch.zeros(r.workspace.numel() + 4096, dtype=torch.uint8, device="cuda")
            guard[size:] = 0xA5
            r.workspace = guard[:size]
        out, lse = torch.zeros_like(q), torch.zeros(b.n_rows, shape.n_q_heads, device="cuda")
        out2, w = torch.zeros_like(q), torch.zeros(b.batch, shape.n_kv_heads, b.max_pages * 128, device="cuda")
        r.attend(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], out, lse)
        r.attend_weigh(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], out2, lse, 16, w)
        torch.cuda.synchronize()
        if kind == "exact":
            assert (guard[size:] == 0xA5).all()
        got.append((out, lse, out2, w))
    assert all(torch.equal(x, y) for x, y in zip(*got))


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [(32, 8, 128, "bf16"), (8, 2, 64, "fp32")])
@pytest.mark.parametrize("seqs", [[(300, 2100), (1, 900), (40, 700)], [(1, 2100), (2, 900), (1, 1)]])
@pytest.mark.parametrize("call", ["quantised", "selected"])
def test_the_other_calls_in_a_workspace_of_exactly_what_they_need(layer, seqs, call):
    from test_paged_quantised import pools8, quantise
    shape = shape_of(*layer)
    b = Batch(shape, seqs, 7, garbage=None, extra_entries=20)
    t, q, r = b.dev(), b.q.to("cuda"), b.runner()
    out, lse = torch.zeros_like(q), torch.zeros(b.n_rows, shape.n_q_heads, device="cuda")
    if call == "quantised":
        pools = pools8(quantise(b, 3, garbage=False))
        run = lambda *o: r.attend_quantised(q, t["row_start"], t["n_ctx"], t["pages"], *pools, *o)
    else:
        idx = torch.arange(b.max_pages, dtype=torch.int32, device="cuda").repeat(b.n_rows, shape.n_kv_heads, 1)
        n_sel = torch.full((b.n_rows, shape.n_kv_heads), b.max_pages, dtype=torch.int32, device="cuda")
        run = lambda *o: r.attend_selected(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], idx, n_sel, *o)
    run(out, lse)
    r.workspace = r.workspace[:16]
    with pytest.raises(B.ActQKVError, match=f"paged_attention_{call} needs") as e:
        run(out, lse)
    size = int(str(e.value).split()[-1])
    guard = torch.zeros(size + 4096, dtype=torch.uint8, device="cuda")
    guard[size:] = 0xA5
    r.workspace = guard[:size]
    again, again_lse = torch.zeros_like(q), torch.zeros_like(lse)
    run(again, again_lse)
    torch.cuda.synchronize()
    assert (guard[size:] == 0xA5).all() and torch.equal(again, out) and torch.equal(again_lse, lse)
