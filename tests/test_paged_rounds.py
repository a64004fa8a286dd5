"""Appends of more items than a launch has workgroups: the workgroups go round."""
import numpy as np
import pytest
import torch

from paper_2502_13542_amd import binding as B
from paper_2502_13542_amd import harness as H

from paged_utils import BS, shape_of
from test_paged_cuts import cut_of

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
ROUND = [(2, 2, 64, "bf16"), (6, 3, 128, "fp32"), (16, 8, 128, "bf16")]


def many(layer):
    """A thousand sequences, each of a few slices of rows and a few pages: more items than a launch has workgroups."""
    rng = np.random.default_rng(layer[1])
    news = rng.integers(20, 150, 1000) if layer[1] == 8 else rng.integers(200, 700, 1000)
    if layer[1] == 3:
        news = news // 2
    return [(int(m), int(m + n)) for m, n in zip(news, rng.integers(0, 200, 1000))]


@pytest.mark.parametrize("layer", ROUND)
def test_items_of_many_sequences_are_more_than_workgroups(layer):
    """And those of the calls of one long sequence elsewhere; of the parts that the results below are compared with they are not."""
    long_one = [("append_quantised", 2 ** 22, 2 ** 15 + 1), ("append_rotated", 2_300_000, 17970)]
    for call, rows, max_pages in long_one:
        items, workgroups, _ = B.paged_cut(B.c_shape(shape_of(1, 1, 64, "bf16")), call, 1, rows, rows, max_pages)
        assert items > workgroups
    seqs = many(layer)
    for call in ("append_rotated", "append_quantised"):
        items, workgroups, _ = cut_of(call, layer[:3], seqs, 0, dtype=layer[3], queries=True)
        assert items > workgroups > 10000
        for at in range(0, 1000, 125):
            items, workgroups, _ = cut_of(call, layer[:3], seqs[at: at + 125], 0, dtype=layer[3], queries=True)
            assert items == workgroups


@pytest.mark.gpu
@pytest.mark.parametrize("layer", ROUND)
@pytest.mark.parametrize("call", ["append_rotated", "append_quantised"])
def test_appends_whose_workgroups_go_round_are_those_of_their_parts(layer, call):
    """Slices of rows, keys and values follow each other in a workgroup: the bits that eight calls of an eighth of the sequences leave."""
    from test_paged_rotated import table_of
    sh, seqs = shape_of(*layer), many(layer)
    g = torch.Generator(device=DEV).manual_seed(5)
    counts = [-(-n // BS) for _, n in seqs]
    max_pages, n_pages = max(counts), sum(counts)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(3)).int()
    pages, start = torch.full((1000, max_pages), -1, dtype=torch.int32), 0
    for s, c in enumerate(counts):
        pages[s, :c] = order[start: start + c]
        start += c
    rows = np.cumsum([0] + [m for m, _ in seqs])
    randn = lambda *n: torch.randn(*n, generator=g, device=DEV).to(sh.torch_dtype)
    loud = torch.exp2(torch.randint(-6, 7, (int(rows[-1]), 1, 1), generator=g, device=DEV).float()).to(sh.torch_dtype)
    k, v = (randn(int(rows[-1]), sh.n_kv_heads, sh.head_dim) * loud for _ in range(2))
    q, table = randn(int(rows[-1]), sh.n_q_heads, sh.head_dim), table_of(64, 1024).to(DEV)
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)
    got = []
    for parts in (1, 8):
        shapes = (n_pages, sh.n_kv_heads, BS, sh.head_dim), (n_pages, sh.n_kv_heads, sh.head_dim, BS)
        if call == "append_quantised":
            codes = [((torch.arange(np.prod(x), device=DEV) * 7 % 120).to(torch.uint8)).reshape(x).view(E4M3) for x in shapes]
            pools = codes + [torch.full((n_pages, sh.n_kv_heads), 2.0 ** -7, device=DEV) for _ in range(2)]
        else:
            pools = [torch.full(x, 3.0, dtype=sh.torch_dtype, device=DEV) for x in shapes]
        q_out, each = torch.full_like(q, 7.0), 1000 // parts
        r = H.PagedRunner(sh, each, int(rows[-1]), max(m for m, _ in seqs), max_pages)
        for s in range(0, 1000, each):
            at = slice(int(rows[s]), int(rows[s + each]))
            args = (k[at], v[at], i32(rows[s: s + each + 1] - rows[s]), i32([n for _, n in seqs[s: s + each]]), pages[s: s + each].to(DEV))
            if call == "append_quantised":
                r.append_quantised(*args, *pools, rotation=table, q=q[at], q_out=q_out[at])
            else:
                r.append_rotated(*args, *pools, table, q=q[at], q_out=q_out[at])
        torch.cuda.synchronize()
        got.append([q_out] + [x.view(torch.uint8) if x.dtype == E4M3 else x for x in pools])
    assert all(torch.equal(x, y) for x, y in zip(*got))
    assert (got[0][0] != 7.0).any(-1).all()
