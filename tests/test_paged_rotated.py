"""Append with rotation against the plain fp64 implementation, on the GPU.

A turned channel is a difference or sum of two products in fp32, one of them rounded by itself, and the result is rounded once more:
off by at most 2 e(fp32) (|a c| + |b s|), and in bf16 half a step more.  Other channels and values are copies."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2502_13542_amd import harness as H

from paged_utils import BS, Batch, f64, shape_of
from test_paged import BATCHES, E16, E32, SHAPES, clamped_batch

pytestmark = pytest.mark.gpu
DEV = "cuda"


def table_of(rotary, n, seed=0):
    """Cosines and sines, some rows larger than 1 (a model's factor)."""
    inv = 10000.0 ** (-np.arange(0, rotary, 2) / rotary)
    angle = np.arange(n)[:, None] * inv
    return torch.tensor(np.stack([np.cos(angle), np.sin(angle)], 1) * 1.1, dtype=torch.float32)


def bound_of(dtype, want, size):
    b = 2 * E32 * size
    return b + E16 * (np.abs(want) + b) if dtype == "bf16" else b


def run(b, rotary, interleaved=False, far=False, keys_alone=False, in_place=False, runner=None, stream=None, **kw):
    t = b.dev()
    table = table_of(rotary, 700 if far else max(int(max(b.n_ctx)), 1))
    places = b.positions()
    row_pos = None
    if far:                                       # places beside the positions, some outside the table
        places = np.random.default_rng(7).integers(-5, 720, b.n_rows)
        places[:: 9] = np.resize([2 ** 31 - 1, -(2 ** 31)], len(places[:: 9]))
        row_pos = torch.tensor(places, dtype=torch.int32, device=DEV)
    q = None if keys_alone else b.q.to(DEV)
    q_out = None if keys_alone else (q if in_place else torch.full_like(q, 7.0))
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    args = (b.k_new.to(DEV), b.v_new.to(DEV), t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], table.to(DEV))
    torch.cuda.synchronize()
    (runner or b.runner()).append_rotated(*args, q=q, q_out=q_out, row_pos=row_pos, interleaved=interleaved, stream=stream, **kw)
    torch.cuda.synchronize()
    turned, size = po.rotate(f64(b.k_new), f64(table), places, interleaved)
    k0, v0 = f64(b.k_pages), f64(b.v_pages)
    kw_, vw = po.append(turned, f64(b.v_new), b.row_start, b.n_ctx, b.pages, k0, v0)
    ks, _ = po.append(size, f64(b.v_new), b.row_start, b.n_ctx, b.pages, np.zeros_like(k0), v0)
    got = f64(t["k_pages"])
    still = ks == 0                               # (written nowhere, or products that are all zero)
    assert np.array_equal(got[still], kw_[still], equal_nan=True), "a slot of nobody's was written"
    off = np.abs(got - kw_)[~still] - bound_of(b.shape.dtype, kw_, ks)[~still]
    assert off.size == 0 or (off <= 0).all(), f"keys off by {off.max():.3e} more than their bound"
    if rotary < b.shape.head_dim:
        assert np.array_equal(got[..., rotary:], kw_[..., rotary:], equal_nan=True)
    assert np.array_equal(f64(t["v_pages"]), vw, equal_nan=True)
    if not keys_alone:
        want, size = po.rotate(f64(b.q), f64(table), places, interleaved)
        pos = b.positions()
        mine = np.zeros(b.n_rows, bool)
        mine[b.row_start[0]: b.row_start[-1]] = True
        mine &= pos >= 0
        off = np.abs(f64(q_out) - want)[mine] - bound_of(b.shape.dtype, want, size)[mine]
        assert (off <= 0).all(), f"queries off by {off.max():.3e} more than their bound"
        left = f64(b.q) if in_place else np.full(b.q.shape, 7.0)
        assert np.array_equal(f64(q_out)[~mine], left[~mine]), "rows of nobody were written"


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("batch", list(BATCHES))
def test_rotated(shape, batch):
    sh = shape_of(*SHAPES[shape])
    run(Batch(sh, BATCHES[batch], 3, extra_rows=(1, 2)), sh.head_dim)


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("rotary", [16, 32, 48, 64])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotated_parts_and_pairs(shape, rotary, interleaved):
    run(Batch(shape_of(*SHAPES[shape]), BATCHES["chunks"], 5, extra_rows=(0, 1)), rotary, interleaved, far=True)


@pytest.mark.parametrize("shape", ["llama", "fp32_64", "g5_64", "fp32_g3"])
@pytest.mark.parametrize("batch", ["steps", "chunks"])
def test_rotated_in_place_and_keys_alone(shape, batch):
    b = Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 7, extra_rows=(2, 0))
    run(b, 64, in_place=True)
    run(b, 64, interleaved=True, keys_alone=True)


@pytest.mark.parametrize("layer", [(8, 1, 128, "bf16"), (7, 1, 64, "fp32"), (48, 6, 64, "bf16"), (5, 1, 128, "fp32")])
def test_rotated_of_other_groups(layer):
    run(Batch(shape_of(*layer), BATCHES["chunks"], 6, extra_rows=(1, 1)), 32, interleaved=True)
    run(Batch(shape_of(*layer), BATCHES["steps"], 6), 64)


MIXED = [[(1, 30)] * 40 + [(100, 300), (8, 200), (9, 140)] + [(2, 129)] * 17 + [(0, 3), (40, 40)],      # more than a launch takes along, and an odd one among them
         [(int(m), int(m + n)) for m, n in zip(np.random.default_rng(3).integers(0, 12, 150), np.random.default_rng(4).integers(0, 140, 150))]]


@pytest.mark.parametrize("shape", ["llama", "mha64", "fp32_g3"])
@pytest.mark.parametrize("seqs", MIXED)
def test_rotated_steps_beside_chunks(shape, seqs):
    run(Batch(shape_of(*SHAPES[shape]), seqs, 8, extra_rows=(1, 2), extra_entries=0), 64)
    run(Batch(shape_of(*SHAPES[shape]), [(1, 60)] * 400 + [(33, 100)], 8, extra_entries=0), 64)


def test_rotated_without_pages_and_at_clamped_lengths():
    b = Batch(shape_of(*SHAPES["llama"]), BATCHES["chunks"], 9, garbage=None)
    b.pages[0, 1] = b.n_pages                     # no page: keys go nowhere, queries are turned
    b.pages[4, 2] = -1
    run(b, 128)
    for shape in ("llama", "fp32_64"):
        run(clamped_batch(shape), 64)


def test_rotated_of_more_rows_than_a_launch_has_workgroups_for():
    """2.3 million rows of one sequence: the workgroups go round.  (Checked on the device, in 64 bits.)"""
    sh = shape_of(1, 1, 64, "bf16")
    m, n = 2_300_000, 2_300_077
    max_pages = -(-n // BS)
    g = torch.Generator(device=DEV).manual_seed(3)
    k, v, q = (torch.randn(m, 1, 64, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(3))
    kp, vp = torch.zeros(max_pages, 1, BS, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(max_pages, 1, 64, BS, dtype=torch.bfloat16, device=DEV)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    table = table_of(64, 50).to(DEV)
    places = torch.randint(0, 50, (m,), dtype=torch.int32, device=DEV)
    pages = torch.randperm(max_pages, device=DEV).int()[None].contiguous()
    H.PagedRunner(sh, 1, m, m, max_pages).append_rotated(k, v, i32([0, m]), i32([n]), pages, kp, vp, table, q=q, q_out=q, row_pos=places)
    torch.cuda.synchronize()
    pos = torch.arange(n - m, n, device=DEV)
    page = pages[0, pos // BS].long()
    assert torch.equal(vp[page, 0, :, pos % BS], v[:, 0])
    cos, sin = (table[places.long(), i].double() for i in (0, 1))
    a, b = k[:, 0, :32].double(), k[:, 0, 32:].double()
    want = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    size = torch.cat([(a * cos).abs() + (b * sin).abs(), (b * cos).abs() + (a * sin).abs()], -1)
    bound = 2 * E32 * size
    bound = bound + E16 * (want.abs() + bound)
    assert ((kp[page, 0, pos % BS].double() - want).abs() <= bound).all()
    assert (kp.reshape(max_pages, -1).abs().sum(1) > 0).sum() == -(-n // BS) - (n - m) // BS


def test_rotated_on_a_side_stream_and_through_a_larger_runner():
    b = Batch(shape_of(*SHAPES["g7"]), BATCHES["few"], 13)
    r = H.PagedRunner(b.shape, 9, 900, 300, 12)
    run(b, 128, runner=r, stream=torch.cuda.Stream(), max_new=4)
    run(b, 128, runner=r)


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_rotated_replayed(shape):
    sh = shape_of(*SHAPES[shape])
    b = Batch(sh, [(1, 600), (4, 300), (90, 90)], 15, garbage=None)
    r, t = b.runner(), b.dev()
    table = table_of(64, 800).to(DEV)
    q, kn, vn = b.q.to(DEV), b.k_new.to(DEV), b.v_new.to(DEV)
    given = t["k_pages"].clone(), t["v_pages"].clone()
    q_out, row_pos = torch.zeros_like(q), torch.zeros(b.n_rows, dtype=torch.int32, device=DEV)

    def step():
        r.append_rotated(kn, vn, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], table, q=q, q_out=q_out, row_pos=row_pos)

    def state():
        torch.cuda.synchronize()
        got = [x.clone() for x in (q_out, t["k_pages"], t["v_pages"])]
        for x, x0 in zip((t["k_pages"], t["v_pages"]), given):
            x.copy_(x0)
        q_out.zero_()
        return got

    step()
    state()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    last = None
    for n_ctx in ([600, 300, 90], [130, 299, 90], [5, 17, 95]):
        t["n_ctx"].copy_(torch.tensor(n_ctx, dtype=torch.int32))
        for x in (q, kn, vn):
            x.copy_(torch.randn(x.shape).to(x.dtype))
        row_pos.copy_(torch.randint(0, 800, (b.n_rows,), dtype=torch.int32))
        step()
        want = state()
        assert last is None or not any(torch.equal(x, y) for x, y in zip(last, want))
        last = want
        for _ in range(2):
            graph.replay()
            assert all(torch.equal(x, y) for x, y in zip(state(), want))
