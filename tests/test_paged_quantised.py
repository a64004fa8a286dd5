"""Append into pages in 8 bits and attention over them against the plain fp64 implementation, on the GPU.

Appended codes and scales are exact: a scale is a power of two, a rotated key is the fp32 value nearest to a sum of two products that 64 bits
hold, and a code the nearest one, ties to even.  Attention is over the values that codes and scales stand for, which enter the
products exactly, so that the bounds of attention over 16- and 32-bit pages hold (test_paged.py)."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2502_13542_amd import harness as H

from paged_utils import BS, Batch, f64, shape_of
from test_paged import BATCHES, CUTS, FORMS, SHAPES, check_out, clamped_batch, form_of, on_device
from test_paged_rotated import MIXED, bound_of, table_of

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4M3 = torch.float8_e4m3fn
NAN_CODE = 0x7f


def to_codes(x):
    """float64 code values as a float8 tensor (exact; NaN as the code of NaN)."""
    c = torch.tensor(np.nan_to_num(x)).float().to(E4M3).view(torch.uint8)
    return torch.where(torch.tensor(np.isnan(x)), NAN_CODE, c).view(E4M3)


def code_values(t):
    return t.detach().cpu().float().double().numpy()


def quantise(b, seed, scales=(-8, -4), garbage=True):
    """Pools of codes and their scales for a batch; behind the last token, and in pages of nobody, codes and scales that are no numbers."""
    g = torch.Generator().manual_seed(seed)
    sh = b.shape
    b.k8, b.v8 = ((torch.randn(x.shape, generator=g) * 60).clamp(-448, 448).to(E4M3) for x in (b.k_pages, b.v_pages))
    b.ks, b.vs = (torch.exp2(torch.randint(*scales, (b.n_pages, sh.n_kv_heads), generator=g).float()) for _ in range(2))
    if garbage:
        k, v = b.k8.view(torch.uint8), b.v8.view(torch.uint8)
        for p in b.free:
            k[p], v[p], b.ks[p], b.vs[p] = NAN_CODE, NAN_CODE, float("nan"), float("inf")
        for s, (_, n) in enumerate(b.seqs):
            if n % BS and 0 <= b.pages[s, n // BS] < b.n_pages:
                k[b.pages[s, n // BS], :, n % BS:] = NAN_CODE
                v[b.pages[s, n // BS], :, :, n % BS:] = NAN_CODE
    return b


def pools8(b):
    return [x.view(torch.uint8).to(DEV).view(E4M3) for x in (b.k8, b.v8)] + [b.ks.to(DEV), b.vs.to(DEV)]


def values64(b):
    """What the pools stand for, finite numbers where nobody may look."""
    return [np.nan_to_num(code_values(x) * f64(s)[..., None, None], nan=0, posinf=0, neginf=0) for x, s in ((b.k8, b.ks), (b.v8, b.vs))]


# ---------------------------------------------------------------- attention
def run_attention(b, kind="plain", seed=0, runner=None, **kw):
    f = form_of(b, kind, seed)
    r, t, q = runner or b.runner(), b.dev(), b.q.to(DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((b.n_rows, b.shape.n_q_heads), 7.0, device=DEV)
    r.attend_quantised(q, t["row_start"], t["n_ctx"], t["pages"], *pools8(b), out, lse, **on_device(f), **kw)
    torch.cuda.synchronize()
    k, v = values64(b)
    want = po.attention(f64(b.q), b.row_start, b.n_ctx, b.pages, k, v, b.shape.head_dim ** -0.5, **f)
    rows = np.arange(b.row_start[0], b.row_start[-1])
    check_out(b, want, out, lse, rows)
    nobody = np.setdiff1d(np.arange(b.n_rows), rows)
    assert (f64(out)[nobody] == 7.0).all() and (f64(lse)[nobody] == 7.0).all(), "rows of nobody were written"
    return out, lse, want


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("batch", list(BATCHES))
def test_attention(shape, batch):
    run_attention(quantise(Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 11, extra_rows=(2, 3)), 1))


@pytest.mark.parametrize("kind", [k for k in FORMS if k != "plain"])
@pytest.mark.parametrize("shape,batch", [("g7", "chunks"), ("g8_64", "chunks"), ("fp32_64", "chunks"), ("llama", "steps"),
                                         ("fp32_g3", "few"), ("mha64", "few"), ("llama", "long_tail"), ("fp32_g3", "long_tail"),
                                         ("fp32_64", "steps")])
def test_attention_forms(shape, batch, kind):
    run_attention(quantise(Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 13, extra_rows=(0, 1)), 2), kind, 3)


@pytest.mark.parametrize("case", range(len(CUTS)))
@pytest.mark.parametrize("kind", ["plain", "cap_slopes_end"])
def test_attention_in_every_cut(case, kind):
    hq, hkv, d, seqs, more = CUTS[case]
    run_attention(quantise(Batch(shape_of(hq, hkv, d, "bf16"), seqs, 79, extra_entries=more), 3), kind, 7)


@pytest.mark.parametrize("shape", ["llama", "g8_64", "fp32_64"])
@pytest.mark.parametrize("kind", ["plain", "all"])
def test_steps_and_chunks_of_a_wide_table(shape, kind):
    run_attention(quantise(Batch(shape_of(*SHAPES[shape]), [(1, 300), (60, 200), (2, 2), (0, 70), (1, 129), (16, 16), (1, 1), (2, 500)], 83,
                                 extra_rows=(1, 2), extra_entries=60 if shape == "llama" else 450), 4), kind, 9)


@pytest.mark.parametrize("shape,n", [("g7", 44), ("llama", 64), ("mha64", 200), ("fp32_64", 300), ("fp32_g3", 250)])
@pytest.mark.parametrize("kind", ["plain", "cap", "slopes", "all"])
def test_steps_of_many_short_sequences(shape, n, kind):
    """More (sequence, KV head) pairs than compute units, of few pages: smaller workgroups."""
    seqs = [(i % 7 != 3, 1 + 97 * i % 724) for i in range(n)]
    run_attention(quantise(Batch(shape_of(*SHAPES[shape]), [(int(m), c) for m, c in seqs], 127), 21), kind, 3)


@pytest.mark.parametrize("shape", ["g7", "fp32_64", "llama", "mha64"])
def test_pages_of_nobody_inside_a_sequence(shape):
    b = Batch(shape_of(*SHAPES[shape]), [(3, 700), (150, 700), (1, 300), (1, 260)], 23)
    quantise(b, 5)
    b.pages[0, 1], b.pages[1, 0], b.pages[1, 3], b.pages[2, 0] = -1, b.n_pages, 2 ** 31 - 1, -(2 ** 31)
    b.pages[3, :2] = b.pages[0, [0, 2]]           # (a page may serve two sequences)
    run_attention(b)
    b.pages[2, :] = -1
    _, _, want = run_attention(b)
    assert np.isneginf(want["lse"][b.row_start[2]]).all()


@pytest.mark.parametrize("shape", ["llama", "g8_64", "fp32_64", "fp32_g3"])
def test_clamped_lengths(shape):
    b = quantise(clamped_batch(shape), 6, garbage=False)
    run_attention(b)
    run_attention(b, "all")


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
@pytest.mark.parametrize("scales", [(-100, -99), (-60, -20), (20, 60)])
@pytest.mark.parametrize("batch", ["steps", "chunks"])
def test_small_and_large_scales(shape, scales, batch):
    """Values over the range of the scales; queries that make the scores ordinary."""
    b = quantise(Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 29), 7, scales=scales)
    b.q = (b.q.float() * 2.0 ** (-sum(scales) / 2 - 5)).to(b.q.dtype)
    if scales == (-100, -99):                     # (of one scale, values so small that bf16 and fp32 results are normal numbers)
        b.q = (b.q.float() * 0.5).to(b.q.dtype)
    run_attention(b)


@pytest.mark.parametrize("seqs", [[(70, 100)], [(128, 128)] * 3, [(128, 128)] * 64])       # (a page each: no cut, which goes by figures of its own)
@pytest.mark.parametrize("layer", [(32, 8, 128), (8, 2, 64), (28, 4, 128)])
@pytest.mark.parametrize("kind", ["plain", "cap", "all"])
def test_chunks_are_those_over_16_bits(seqs, layer, kind):
    """Codes are bf16 values: attention of chunks gives the bits that it gives over pages that hold those."""
    b = quantise(Batch(shape_of(*layer, "bf16"), seqs, 31, extra_entries=0), 8, garbage=False)
    b.k_pages, b.v_pages = (torch.tensor(x).to(torch.bfloat16) for x in values64(b))
    f = on_device(form_of(b, kind, 3))
    r, t, q = b.runner(), b.dev(), b.q.to(DEV)
    got = [[torch.zeros_like(q), torch.zeros(b.n_rows, layer[0], device=DEV)] for _ in range(2)]
    r.attend(q, t["row_start"], t["n_ctx"], t["pages"], t["k_pages"], t["v_pages"], *got[0], **f)
    r.attend_quantised(q, t["row_start"], t["n_ctx"], t["pages"], *pools8(b), *got[1], **f)
    torch.cuda.synchronize()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


# ---------------------------------------------------------------- append
def run_append(b, rotary=0, interleaved=False, far=False, with_q=True, runner=None, stream=None):
    t = b.dev()
    pools = pools8(b)
    k, kw = f64(b.k_new), {}
    if rotary:
        table = table_of(rotary, 700)
        places = np.random.default_rng(7).integers(-5, 720, b.n_rows) if far else b.positions()
        k, _ = po.rotate(k, f64(table), places, interleaved)
        k = k.astype(np.float32).astype(np.float64)
        kw = dict(rotation=table.to(DEV), interleaved=interleaved)
        if far:
            kw["row_pos"] = torch.tensor(places, dtype=torch.int32, device=DEV)
        if with_q:
            kw["q"] = b.q.to(DEV)
            kw["q_out"] = torch.full_like(kw["q"], 7.0)
    args = b.k_new.to(DEV), b.v_new.to(DEV)
    torch.cuda.synchronize()
    (runner or b.runner()).append_quantised(*args, t["row_start"], t["n_ctx"], t["pages"], *pools, stream=stream, **kw)
    torch.cuda.synchronize()
    want = po.quantised_append(k, f64(b.v_new), b.row_start, b.n_ctx, b.pages, code_values(b.k8), code_values(b.v8), f64(b.ks), f64(b.vs))
    for name, got, w in zip(("k_pages", "v_pages", "k_scales", "v_scales"), pools, want):
        got = code_values(got) if "pages" in name else f64(got)
        assert np.array_equal(got, w, equal_nan=True), f"{name}: {np.sum(~((got == w) | (np.isnan(got) & np.isnan(w))))} differ"
    if "q" in kw:
        want, size = po.rotate(f64(b.q), f64(table), places, interleaved)
        mine = (np.arange(b.n_rows) >= b.row_start[0]) & (np.arange(b.n_rows) < b.row_start[-1]) & (b.positions() >= 0)
        assert (np.abs(f64(kw["q_out"]) - want)[mine] <= bound_of(b.shape.dtype, want, size)[mine]).all()
        assert (f64(kw["q_out"])[~mine] == 7.0).all()
    return pools


def loud(b, seed):
    """New tokens of very different size: some pages' scales grow by much, others not at all."""
    g = torch.Generator().manual_seed(seed)
    by = torch.exp2(torch.randint(-12, 9, (b.n_rows, 1, 1), generator=g).float())
    b.k_new, b.v_new = (b.k_new.float() * by).to(b.k_new.dtype), (b.v_new.float() * by.flip(0)).to(b.v_new.dtype)
    return b


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("kind", ["quiet", "loud"])
def test_append(shape, batch, kind):
    b = quantise(Batch(shape_of(*SHAPES[shape]), BATCHES[batch], 31, extra_rows=(1, 2)), 9, scales=(-9, -3), garbage=kind == "loud")
    for s, (m, n) in enumerate(b.seqs):           # (a page that holds tokens has a scale)
        if m and (n - m) % BS:
            assert torch.isfinite(b.ks[b.pages[s, (n - m) // BS]]).all()
    run_append(loud(b, 3) if kind == "loud" else b)


@pytest.mark.parametrize("shape", ["llama", "mha64", "fp32_g3"])
@pytest.mark.parametrize("seqs", MIXED)
def test_append_of_steps_beside_chunks(shape, seqs):
    run_append(loud(quantise(Batch(shape_of(*SHAPES[shape]), seqs, 8, extra_rows=(1, 2), extra_entries=0), 9), 3), 64)


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("rotary,interleaved", [(64, False), (48, True), (16, False), (128, False), (128, True)])
def test_append_rotated(shape, rotary, interleaved):
    sh = shape_of(*SHAPES[shape])
    for i, batch in enumerate(("chunks", "steps", "few")):
        b = loud(quantise(Batch(sh, BATCHES[batch], 33 + i, extra_rows=(1, 0)), 10), i)
        run_append(b, min(rotary, sh.head_dim), interleaved, far=i != 1, with_q=i != 2)


def test_append_of_more_rows_than_a_launch_has_workgroups_for():
    """As many rows as a call may bring, of one sequence: the workgroups go round.  (Checked on the device, exactly.)"""
    sh = shape_of(1, 1, 64, "bf16")
    m = 2 ** 22
    n, max_pages = m + 77, m // BS + 1
    g = torch.Generator(device=DEV).manual_seed(3)
    k, v = (torch.randn(m, 1, 64, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    pools = [torch.zeros(s, dtype=torch.uint8, device=DEV).view(E4M3) for s in ((max_pages, 1, BS, 64), (max_pages, 1, 64, BS))]
    pools += [torch.full((max_pages, 1), 2.0 ** -9, device=DEV) for _ in range(2)]
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    pages = torch.randperm(max_pages, device=DEV).int()[None].contiguous()
    H.PagedRunner(sh, 1, m, m, max_pages).append_quantised(k, v, i32([0, m]), i32([n]), pages, *pools)
    torch.cuda.synchronize()
    order = pages[0].long()
    for x, codes, scales in ((k, pools[0], pools[2]), (v, pools[1].transpose(2, 3), pools[3])):
        full = torch.cat([torch.zeros(77, 64, device=DEV), x[:, 0].float(), torch.zeros(max_pages * BS - n, 64, device=DEV)]).reshape(max_pages, BS, 64)
        e = torch.ceil(torch.log2(full.abs().amax((1, 2)).double() / 448))
        e[0] = max(e[0], torch.tensor(-9.0, device=DEV, dtype=torch.float64))
        assert torch.equal(scales[order, 0], torch.exp2(e).float())
        want = (full * torch.exp2(-e).float()[:, None, None]).to(E4M3)
        assert torch.equal(codes[:, 0].float()[order], want.float())


@pytest.mark.parametrize("layer", [(8, 1, 128, "bf16"), (7, 1, 64, "fp32"), (48, 6, 64, "bf16"), (5, 1, 128, "fp32")])
def test_other_groups(layer):
    for batch in ("steps", "chunks"):
        b = quantise(Batch(shape_of(*layer), BATCHES[batch], 32, extra_rows=(1, 1)), 9)
        run_append(loud(b, 4), 48, True)
        run_attention(b)


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_append_of_the_scales_edges(shape):
    """Largest values at and next to 448 times a power of two, zeros, subnormals, infinities and NaN, scales that hold anything."""
    sh = shape_of(*SHAPES[shape])
    b = quantise(Batch(sh, [(1, 1), (1, 130), (2, 200), (5, 133), (3, 3), (140, 300), (1, 250), (1, 140)], 35, garbage=None), 11, garbage=False)
    k = torch.zeros_like(b.k_new)
    at = b.row_start
    k[at[0], :, 3] = 448.0
    k[at[1], :, 3], k[at[1], :, 4] = 450.0, -1.75
    k[at[2], :, 5], k[at[2] + 1, :, 6] = 1e-30, -3e-38
    k[at[3]: at[4]] = 0
    k[at[4], :, 1], k[at[4] + 1, :, 2], k[at[4] + 2, :, 3] = float("inf"), float("nan"), 2.0 ** 100
    k[at[5]: at[6]] = (torch.randn(140, sh.n_kv_heads, sh.head_dim) * 1e-35).to(k.dtype)
    k[at[6], :, 0] = 2.0 ** 126
    b.k_new, b.v_new = k, k.flip(2).contiguous()
    run_append(b)


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_append_without_pages_and_at_clamped_lengths(shape):
    b = quantise(Batch(shape_of(*SHAPES[shape]), BATCHES["chunks"], 37), 12, garbage=False)
    b.pages[0, 1], b.pages[4, 2] = b.n_pages, -1
    run_append(b, 64)
    run_append(quantise(clamped_batch(shape), 13, garbage=False), 64)


@pytest.mark.parametrize("shape", ["g7", "fp32_64"])
def test_append_token_by_token_is_within_two_roundings_of_the_token(shape):
    """A page filled by steps whose tokens grow: a value was rounded to the scale of its time and again to the last one."""
    sh = shape_of(*SHAPES[shape])
    g = torch.Generator().manual_seed(17)
    b = Batch(sh, [(1, 1)], 39, garbage=None)
    quantise(b, 14, garbage=False)
    r, pools = H.PagedRunner(sh, 1, 1, 1, b.max_pages), pools8(b)
    pages, start = b.dev()["pages"], torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    held = []
    for n in range(1, BS + 1):
        x = [(torch.randn(1, sh.n_kv_heads, sh.head_dim, generator=g) * 1.07 ** n).to(sh.torch_dtype) for _ in range(2)]
        held.append(x)
        r.append_quantised(x[0].to(DEV), x[1].to(DEV), start, torch.tensor([n], dtype=torch.int32, device=DEV), pages, *pools)
    torch.cuda.synchronize()
    p = b.pages[0, 0]
    k, v = (code_values(x)[p] * f64(s)[p][:, None, None] for x, s in zip(pools[:2], pools[2:]))
    for i, (got, scale) in enumerate(((k, f64(pools[2])[p]), (v.swapaxes(1, 2), f64(pools[3])[p]))):
        want = np.stack([f64(x[i])[0] for x in held], 1)
        # half a step each time: 2^-4 of the value, or half of the least code's step times the scale
        bound = 2 * np.maximum(2.0 ** -4 * np.abs(want) * 1.07, 2.0 ** -10 * scale[:, None, None])
        assert (np.abs(got - want) <= bound).all()
        assert (np.abs(want).max((1, 2)) <= 448 * scale).all() and (np.abs(want).max((1, 2)) > 224 * scale * (1 - 2.0 ** -9)).all()


# ---------------------------------------------------------------- both, as they are used
@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_a_cache_in_use(shape):
    """Prompts in chunks and steps, rotated on the way: every call's attention over what the pools hold by their own definition."""
    sh = shape_of(*SHAPES[shape])
    g = torch.Generator().manual_seed(41)
    batch, max_pages, n_pages = 3, 6, 20
    pages = np.random.default_rng(3).permutation(n_pages)[: batch * max_pages].reshape(batch, max_pages)
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)
    r = H.PagedRunner(sh, batch, 700, 300, max_pages)
    pools = [torch.full(s, NAN_CODE, dtype=torch.uint8, device=DEV).view(E4M3) for s in
             ((n_pages, sh.n_kv_heads, BS, sh.head_dim), (n_pages, sh.n_kv_heads, sh.head_dim, BS))]
    pools += [torch.full((n_pages, sh.n_kv_heads), float("nan"), device=DEV) for _ in range(2)]
    mirror = [code_values(pools[0]), code_values(pools[1]), f64(pools[2]), f64(pools[3])]
    table = table_of(64, 1024)
    n_ctx = np.zeros(batch, int)
    for news in [(150, 1, 0), (300, 200, 129), (1, 1, 1), (7, 1, 90), (1, 1, 1)]:
        n_rows, start = sum(news), np.cumsum([0, *news])
        n_ctx = n_ctx + np.array(news)
        k_new, v_new = (torch.randn(n_rows, sh.n_kv_heads, sh.head_dim, generator=g).to(sh.torch_dtype) for _ in range(2))
        q = torch.randn(n_rows, sh.n_q_heads, sh.head_dim, generator=g).to(sh.torch_dtype)
        qd, out, lse = q.to(DEV), torch.zeros_like(q, device=DEV), torch.zeros(n_rows, sh.n_q_heads, device=DEV)
        call = (i32(start), i32(n_ctx), i32(pages))
        r.append_quantised(k_new.to(DEV), v_new.to(DEV), *call, *pools, rotation=table.to(DEV), q=qd, q_out=qd)
        r.attend_quantised(qd, *call, *pools, out, lse, softcap=25.0)
        torch.cuda.synchronize()
        places = np.concatenate([np.arange(n - m, n) for n, m in zip(n_ctx, news)])
        k = po.rotate(f64(k_new), f64(table), places, False)[0].astype(np.float32).astype(np.float64)
        mirror = po.quantised_append(k, f64(v_new), start, n_ctx, pages, *mirror)
        for got, w in zip(pools, mirror):
            got = code_values(got) if got.dtype == E4M3 else f64(got)
            assert np.array_equal(got, w, equal_nan=True)
        k64, v64 = (np.nan_to_num(x * s[..., None, None]) for x, s in zip(mirror[:2], mirror[2:]))
        want = po.attention(f64(qd), start, n_ctx, pages, k64, v64, sh.head_dim ** -0.5, softcap=25.0)
        check_out(type("B", (), dict(shape=sh, n_ctx=n_ctx)), want, out, lse, np.arange(n_rows))


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_replayed_graph(shape):
    sh = shape_of(*SHAPES[shape])
    b = quantise(Batch(sh, [(1, 600), (4, 300), (90, 90), (2, 131)], 43), 15, garbage=False)
    r, t = b.runner(), b.dev()
    given = pools8(b)
    pools = [x.clone() for x in given]
    table = table_of(64, 800).to(DEV)
    q, kn, vn = b.q.to(DEV), b.k_new.to(DEV), b.v_new.to(DEV)
    q_out, out, lse = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(b.n_rows, sh.n_q_heads, device=DEV)

    def step():
        r.append_quantised(kn, vn, t["row_start"], t["n_ctx"], t["pages"], *pools, rotation=table, q=q, q_out=q_out)
        r.attend_quantised(q_out, t["row_start"], t["n_ctx"], t["pages"], *pools, out, lse)

    def start():
        for x, x0 in zip(pools, given):
            x.view(torch.uint8).copy_(x0.view(torch.uint8))
        for x in (q_out, out, lse):
            x.zero_()

    def state():
        torch.cuda.synchronize()
        return [x.view(torch.uint8).clone() for x in (*pools, q_out, out, lse)]

    start(), step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    last = None
    for n_ctx in ([600, 300, 90, 131], [130, 299, 90, 140], [5, 141, 90, 142], [600, 17, 95, 256]):
        t["n_ctx"].copy_(torch.tensor(n_ctx, dtype=torch.int32))
        for i, x in enumerate((q, kn, vn)):
            x.copy_((torch.randn(x.shape) * (1, 8, 3)[i]).to(x.dtype))
        start(), step()
        want = state()
        assert last is None or not any(torch.equal(x, y) for x, y in zip(last, want))
        last = want
        for _ in range(2):
            start()
            graph.replay()
            assert all(torch.equal(x, y) for x, y in zip(state(), want))


@pytest.mark.parametrize("shape", ["llama", "fp32_g3"])
@pytest.mark.parametrize("seqs", [[(1, 300), (2, 140)], [(150, 300), (3, 140)]])
def test_pages_past_32_bits(shape, seqs):
    """A pool of more than 2^32 bytes: the same bits as from a small one."""
    sh = shape_of(*SHAPES[shape])
    b = quantise(Batch(sh, seqs, 97), 16, garbage=False)
    r, t, small = b.runner(), b.dev(), pools8(b)
    page = sh.n_kv_heads * BS * sh.head_dim
    n_far = 2 ** 32 // page + 40
    move = torch.tensor([n_far - 1 - 7 * i for i in range(b.n_pages)], device=DEV)
    far = []
    for x in small:
        pool = torch.empty(n_far, *x.shape[1:], dtype=x.dtype, device=DEV)
        (pool.view(torch.uint8) if x.dtype == E4M3 else pool)[move] = x.view(torch.uint8) if x.dtype == E4M3 else x
        far.append(pool)
    far_pages = torch.where(t["pages"] >= 0, move[t["pages"].clamp(min=0).long()].int(), -1).contiguous()
    got = []
    for pools, pages in ((small, t["pages"]), (far, far_pages)):
        q = b.q.to(DEV)
        out, lse = torch.zeros_like(q), torch.zeros(b.n_rows, sh.n_q_heads, device=DEV)
        r.append_quantised(b.k_new.to(DEV) * 3, b.v_new.to(DEV) * 3, t["row_start"], t["n_ctx"], pages, *pools)
        r.attend_quantised(q, t["row_start"], t["n_ctx"], pages, *pools, out, lse)
        torch.cuda.synchronize()
        got.append([out, lse] + [(x.view(torch.uint8) if x.dtype == E4M3 else x)[move if pools is far else slice(None)] for x in pools])
    assert all(torch.equal(x, y) for x, y in zip(*got))


@pytest.mark.parametrize("shape", ["llama", "fp32_64"])
def test_two_calls_at_once(shape):
    sh = shape_of(*SHAPES[shape])
    prepared, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for i, seqs in enumerate(([(1, 900), (1, 40)], [(120, 900), (1, 40)])):
        b = quantise(Batch(sh, seqs, 101 + i), 17)
        t, q = b.dev(), b.q.to(DEV)
        args = (q, t["row_start"], t["n_ctx"], t["pages"], *pools8(b))
        outs = [torch.zeros_like(q) for _ in range(9)]
        r = b.runner()
        r.attend_quantised(*args, outs[0])
        prepared.append((r, args, outs))
    torch.cuda.synchronize()
    for i in range(1, 9):
        for (r, args, outs), stream in zip(prepared, streams):
            r.attend_quantised(*args, outs[i], stream=stream)
    torch.cuda.synchronize()
    for _, _, outs in prepared:
        assert all(torch.equal(o, outs[0]) for o in outs[1:])


def test_a_runner_made_for_more():
    sh = shape_of(*SHAPES["llama"])
    b = quantise(Batch(sh, [(1, 300), (1, 129), (1, 1)], 107), 18)
    made_for = H.PagedRunner(sh, 5, 500, 400, b.max_pages + 3)
    run_attention(b, runner=made_for, max_new=1)
    run_attention(b, runner=made_for)
    run_append(b, 64, runner=made_for, stream=torch.cuda.Stream())
