"""The paged key-value cache on the GPU (fusion_cache_append, fusion_cache_attention, fusion_cache_evict) against the
definitions in 64 bits (cache_reference.py, where the tolerances are derived).  Copies are compared bit by bit, and
whatever no call may touch holds NaN, so that a read of it shows in a result and a write in the comparison."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import cache_reference as ref  # noqa: E402
import paper_2607_02612_gb300 as fz  # noqa: E402
from paper_2607_02612_gb300 import runner  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda"


def on_device(dtype, c, heads):
    d = {k: None if t is None else t.to(DEV) for k, t in c.items()}
    return runner.cache_of(dtype, d["k"], d["v"], d["table"], d["lengths"], heads=heads, sizes=d["sizes"], weights=d["weights"])


def same(dc, c, lengths=None):
    """The device's cache equals the host's, bit by bit."""
    for name in ("k", "v", "sizes", "weights"):
        got, want = getattr(dc, name), c[name]
        if want is not None:
            assert torch.equal(ref.bits(got.cpu()), ref.bits(want)), name
    assert torch.equal(dc.lengths.cpu(), c["lengths"] if lengths is None else lengths)


def status(f):
    torch.cuda.synchronize()
    return int(f.status.item())


# ---- append ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_heads,dim,page", [(1, 8, 1), (3, 64, 16), (2, 80, 8), (8, 128, 64), (5, 256, 4)])
@pytest.mark.parametrize("in_place", [True, False])
def test_append(dtype, kv_heads, dim, page, in_place):
    """Ragged samples (one without rows, one that fills its pages) to sequences in another order, from slices of packed
    projections; the other sequences keep their tokens."""
    lengths, counts, ids = [5, 0, 17, 3, 40], [33, 0, 1, 24], [3, 0, 1, 4]
    c = ref.make(dtype, lengths, kv_heads, dim, page, room=24, sizes="whole", weights=True, seed=1)
    rows, width = sum(counts) + 2, kv_heads * dim
    g = torch.Generator().manual_seed(2)
    packed = torch.randn((rows, 3 * width), generator=g).to(ref.TYPES[dtype])
    sizes, scores = torch.rand(rows, generator=g), torch.rand(rows, generator=g)
    offsets = torch.tensor([1, *(1 + torch.tensor(counts).cumsum(0)).tolist()], dtype=torch.int32)
    dc, f = on_device(dtype, c, kv_heads), runner.Fusion(5)
    p = packed.to(DEV)
    rr = runner.RaggedRows(4, max(counts), rows, offsets.to(DEV), ids=torch.tensor(ids, dtype=torch.int32, device=DEV))
    out = None if in_place else torch.full((5,), -7, dtype=torch.int32, device=DEV)
    f.cache_append(dc, p[:, width:2 * width], p[:, 2 * width:], rr, sizes=sizes.to(DEV), scores=scores.to(DEV), lengths_out=out)
    assert status(f) == 0
    new = ref.append(c, packed[:, width:2 * width], packed[:, 2 * width:], offsets, ids, sizes, scores)
    same(dc, c, new if in_place else None)
    if not in_place:
        assert torch.equal(out.cpu(), new)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_one_row_each_and_defaults(dtype):
    """A token per sequence (no offsets given), sizes 1 and scores 0 by default, twice; and long samples of many CTAs."""
    c = ref.make(dtype, [0, 1, 15, 16, 17, 31], 2, 64, 16, room=700, sizes="whole", weights=True, seed=3)
    dc, f = on_device(dtype, c, 2), runner.Fusion(6)
    g = torch.Generator().manual_seed(4)
    for _ in range(2):
        k, v = (torch.randn((6, 2, 64), generator=g).to(ref.TYPES[dtype]) for _ in range(2))
        f.cache_append(dc, k.to(DEV), v.to(DEV))
        c["lengths"] = ref.append(c, k, v, range(7))
    offsets = [0, 650, 651, 1300, 1300, 1901, 2000]
    k, v = (torch.randn((2000, 128), generator=g).to(ref.TYPES[dtype]) for _ in range(2))
    for _ in range(2):   # the second time there is no room for three of them
        f.cache_append(dc, k.to(DEV), v.to(DEV), runner.RaggedRows(6, 650, 2000, torch.tensor(offsets, dtype=torch.int32, device=DEV)))
        if status(f) == 0:
            c["lengths"] = ref.append(c, k, v, offsets)
    assert status(f) == fz.FUSION_DEV_BAD_CACHE
    fits = [b for b in range(6) if int(c["lengths"][b]) + offsets[b + 1] - offsets[b] <= dc.max_pages * dc.page_tokens]
    assert 0 < len(fits) < 6
    for b in fits:
        new = ref.append(c, k, v, [offsets[b], offsets[b + 1]], [b])
        c["lengths"][b] = new[b]
    same(dc, c)


@pytest.mark.parametrize("dtype,kv_heads,dim", [("bf16", 1, 8), ("f32", 1, 8), ("f32", 9, 256)])
def test_append_narrow_and_wide_rows(dtype, kv_heads, dim):
    """Rows of 16 bytes, of which a CTA takes many more than it has threads, and of more chunks than it has threads."""
    c = ref.make(dtype, [3, 0], kv_heads, dim, 32, room=3000, sizes="whole", weights=True, seed=33)
    dc, f = on_device(dtype, c, kv_heads), runner.Fusion(2)
    g = torch.Generator().manual_seed(34)
    k, v = (torch.randn((4001, kv_heads * dim), generator=g).to(ref.TYPES[dtype]) for _ in range(2))
    sizes, scores = torch.rand(4001, generator=g), torch.rand(4001, generator=g)
    offsets = [0, 2500, 4001]
    f.cache_append(dc, k.to(DEV), v.to(DEV), runner.RaggedRows(2, 2500, 4001, torch.tensor(offsets, dtype=torch.int32, device=DEV)),
                   sizes=sizes.to(DEV), scores=scores.to(DEV))
    assert status(f) == 0
    same(dc, c, ref.append(c, k, v, offsets, sizes=sizes, scores=scores))


@pytest.mark.parametrize("in_place", [True, False])
def test_append_leaves_bad_samples_out(in_place):
    """A sample that is out of range in some way is left out, and the others are appended."""
    bits = fz.FUSION_DEV_BAD_OFFSETS, fz.FUSION_DEV_BAD_IDS, fz.FUSION_DEV_BAD_CACHE, fz.FUSION_DEV_BAD_BATCH
    offs, ids_bit, cache_bit, batch_bit = bits
    for what, bit in (("decreasing", offs), ("long", offs), ("id", ids_bit), ("twice", ids_bit), ("room", cache_bit),
                      ("page", cache_bit), ("length", cache_bit), ("batch", batch_bit), ("count", 0)):
        c = ref.make("bf16", [4, 9, 2, 30], 2, 16, 8, room=20, sizes="whole", weights=True, seed=5)
        offsets, ids, count, good = [0, 10, 12, 20, 25], [2, 1, 0, 3], None, [0, 1, 2, 3]
        longest = 10
        if what == "decreasing":
            offsets, good = [0, 10, 8, 16, 21], [0, 2, 3]
        elif what == "long":
            longest, good = 9, [1, 2, 3]
        elif what == "id":
            ids, good = [2, 1, 4, -1], [0, 1]
        elif what == "twice":
            ids, good = [2, 1, 2, 3], [1, 3]
        elif what == "room":
            c["lengths"][1], good = 7 * 8 - 1, [0, 2, 3]
        elif what == "page":
            c["table"][2, 1], good = c["k"].shape[0], [1, 2, 3]
        elif what == "length":
            c["lengths"][3], good = -2, [0, 1, 2]
        elif what == "batch":
            count, good = 5, []
        elif what == "count":
            count, good = 2, [0, 1]
        k, v = (torch.randn((25, 32)).to(torch.bfloat16) for _ in range(2))
        dc, f = on_device("bf16", c, 2), runner.Fusion(4)
        rr = runner.RaggedRows(4, longest, 25, torch.tensor(offsets, dtype=torch.int32, device=DEV),
                               None if count is None else torch.tensor([count], dtype=torch.int32, device=DEV),
                               torch.tensor(ids, dtype=torch.int32, device=DEV))
        out = None if in_place else torch.full((4,), -7, dtype=torch.int32, device=DEV)
        f.cache_append(dc, k.to(DEV), v.to(DEV), rr, lengths_out=out)
        assert status(f) == bit, what
        new = c["lengths"].clone()
        for i in good:
            new[ids[i]] = ref.append(c, k, v, offsets[i:i + 2], ids[i:i + 1])[ids[i]]
        same(dc, c, new if in_place else None)
        if not in_place:
            assert torch.equal(out.cpu(), new), what


# ---- attention -----------------------------------------------------------------------------------------------------
def attend(dtype, c, heads, *, window=0, sinks=0, scale=None, seed=9, spread=1.0, q=None, expect=0):
    """One call checked against the definition; returns the outputs."""
    batch, dim = len(c["lengths"]), c["k"].shape[3]
    if q is None:
        q = (torch.randn((batch, heads, dim), generator=torch.Generator().manual_seed(seed)) * spread).to(ref.TYPES[dtype])
    dc, f = on_device(dtype, c, heads), runner.Fusion(max(batch, 1))
    out = torch.full((batch, heads, dim), 7.0, dtype=ref.TYPES[dtype], device=DEV)
    f.cache_attention(dc, q.to(DEV), window=window, sinks=sinks, scale=scale, out=out)
    assert status(f) == expect
    want, tol, w, wtol = ref.attention(c, q, dtype, scale=scale, window=window, sinks=sinks)
    got = out.cpu().double()
    err = (got - want).abs()
    assert torch.isfinite(got).all() and (err <= tol).all(), float((err / tol).max())
    if w is not None:
        gw = dc.weights.cpu().double()
        held = torch.isfinite(w)
        assert torch.equal(torch.isfinite(gw), held)
        assert ((gw - w).abs()[held] <= wtol[held]).all(), float(((gw - w).abs() - wtol)[held].max())
    keep = ref.copy(c)
    keep["weights"] = None
    same(dc, keep)
    assert int(dc.workspace[:1 << 18].max()) == 0   # the counters are zero again
    return out, dc


LENGTHS = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 513]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [
    (1, 1, 64, 16), (6, 6, 64, 16), (8, 2, 128, 16), (8, 1, 128, 32), (7, 1, 64, 8), (12, 4, 80, 4), (4, 4, 8, 1), (16, 2, 256, 16),
    (9, 1, 128, 128), (40, 2, 64, 64), (33, 1, 128, 16), (70, 1, 96, 16), (18, 1, 256, 16), (2, 2, 200, 256)])
def test_attention_shapes(dtype, heads, kv_heads, dim, page):
    """Groups of 1 to 70 query heads, widths on and off the kernel's 64 / 128 / 256, lengths around its tiles, with sizes
    (some tokens masked, holding NaN and infinity) and weights."""
    attend(dtype, ref.make(dtype, LENGTHS, kv_heads, dim, page, sizes="masked", weights=True, seed=6), heads)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sizes,weights", [(None, False), (None, True), ("whole", False)])
def test_attention_optional_inputs(dtype, sizes, weights):
    attend(dtype, ref.make(dtype, LENGTHS, 2, 64, 16, sizes=sizes, weights=weights, seed=7), 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (64, 4), (100, 0), (200, 13), (0, 5), (2 ** 31 - 1, 2 ** 31 - 1), (3, 500)])
def test_attention_window_and_sinks(dtype, window, sinks):
    attend(dtype, ref.make(dtype, LENGTHS, 2, 128, 16, sizes="masked", weights=True, seed=8), 8, window=window,
           sinks=sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim,n", [(32, 8, 128, [3000]), (8, 1, 64, [5001, 3]), (64, 1, 128, [9000]), (4, 4, 256, [1, 2500])])
def test_attention_split_over_many_ctas(dtype, heads, kv_heads, dim, n):
    """Few long sequences: every (sequence, key head) is shared by many CTAs and joined; three calls give the same bits."""
    c = ref.make(dtype, n, kv_heads, dim, 32, sizes="whole", weights=True, seed=10)
    outs = [attend(dtype, c, heads) for _ in range(3)]
    for o, dc in outs[1:]:
        assert torch.equal(ref.bits(o), ref.bits(outs[0][0])) and torch.equal(ref.bits(dc.weights), ref.bits(outs[0][1].weights))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_many_short_sequences(dtype):
    attend(dtype, ref.make(dtype, [(37 * i) % 90 for i in range(700)], 3, 64, 16, weights=True, seed=11), 6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(1, 1, 64, 16), (8, 2, 128, 16), (16, 1, 64, 8), (21, 1, 128, 4), (4, 4, 80, 32), (3, 1, 8, 128)])
def test_attention_short_sequences_a_warp_each(dtype, heads, kv_heads, dim, page):
    """Sequences of at most 128 tokens, enough of them that every warp works alone: masked tokens, weights, a window; and one
    sequence with a bad page among them."""
    n = [(29 * i) % 128 for i in range(260)]
    c = ref.make(dtype, n, kv_heads, dim, page, sizes="masked", weights=True, seed=41)
    attend(dtype, c, heads)
    attend(dtype, c, heads, window=40, sinks=3)
    q = torch.randn((260, heads, dim), generator=torch.Generator().manual_seed(42)).to(ref.TYPES[dtype])
    want, tol, w, wtol = ref.attention(c, q, dtype)
    bad = 123
    assert n[bad] > 0
    table = c["table"].clone()
    table[bad, 0] = -1
    dc, f = on_device(dtype, dict(c, table=table), heads), runner.Fusion(260)
    out = torch.full((260, heads, dim), 7.0, dtype=ref.TYPES[dtype], device=DEV)
    f.cache_attention(dc, q.to(DEV), out=out)
    assert status(f) == fz.FUSION_DEV_BAD_CACHE
    got, gw, good = out.cpu().double(), dc.weights.cpu().double(), [b for b in range(260) if b != bad]
    assert ((got[good] - want[good]).abs() <= tol[good]).all() and (got[bad] == 7.0).all()
    for b in good:
        at = ref.places(c, b, torch.arange(n[b]))
        assert ((gw[at] - w[at]).abs() <= wtol[at]).all()
    at = ref.places(c, bad, torch.arange(n[bad]))
    assert torch.equal(gw[at], c["weights"][at].double())
    assert int(dc.workspace[:1 << 18].max()) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_thousands_of_sequences(dtype):
    """More sequences than threads: most of them empty, a few with tokens; and the same batch appended to in one call."""
    n = [(i % 11) * (i % 3 == 0) for i in range(9000)]
    c = ref.make(dtype, n, 1, 8, 16, room=1, weights=True, seed=38)
    _, dc = attend(dtype, c, 2)
    k, v = (torch.randn((9000, 8), generator=torch.Generator().manual_seed(39)).to(ref.TYPES[dtype]) for _ in range(2))
    f = runner.Fusion(1)
    f.cache_append(dc, k.to(DEV), v.to(DEV))
    c["weights"] = dc.weights.cpu()
    new = ref.append(c, k, v, range(9001))
    want = ref.copy(c)
    for b in range(9000):
        pg, off = ref.places(want, b, torch.tensor([n[b]]))
        want["weights"][pg, off] = 0.0
    assert status(f) == 0
    same(dc, want, new)
    want["lengths"] = new
    budget = [i % 7 for i in range(9000)]
    f.cache_evict(dc, torch.tensor(budget, dtype=torch.int32, device=DEV), recent=1)
    want["lengths"], _ = ref.evict(want, budget, recent=1)
    assert status(f) == 0
    same(dc, want)


def test_a_cache_of_no_sequences():
    dc, f = runner.device_cache("f32", 0, 64, 4, 2, 16, sizes=True, weights=True), runner.Fusion(1)
    f.cache_append(dc, torch.zeros((0, 32), device=DEV), torch.zeros((0, 32), device=DEV))
    assert f.cache_attention(dc, torch.zeros((0, 4, 16), device=DEV)).shape == (0, 4, 16)
    f.cache_evict(dc, torch.zeros(0, dtype=torch.int32, device=DEV))
    assert status(f) == 0


@pytest.mark.parametrize("heads,dim", [(1024, 8), (640, 64)])
def test_attention_many_query_heads(heads, dim):
    attend("bf16", ref.make("bf16", [130, 17], 1, dim, 16, weights=True, seed=40), heads)
    attend("f32", ref.make("f32", [130, 17], 1, dim, 16, weights=True, seed=40), heads)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_peaked_and_rising_logits(dtype):
    """Logits of hundreds, rising along the sequence (every tile rescales) or falling; a negative and a zero scale."""
    for sign in (1.0, -1.0):
        c = ref.make(dtype, [700, 65], 2, 64, 16, weights=True, seed=12)
        for b, n in enumerate([700, 65]):
            pg, off = ref.places(c, b, torch.arange(n))
            c["k"][pg, :, off, 0] = (sign * torch.arange(n) / 4)[:, None].to(ref.TYPES[dtype])
        q = torch.zeros((2, 4, 64))
        q[..., 0] = 4.0
        q[..., 1:] = torch.randn((2, 4, 63), generator=torch.Generator().manual_seed(13)) / 4
        attend(dtype, c, 4, q=q.to(ref.TYPES[dtype]), scale=1.0)
        attend(dtype, c, 4, q=q.to(ref.TYPES[dtype]), scale=-0.25)
        attend(dtype, c, 4, q=q.to(ref.TYPES[dtype]), scale=0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_all_masked(dtype):
    """Every token of size 0 (with NaN keys and infinite values): a zero row, untouched weights; the same for a window that
    sees only masked tokens."""
    c = ref.make(dtype, [40, 200, 5], 2, 64, 16, sizes="whole", weights=True, seed=14)
    for b, pos in ((0, torch.arange(40)), (1, torch.arange(150, 200))):
        pg, off = ref.places(c, b, pos)
        c["sizes"][pg, off] = 0.0
        c["k"][pg, :, off], c["v"][pg, :, off] = math.nan, math.inf
    out, _ = attend(dtype, c, 4)
    assert (out[0] == 0).all()
    out, _ = attend(dtype, c, 4, window=50)
    assert (out[:2] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_minus_infinity_and_nan(dtype):
    """Logits that overflow to -inf weigh nothing, wherever their tile lies; a row of nothing else is zero; a NaN in a
    visible token reaches its sequence's heads and no other."""
    c = ref.make(dtype, [300, 64, 100], 1, 64, 16, seed=15)
    q = torch.randn((3, 2, 64), generator=torch.Generator().manual_seed(16))
    q[..., 0] = -4.0
    for b, pos in ((0, torch.arange(0, 128)), (1, torch.arange(64))):
        pg, off = ref.places(c, b, pos)
        c["k"][pg, :, off, 0] = 3e38
    dc, f = on_device(dtype, c, 2), runner.Fusion(3)
    out = f.cache_attention(dc, q.to(ref.TYPES[dtype]).to(DEV), scale=1.0).cpu()
    assert status(f) == 0 and (out[1] == 0).all()
    for b, pos in ((0, torch.arange(128)),):
        pg, off = ref.places(c, b, pos)
        c["sizes"] = torch.ones(c["k"].shape[0], 16)
        c["sizes"][pg, off] = 0.0
    want, tol, _, _ = ref.attention(c, q.to(ref.TYPES[dtype]), dtype, scale=1.0)
    assert ((out[0].double() - want[0]).abs() <= tol[0]).all()
    pg, off = ref.places(c, 0, torch.tensor([200]))
    dc.v[int(pg), :, int(off), 5] = math.nan
    out = f.cache_attention(dc, q.to(ref.TYPES[dtype]).to(DEV), scale=1.0).cpu()
    assert torch.isnan(out[0, :, 5]).all() and torch.isfinite(out[1:]).all()
    dc.k[int(pg), :, int(off), 5] = math.nan
    out = f.cache_attention(dc, q.to(ref.TYPES[dtype]).to(DEV), scale=1.0).cpu()
    assert torch.isnan(out[0]).all() and torch.isfinite(out[1:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_bad_pages_and_lengths(dtype):
    """A visible token whose page id is out of range, and a length out of range: that sequence's row and weights stay as
    they are, the others are right; a bad id that no visible token needs is not read."""
    lengths = [600, 70, 300, 5, 64]
    c = ref.make(dtype, lengths, 2, 64, 16, room=16, weights=True, seed=17)
    good = ref.copy(c)
    c["table"][0, 20], c["table"][2, 0], c["table"][3, 1] = c["k"].shape[0], -1, -5
    c["lengths"][4] = c["table"].shape[1] * 16 + 1
    q = torch.randn((5, 4, 64), generator=torch.Generator().manual_seed(18)).to(ref.TYPES[dtype])
    dc, f = on_device(dtype, c, 4), runner.Fusion(5)
    out = torch.full((5, 4, 64), 7.0, dtype=ref.TYPES[dtype], device=DEV)
    f.cache_attention(dc, q.to(DEV), out=out)
    assert status(f) == fz.FUSION_DEV_BAD_CACHE
    want, tol, w, wtol = ref.attention(good, q, dtype)
    got, gw = out.cpu().double(), dc.weights.cpu().double()
    for b in range(5):
        at = ref.places(good, b, torch.arange(lengths[b]))
        if b in (1, 3):
            assert ((got[b] - want[b]).abs() <= tol[b]).all() and ((gw[at] - w[at]).abs() <= wtol[at]).all()
        else:
            assert (got[b] == 7.0).all()
            assert torch.equal(gw[at], good["weights"][at].double())
    assert int(dc.workspace[:1 << 18].max()) == 0
    c["lengths"][4] = -1
    c["lengths"][0], c["lengths"][2] = 320, 0     # the bad entries are out of sight now
    dc = on_device(dtype, c, 4)
    f.status.zero_()
    out = f.cache_attention(dc, q.to(DEV)).cpu()
    assert status(f) == fz.FUSION_DEV_BAD_CACHE and (out[2] == 0).all()


def test_attention_strided_queries_other_stream_and_graph():
    """Queries as a slice of a packed projection, a call on another stream, and a captured call replayed on other lengths,
    pages and queries."""
    c = ref.make("bf16", [100, 37, 64], 2, 64, 16, room=300, sizes="whole", weights=False, seed=19)
    dc, f = on_device("bf16", c, 4), runner.Fusion(3)
    packed = torch.randn((3, 8 * 64), generator=torch.Generator().manual_seed(20)).to(torch.bfloat16)
    p = packed.to(DEV)
    q = packed[:, :256].reshape(3, 4, 64)
    want, tol, _, _ = ref.attention(c, q, "bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = f.cache_attention(dc, p[:, :256])
    side.synchronize()
    assert ((out.cpu().double() - want).abs() <= tol).all()
    graph, staged, result = torch.cuda.CUDAGraph(), torch.zeros_like(p), torch.zeros_like(out)
    with torch.cuda.graph(graph):   # (between kernels of torch's)
        p.copy_(staged)
        p.mul_(2.0)
        f.cache_attention(dc, p[:, :256], window=90, sinks=2, out=out)
        result.copy_(out)
        p.zero_()
    for seed in (21, 22):
        n = [399 - seed, seed, 0]
        c2 = ref.make("bf16", n, 2, 64, 16, room=400 - max(n), sizes="whole", seed=seed)
        assert c2["table"].shape == c["table"].shape and c2["k"].shape == c["k"].shape
        dc.k.copy_(c2["k"]), dc.v.copy_(c2["v"]), dc.sizes.copy_(c2["sizes"])
        dc.page_table.copy_(c2["table"]), dc.lengths.copy_(c2["lengths"])
        staged.copy_(torch.randn((3, 512), generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        q = (staged * 2.0).cpu()[:, :256].reshape(3, 4, 64)
        want, tol, _, _ = ref.attention(c2, q, "bf16", window=90, sinks=2)
        assert ((result.cpu().double() - want).abs() <= tol).all()
    assert status(f) == 0


def test_attention_rows_past_two_to_the_31():
    """Pools of more than 2^31 elements: the first and the last pages of each."""
    kv, dim, page = 1, 256, 1024
    pages = (1 << 31) // (kv * dim * page) + 8
    c = ref.make("bf16", [2000, 1024], kv, dim, page, seed=23, spare=0)
    k, v = (torch.empty((pages, kv, page, dim), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    where = torch.tensor([[pages - 1, 0], [pages - 2, 1]], dtype=torch.int32)
    for b in range(2):
        for e in range(2):
            k[int(where[b, e])] = c["k"][int(c["table"][b, e])].to(DEV)
            v[int(where[b, e])] = c["v"][int(c["table"][b, e])].to(DEV)
    q = torch.randn((2, 4, dim), generator=torch.Generator().manual_seed(24)).to(torch.bfloat16)
    f = runner.Fusion(2)
    dc = runner.cache_of("bf16", k, v, where.to(DEV), c["lengths"].to(DEV), heads=4)
    out = f.cache_attention(dc, q.to(DEV))
    want, tol, _, _ = ref.attention(c, q, "bf16")
    assert status(f) == 0 and ((out.cpu().double() - want).abs() <= tol).all()
    row = torch.randn((2, dim), generator=torch.Generator().manual_seed(25)).to(torch.bfloat16).to(DEV)
    dc.lengths.fill_(1000)
    f.cache_append(dc, row, row)
    assert status(f) == 0 and torch.equal(k[pages - 1, 0, 1000], row[0]) and torch.equal(v[pages - 2, 0, 1000], row[1])


# ---- eviction --------------------------------------------------------------------------------------------------------
def evicts(dtype, c, budget, *, sinks=0, recent=0, outside=False, keep=True):
    batch = len(c["lengths"])
    b = torch.tensor(budget, dtype=torch.int32)
    table_out = None
    if outside:   # pages of their own, fewer than the sequences have
        page, longest = c["k"].shape[2], max(1, max(min(max(x, 0), n) for x, n in zip(budget, c["lengths"].tolist())))
        per, first = -(-longest // page), c["k"].shape[0]
        table_out = (first + torch.randperm(batch * per, generator=torch.Generator().manual_seed(1))).view(batch, per).to(torch.int32)
        for name in ("k", "v", "sizes", "weights"):
            if c[name] is not None:
                c[name] = torch.cat([c[name], torch.full((batch * per, *c[name].shape[1:]), math.nan, dtype=c[name].dtype)])
    dc, f = on_device(dtype, c, c["k"].shape[1]), runner.Fusion(batch)
    kept = torch.full((batch, max(1, int(c["lengths"].max()))), -3, dtype=torch.int32, device=DEV) if keep else None
    out = torch.full((batch,), -7, dtype=torch.int32, device=DEV) if outside else None
    f.cache_evict(dc, b.to(DEV), sinks=sinks, recent=recent, page_table_out=None if table_out is None else table_out.to(DEV),
                  lengths_out=out, keep_idx=kept)
    assert status(f) == 0
    new, keeps = ref.evict(c, budget, sinks=sinks, recent=recent, table_out=table_out)
    same(dc, c, None if outside else new)
    if outside:
        assert torch.equal(out.cpu(), new)
    if keep:
        for i, k in enumerate(keeps):
            row = kept[i].tolist()
            assert row[:len(k)] == k and all(x == -3 for x in row[len(k):])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_heads,dim,page", [(1, 8, 1), (3, 64, 16), (2, 80, 8), (8, 128, 64), (5, 256, 4)])
@pytest.mark.parametrize("outside", [False, True])
def test_evict(dtype, kv_heads, dim, page, outside):
    """Budgets of nothing, one, a few, all and more, with sinks and a recent window that may exceed them."""
    lengths = [0, 1, 40, 257, 600, 64, 513, 33]
    budget = [5, 0, 41, 100, 333, -2, 1, 32]
    for sinks, recent in ((0, 0), (4, 16), (1, 400)):
        c = ref.make(dtype, lengths, kv_heads, dim, page, sizes="masked", weights=True, seed=26)
        evicts(dtype, c, budget, sinks=sinks, recent=recent, outside=outside)


@pytest.mark.parametrize("outside", [False, True])
def test_evict_ties_go_to_the_lowest_position(outside):
    """Weights of few values, zeros of both signs, all equal, negative and denormal; no sizes, no kept positions wanted."""
    for values in ([0.0, -0.0], [1.5], [0.25, 0.5, 0.75], [-1.0, 0.0, 1e-40, -1e-40, 3e38, -3e38]):
        c = ref.make("bf16", [700, 90, 1200, 3], 2, 32, 16, weights=True, seed=27)
        g = torch.Generator().manual_seed(28)
        for b, n in enumerate(c["lengths"].tolist()):
            at = ref.places(c, b, torch.arange(n))
            c["weights"][at] = torch.tensor(values)[torch.randint(0, len(values), (n,), generator=g)]
        evicts("bf16", c, [300, 89, 37, 1], sinks=2, recent=3, outside=outside, keep=values != [1.5])


@pytest.mark.parametrize("n,budget", [(1100, 600), (3000, 1200), (5000, 2500), (9001, 8999), (20000, 77), (40000, 30000), (70000, 35000)])
@pytest.mark.parametrize("outside", [False, True])
def test_evict_long_sequences(n, budget, outside):
    c = ref.make("bf16", [n, n // 3], 2, 64, 64, weights=True, sizes="whole", seed=29)
    evicts("bf16", c, [budget, budget // 4], sinks=4, recent=16, outside=outside)


@pytest.mark.parametrize("n,budget,values", [(150001, 149000, 0), (150001, 70000, 3), (300000, 5, 0)])
def test_evict_sequences_longer_than_the_registers(n, budget, values):
    """More weights than the threads of a cluster hold: the rest are read again; with ties across both parts."""
    c = ref.make("bf16", [n, 40], 1, 8, 256, weights=True, seed=35)
    if values:
        at = ref.places(c, 0, torch.arange(n))
        c["weights"][at] = torch.randint(0, values, (n,), generator=torch.Generator().manual_seed(36)).float()
    evicts("bf16", c, [budget, 17], sinks=3, recent=100)


def test_evict_compares_nothing_where_all_places_are_given():
    """Budgets that the sinks and the recent tokens fill, and a budget of nothing: no weight is compared, so NaN is none's
    concern."""
    c = ref.make("f32", [50, 60, 70], 2, 16, 16, weights=True, seed=37)
    c["weights"][:] = math.nan
    dc, f = on_device("f32", c, 2), runner.Fusion(3)
    f.cache_evict(dc, torch.tensor([12, 0, 70], dtype=torch.int32, device=DEV), sinks=4, recent=8)
    assert status(f) == 0
    for b, keep in ((0, [*range(4), *range(42, 50)]), (1, []), (2, list(range(70)))):
        src, dst = ref.places(c, b, torch.tensor(keep, dtype=torch.long)), ref.places(c, b, torch.arange(len(keep)))
        for name in ("k", "v"):
            c[name][dst[0], :, dst[1]] = c[name][src[0], :, src[1]]
    same(dc, c, torch.tensor([12, 0, 70], dtype=torch.int32))


@pytest.mark.parametrize("outside", [False, True])
def test_evict_leaves_bad_sequences_as_they_are(outside):
    c = ref.make("f32", [50, 60, 70, 80, 90, 64], 2, 16, 16, room=16, weights=True, seed=30)
    good = ref.copy(c)
    for b, pos, value in ((0, 20, math.nan), (1, 30, math.inf), (5, 0, math.nan)):   # (the last one is not compared)
        pg, off = ref.places(c, b, torch.tensor([pos]))
        c["weights"][pg, off] = value
        good["weights"][pg, off] = value
    c["table"][2, 3] = -1
    c["lengths"][3] = 1000
    c["table"][4, 6] = 10 ** 6      # past its length: not read
    good["table"], good["lengths"] = c["table"].clone(), c["lengths"].clone()
    table_out = None
    if outside:
        table_out = (c["k"].shape[0] + torch.arange(12)).view(6, 2).to(torch.int32)
        for name in ("k", "v", "weights"):
            for x in (c, good):
                x[name] = torch.cat([x[name], torch.full((12, *x[name].shape[1:]), math.nan)])
    dc, f = on_device("f32", c, 2), runner.Fusion(6)
    out = torch.full((6,), -7, dtype=torch.int32, device=DEV) if outside else None
    budget = [30] * 6
    f.cache_evict(dc, torch.tensor(budget, dtype=torch.int32, device=DEV), sinks=1, recent=2, lengths_out=out,
                  page_table_out=None if table_out is None else table_out.to(DEV))
    assert status(f) == fz.FUSION_DEV_BAD_CACHE | fz.FUSION_DEV_NONFINITE
    new = torch.tensor([0, 0, 0, 0, 30, 30] if outside else [50, 60, 70, 1000, 30, 30], dtype=torch.int32)
    for b in (4, 5):
        one = {k: t for k, t in good.items()}
        one["table"], one["lengths"] = good["table"][b:b + 1], good["lengths"][b:b + 1]
        ref.evict(one, budget[b:b + 1], sinks=1, recent=2, table_out=None if table_out is None else table_out[b:b + 1])
    same(dc, good, good["lengths"] if outside else new)
    if outside:
        assert torch.equal(out.cpu(), new)


def test_evict_without_room_outside():
    c = ref.make("f32", [50, 10], 2, 16, 16, weights=True, seed=31, spare=4)
    spare = [p for p in range(c["k"].shape[0]) if p not in c["table"].flatten().tolist()]
    dc, f = on_device("f32", c, 2), runner.Fusion(2)
    out = torch.full((2,), -7, dtype=torch.int32, device=DEV)
    f.cache_evict(dc, torch.tensor([17, 17], dtype=torch.int32, device=DEV), lengths_out=out,
                  page_table_out=torch.tensor([spare[:1], spare[1:2]], dtype=torch.int32, device=DEV))
    assert status(f) == fz.FUSION_DEV_BAD_CACHE and out.tolist() == [0, 10]


# ---- together --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_decoder_over_a_compacted_batch(dtype):
    """A stage's output batch (ids, offsets, sizes and scores on the device) becomes the prefix of its sequences; decoder
    steps append a token, attend and accumulate weights; an eviction prunes; steps follow.  The steps are one graph."""
    from workloads import make_workload
    w = make_workload("ragged_b8192_n65_chain4_bf16" if dtype == "bf16" else "ragged_b8192_n65_chain4_f32", batch=12)
    b, spec = w.batch, w.stages[0]
    f = runner.Fusion(b.batch, spec.head.classes)
    db = runner.device_batch(b.dtype, b.offsets, b.x, b.keys, b.sizes, b.scores, device=DEV)
    flags = fz.FUSION_STAGE_MERGE | fz.FUSION_STAGE_EXIT | fz.FUSION_STAGE_PRUNE
    o = f.stage(db, flags, torch.from_numpy(spec.r).to(DEV), torch.from_numpy(spec.rho).to(DEV),
                runner.head_tensors(spec.head, b.dtype, DEV))
    nb = runner.output_batch(db, o)
    heads, kv, dim = 6, 2, 64
    dc = runner.device_cache(dtype, b.batch, 100, heads, kv, dim, page_tokens=16, sizes=True, weights=True)
    g = torch.Generator(device=DEV).manual_seed(32)
    qkv = torch.randn((nb.max_rows, (heads + 2 * kv) * dim), generator=g, device=DEV).to(ref.TYPES[dtype])
    cut = [heads * dim, (heads + kv) * dim]
    f.cache_append(dc, qkv[:, cut[0]:cut[1]], qkv[:, cut[1]:], nb, sizes=nb.sizes, scores=nb.scores)
    c = dict(k=torch.zeros_like(dc.k).cpu(), v=torch.zeros_like(dc.v).cpu(), sizes=torch.zeros_like(dc.sizes).cpu(),
             weights=torch.zeros_like(dc.weights).cpu(), table=dc.page_table.cpu(), lengths=torch.zeros(b.batch, dtype=torch.int32))
    n_out = int(o["batch"].item())
    assert 0 < n_out < b.batch
    host = qkv.cpu()
    c["lengths"] = ref.append(c, host[:, cut[0]:cut[1]], host[:, cut[1]:], o["offsets"].tolist(), o["ids"].tolist(),
                              o["sizes"].cpu(), o["scores"].cpu(), count=n_out)
    same(dc, c)
    step = torch.empty((b.batch, (heads + 2 * kv) * dim), dtype=ref.TYPES[dtype], device=DEV)
    out = torch.empty((b.batch, heads, dim), dtype=ref.TYPES[dtype], device=DEV)
    budget = torch.full((b.batch,), 20, dtype=torch.int32, device=DEV)

    def one_step():
        f.cache_append(dc, step[:, cut[0]:cut[1]], step[:, cut[1]:])
        f.cache_attention(dc, step[:, :cut[0]], out=out)

    graph = None
    for k in range(9):
        step.copy_(torch.randn(step.shape, generator=g, device=DEV))
        if k == 3:
            held = dc.lengths.clone()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                one_step()
            assert torch.equal(held, dc.lengths)
        graph.replay() if graph else one_step()
        hs = step.cpu()
        c["lengths"] = ref.append(c, hs[:, cut[0]:cut[1]], hs[:, cut[1]:], range(b.batch + 1))
        want, tol, wt, wtol = ref.attention(c, hs[:, :cut[0]].reshape(b.batch, heads, dim), dtype)
        assert ((out.cpu().double() - want).abs() <= tol).all()
        gw = dc.weights.cpu()
        assert ((gw.double() - wt).abs() <= wtol + 1e-45).all()
        c["weights"] = gw    # the device's own from here: the eviction compares them
        same(dc, c)
        if k == 5:
            f.cache_evict(dc, budget, sinks=1, recent=4)
            c["lengths"], _ = ref.evict(c, [20] * b.batch, sinks=1, recent=4)
            same(dc, c)
    assert status(f) == 0


# ---- bounds ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_batch(dtype):
    """FUSION_CACHE_MAX_BATCH sequences, and one fewer: a row each in place and with the lengths elsewhere, by ids in
    another order with the last sample left out, attention of one token (its value), eviction of every other one."""
    for batch in (fz.FUSION_CACHE_MAX_BATCH, fz.FUSION_CACHE_MAX_BATCH - 1):
        g = torch.Generator(device=DEV).manual_seed(50)
        dc, f = runner.device_cache(dtype, batch, 2, 1, 1, 8, page_tokens=1, weights=True), runner.Fusion(1)
        k, v = (torch.randn((batch, 8), generator=g, device=DEV).to(ref.TYPES[dtype]) for _ in range(2))
        out = torch.full((batch,), -7, dtype=torch.int32, device=DEV)
        f.cache_append(dc, k, v, lengths_out=out)
        assert status(f) == 0 and (out == 1).all() and (dc.lengths == 0).all()
        assert torch.equal(dc.k[::2, 0, 0], k) and torch.equal(dc.v[::2, 0, 0], v)
        ids = torch.randperm(batch, generator=g, device=DEV).to(torch.int32)
        last = int(ids[-1])
        rows = runner.RaggedRows(batch, 1, batch, torch.arange(batch + 1, dtype=torch.int32, device=DEV),
                                 torch.tensor([batch - 1], dtype=torch.int32, device=DEV), ids)
        out.fill_(-7)
        f.cache_append(dc, k, v, rows, lengths_out=out)
        want = torch.ones_like(out)
        want[last] = 0
        assert status(f) == 0 and torch.equal(out, want) and (dc.lengths == 0).all()
        f.cache_append(dc, k, v, rows)
        assert status(f) == 0 and torch.equal(dc.lengths, want)
        held = ids[:-1].long()
        assert torch.equal(dc.k[::2, 0, 0][held], k[:-1]) and torch.equal(dc.v[::2, 0, 0][held], v[:-1])
        got = f.cache_attention(dc, k.view(batch, 1, 8))
        assert status(f) == 0 and torch.equal(got[held, 0], v[:-1]) and (got[last] == 0).all()
        assert (dc.weights[::2, 0][held] == 1).all()
        f.cache_evict(dc, (torch.arange(batch, device=DEV) % 2).to(torch.int32))
        want[::2] = 0
        assert status(f) == 0 and torch.equal(dc.lengths, want)
        assert int(dc.workspace[:1 << 18].max()) == 0
        rows = runner.RaggedRows(batch, 1, batch, rows.offsets, torch.tensor([batch + 1], dtype=torch.int32, device=DEV), ids)
        f.cache_append(dc, k, v, rows)
        assert status(f) == fz.FUSION_DEV_BAD_BATCH and torch.equal(dc.lengths, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_capacity(dtype):
    """A page table with room for 2^30 tokens (of which a few pages are there): windows and sinks of everything, an append,
    an eviction."""
    c = ref.make(dtype, [1500], 1, 8, 1024, room=500, weights=True, seed=51)
    table = torch.full((1, 1 << 20), -1, dtype=torch.int32)
    table[:, :2] = c["table"]
    c["table"] = table
    for window, sinks in ((2 ** 31 - 1, 2 ** 31 - 1), (2 ** 30, 0), (2 ** 30 - 1, 2 ** 31 - 1), (700, 2 ** 31 - 1), (700, 9)):
        _, dc = attend(dtype, c, 2, window=window, sinks=sinks)
        c["weights"] = dc.weights.cpu()
    f = runner.Fusion(1)
    k, v = (torch.randn((1, 8), generator=torch.Generator().manual_seed(52)).to(ref.TYPES[dtype]) for _ in range(2))
    f.cache_append(dc, k.to(DEV), v.to(DEV))
    c["lengths"] = ref.append(c, k, v, [0, 1])
    f.cache_evict(dc, torch.tensor([601], dtype=torch.int32, device=DEV), sinks=4, recent=2 ** 31 - 1)
    c["lengths"], _ = ref.evict(c, [601], sinks=4, recent=2 ** 31 - 1)
    assert status(f) == 0
    same(dc, c)


# ---- sequences that are left out -------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [[600, 70, 300], [40] * 260])
def test_attention_leaves_the_weights_of_a_refused_sequence(dtype, lengths):
    """A bad page, and a NaN or an infinity among the sequence's queries or keys, whose logits are no numbers: its weights
    keep their bits, -0 among them, and so does every page that it names and another sequence holds."""
    for what in ("query", "infinite query", "key", "infinite key"):
        c = ref.make(dtype, lengths, 2, 64, 16, room=16, weights=True, seed=53)
        good = ref.copy(c)
        at0 = ref.places(c, 0, torch.arange(lengths[0]))
        c["weights"][at0[0][::2], at0[1][::2]] = -0.0
        q = torch.randn((len(lengths), 4, 64), generator=torch.Generator().manual_seed(54)).to(ref.TYPES[dtype])
        value = math.inf if "infinite" in what else math.nan
        if "query" in what:
            q[0, 1:3, 7] = value
        else:
            c["k"][at0[0][5:9], :, at0[1][5:9], 3] = value
        held = c["weights"].clone()
        c["table"][0, 2] = -1                       # position 32 on
        c["table"][0, 1] = c["table"][2, 0]         # the third sequence's by now
        dc, f = on_device(dtype, c, 4), runner.Fusion(len(lengths))
        out = torch.full((len(lengths), 4, 64), 7.0, dtype=ref.TYPES[dtype], device=DEV)
        f.cache_attention(dc, q.to(DEV), out=out)
        assert status(f) == fz.FUSION_DEV_BAD_CACHE, what
        assert (out[0] == 7.0).all()
        good["k"], good["lengths"][0] = c["k"], 0
        want, tol, w, wtol = ref.attention(good, torch.nan_to_num(q), dtype)
        got, gw = out.cpu().double(), dc.weights.cpu()
        assert torch.equal(ref.bits(gw[at0]), ref.bits(held[at0])), what
        for b in range(1, len(lengths)):
            at = ref.places(good, b, torch.arange(lengths[b]))
            assert ((got[b] - want[b]).abs() <= tol[b]).all() and ((gw[at].double() - w[at]).abs() <= wtol[at]).all(), (what, b)


@pytest.mark.parametrize("n,dtype", [(70, "f32"), (3000, "bf16"), (9000, "bf16"), (150001, "bf16")])
def test_evict_compares_nothing_whatever_the_weights_hold(n, dtype):
    """Where the sinks and the recent tokens fill the budget, weights of any bits: NaN of all ones (memory that nobody has
    written), of either sign, infinities; and a budget of nothing."""
    for word in (-1, 0x7FFFFFFF, -0x800000, 0x7F800000, 0):
        c = ref.make(dtype, [n, 60, 45], 1, 8, 16, weights=True, seed=55)
        c["weights"] = torch.full(c["weights"].shape, word, dtype=torch.int32).view(torch.float32)
        dc, f = on_device(dtype, c, 1), runner.Fusion(3)
        f.cache_evict(dc, torch.tensor([n - 20, 0, 12], dtype=torch.int32, device=DEV), sinks=4, recent=n - 24)
        assert status(f) == 0
        for b, keep in ((0, [*range(4), *range(24, n)]), (1, []), (2, [*range(4), *range(37, 45)])):
            src, dst = ref.places(c, b, torch.tensor(keep, dtype=torch.long)), ref.places(c, b, torch.arange(len(keep)))
            for name in ("k", "v"):
                c[name][dst[0], :, dst[1]] = c[name][src[0], :, src[1]]
        same(dc, c, torch.tensor([n - 20, 0, 12], dtype=torch.int32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_of_no_rows(dtype):
    """Batches without rows, whose tensors have no address: samples of no tokens, and no samples; in place and elsewhere."""
    c = ref.make(dtype, [5, 0, 17], 2, 16, 8, room=4, sizes="whole", weights=True, seed=56)
    dc, f = on_device(dtype, c, 2), runner.Fusion(3)
    none = torch.empty((0, 32), dtype=ref.TYPES[dtype], device=DEV)
    per_row = torch.empty(0, device=DEV)
    for batch in (3, 1, 0):
        ids = torch.arange(batch, dtype=torch.int32, device=DEV).flip(0)
        for rows in (runner.RaggedRows(batch, 1, 0, torch.zeros(batch + 1, dtype=torch.int32, device=DEV)),
                     runner.RaggedRows(batch, 7, 0, torch.zeros(batch + 1, dtype=torch.int32, device=DEV), ids=ids)):
            out = torch.full((3,), -7, dtype=torch.int32, device=DEV)
            assert f.cache_append(dc, none, none, rows, sizes=per_row, scores=per_row, lengths_out=out) is out
            assert out.tolist() == [5, 0, 17]
            f.cache_append(dc, none.view(0, 2, 16), none, rows)
    assert status(f) == 0
    same(dc, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_behind_copies_fills_and_other_streams(dtype):
    """A graph in which each of the three calls follows a copy, a fill or a join with another stream's kernel that writes what
    it reads, and is followed by a copy of what it wrote; replayed on other rows, lengths and budgets, calls of its own between."""
    lengths = [100, 37, 0, 64, 300]
    c = ref.make(dtype, lengths, 2, 64, 16, room=40, sizes="whole", weights=True, seed=57)
    dc, f = on_device(dtype, c, 4), runner.Fusion(5)
    t = ref.TYPES[dtype]
    rows, offsets = 60, torch.tensor([0, 13, 13, 30, 31, 60], dtype=torch.int32)
    rr = runner.RaggedRows(5, 30, rows, offsets.to(DEV))
    k, v = (torch.zeros((rows, 2, 64), dtype=t, device=DEV) for _ in range(2))
    q, out = (torch.zeros((5, 4, 64), dtype=t, device=DEV) for _ in range(2))
    kept, budget = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in ((5, 64), 5))
    src = {n: torch.zeros_like(x) for n, x in dict(k=k, v=v, q=q, budget=budget).items()}
    copies = {n: torch.zeros_like(x) for n, x in dict(lengths=dc.lengths, out=out, weights=dc.weights, kept=kept).items()}
    side = torch.cuda.Stream()
    lens = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            v.copy_(src["v"])
            v.mul_(2.0)                       # another stream's kernel, joined just before the append
        dc.lengths.copy_(lens)
        k.copy_(src["k"])
        main.wait_stream(side)
        f.cache_append(dc, k, v, rr)
        copies["lengths"].copy_(dc.lengths)
        k.zero_()
        dc.weights.zero_()
        q.copy_(src["q"])
        f.cache_attention(dc, q, out=out)
        q.zero_()
        copies["out"].copy_(out)
        copies["weights"].copy_(dc.weights)
        kept.zero_()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            budget.copy_(src["budget"])
            budget.add_(1)
        main.wait_stream(side)
        f.cache_evict(dc, budget, sinks=2, recent=8, keep_idx=kept)
        copies["kept"].copy_(kept)
        budget.zero_()
    for seed in (58, 59, 60):
        g = torch.Generator().manual_seed(seed)
        c = ref.make(dtype, lengths, 2, 64, 16, room=40, sizes="whole", weights=True, seed=seed)
        for name, x in (("k", dc.k), ("v", dc.v), ("sizes", dc.sizes), ("table", dc.page_table)):
            x.copy_(c[name])
        host = {n: torch.randn(x.shape, generator=g).to(t) for n, x in src.items() if n != "budget"}
        host["budget"] = torch.randint(0, 200, (5,), generator=g).to(torch.int32)
        for n, x in host.items():
            src[n].copy_(x)
        graph.replay()
        c["lengths"] = ref.append(c, host["k"], host["v"] * 2.0, offsets)
        assert torch.equal(copies["lengths"].cpu(), c["lengths"])
        c["weights"] = torch.zeros_like(c["weights"])
        want, tol, w, wtol = ref.attention(c, host["q"], dtype)
        assert ((copies["out"].cpu().double() - want).abs() <= tol).all()
        gw = copies["weights"].cpu()
        assert ((gw.double() - w).abs() <= wtol + 1e-45).all()
        c["weights"] = gw
        c["lengths"], keeps = ref.evict(c, host["budget"] + 1, sinks=2, recent=8)
        same(dc, c)
        for b, keep in enumerate(keeps):
            assert copies["kept"][b].tolist() == (keep + [0] * 64)[:64]
        f.cache_attention(dc, q)     # (a call of its own between two replays)
    assert status(f) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_streams_at_once(dtype):
    """Calls that overlap on two streams, a cache object each over the same pools (other sequences' pages): steps of append,
    attention with weights and, at the end, an eviction give the bits that they give one after the other."""
    lengths = [700, 33, 2500, 64, 5, 900]
    c = ref.make(dtype, lengths, 2, 64, 16, room=40, sizes="whole", weights=True, seed=61)
    g = torch.Generator().manual_seed(62)
    rows = [torch.randn((20, 3, 8 * 64), generator=g).to(ref.TYPES[dtype]).to(DEV) for _ in range(2)]   # queries, keys, values
    budget = torch.tensor([300, 40, 1100], dtype=torch.int32, device=DEV)

    def run(streams):
        d = {k: None if t is None else t.to(DEV) for k, t in c.items()}
        halves = [runner.cache_of(dtype, d["k"], d["v"], d["table"][3 * s:3 * s + 3].contiguous(), d["lengths"][3 * s:3 * s + 3].contiguous(), heads=4,
                                  sizes=d["sizes"], weights=d["weights"]) for s in range(2)]
        f, outs = runner.Fusion(6), [[], []]
        torch.cuda.synchronize()
        for step in range(21):
            for s, dc in enumerate(halves):
                with torch.cuda.stream(streams[s]):
                    if step == 20:
                        f.cache_evict(dc, budget, sinks=2, recent=16)
                        continue
                    x = rows[s][step]
                    f.cache_append(dc, x[:, 256:384], x[:, 384:])
                    outs[s].append(f.cache_attention(dc, x[:, :256]))
        assert status(f) == 0
        bits = [ref.bits(t.cpu()) for t in (d["k"], d["v"], d["sizes"], d["weights"], *outs[0], *outs[1])]
        return [*bits, halves[0].lengths.cpu(), halves[1].lengths.cpu()]

    main = torch.cuda.current_stream()
    want = run([main, main])
    for _ in range(3):
        got = run([torch.cuda.Stream(), torch.cuda.Stream()])
        assert all(torch.equal(a, b) for a, b in zip(got, want, strict=True))
