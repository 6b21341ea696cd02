"""The cache in 4 bits, appends that rotate keys and queries, and reading rows back, on the GPU against the definitions on the
host (packed_reference.py, where the tolerances are derived).  What is copied, rotated or rounded to 4 bits is compared bit by
bit; whatever no call may touch or use holds NaN."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import cache_reference as ref  # noqa: E402
import packed_reference as pk  # noqa: E402
import paper_2607_02612_gb300 as fz  # noqa: E402
from paper_2607_02612_gb300 import runner  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda"
POOLS = ("k", "v", "k_scales", "v_scales")


def packed(dtype, c, heads):
    d = {k: None if t is None else t.to(DEV) for k, t in c.items()}
    return runner.packed_cache_of(dtype, d["k"], d["v"], d["k_scales"], d["v_scales"], d["table"], d["lengths"], heads=heads,
                                  sizes=d["sizes"], weights=d["weights"])


def plain(dtype, c, heads):
    d = {k: None if t is None else t.to(DEV) for k, t in c.items()}
    return runner.cache_of(dtype, d["k"], d["v"], d["table"], d["lengths"], heads=heads, sizes=d["sizes"], weights=d["weights"])


def same(dc, c, lengths=None):
    """The device's cache equals the host's, bit by bit."""
    for name in (*POOLS, "sizes", "weights"):
        want = c.get(name)
        if want is not None:
            got = getattr(dc, name).cpu()
            assert torch.equal(got, want) if got.dtype == torch.uint8 else torch.equal(ref.bits(got), ref.bits(want)), name
    assert torch.equal(dc.lengths.cpu(), c["lengths"] if lengths is None else lengths)


def equal_bits(a, b):
    return torch.equal(ref.bits(a.cpu()), ref.bits(b.cpu()))


def status(f):
    torch.cuda.synchronize()
    return int(f.status.item())


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def ragged(offsets, ids=None, longest=None, batch=None):
    n = len(offsets) - 1
    longest = longest or max([1, *(b - a for a, b in zip(offsets, offsets[1:]))])
    return runner.RaggedRows(n, longest, offsets[-1], ints(offsets), ints(batch), ints(ids))


def hard_rows(g, rows, kv, dim, dtype):
    """Rows with every kind of group: ties between two codes, zeros, tiny, huge and mixed magnitudes, NaN and infinities."""
    x = torch.randn((rows, kv, dim), generator=g)
    a = x.view(-1, 16)
    kind = torch.randint(0, 10, (a.shape[0],), generator=g)
    top = torch.randint(8, 16, (a.shape[0], 1), generator=g) * 2.0 ** torch.randint(-6, 7, (a.shape[0], 1), generator=g)
    ties = pk.MIDDLES.float()[torch.randint(0, 7, a.shape, generator=g)] * torch.sign(a)
    ties[:, 0] = 6.0
    a[kind == 1] = (ties * top / 8)[kind == 1]                      # x / scale lies between two codes
    a[kind == 2] = 0.0
    a[kind == 3] *= 2.0 ** -11                                      # scales at e4m3's lower end
    a[kind == 4] *= 2.0 ** -16                                      # scale 0
    a[kind == 5] *= 3000.0                                          # scale 448, codes cut off
    a[kind == 6] *= torch.exp(torch.randn(a[kind == 6].shape, generator=g) * 4)
    a[kind == 7, 3] = math.nan if rows > 2 else 1.0
    a[kind == 8, 9] = -math.inf if rows > 2 else 1.0
    a[kind == 2, 5] = -0.0
    return x.to(ref.TYPES[dtype])


# ---- append in 4 bits -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_heads,dim,page", [(1, 32, 1), (3, 64, 16), (2, 96, 8), (8, 128, 64), (5, 256, 4), (17, 160, 2)])
@pytest.mark.parametrize("in_place", [True, False])
def test_append(dtype, kv_heads, dim, page, in_place):
    """Ragged samples (one without rows, one that fills its pages) to sequences in another order, from slices of packed
    projections; the other sequences keep their tokens, and what lies behind a row's scales is zero where a row was written."""
    counts, ids = [33, 0, 1, 24], [3, 0, 1, 4]
    c = pk.make([5, 0, 17, 3, 40], kv_heads, dim, page, room=24, sizes="whole", weights=True, seed=1)
    dc, f = packed(dtype, c, kv_heads), runner.Fusion(8)
    g = torch.Generator().manual_seed(2)
    offsets, width = [0, 33, 33, 34, 58], kv_heads * dim
    both = torch.randn((58 + 3, 3 * width), generator=g).to(ref.TYPES[dtype])
    both[:58, width:2 * width] = hard_rows(g, 58, kv_heads, dim, dtype).view(58, width)
    both[:58, 2 * width:] = hard_rows(g, 58, kv_heads, dim, dtype).view(58, width)
    sizes, scores = torch.rand(58, generator=g), torch.rand(58, generator=g)
    assert counts == [b - a for a, b in zip(offsets, offsets[1:])]
    dev = both.to(DEV)
    out = torch.full((5,), -7, dtype=torch.int32, device=DEV)
    got = f.cache_append(dc, dev[:, width:2 * width], dev[:, 2 * width:], ragged(offsets, ids), sizes=sizes.to(DEV), scores=scores.to(DEV),
                         lengths_out=None if in_place else out)
    assert got is (dc.lengths if in_place else out) and status(f) == 0
    rows = both[:58].float()
    new = pk.append(c, rows[:, width:2 * width].reshape(58, kv_heads, dim), rows[:, 2 * width:].reshape(58, kv_heads, dim), offsets, ids,
                    sizes, scores)
    same(dc, c, new if in_place else None)
    if not in_place:
        assert torch.equal(out.cpu(), new)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_every_value_of_a_group(dtype):
    """All bf16 numbers (in float32 also those next to a tie) beside each of the e4m3 scales."""
    g = torch.Generator().manual_seed(3)
    every = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    every = every[torch.isfinite(every)]
    tops = pk.E4M3[1:] * 6
    small = [m * s * (1 + e) for s in pk.E4M3[1:] for m in pk.MIDDLES for e in (0, 2.0 ** -23, -2.0 ** -23)]
    small = torch.cat([torch.tensor(small, dtype=torch.float64).float(), every])
    rows = -(-len(small) // (15 * 8))
    x = torch.zeros((rows * 8, 16))
    x[:, 1:] = torch.nn.functional.pad(small, (0, rows * 8 * 15 - len(small)))[torch.randperm(rows * 8 * 15, generator=g)].view(-1, 15)
    x[:, 0] = tops[torch.randint(0, len(tops), (rows * 8,), generator=g)].float()
    # and each tie beside its own scale
    n = min(len(small) // 21 * 21, 126 * 21)
    own = small[:n].view(126, 21)
    for i in range(2):
        x[i * 126:(i + 1) * 126, 1:] = own[:, i * 6:i * 6 + 15]
        x[i * 126:(i + 1) * 126, 0] = tops.float()
    x = x.view(rows, 1, 128).to(ref.TYPES[dtype])
    c = pk.make([0], 1, 128, 16, room=rows, seed=4)
    dc, f = packed(dtype, c, 1), runner.Fusion(1)
    f.cache_append(dc, x.to(DEV), x.flip(0).contiguous().to(DEV), ragged([0, rows]))
    assert status(f) == 0
    same(dc, c, pk.append(c, x.float(), x.flip(0).float(), [0, rows]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_one_row_each_and_long_samples(dtype):
    """A token per sequence (no offsets given), sizes 1 and scores 0 by default, twice; then samples of many CTAs and one whose
    rows the CTAs take in several turns; the second time there is no room for some."""
    c = pk.make([0, 1, 15, 16, 17, 31], 2, 64, 16, room=700, sizes="whole", weights=True, seed=3)
    dc, f = packed(dtype, c, 2), runner.Fusion(6)
    g = torch.Generator().manual_seed(4)
    for _ in range(2):
        k, v = (torch.randn((6, 2, 64), generator=g).to(ref.TYPES[dtype]) for _ in range(2))
        f.cache_append(dc, k.to(DEV), v.to(DEV))
        c["lengths"] = pk.append(c, k.float(), v.float(), range(7))
    offsets = [0, 650, 651, 1300, 1300, 1901, 2000]
    k, v = (torch.randn((2000, 2, 64), generator=g).to(ref.TYPES[dtype]) for _ in range(2))
    for _ in range(2):
        f.cache_append(dc, k.to(DEV), v.to(DEV), ragged(offsets))
        if status(f) == 0:
            c["lengths"] = pk.append(c, k.float(), v.float(), offsets)
    assert status(f) == fz.FUSION_DEV_BAD_CACHE
    fits = [b for b in range(6) if int(c["lengths"][b]) + offsets[b + 1] - offsets[b] <= dc.max_pages * dc.page_tokens]
    assert 0 < len(fits) < 6
    for b in fits:
        c["lengths"][b] = pk.append(c, k.float(), v.float(), [offsets[b], offsets[b + 1]], [b])[b]
    same(dc, c)
    assert int(dc.workspace[:1 << 18].max()) == 0
    n = 90001   # more rows than 2432 CTAs take at once
    c = pk.make([3], 1, 128, 128, room=n, seed=5)
    dc = packed(dtype, c, 1)
    k, v = (torch.randn((n, 1, 128), generator=g).to(ref.TYPES[dtype]) for _ in range(2))
    f = runner.Fusion(1)
    f.cache_append(dc, k.to(DEV), v.to(DEV), ragged([0, n]))
    assert status(f) == 0
    same(dc, c, pk.append(c, k.float(), v.float(), [0, n]))


# ---- rotation -----------------------------------------------------------------------------------------------------------
TURNS = [(2, 64, 64, 4), (1, 80, 80, 3), (3, 96, 32, 1), (2, 128, 128, 16), (4, 8 * 23, 176, 5), (1, 256, 128, 1), (2, 16, 16, 2)]


def rotated(dtype, four, kv, dim, turned, heads, pairs, where, seed, in_place=True, queries=True):
    g = torch.Generator().manual_seed(seed)
    lengths, offsets, ids = [5, 0, 17, 3, 40], [0, 33, 33, 34, 58], [3, 0, 1, 4]
    make = dict(room=24, sizes="whole", weights=True, seed=seed)
    c = pk.make(lengths, kv, dim, 16, **make) if four else ref.make(dtype, lengths, kv, dim, 16, **make)
    dc, f = (packed if four else plain)(dtype, c, kv), runner.Fusion(8)
    table = torch.randn((5000, turned), generator=g)   # (any numbers serve as cosines and sines)
    k, v = (torch.randn((60, kv, dim), generator=g).to(ref.TYPES[dtype]) for _ in range(2))
    wide = torch.randn((61, heads + 2, dim), generator=g).to(ref.TYPES[dtype])
    place = torch.cat([torch.arange(b - a) + lengths[t] for a, b, t in zip(offsets, offsets[1:], ids)])
    pos = None if where == "places" else torch.randint(0, 5000, (58,), generator=g) if where == "given" else torch.full((58,), 4999)
    q = wide[:58, 1:heads + 1]
    rows = dict(sizes=torch.rand(58, generator=g), scores=torch.rand(58, generator=g))
    q_out = torch.full((61, heads, dim), math.nan, dtype=ref.TYPES[dtype], device=DEV)
    out = torch.full((5,), -7, dtype=torch.int32, device=DEV)
    got = f.cache_append_rotated(dc, k.to(DEV), v.to(DEV), runner.Rotation(table.to(DEV), pairs), ragged(offsets, ids),
                                 positions=None if pos is None else pos.to(torch.int32).to(DEV),
                                 q=wide.to(DEV)[:, 1:heads + 1] if queries else None, q_out=q_out if queries else None,
                                 lengths_out=None if in_place else out, **{n: t.to(DEV) for n, t in rows.items()})
    assert status(f) == 0 and got is (q_out if queries else None)
    at = place if pos is None else pos
    kt = pk.turn(k[:58].float(), table, at, pairs)
    if queries:
        assert equal_bits(q_out[:58], pk.turn(q.float(), table, at, pairs).to(ref.TYPES[dtype])) and torch.isnan(q_out[58:]).all()
    new = pk.append(c, kt, v[:58].float(), offsets, ids, **rows) if four else ref.append(c, kt.to(ref.TYPES[dtype]), v, offsets, ids, **rows)
    same(dc, c, new if in_place else None)
    if not in_place:
        assert torch.equal(out.cpu(), new)
    assert int(dc.workspace[:1 << 18].max()) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", ["halves", "adjacent"])
@pytest.mark.parametrize("kv,dim,turned,heads", TURNS)
def test_rotated_append(dtype, pairs, kv, dim, turned, heads):
    rotated(dtype, False, kv, dim, turned, heads, pairs, "given", 6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", ["halves", "adjacent"])
@pytest.mark.parametrize("kv,dim,turned,heads", [(1, 80, 32, 3), (16, 80, 32, 64), (3, 40, 16, 7), (2, 40, 32, 1), (2, 24, 16, 5), (5, 48, 16, 2),
                                                 (2, 112, 48, 4), (1, 56, 32, 9), (2, 144, 16, 3), (2, 208, 192, 2), (1, 16, 16, 1), (1, 240, 240, 2)])
def test_rotated_append_odd_numbers_of_segments(dtype, pairs, kv, dim, turned, heads):
    rotated(dtype, False, kv, dim, turned, heads, pairs, "given", 40)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", ["halves", "adjacent"])
@pytest.mark.parametrize("kv,dim,turned,heads", [t for t in TURNS if t[1] % 32 == 0 and t[2] % 32 == 0] + [(3, 160, 96, 6), (2, 32, 32, 2)])
def test_rotated_append_in_4_bits(dtype, pairs, kv, dim, turned, heads):
    rotated(dtype, True, kv, dim, turned, heads, pairs, "given", 7)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("where", ["places", "last"])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("queries", [True, False])
def test_rotated_append_positions_and_optional_arguments(four, where, in_place, queries):
    rotated("bf16", four, 2, 64, 32, 8, "halves", where, 8, in_place, queries)


def test_rotated_queries_in_place_and_many_heads():
    """q_out is q; 1024 query heads beside one key head, and 300 key heads beside one query head."""
    for kv, heads, dim in ((1, 1024, 32), (300, 1, 32), (2, 64, 256)):
        g = torch.Generator().manual_seed(9)
        c = ref.make("bf16", [0, 2], kv, dim, 4, room=4, seed=9)
        dc, f = plain("bf16", c, kv), runner.Fusion(2)
        table = torch.randn((6, dim), generator=g)
        k, v = (torch.randn((2, kv, dim), generator=g).to(torch.bfloat16) for _ in range(2))
        q = torch.randn((2, heads, dim), generator=g).to(torch.bfloat16)
        dq = q.to(DEV)
        assert f.cache_append_rotated(dc, k.to(DEV), v.to(DEV), runner.Rotation(table.to(DEV)), q=dq, q_out=dq) is dq and status(f) == 0
        at = torch.tensor([0, 2])
        assert equal_bits(dq, pk.turn(q.float(), table, at, "halves").to(torch.bfloat16))
        same(dc, c, ref.append(c, pk.turn(k.float(), table, at, "halves").to(torch.bfloat16), v, [0, 1, 2]))


def test_rotation_table():
    """Its angles, against the C library's functions, and that rotated dot products depend on differences of positions."""
    t = runner.rotation_table(70000, 64, base=500.0, device=DEV).cpu()
    for p in (0, 1, 69999):
        for i in (0, 7, 31):
            a = p * 500.0 ** (-2 * i / 64)
            assert abs(t[p, i].item() - math.cos(a)) <= 2.0 ** -24 + 2e-11 and abs(t[p, 32 + i].item() - math.sin(a)) <= 2.0 ** -24 + 2e-11
    g = torch.Generator().manual_seed(10)
    x, y = (torch.randn((1, 1, 64), generator=g) for _ in range(2))
    for pairs in ("halves", "adjacent"):
        dots = [(pk.turn(x, t, torch.tensor([p]), pairs).double() * pk.turn(y, t, torch.tensor([p + 30]), pairs).double()).sum() for p in (0, 1000, 60000)]
        # 64 products of dims below 5, each dim off by at most 3 2^-24 of its size and the table's 2^-24
        assert max(abs(d - dots[0]) for d in dots) <= 2 * 64 * 25 * 8 * 2.0 ** -24


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("in_place", [True, False])
def test_rotated_append_bad_positions(four, in_place):
    """A position that the table does not have leaves its sequence as it is, whatever CTA meets it; the others are appended."""
    for bad in (-1, 700, 2 ** 31 - 1, -2 ** 31):
        g = torch.Generator().manual_seed(11)
        lengths, offsets = [5, 0, 17], [0, 600, 601, 640]
        make = dict(room=610, sizes="whole", weights=True, seed=11)
        c = pk.make(lengths, 2, 64, 16, **make) if four else ref.make("bf16", lengths, 2, 64, 16, **make)
        dc, f = (packed if four else plain)("bf16", c, 4), runner.Fusion(3)
        table = torch.randn((700, 64), generator=g)
        pos = torch.randint(0, 700, (640,), generator=g)
        k, v = (torch.randn((640, 2, 64), generator=g).to(torch.bfloat16) for _ in range(2))
        given = pos.clone()
        given[433] = bad
        out = torch.full((3,), -7, dtype=torch.int32, device=DEV)
        f.cache_append_rotated(dc, k.to(DEV), v.to(DEV), runner.Rotation(table.to(DEV)), ragged(offsets), positions=ints(given.tolist()),
                               lengths_out=None if in_place else out)
        assert status(f) == fz.FUSION_DEV_BAD_POSITION
        kt = pk.turn(k.float(), table, pos, "halves")
        rows = [(kt, v.float()), pk.append] if four else [(kt.to(torch.bfloat16), v), ref.append]
        before = ref.copy(c)
        new = rows[1](c, *rows[0], offsets)
        assert (dc.lengths if in_place else out).tolist() == [5, *new.tolist()[1:]]
        for b in (0, 1, 2):   # sequence 0's tokens as before, the others' as appended
            want, n = (before, 5) if b == 0 else (c, int(new[b]))
            at = ref.places(c, b, torch.arange(n))
            for name in (POOLS if four else ("k", "v")):
                got, w = getattr(dc, name).cpu()[at[0], :, at[1]], want[name][at[0], :, at[1]]
                assert torch.equal(got, w) if four else equal_bits(got, w)
        assert int(dc.workspace[:1 << 18].max()) == 0
        # positions as places run out of the table too
        f = runner.Fusion(3)
        f.cache_append_rotated(dc, k.to(DEV), v.to(DEV), runner.Rotation(table[:600].to(DEV)), ragged(offsets), lengths_out=out)
        assert status(f) & fz.FUSION_DEV_BAD_POSITION and out[0] == 5


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("in_place", [True, False])
def test_rotated_append_leaves_bad_samples_out(four, in_place):
    offs, ids_bit, cache_bit, batch_bit = fz.FUSION_DEV_BAD_OFFSETS, fz.FUSION_DEV_BAD_IDS, fz.FUSION_DEV_BAD_CACHE, fz.FUSION_DEV_BAD_BATCH
    for what, bit in (("decreasing", offs), ("long", offs), ("id", ids_bit), ("twice", ids_bit), ("room", cache_bit),
                      ("page", cache_bit), ("length", cache_bit), ("batch", batch_bit), ("count", 0)):
        make = dict(room=20, sizes="whole", weights=True, seed=5)
        c = pk.make([4, 9, 2, 30], 2, 32, 8, **make) if four else ref.make("bf16", [4, 9, 2, 30], 2, 32, 8, **make)
        offsets, ids, count, good, longest = [0, 10, 12, 20, 25], [2, 1, 0, 3], None, [0, 1, 2, 3], 10
        if what == "decreasing":
            offsets, good = [0, 10, 8, 16, 21], [0, 2, 3]
        elif what == "long":
            longest, good = 9, [1, 2, 3]
        elif what == "id":
            ids, good = [2, 4, -1, 3], [0, 3]
        elif what == "twice":
            ids, good = [2, 1, 2, 3], [1, 3]
        elif what == "room":
            c["lengths"][2], good = 8 * c["table"].shape[1] - 9, [1, 2, 3]
        elif what == "page":
            c["table"][1, 1], good = 10 ** 6, [0, 2, 3]
        elif what == "length":
            c["lengths"][0], good = -3, [0, 1, 3]
        elif what == "batch":
            count, good = [5], []
        elif what == "count":
            count, good = [2], [0, 1]
        dc, f = (packed if four else plain)("bf16", c, 2), runner.Fusion(4)
        g = torch.Generator().manual_seed(6)
        k, v, q = (torch.randn((25, 2, 32), generator=g).to(torch.bfloat16) for _ in range(3))
        table = torch.randn((100, 32), generator=g)
        q_out = torch.full((25, 2, 32), math.nan, dtype=torch.bfloat16, device=DEV)
        out = torch.full((4,), -7, dtype=torch.int32, device=DEV)
        rows = runner.RaggedRows(4, longest, 25, ints(offsets), ints(count), ints(ids))
        f.cache_append_rotated(dc, k.to(DEV), v.to(DEV), runner.Rotation(table.to(DEV)), rows, positions=ints(list(range(25))),
                               q=q.to(DEV), q_out=q_out, lengths_out=None if in_place else out)
        assert status(f) == bit, what
        at = torch.arange(25)
        kt, qt = pk.turn(k.float(), table, at, "halves"), pk.turn(q.float(), table, at, "halves").to(torch.bfloat16)
        wrote = torch.zeros(25, dtype=torch.bool)
        new = c["lengths"].clone()
        for i in good:
            a, b = offsets[i], offsets[i + 1]
            wrote[a:b] = True
            one = [kt[a:b], v[a:b].float()] if four else [kt[a:b].to(torch.bfloat16), v[a:b]]
            new[ids[i]] = (pk if four else ref).append(c, *one, [0, b - a], [ids[i]])[ids[i]]
        if what != "batch" or in_place:
            assert torch.equal((dc.lengths if in_place else out).cpu(), new), what
        same(dc, c, new if in_place else None)
        assert equal_bits(q_out[wrote.to(DEV)], qt[wrote]) and torch.isnan(q_out[~wrote.to(DEV)]).all(), what
        assert int(dc.workspace[:1 << 18].max()) == 0


# ---- reading back ---------------------------------------------------------------------------------------------------------
READS = [(1, 32, 1), (3, 64, 16), (2, 96, 8), (8, 128, 64), (40, 256, 4), (2, 8, 2)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("four,kv_heads,dim,page", [(four, *r) for four in (False, True) for r in READS if not four or r[1] % 32 == 0])
def test_read(dtype, four, kv_heads, dim, page):
    """Ragged pieces of sequences, one twice, one without rows; rows of no sample stay."""
    lengths, counts, ids, starts = [5, 0, 170, 3, 40], [33, 0, 1, 24, 150, 5], [4, 1, 3, 2, 2, 0], [7, 0, 2, 100, 20, 0]
    make = dict(sizes="whole", weights=True, seed=12)
    c = pk.make(lengths, kv_heads, dim, page, **make) if four else ref.make(dtype, lengths, kv_heads, dim, page, **make)
    dc, f = (packed if four else plain)(dtype, c, kv_heads), runner.Fusion(8)
    offsets = [0, *torch.tensor(counts).cumsum(0).tolist()]
    n = offsets[-1]
    outs = [torch.full((n + 2, kv_heads, dim), 7.0, dtype=ref.TYPES[dtype], device=DEV) for _ in range(2)]
    per = [torch.full((n + 2,), 7.0, device=DEV) for _ in range(2)]
    got = f.cache_read(dc, ragged(offsets, ids), starts=ints(starts), k_out=outs[0], v_out=outs[1], sizes_out=per[0], weights_out=per[1])
    assert got == (outs[0], outs[1]) and status(f) == 0
    for i, t in enumerate(ids):
        at = ref.places(c, t, torch.arange(starts[i], starts[i] + counts[i]))
        a, b = offsets[i], offsets[i + 1]
        for name, out in (("k", outs[0]), ("v", outs[1])):
            if four:
                want = pk.unpack(c[name][at[0], :, at[1]], c[name + "_scales"][at[0], :, at[1]])
                assert torch.equal(out[a:b].cpu().double(), want)
            else:
                assert equal_bits(out[a:b], c[name][at[0], :, at[1]])
        assert torch.equal(per[0][a:b].cpu(), c["sizes"][at]) and torch.equal(per[1][a:b].cpu(), c["weights"][at])
    assert all((t[n:] == 7).all() for t in (*outs, *per))
    same(dc, c)
    c["sizes"] = c["weights"] = None
    dc = (packed if four else plain)(dtype, c, kv_heads)
    k, v = f.cache_read(dc, ragged([0, 5]), sizes_out=per[0], weights_out=per[1])
    assert status(f) == 0 and equal_bits(k, outs[0][offsets[5]:n]) and equal_bits(v, outs[1][offsets[5]:n])
    assert (per[0][:5] == 1).all() and (per[1][:5] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [None, "halves", "adjacent"])
@pytest.mark.parametrize("moved", ["k", "v", "q", "stride"])
def test_rows_aligned_to_16_bytes_only(dtype, pairs, moved):
    """One of the row tensors, or their strides, 16 bytes off a multiple of 32."""
    kv, dim, heads, rows = 3, 96, 6, 41
    g = torch.Generator().manual_seed(30)
    c = pk.make([5, 0], kv, dim, 8, room=rows, seed=31)
    dc, f = packed(dtype, c, kv), runner.Fusion(2)
    off = 16 // torch.empty(0, dtype=ref.TYPES[dtype]).element_size()
    given, host = {}, {}
    for name, n in (("k", kv), ("v", kv), ("q", heads)):
        x = hard_rows(g, rows, n, dim, dtype) if name == "v" else torch.randn((rows, n, dim), generator=g).to(ref.TYPES[dtype])
        wide = torch.full((rows * (n * dim + 2 * off) + off,), math.nan, dtype=x.dtype, device=DEV)
        wide = wide[off * (moved == name):].as_strided((rows, n, dim), ((n * dim + off * (2 - (moved == "stride"))), dim, 1))
        assert wide.data_ptr() % 32 == 16 * (moved == name) and wide.data_ptr() % 16 == 0
        wide.copy_(x)
        given[name], host[name] = wide, x
    offsets, ids = [0, 30, rows], [1, 0]
    if pairs is None:
        f.cache_append(dc, given["k"], given["v"], ragged(offsets, ids))
        kt = host["k"].float()
    else:
        table = torch.randn((64, dim), generator=g)
        at = torch.cat([torch.arange(30), torch.arange(11) + 5])
        q = f.cache_append_rotated(dc, given["k"], given["v"], runner.Rotation(table.to(DEV), pairs), ragged(offsets, ids), q=given["q"])
        kt = pk.turn(host["k"].float(), table, at, pairs)
        assert equal_bits(q, pk.turn(host["q"].float(), table, at, pairs).to(ref.TYPES[dtype]))
    assert status(f) == 0
    new = pk.append(c, kt, host["v"].float(), offsets, ids)
    same(dc, c, new)
    # and back
    n = 46
    flat = [torch.full((n * kv * dim + 2 * off,), 7.0, dtype=ref.TYPES[dtype], device=DEV) for _ in range(2)]
    outs = [x[off * (moved == name):][:n * kv * dim].view(n, kv, dim) for x, name in zip(flat, "kv")]
    f.cache_read(dc, ragged([0, 30, n], ids), k_out=outs[0], v_out=outs[1])
    assert status(f) == 0
    for i, t in enumerate(ids):
        places = ref.places(c, t, torch.arange(int(new[t])))
        for name, out in zip("kv", outs):
            want = pk.unpack(c[name][places[0], :, places[1]], c[name + "_scales"][places[0], :, places[1]])
            got = out[[0, 30][i]:[30, n][i]].cpu().double()
            assert torch.equal(got[want.isfinite()], want[want.isfinite()]) and torch.isnan(got[~want.isfinite()]).all()
    for x, name in zip(flat, "kv"):
        assert (x[:off * (moved == name)] == 7).all() and (x[off * (moved == name) + n * kv * dim:] == 7).all()


@pytest.mark.parametrize("four", [False, True])
def test_read_leaves_bad_samples_out(four):
    cache_bit, offs, ids_bit = fz.FUSION_DEV_BAD_CACHE, fz.FUSION_DEV_BAD_OFFSETS, fz.FUSION_DEV_BAD_IDS
    for what, bit, good in (("past the end", cache_bit, [0, 2]), ("before the start", cache_bit, [0, 2]), ("page", cache_bit, [0, 2]),
                            ("length", cache_bit, [0, 2]), ("id", ids_bit, [0, 2]), ("decreasing", offs, [0, 2]), ("far start", cache_bit, [0, 2]),
                            ("batch", fz.FUSION_DEV_BAD_BATCH, []), ("count", 0, [0])):
        c = pk.make([9, 20, 6], 2, 32, 8, seed=13) if four else ref.make("bf16", [9, 20, 6], 2, 32, 8, seed=13)
        offsets, ids, starts, batch = [0, 4, 10, 16], [0, 1, 2], [0, 3, 0], None
        if what == "past the end":
            starts[1] = 15
        elif what == "before the start":
            starts[1] = -1
        elif what == "far start":
            starts[1] = 2 ** 31 - 1
        elif what == "page":
            c["table"][1, 0] = -1
        elif what == "length":
            c["lengths"][1] = 10 ** 6
        elif what == "id":
            ids[1] = 3
        elif what == "decreasing":
            offsets = [0, 4, 3, 9, 16]
            offsets = offsets[:4]
        elif what == "batch":
            batch = [4]
        elif what == "count":
            batch = [1]
        dc, f = (packed if four else plain)("bf16", c, 2), runner.Fusion(3)
        outs = [torch.full((16, 2, 32), math.inf, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        rows = runner.RaggedRows(3, 10, 16, ints(offsets), ints(batch), ints(ids))
        f.cache_read(dc, rows, starts=ints(starts), k_out=outs[0], v_out=outs[1])
        assert status(f) == bit, what
        wrote = torch.zeros(16, dtype=torch.bool)
        for i in good:
            wrote[offsets[i]:offsets[i + 1]] = True
        for out in outs:
            assert torch.isfinite(out[wrote.to(DEV)]).all() and torch.isinf(out[~wrote.to(DEV)]).all(), what


# ---- attention --------------------------------------------------------------------------------------------------------------
def attend(dtype, c, heads, *, q=None, seed=20, rounds=1, **kw):
    """Runs the attention `rounds` times and compares; returns (out, cache)."""
    batch, dim = len(c["lengths"]), c["k"].shape[3] * 2
    if q is None:
        q = (torch.randn((batch, heads, dim), generator=torch.Generator().manual_seed(seed)) * 2).to(ref.TYPES[dtype])
    dc, f = packed(dtype, c, heads), runner.Fusion(1)
    before = ref.copy(c)
    for _ in range(rounds):
        want, tol, w, wtol = pk.attention(c, q, dtype, **kw)
        out = f.cache_attention(dc, q.to(DEV), **kw)
        assert status(f) == 0
        off = (out.cpu().double() - want).abs()
        assert (off <= tol).all(), float((off / tol).max())
        if w is not None:
            got = dc.weights.cpu()
            known = ~torch.isnan(w)
            assert ((got.double() - w).abs() <= wtol + 1e-45)[known].all() and torch.isnan(got[~known]).all()
            c["weights"] = got
    for name in POOLS:
        assert torch.equal(getattr(dc, name).cpu(), before[name])
    assert int(dc.workspace[:1 << 18].max()) == 0
    return out, dc


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [
    (1, 1, 32, 1), (6, 6, 64, 16), (8, 2, 96, 8), (32, 4, 128, 16), (9, 1, 128, 64), (16, 1, 64, 4), (34, 2, 160, 32), (4, 4, 192, 2),
    (3, 1, 224, 128), (20, 2, 256, 16)])
def test_attention_shapes(dtype, heads, kv_heads, dim, page):
    c = pk.make([1, 0, 15, 16, 17, 129, 300, 64], kv_heads, dim, page, sizes="masked", weights=True, seed=14)
    attend(dtype, c, heads, rounds=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sizes,weights", [(None, False), (None, True), ("whole", False)])
def test_attention_optional_inputs(dtype, sizes, weights):
    attend(dtype, pk.make([70, 3, 200], 2, 64, 16, sizes=sizes, weights=weights, seed=15), 6, scale=0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (64, 4), (100, 0), (200, 13), (0, 5), (2 ** 31 - 1, 2 ** 31 - 1), (3, 500)])
def test_attention_window_and_sinks(dtype, window, sinks):
    attend(dtype, pk.make([1, 4, 63, 64, 65, 250, 0], 2, 128, 16, sizes="masked", weights=True, seed=16), 4, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim,n", [(32, 8, 128, [3000]), (8, 1, 64, [5001, 3]), (64, 1, 128, [9000]), (4, 4, 256, [1, 2500]), (5, 1, 32, [20011])])
def test_attention_split_over_many_ctas(dtype, heads, kv_heads, dim, n):
    """Runs that share a (sequence, key head), in one step and in two, twice with the same result."""
    c = pk.make(n, kv_heads, dim, 16, weights=True, seed=17)
    first, _ = attend(dtype, ref.copy(c), heads)
    second, _ = attend(dtype, c, heads)
    assert equal_bits(first, second)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(1, 1, 64, 16), (8, 2, 128, 16), (16, 1, 64, 8), (21, 1, 128, 4), (4, 4, 96, 32), (3, 1, 32, 128)])
def test_attention_short_sequences_a_warp_each(dtype, heads, kv_heads, dim, page):
    """Batches large enough, of sequences short enough, for warps that work alone."""
    g = torch.Generator().manual_seed(18)
    lengths = torch.randint(0, 129, (300,), generator=g).tolist()
    c = pk.make(lengths, kv_heads, dim, page, sizes="masked", weights=True, seed=18)
    assert c["table"].shape[1] * page <= 128
    attend(dtype, c, heads)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_peaked_and_rising_logits(dtype):
    """Logits that grow along the sequence by far more than a shift lags, that fall, that are equal, and one that takes all;
    keys of different magnitudes, whose groups have scales from the smallest to the largest."""
    for kind in ("rising", "falling", "equal", "one"):
        c = pk.make([600], 1, 64, 16, weights=True, seed=19)
        at = ref.places(c, 0, torch.arange(600))
        k = torch.randn((600, 1, 64), generator=torch.Generator().manual_seed(19)) * 0.1
        k[..., 0] += {"rising": torch.arange(600.0), "falling": 600 - torch.arange(600.0), "equal": torch.zeros(600),
                      "one": (torch.arange(600) == 331) * 500.0}[kind][:, None]
        k *= torch.tensor([1.0, 0.01, 0.0, 2.0 ** -8]).repeat_interleave(16)
        c["k"][at[0], :, at[1]], c["k_scales"][at[0], :, at[1]] = pk.pack(k)
        q = torch.randn((1, 3, 64), generator=torch.Generator().manual_seed(20))
        q[..., 0] = 3.0
        attend(dtype, c, 3, q=q.to(ref.TYPES[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [2.0 ** -120, 1e-30, 2.0 ** -20, 1.0, 2.0 ** 30, 1e30, 1e36])
def test_attention_queries_of_any_magnitude(dtype, size):
    """Large queries beside a scale that makes up for them, tiny ones, dims of one query far apart, a query of zeros."""
    c = pk.make([150, 7], 2, 96, 8, seed=21)
    q = torch.randn((2, 4, 96), generator=torch.Generator().manual_seed(21))
    q[0, 0, ::3] *= 2.0 ** -18
    q[0, 1] = 0.0
    q[1, 2, 5:] *= 2.0 ** -30
    attend(dtype, c, 4, q=(q.clamp(-3, 3) * size).to(ref.TYPES[dtype]), scale=min(0.2 / size, 2e38))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_all_masked(dtype):
    """Sequences of masked tokens alone, of any number of rounds, are zeros and leave the weights."""
    for lengths in ([40, 700, 3], [60] * 300):
        c = pk.make(lengths, 2, 64, 16, sizes="masked", weights=True, seed=22)
        for b in range(0, len(lengths), 2):
            at = ref.places(c, b, torch.arange(lengths[b]))
            c["sizes"][at] = 0.0
            for name in POOLS:
                c[name][at[0], :, at[1]] = pk.JUNK
        out, _ = attend(dtype, c, 4)
        assert (out[::2] == 0).all() and torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_nan_and_infinities_stay_where_they_are(dtype):
    """A NaN or infinite query spoils its head, a group that holds NaN in a value the group's dims of the key head's queries, in a key
    the key head; everything else is as it was."""
    c = pk.make([200, 90], 2, 64, 16, seed=23)
    q = torch.randn((2, 6, 64), generator=torch.Generator().manual_seed(23)).to(ref.TYPES[dtype])
    want, tol, _, _ = pk.attention(c, q, dtype)
    at = ref.places(c, 0, torch.arange(200))
    for what in ("nan query", "infinite query", "value", "key"):
        d, p = ref.copy(c), q.clone()
        spoilt = torch.zeros(want.shape, dtype=torch.bool)
        if "query" in what:
            p[0, 4, 3] = math.nan if "nan" in what else math.inf
            spoilt[0, 4] = True
        elif what == "value":
            d["v_scales"][at[0][7], 1, at[1][7], 2] = pk.NAN_SCALE
            spoilt[0, 3:, 32:48] = True
        else:
            d["k_scales"][at[0][7], 1, at[1][7], 0] = pk.NAN_SCALE
            spoilt[0, 3:] = True
        dc, f = packed(dtype, d, 6), runner.Fusion(1)
        out = f.cache_attention(dc, p.to(DEV)).cpu()
        assert status(f) == 0 and torch.isnan(out[spoilt]).all(), what
        assert ((out.double() - want).abs() <= tol)[~spoilt].all(), what


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [[600, 70, 300], [40] * 260])
def test_attention_bad_pages_and_lengths(dtype, lengths):
    """A page or a length out of range is told, and its sequence's row and weights are left; the others are as they would be."""
    for what in ("page", "length", "negative length"):
        c = pk.make(lengths, 2, 64, 16, room=16, weights=True, seed=24)
        q = torch.randn((len(lengths), 4, 64), generator=torch.Generator().manual_seed(24)).to(ref.TYPES[dtype])
        want, tol, w, wtol = pk.attention(c, q, dtype)
        old = c["weights"].clone()
        mine = ref.places(c, 0, torch.arange(lengths[0]))
        if what == "page":
            c["table"][0, (lengths[0] - 1) // 16] = c["k"].shape[0]
        else:
            c["lengths"][0] = c["table"].shape[1] * 16 + 1 if what == "length" else -1
        dc, f = packed(dtype, c, 4), runner.Fusion(1)
        out = torch.full((len(lengths), 4, 64), math.nan, dtype=ref.TYPES[dtype], device=DEV)
        f.cache_attention(dc, q.to(DEV), out=out)
        assert status(f) == fz.FUSION_DEV_BAD_CACHE and torch.isnan(out[0]).all()
        assert ((out[1:].cpu().double() - want[1:]).abs() <= tol[1:]).all()
        got = dc.weights.cpu()
        assert equal_bits(got[mine], old[mine])
        got[mine], w[mine], wtol[mine] = 0.0, 0.0, 1.0
        known = ~torch.isnan(w)
        assert ((got.double() - w).abs() <= wtol + 1e-45)[known].all()
        assert int(dc.workspace[:1 << 18].max()) == 0


def test_attention_and_reads_past_two_to_the_31():
    """Rows whose bytes lie past 2^31 and 2^32 in the pools of codes, and their scales."""
    dim, page, pages = 256, 64, 600000   # 38.4 M rows of 128 bytes, of 16 bytes of scales
    g = torch.Generator(device=DEV).manual_seed(25)
    pools = [torch.zeros((pages, 1, page, n), dtype=torch.uint8, device=DEV) for n in (128, 128, 16, 16)]
    table = torch.tensor([[599999, 3, 262150], [131080, 524300, 262143]], dtype=torch.int32)
    c = dict(table=table, lengths=torch.tensor([170, 192], dtype=torch.int32), sizes=None, weights=None)
    used = table.flatten().long().to(DEV)
    for p in pools:
        p[used] = torch.randint(0, 256 if p.shape[3] == 128 else 0x50, p[used].shape, generator=g, device=DEV, dtype=torch.int32).to(torch.uint8)
    dc = runner.packed_cache_of("bf16", *pools, table.to(DEV), c["lengths"].to(DEV), heads=4)
    f = runner.Fusion(2)
    q = (torch.randn((2, 4, dim), generator=torch.Generator().manual_seed(25)) * 1e-3).to(torch.bfloat16)
    small = {n: p[used].cpu() for n, p in zip(("k", "v", "k_scales", "v_scales"), pools)}
    host = dict(c, **small, table=torch.arange(6, dtype=torch.int32).view(2, 3))
    want, tol, _, _ = pk.attention(host, q, "bf16")
    out = f.cache_attention(dc, q.to(DEV))
    assert status(f) == 0 and ((out.cpu().double() - want).abs() <= tol).all()
    k, v = f.cache_read(dc, ragged([0, 170, 362]))
    assert status(f) == 0
    for b, (a, e) in enumerate(((0, 170), (170, 362))):
        at = ref.places(host, b, torch.arange(e - a))
        for name, got in (("k", k), ("v", v)):
            assert torch.equal(got[a:e].cpu().double(), pk.unpack(host[name][at[0], :, at[1]], host[name + "_scales"][at[0], :, at[1]]))
    dc.lengths.copy_(ints([100, 100]))
    x = torch.randn((92 + 60, 1, dim), generator=torch.Generator().manual_seed(26)).to(torch.bfloat16)
    f.cache_append(dc, x.to(DEV), x.to(DEV), ragged([0, 60, 152]))
    host["lengths"] = torch.tensor([100, 100], dtype=torch.int32)
    new = pk.append(host, x.float(), x.float(), [0, 60, 152])
    assert status(f) == 0 and torch.equal(dc.lengths.cpu(), new)
    for name, p in zip(("k", "v", "k_scales", "v_scales"), pools):
        assert torch.equal(p[used].cpu(), host[name]), name


# ---- eviction -----------------------------------------------------------------------------------------------------------------
EVICTIONS = [(1, 32, 1), (3, 64, 16), (2, 96, 8), (8, 128, 64), (5, 256, 4), (40, 160, 2)]
LENGTHS = [[0, 1, 9, 40, 130, 77], [17] * 140, [3000, 100]]


@pytest.mark.parametrize("outside", [False, True])
@pytest.mark.parametrize("kv_heads,dim,page,lengths", [(*e, n) for n in LENGTHS for e in EVICTIONS if n[0] < 1000 or e[2] >= 4])
def test_evict(kv_heads, dim, page, outside, lengths):
    c = pk.make(lengths, kv_heads, dim, page, sizes="whole", weights=True, spare=1 if not outside else sum(-(-n // page) + 1 for n in lengths), seed=27)
    budgets = [max(0, n // 2 + (i % 3) * 7 - 5) for i, n in enumerate(lengths)]
    dc, f = packed("bf16", c, kv_heads), runner.Fusion(1)
    table_out = None
    if outside:
        used = set(c["table"].flatten().tolist())
        free = [p for p in range(c["k"].shape[0]) if p not in used]
        per = max(1, max(-(-min(b, n) // page) for b, n in zip(budgets, lengths)))
        while len(free) < per * len(lengths):   # more pages than there are: grow the pools
            free.append(c["k"].shape[0])
            for name in (*POOLS, "sizes", "weights"):
                c[name] = torch.cat([c[name], c[name][:1]])
        dc = packed("bf16", c, kv_heads)
        table_out = torch.tensor(free[:per * len(lengths)], dtype=torch.int32).view(len(lengths), per)
    keep = torch.full((len(lengths), max(lengths)), -9, dtype=torch.int32, device=DEV)
    out = torch.full((len(lengths),), -7, dtype=torch.int32, device=DEV)
    f.cache_evict(dc, ints(budgets), sinks=2, recent=5, page_table_out=None if table_out is None else table_out.to(DEV), lengths_out=out,
                  keep_idx=keep)
    assert status(f) == 0
    new, keeps = pk.evict(c, budgets, sinks=2, recent=5, table_out=table_out)
    assert torch.equal(out.cpu(), new)
    for b, kept in enumerate(keeps):
        assert keep[b, :len(kept)].tolist() == kept and (keep[b, len(kept):] == -9).all()
    same(dc, c)


# ---- together -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_decoder_over_a_packed_cache(dtype):
    """A compacted prefix with its own positions, rotated on its way; steps of a rotated token with attention, replayed as a graph;
    an eviction, after which positions and places part; the rows read back at last."""
    heads, kv, dim, batch = 8, 2, 64, 5
    g = torch.Generator().manual_seed(28)
    counts = [30, 1, 77, 50, 12]
    offsets, ids = [0, *torch.tensor(counts).cumsum(0).tolist()], [4, 2, 0, 1, 3]
    rows = offsets[-1]
    dc = runner.device_packed_cache(dtype, batch, 160, heads, kv, dim, sizes=True, weights=True)
    f = runner.Fusion(batch)
    table = runner.rotation_table(2000, dim, device=DEV)
    rot, host = runner.Rotation(table, "adjacent"), table.cpu()
    t = ref.TYPES[dtype]
    k, v = (torch.randn((rows, kv, dim), generator=g).to(t) for _ in range(2))
    pos = torch.randint(0, 900, (rows,), generator=g).sort().values
    sizes, scores = torch.randint(1, 4, (rows,), generator=g).float(), torch.rand(rows, generator=g)
    f.cache_append_rotated(dc, k.to(DEV), v.to(DEV), rot, ragged(offsets, ids), positions=ints(pos.tolist()), sizes=sizes.to(DEV),
                           scores=scores.to(DEV))
    c = {name: torch.zeros_like(getattr(dc, name)).cpu() for name in (*POOLS, "sizes", "weights")}
    c.update(table=dc.page_table.cpu(), lengths=torch.zeros(batch, dtype=torch.int32))
    c["lengths"] = pk.append(c, pk.turn(k.float(), host, pos, "adjacent"), v.float(), offsets, ids, sizes, scores)
    same(dc, c)
    step = torch.empty((batch, (heads + 2 * kv) * dim), dtype=t, device=DEV)
    at = torch.empty(batch, dtype=torch.int32, device=DEV)
    q_out, out = (torch.empty((batch, heads, dim), dtype=t, device=DEV) for _ in range(2))
    cut = [heads * dim, (heads + kv) * dim]

    def one_step():
        f.cache_append_rotated(dc, step[:, cut[0]:cut[1]], step[:, cut[1]:], rot, positions=at, q=step[:, :cut[0]].unflatten(1, (heads, dim)),
                               q_out=q_out)
        f.cache_attention(dc, q_out, window=90, sinks=4, out=out)

    graph = None
    for i in range(8):
        step.copy_(torch.randn(step.shape, generator=g))
        at.copy_(torch.arange(batch) * 3 + 900 + i)
        if i == 2:
            held = dc.lengths.clone()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                one_step()
            assert torch.equal(held, dc.lengths)
        graph.replay() if graph else one_step()
        hs, ha = step.cpu().float(), at.cpu().long()
        kt = pk.turn(hs[:, cut[0]:cut[1]].reshape(batch, kv, dim), host, ha, "adjacent")
        c["lengths"] = pk.append(c, kt, hs[:, cut[1]:].reshape(batch, kv, dim), range(batch + 1))
        qt = pk.turn(hs[:, :cut[0]].reshape(batch, heads, dim), host, ha, "adjacent").to(t)
        assert equal_bits(q_out, qt)
        want, tol, wt, wtol = pk.attention(c, qt, dtype, window=90, sinks=4)
        assert ((out.cpu().double() - want).abs() <= tol).all()
        got = dc.weights.cpu()
        assert ((got.double() - wt).abs() <= wtol + 1e-45).all()
        c["weights"] = got    # the device's own from here: the eviction compares them
        same(dc, c)
        if i == 4:
            f.cache_evict(dc, torch.full((batch,), 20, dtype=torch.int32, device=DEV), sinks=1, recent=4)
            c["lengths"], _ = pk.evict(c, [20] * batch, sinks=1, recent=4)
            same(dc, c)
    n = c["lengths"].tolist()
    offsets = [0, *torch.tensor(n).cumsum(0).tolist()]
    kr, vr = f.cache_read(dc, ragged(offsets))
    assert status(f) == 0
    for b in range(batch):
        where = ref.places(c, b, torch.arange(n[b]))
        for name, got in (("k", kr), ("v", vr)):
            want = pk.unpack(c[name][where[0], :, where[1]], c[name + "_scales"][where[0], :, where[1]])
            assert torch.equal(got[offsets[b]:offsets[b + 1]].cpu().double(), want)


def test_two_streams_at_once():
    """Calls on two caches from two streams that overlap, replayed many times, and the same one after the other."""
    def work(seed):
        c = pk.make([700, 3000, 20, 5], 2, 128, 16, room=64, weights=True, seed=seed)
        q = torch.randn((4, 8, 128), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)
        return packed("bf16", c, 8), runner.Fusion(4), q.to(DEV), runner.Rotation(runner.rotation_table(4000, 128, device=DEV))

    def steps(dc, f, q, rot):
        outs = []
        for _ in range(12):
            turned = f.cache_append_rotated(dc, q[:, :2], q[:, 2:4], rot, q=q)
            outs.append(f.cache_attention(dc, turned))
        return outs

    alone = [steps(*work(s)) for s in (30, 31)]
    torch.cuda.synchronize()
    both, streams = [work(s) for s in (30, 31)], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = []
    for w, s in zip(both, streams):
        with torch.cuda.stream(s):
            outs.append(steps(*w))
    torch.cuda.synchronize()
    for got, want, w in zip(outs, alone, both):
        assert all(equal_bits(a, b) for a, b in zip(got, want)) and int(w[1].status.item()) == 0


def test_the_largest_batch():
    """FUSION_CACHE_MAX_BATCH sequences: a row each in place and with the lengths elsewhere, attention, a read, an eviction."""
    batch = fz.FUSION_CACHE_MAX_BATCH
    g = torch.Generator(device=DEV).manual_seed(32)
    dc, f = runner.device_packed_cache("bf16", batch, 2, 1, 1, 32, page_tokens=1, weights=True), runner.Fusion(1)
    k, v = (torch.randint(-3, 4, (batch, 1, 32), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    k[:, :, ::16], v[:, :, ::16] = 6.0, 6.0   # whole numbers up to 3 are codes beside 6
    rot = runner.Rotation(torch.tensor([[1.0] * 16 + [0.0] * 16] * 2, device=DEV))
    out = torch.full((batch,), -7, dtype=torch.int32, device=DEV)
    f.cache_append_rotated(dc, k, v, rot, lengths_out=out)
    assert status(f) == 0 and (out == 1).all() and (dc.lengths == 0).all()
    f.cache_append_rotated(dc, k, v, rot)
    assert (dc.lengths == 1).all()
    got = f.cache_attention(dc, k)
    assert status(f) == 0 and torch.equal(got, v) and (dc.weights[::2, 0] == 1).all()
    rows = runner.RaggedRows(batch, 1, batch, torch.arange(batch + 1, dtype=torch.int32, device=DEV))
    kr, vr = f.cache_read(dc, rows)
    assert torch.equal(kr, k) and torch.equal(vr, v)
    f.cache_evict(dc, (torch.arange(batch, device=DEV) % 2).to(torch.int32))
    assert status(f) == 0 and torch.equal(dc.lengths, (torch.arange(batch, device=DEV) % 2).to(torch.int32))
    assert int(dc.workspace[:1 << 18].max()) == 0


def test_empty_calls():
    """Caches of no sequences, batches of no samples and samples of no rows."""
    for four in (False, True):
        new = runner.device_packed_cache if four else runner.device_cache
        f = runner.Fusion(3)
        rot = runner.Rotation(runner.rotation_table(8, 32, device=DEV))
        none = torch.zeros((0, 2, 32), dtype=torch.bfloat16, device=DEV)
        dc = new("bf16", 0, 8, 2, 2, 32, weights=True)
        assert f.cache_append_rotated(dc, none, none, rot, q=none).shape == (0, 2, 32)
        assert f.cache_append(dc, none, none).shape == (0,) and f.cache_attention(dc, none).shape == (0, 2, 32)
        dc = new("bf16", 3, 8, 2, 2, 32, weights=True)
        out = torch.full((3,), -7, dtype=torch.int32, device=DEV)
        for offsets in ([0], [0, 0, 0]):
            rows = runner.RaggedRows(len(offsets) - 1, 1, 0, ints(offsets))
            out.fill_(-7)
            assert f.cache_append_rotated(dc, none, none, rot, rows, q=none, lengths_out=out).shape == (0, 2, 32)
            assert out.tolist() == [0, 0, 0]
            k, v = f.cache_read(dc, rows)
            assert k.shape == v.shape == (0, 2, 32)
        f.cache_evict(dc, ints([1, 2, 3]))
        assert (f.cache_attention(dc, torch.ones((3, 2, 32), dtype=torch.bfloat16, device=DEV)) == 0).all() and status(f) == 0
