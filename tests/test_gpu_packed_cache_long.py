"""Rotated and packed appends whose CTAs take several rows: queries rotated in place, and more rows than the CTAs of a sample take at
once, on the GPU against the definitions on the host (packed_reference.py) and against shorter calls, bit by bit."""
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


def status(f):
    torch.cuda.synchronize()
    return int(f.status.item())


def ragged(offsets, longest):
    return runner.RaggedRows(len(offsets) - 1, longest, offsets[-1], torch.tensor(offsets, dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("pairs", ["halves", "adjacent"])
@pytest.mark.parametrize("dim,turned,longest", [(64, 64, 1000), (96, 32, 800), (256, 128, 300)])
def test_queries_in_place(dtype, four, pairs, dim, turned, longest):
    """q_out is q, in 200 samples of 0 to `longest` rows, of which a thread has up to 2 to 4 one after another: it asks for rows
    ahead and writes the ones before them to the same tensor."""
    kv, heads, batch = 2, 3, 200
    g = torch.Generator().manual_seed(dim + turned)
    counts = torch.randint(2, longest, (batch,), generator=g).tolist()
    counts[3], counts[50], counts[51], counts[199] = longest, 0, 1, longest
    offsets = [0, *torch.tensor(counts).cumsum(0).tolist()]
    n = offsets[-1]
    t = ref.TYPES[dtype]
    dc, f = (runner.device_packed_cache if four else runner.device_cache)(dtype, batch, longest, kv, kv, dim), runner.Fusion(1)
    k, v = (torch.randn((n, kv, dim), generator=g).to(t) for _ in range(2))
    q = torch.randn((n, heads, dim), generator=g).to(t)
    table, pos = torch.randn((700, turned), generator=g), torch.randint(0, 700, (n,), generator=g)
    dq = q.to(DEV)
    got = f.cache_append_rotated(dc, k.to(DEV), v.to(DEV), runner.Rotation(table.to(DEV), pairs), ragged(offsets, longest),
                                 positions=pos.to(torch.int32).to(DEV), q=dq, q_out=dq)
    assert got is dq and status(f) == 0
    assert torch.equal(ref.bits(dq.cpu()), ref.bits(pk.turn(q.float(), table, pos, pairs).to(t)))
    assert dc.lengths.tolist() == counts and int(dc.workspace[:1 << 18].max()) == 0
    kt = pk.turn(k.float(), table, pos, pairs)
    sample = torch.repeat_interleave(torch.arange(batch), torch.tensor(counts))
    place = torch.arange(n) - torch.tensor(offsets)[sample]
    page, off = dc.page_table.cpu()[sample, place // dc.page_tokens].long(), place % dc.page_tokens
    for name, rows in (("k", kt), ("v", v.float())):
        held = getattr(dc, name).cpu()[page, :, off]
        if four:
            codes, scales = pk.pack(rows)
            assert torch.equal(held, codes) and torch.equal(getattr(dc, name + "_scales").cpu()[page, :, off], scales)
        else:
            assert torch.equal(ref.bits(held), ref.bits(rows.to(t)))


# 12 key heads of 256 dims: rows that a CTA has side by side, whose 24 units a row are all that it takes
@pytest.mark.parametrize("dtype,four,turned,side", [("f32", False, 256, 8), ("bf16", False, 128, 16), ("f32", True, 256, 16), ("bf16", True, 256, 32),
                                                    ("f32", True, 0, 16), ("bf16", True, 0, 32)])
def test_more_rows_than_the_ctas_of_a_sample_take_at_once(dtype, four, turned, side):
    """One sample of 2500 times as many rows as a CTA has at once, of which 2432 CTAs take some in a second turn, against the same rows in
    calls that need no such turn.  Then positions that the table does not have, in one CTA and in most of them."""
    kv, dim, n = 12, 256, 2500 * side
    g = torch.Generator(device=DEV).manual_seed(side)
    new = runner.device_packed_cache if four else runner.device_cache
    (dc, parts), f = (new(dtype, 1, n, kv, kv, dim, page_tokens=1024) for _ in range(2)), runner.Fusion(1)
    k, v = (torch.randn((n, kv, dim), generator=g, device=DEV, dtype=ref.TYPES[dtype]) for _ in range(2))
    rot = runner.Rotation(torch.randn((700, turned), generator=g, device=DEV)) if turned else None
    pos = torch.randint(0, 700, (n,), generator=g, device=DEV, dtype=torch.int32)

    def append(c, a, b, at=pos):
        if rot is None:
            f.cache_append(c, k[a:b], v[a:b], ragged([0, b - a], b - a))
        else:
            f.cache_append_rotated(c, k[a:b], v[a:b], rot, ragged([0, b - a], b - a), positions=at[a:b])

    append(dc, 0, n)
    step = 900 * side + 7
    for a in range(0, n, step):
        append(parts, a, min(n, a + step))
    assert status(f) == 0 and dc.lengths.tolist() == parts.lengths.tolist() == [n]
    pools = ("k", "v", "k_scales", "v_scales") if four else ("k", "v")

    def same():
        return all(torch.equal(getattr(dc, name).view(torch.uint8), getattr(parts, name).view(torch.uint8)) for name in pools)

    assert same() and int(dc.workspace[:1 << 18].max()) == 0
    if rot is None:
        return
    for bad in ([n - 1], range(3, n, 11), [0]):
        wrong = pos.clone()
        wrong[torch.tensor(bad, device=DEV)] = 700
        f = runner.Fusion(1)
        dc.lengths.zero_()
        for name in pools:
            getattr(dc, name).zero_()
        append(dc, 0, n, wrong)
        assert status(f) == fz.FUSION_DEV_BAD_POSITION and dc.lengths.tolist() == [0] and int(dc.workspace[:1 << 18].max()) == 0
    f = runner.Fusion(1)
    append(dc, 0, n)
    assert status(f) == 0 and dc.lengths.tolist() == [n] and same()
