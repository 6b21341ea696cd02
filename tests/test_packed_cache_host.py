"""The cache in 4 bits, rotated appends and reads on the host: what the calls refuse before anything is enqueued, the runner's
checks, and the reference that the GPU tests compare with, against itself (no GPU needed)."""
import inspect
import math
import os
import re
import sys
import types

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import packed_reference as pk  # noqa: E402
import paper_2607_02612_gb300 as fz  # noqa: E402
from paper_2607_02612_gb300 import _binding as fb, runner  # noqa: E402

FAKE = 0x100000   # never dereferenced: every call below fails a host check first
SHAPE = dict(max_batch=4, max_pages=10, page_tokens=16, kv_heads=2, head_dim=64, num_pages=40, k=FAKE, v=FAKE, sizes=None,
             weights=FAKE, page_table=FAKE, lengths=FAKE)
CSRC = os.path.join(os.path.dirname(fz.__file__), "csrc")


@pytest.fixture(scope="module", autouse=True)
def lib():
    fz.build()


def cache(**kw):
    return fz.cache(**{**SHAPE, **kw})


def four(k_scales=FAKE, v_scales=FAKE, **kw):
    return fz.packed_cache(cache(**kw), k_scales, v_scales)


def turns(table=FAKE, table_rows=100, dims=64, pairs=fz.FUSION_PAIRS_HALVES, positions=None):
    return fz.rotation(table, table_rows, dims, pairs, positions)


WS = 1 << 26
ROWS = dict(dtype=fz.FUSION_BF16, cache=None, in_=None, k=FAKE, k_stride=128, v=FAKE, v_stride=128, sizes=None, scores=None)
END = dict(lengths_out=FAKE, workspace=FAKE, workspace_bytes=WS, dev_status=FAKE, stream=0)
TURN = dict(rotation=None, q=FAKE, q_stride=512, heads=8, q_out=FAKE)
ATTEND = dict(dtype=fz.FUSION_BF16, cache=None, q=FAKE, q_stride=512, heads=8, scale=0.125, window=0, sinks=0, out=FAKE,
              workspace=FAKE, workspace_bytes=WS, dev_status=FAKE, stream=0)
EVICT = dict(cache=None, budget=FAKE, sinks=1, recent=2, page_table_out=None, max_pages_out=0, lengths_out=FAKE, keep_idx=None,
             keep_stride=0, workspace=FAKE, workspace_bytes=WS, dev_status=FAKE, stream=0)
READ = dict(dtype=fz.FUSION_BF16, cache=None, in_=None, starts=None, k_out=FAKE, v_out=FAKE, sizes_out=None, weights_out=None,
            dev_status=FAKE, stream=0)
CALLS = {"fusion_cache_append_rotated": {**ROWS, **TURN, **END}, "fusion_cache_read": READ, "fusion_packed_append": {**ROWS, **END},
         "fusion_packed_append_rotated": {**ROWS, **TURN, **END}, "fusion_packed_attention": ATTEND, "fusion_packed_evict": EVICT,
         "fusion_packed_read": READ}
PACKED = [n for n in CALLS if "packed" in n]
ROTATED = [n for n in CALLS if "rotated" in n]
APPENDS = [n for n in CALLS if "append" in n]
READS = [n for n in CALLS if "read" in n]


def call(name, **kw):
    a = dict(CALLS[name])
    if "in_" in a:
        a["in_"] = fz.ragged(4, 5000, 20000, FAKE)
    if "rotation" in a:
        a["rotation"] = turns()
    a["cache"] = four() if name in PACKED else cache()
    a.update(kw)
    return getattr(fz, name)(*a.values())


def with_cache(name, **kw):
    return call(name, cache=four(**kw) if name in PACKED else cache(**kw))


@pytest.mark.parametrize("name", CALLS)
def test_argument_lists(name):
    """The binding's functions take what the tests pass, in this order."""
    assert list(inspect.signature(getattr(fz, name)).parameters) == list(CALLS[name])


BAD_SHAPES = [dict(max_batch=-1), dict(max_batch=fz.FUSION_CACHE_MAX_BATCH + 1), dict(page_tokens=0), dict(page_tokens=24),
              dict(page_tokens=2 * fz.FUSION_CACHE_MAX_PAGE_TOKENS), dict(kv_heads=0), dict(head_dim=4), dict(head_dim=12),
              dict(head_dim=fz.FUSION_CACHE_MAX_HEAD_DIM + 32), dict(max_pages=0), dict(max_pages=(1 << 26) + 1), dict(num_pages=0),
              dict(num_pages=1 << 27), dict(num_pages=1 << 40)]


@pytest.mark.parametrize("name", CALLS)
def test_bad_caches_are_refused(name):
    for kw in BAD_SHAPES + ([dict(head_dim=d) for d in (8, 16, 48, 80, 144)] if name in PACKED else []):
        assert with_cache(name, **kw) == fz.FUSION_ERR_SHAPE, kw
    for kw in (dict(k=None), dict(v=None), dict(page_table=None), dict(lengths=None), dict(k=FAKE + 8), dict(v=FAKE + 2)):
        assert with_cache(name, **kw) == fz.FUSION_ERR_INVALID_ARG, kw
    if name in PACKED:
        for kw in (dict(k_scales=None), dict(v_scales=None), dict(k_scales=FAKE + 8), dict(v_scales=FAKE + 4)):
            assert with_cache(name, **kw) == fz.FUSION_ERR_INVALID_ARG, kw
    for off in (1, 2, 3, 6):
        for what in ("sizes", "weights", "page_table", "lengths"):
            assert with_cache(name, **{what: FAKE + off}) == fz.FUSION_ERR_INVALID_ARG, (what, off)
        assert call(name, dev_status=FAKE + off) == fz.FUSION_ERR_INVALID_ARG
    if "dtype" in CALLS[name]:
        assert call(name, dtype=2) == fz.FUSION_ERR_DTYPE
    if "workspace" in CALLS[name]:
        for kw in (dict(workspace=None), dict(workspace=FAKE + 8), dict(workspace_bytes=1000)):
            assert call(name, **kw) == fz.FUSION_ERR_WORKSPACE, kw


@pytest.mark.parametrize("name", APPENDS)
def test_appends_reject_bad_rows(name):
    for in_ in (fz.ragged(5, 10, 100, FAKE), fz.ragged(-1, 10, 100, FAKE), fz.ragged(4, 0, 100, FAKE), fz.ragged(4, 10, -1, FAKE),
                fz.ragged(4, 10, 1 << 31, FAKE)):
        assert call(name, in_=in_) == fz.FUSION_ERR_SHAPE
    for kw in (dict(k=None), dict(v=None), dict(lengths_out=None), dict(k=FAKE + 4), dict(v=FAKE + 8), dict(k_stride=-128),
               dict(v_stride=132), dict(in_=fz.ragged(4, 10, 100, None)), dict(sizes=FAKE + 2), dict(scores=FAKE + 1),
               dict(lengths_out=FAKE + 3), dict(in_=fz.ragged(4, 10, 100, FAKE + 2)), dict(in_=fz.ragged(4, 10, 100, FAKE, FAKE + 2)),
               dict(in_=fz.ragged(4, 10, 100, FAKE, None, FAKE + 2))):
        assert call(name, **kw) == fz.FUSION_ERR_INVALID_ARG, kw
    assert call(name, dtype=fz.FUSION_F32, k_stride=130) == fz.FUSION_ERR_INVALID_ARG


@pytest.mark.parametrize("name", ROTATED)
def test_rotations_are_checked(name):
    for kw in (dict(table_rows=0), dict(table_rows=-5), dict(dims=0), dict(dims=8), dict(dims=24), dict(dims=96), dict(dims=-32),
               *([dict(dims=16), dict(dims=48)] if name in PACKED else [])):
        assert call(name, rotation=turns(**kw)) == fz.FUSION_ERR_SHAPE, kw
    for kw in (dict(table=None), dict(table=FAKE + 8), dict(pairs=2), dict(pairs=-1), dict(positions=FAKE + 2)):
        assert call(name, rotation=turns(**kw)) == fz.FUSION_ERR_INVALID_ARG, kw
    for heads in (0, -1, fz.FUSION_CACHE_MAX_HEADS + 1):
        assert call(name, heads=heads) == fz.FUSION_ERR_SHAPE
    for kw in (dict(q_out=None), dict(q=FAKE + 8), dict(q_out=FAKE + 4), dict(q_stride=-512), dict(q_stride=516), dict(q_out=FAKE, q_stride=1024)):
        assert call(name, **kw) == fz.FUSION_ERR_INVALID_ARG, kw


def test_packed_attention_rejects_bad_arguments():
    for heads in (0, 1, 9, -2, fz.FUSION_CACHE_MAX_HEADS + 2):
        assert call("fusion_packed_attention", heads=heads) == fz.FUSION_ERR_SHAPE, heads
    for kw in (dict(q=None), dict(out=None), dict(q=FAKE + 2), dict(out=FAKE + 8), dict(q_stride=-8), dict(q_stride=516),
               dict(scale=math.nan), dict(scale=math.inf), dict(scale=2.4e38), dict(window=-1), dict(sinks=-1)):
        assert call("fusion_packed_attention", **kw) == fz.FUSION_ERR_INVALID_ARG, kw
    need = fz.fusion_packed_workspace_size(four(), 8)
    assert call("fusion_packed_attention", workspace_bytes=need - 1) == fz.FUSION_ERR_WORKSPACE


def test_packed_eviction_rejects_bad_arguments():
    assert with_cache("fusion_packed_evict", weights=None) == fz.FUSION_ERR_INVALID_ARG
    for kw in (dict(budget=None), dict(lengths_out=None), dict(sinks=-1), dict(recent=-1), dict(keep_idx=FAKE, keep_stride=0),
               dict(budget=FAKE + 2), dict(keep_idx=FAKE + 1, keep_stride=3), dict(page_table_out=FAKE + 2, max_pages_out=2)):
        assert call("fusion_packed_evict", **kw) == fz.FUSION_ERR_INVALID_ARG, kw
    assert call("fusion_packed_evict", page_table_out=FAKE + 64, max_pages_out=0) == fz.FUSION_ERR_SHAPE


@pytest.mark.parametrize("name", READS)
def test_reads_reject_bad_arguments(name):
    for in_ in (fz.ragged(fz.FUSION_CACHE_MAX_BATCH + 1, 10, 100, FAKE), fz.ragged(-1, 10, 100, FAKE), fz.ragged(4, 0, 100, FAKE),
                fz.ragged(4, 10, -1, FAKE), fz.ragged(4, 10, 1 << 31, FAKE)):
        assert call(name, in_=in_) == fz.FUSION_ERR_SHAPE
    for kw in (dict(in_=fz.ragged(4, 10, 100, None)), dict(k_out=FAKE + 8), dict(v_out=FAKE + 4), dict(starts=FAKE + 2), dict(sizes_out=FAKE + 1),
               dict(weights_out=FAKE + 3), dict(in_=fz.ragged(4, 10, 100, FAKE, None, FAKE + 2))):
        assert call(name, **kw) == fz.FUSION_ERR_INVALID_ARG, kw


def test_workspace_and_constants():
    assert fz.fusion_packed_workspace_size(four(), 8) == fz.fusion_cache_workspace_size(cache(), 8) > 0
    for kw in (*BAD_SHAPES, dict(head_dim=80)):
        assert fz.fusion_packed_workspace_size(four(**kw), 8) == 0
    assert fz.fusion_packed_workspace_size(four(), 9) == 0
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "fusion.h")).read()
    for name in ("FUSION_DEV_BAD_POSITION", "FUSION_PAIRS_HALVES", "FUSION_PAIRS_ADJACENT"):
        assert f"#define {name} {getattr(fz, name)} " in text
    assert "position" in fz.fusion_status_string(fz.FUSION_DEV_BAD_POSITION)
    assert "#define FUSION_PACKED_SCALE_BYTES(head_dim) (((head_dim) / 16 + 3) / 4 * 4)" in text
    assert [fz.packed_scale_bytes(d) for d in (32, 64, 96, 128, 160, 192, 224, 256)] == [4, 4, 8, 8, 12, 12, 16, 16]
    # (names with digits, which the list of exported symbols is compared without)
    assert set(re.findall(r"\b(fusion_\w+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S))) == set(fb.EXPORTED)


# ---- the runner ------------------------------------------------------------------------------------------------------
def stub_cache(**kw):
    """What Fusion's calls look at in a cache, on the host."""
    return types.SimpleNamespace(**{**dict(max_batch=3, kv_heads=2, head_dim=64, heads=4, index=-1, torch_dtype=torch.float32, device="cpu",
                                           lengths=torch.zeros(3, dtype=torch.int32), code=0, _ws=0, ws_bytes=0, c_struct=lambda: None), **kw})


def stub_rows(n=3, **kw):
    return types.SimpleNamespace(**{**dict(max_batch=3, max_tokens=n, max_rows=n, offsets=torch.zeros(4, dtype=torch.int32), batch=None,
                                           ids=None, ragged=lambda: None), **kw})


def test_runner_checks_rotated_appends(monkeypatch):
    seen = []
    monkeypatch.setattr(runner, "_enqueue", lambda call, device, status, *args: seen.append(args))
    f, c = types.SimpleNamespace(status=None), stub_cache(lib=types.SimpleNamespace(fusion_cache_append_rotated=None))
    rot = types.SimpleNamespace(table=torch.zeros(9, 64), c_struct=lambda p: ("rotation", p))
    k, q = torch.zeros(3, 2, 64), torch.zeros(3, 7, 64)
    go = lambda **kw: runner.Fusion.cache_append_rotated(f, c, k, k, rot, **{**dict(rows=stub_rows()), **kw})   # noqa: E731
    assert go() is None and seen[-1][10:14] == (None, 0, 0, None)
    pos = torch.zeros(3, dtype=torch.int32)
    out = go(q=q, positions=pos)
    assert out.shape == q.shape and seen[-1][9] == ("rotation", pos.data_ptr())
    assert seen[-1][10:14] == (q.data_ptr(), 7 * 64, 7, out.data_ptr())
    wide = torch.zeros(3, 9, 64)
    assert go(q=wide[:, 1:8], q_out=q) is q and seen[-1][10:14] == (wide.data_ptr() + 256, 9 * 64, 7, q.data_ptr())
    n = len(seen)
    for kw in (dict(q=q[:2]), dict(q=q.bfloat16()), dict(q=q[..., :32]), dict(q=q.flatten(1)), dict(q=q, q_out=q[:2]), dict(q=q, q_out=q[:, :6]),
               dict(q=q, q_out=q.bfloat16()), dict(q=q, q_out=q.flatten(1)), dict(q_out=q), dict(positions=pos[:2]), dict(positions=pos.long()),
               dict(lengths_out=pos[:2]), dict(sizes=torch.zeros(2)), dict(scores=torch.zeros(3, dtype=torch.float64)),
               dict(q=torch.zeros(3, 64, 7).transpose(1, 2))):
        with pytest.raises(fz.FusionError):
            go(**kw)
    with pytest.raises(fz.FusionError):
        runner.Fusion.cache_append_rotated(f, c, k[:2], k, rot, stub_rows())
    elsewhere = types.SimpleNamespace(get_device=lambda: 0)
    with pytest.raises(fz.FusionError):
        runner.Fusion.cache_append_rotated(f, c, k, k, types.SimpleNamespace(table=elsewhere), stub_rows())
    for where in ("offsets", "batch", "ids"):
        with pytest.raises(fz.FusionError):
            go(rows=stub_rows(**{where: elsewhere}))
    assert len(seen) == n


def test_runner_checks_reads(monkeypatch):
    seen = []
    monkeypatch.setattr(runner, "_enqueue", lambda call, device, status, *args: seen.append(args))
    f, c = types.SimpleNamespace(status=None), stub_cache(lib=types.SimpleNamespace(fusion_cache_read=None))
    k, v = runner.Fusion.cache_read(f, c, stub_rows(5))
    assert k.shape == v.shape == (5, 2, 64) and seen[-1][3:] == (None, k.data_ptr(), v.data_ptr(), None, None)
    starts, per = torch.zeros(3, dtype=torch.int32), torch.zeros(5)
    runner.Fusion.cache_read(f, c, stub_rows(5), starts=starts, k_out=v, v_out=k, sizes_out=per, weights_out=per)
    assert seen[-1][3:] == (starts.data_ptr(), v.data_ptr(), k.data_ptr(), per.data_ptr(), per.data_ptr())
    n = len(seen)
    for kw in (dict(starts=starts[:2]), dict(starts=starts.long()), dict(k_out=k[:4]), dict(v_out=v[:, :1]), dict(k_out=k.bfloat16()),
               dict(v_out=v.flatten(1)), dict(sizes_out=per[:4]), dict(weights_out=per.double()), dict(k_out=torch.zeros(5, 64, 2).transpose(1, 2))):
        with pytest.raises(fz.FusionError):
            runner.Fusion.cache_read(f, c, stub_rows(5), **kw)
    with pytest.raises(fz.FusionError):
        runner.Fusion.cache_read(f, c, stub_rows(5, ids=types.SimpleNamespace(get_device=lambda: 0)))
    runner.Fusion.cache_read(f, c, stub_rows(0))   # no rows: nothing to enqueue
    assert len(seen) == n


def test_runner_refuses_packed_tensors_that_do_not_fit():
    pool, per, table, n = torch.zeros(6, 2, 16, 32, dtype=torch.uint8), torch.zeros(6, 16), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    z = torch.zeros(6, 2, 16, 4, dtype=torch.uint8)
    for bad in ((pool, pool[:5], z, z, table, n, None), (pool.int(), pool.int(), z, z, table, n, None), (pool, pool, z[..., :3], z, table, n, None),
                (pool, pool, z, z.bool(), table, n, None), (pool, pool, z, z, table.long(), n, None), (pool, pool, z, z, table, n, per[:5]),
                (pool, pool, z, None, table, n, None)):
        with pytest.raises(fz.FusionError):
            runner.packed_cache_of("bf16", *bad[:6], heads=4, sizes=bad[6])
    for pairs in ("thirds", "", None):
        with pytest.raises(fz.FusionError):
            runner.Rotation(torch.zeros(4, 32), pairs)
    with pytest.raises(fz.FusionError):
        runner.Rotation(torch.zeros(4, 32))   # not on a device


def test_rotation_table_on_the_host():
    t = runner.rotation_table(1000, 48, base=77.0, device="cpu")
    assert t.shape == (1000, 48) and t.dtype == torch.float32
    for p, i in ((0, 0), (999, 0), (999, 23), (17, 5)):
        a = p * 77.0 ** (-2 * i / 48)
        # 2^-25 from the rounding, and the angle's own 2^-53 of up to 999, twice
        assert abs(t[p, i].item() - math.cos(a)) <= 2.0 ** -25 + 4e-13 and abs(t[p, 24 + i].item() - math.sin(a)) <= 2.0 ** -25 + 4e-13


# ---- the sources -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("name", ["cache_rows.cuh", "cache_store.cu", "cache_read.cu", "packed_attn.cu", "fp4.cuh"])
def test_no_read_only_loads_in_kernels_that_start_early(name):
    """As in the other kernels of the cache: they are resident while the kernel before them still writes what they read."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    found = re.findall(r"\bldg16\(|\b__ldg\(|\.nc\b|__restrict__", text)
    assert len(text) > 900 and not found, found


# ---- the reference itself ----------------------------------------------------------------------------------------------
def test_reference_scales_are_the_nearest():
    """Against torch's own conversion, over every interval between two e4m3 numbers."""
    x = torch.cat([torch.linspace(float(a), float(b), 9, dtype=torch.float64) for a, b in zip(pk.E4M3, pk.E4M3[1:])])
    x = torch.cat([x, x * (1 + 2.0 ** -23), torch.tensor([449.0, 1e6], dtype=torch.float64)]).float().double()
    want = x.float().clamp(max=448.0).to(torch.float8_e4m3fn)
    assert torch.equal(pk.e4m3_byte(x), want.view(torch.uint8))
    every = torch.arange(256, dtype=torch.int16).to(torch.uint8)
    back = every.view(torch.float8_e4m3fn).double()
    assert torch.equal(torch.nan_to_num(pk.e4m3_value(every), 9e9), torch.nan_to_num(back, 9e9))


def test_reference_codes_are_the_nearest():
    """Every code against all sixteen by distance, ties to the even code."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn((400, 64), generator=g) * 2.0 ** torch.randint(-9, 9, (400, 1), generator=g)
    x[::7, 3::5] = x[::7, :1] / 6 * 1.25
    codes, scales = pk.pack(x)
    scale = pk.e4m3_value(scales[:, :4]).repeat_interleave(16, dim=1)
    code = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).long()
    off = (x.double().abs()[..., None] - pk.MAGNITUDES * scale[..., None]).abs()
    best = off.min(-1).values
    mine = off.gather(-1, (code % 8)[..., None])[..., 0]
    assert torch.equal(mine, best)
    tie = (off == best[..., None]).sum(-1) > 1
    assert ((code % 2 == 0) | ~tie)[scale > 0].all() and ((code >= 8) == torch.signbit(x))[scale > 0].all()
    assert torch.equal(pk.unpack(codes, scales).float().double(), pk.unpack(codes, scales))


def test_reference_rotation_is_one_of_complex_numbers():
    """(a + i b) times (cos + i sin), to the three roundings of a result: half a step of each product and of the sum."""
    g = torch.Generator().manual_seed(2)
    x, angle = torch.randn((50, 3, 80), generator=g), torch.rand((50, 24), generator=g).double() * 6
    table = torch.cat([angle.cos(), angle.sin()], dim=1).float()
    e = torch.complex(table[:, :24].double(), table[:, 24:].double())[:, None]
    for pairs in ("halves", "adjacent"):
        y = pk.turn(x, table, torch.arange(50), pairs)
        pick = (slice(0, 24), slice(24, 48)) if pairs == "halves" else (slice(0, 48, 2), slice(1, 48, 2))
        z = torch.complex(x[..., pick[0]].double(), x[..., pick[1]].double()) * e
        bound = 2 * 2.0 ** -24 * (x[..., pick[0]].abs() + x[..., pick[1]].abs()).double()
        assert ((y[..., pick[0]] - z.real).abs() <= bound).all() and ((y[..., pick[1]] - z.imag).abs() <= bound).all()
        assert torch.equal(y[..., 48:], x[..., 48:])
