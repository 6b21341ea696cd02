"""The key-value cache calls on the host: what they refuse before anything is enqueued, the workspace's size, the runner's
checks; and the reference that the GPU tests compare with, against itself (no GPU needed)."""
import importlib
import itertools
import math
import os
import re
import subprocess
import sys
import types

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import cache_reference as ref  # noqa: E402
import paper_2607_02612_gb300 as fz  # noqa: E402
from paper_2607_02612_gb300 import runner  # noqa: E402

FAKE = 0x100000   # never dereferenced: every call below fails a host check first
SHAPE = dict(max_batch=4, max_pages=10, page_tokens=16, kv_heads=2, head_dim=64, num_pages=40, k=FAKE, v=FAKE, sizes=None,
             weights=FAKE, page_table=FAKE, lengths=FAKE)


@pytest.fixture(scope="module", autouse=True)
def lib():
    fz.build()


def cache(**kw):
    return fz.cache(**{**SHAPE, **kw})


def size(heads=8, **kw):
    return fz.fusion_cache_workspace_size(cache(**kw), heads)


def append(c=None, **kw):
    a = dict(dtype=fz.FUSION_BF16, cache=c if c is not None else cache(), in_=fz.ragged(4, 5000, 20000, FAKE), k=FAKE,
             k_stride=128, v=FAKE, v_stride=128, sizes=None, scores=None, lengths_out=FAKE, workspace=FAKE,
             workspace_bytes=size(), dev_status=FAKE, stream=0)
    a.update(kw)
    return fz.fusion_cache_append(*a.values())


def attention(c=None, **kw):
    a = dict(dtype=fz.FUSION_BF16, cache=c if c is not None else cache(), q=FAKE, q_stride=512, heads=8, scale=0.125, window=0,
             sinks=0, out=FAKE, workspace=FAKE, workspace_bytes=size(), dev_status=FAKE, stream=0)
    a.update(kw)
    return fz.fusion_cache_attention(*a.values())


def evict(c=None, **kw):
    a = dict(dtype=fz.FUSION_BF16, cache=c if c is not None else cache(), budget=FAKE, sinks=1, recent=2, page_table_out=None,
             max_pages_out=0, lengths_out=FAKE, keep_idx=None, keep_stride=0, workspace=FAKE, workspace_bytes=size(),
             dev_status=FAKE, stream=0)
    a.update(kw)
    return fz.fusion_cache_evict(*a.values())


BAD_SHAPES = [dict(max_batch=-1), dict(max_batch=fz.FUSION_CACHE_MAX_BATCH + 1), dict(page_tokens=0), dict(page_tokens=24),
              dict(page_tokens=2 * fz.FUSION_CACHE_MAX_PAGE_TOKENS), dict(kv_heads=0), dict(head_dim=4), dict(head_dim=12),
              dict(head_dim=fz.FUSION_CACHE_MAX_HEAD_DIM + 8), dict(max_pages=0), dict(max_pages=(1 << 26) + 1),
              dict(num_pages=0), dict(num_pages=1 << 27), dict(num_pages=1 << 40)]


@pytest.mark.parametrize("call", [append, attention, evict])
def test_bad_shapes_are_refused(call):
    for kw in BAD_SHAPES:
        assert call(cache(**kw)) == fz.FUSION_ERR_SHAPE, kw
        assert size(**kw) == 0, kw
    for kw in (dict(k=None), dict(v=None), dict(page_table=None), dict(lengths=None), dict(k=FAKE + 8), dict(v=FAKE + 2)):
        assert call(cache(**kw)) == fz.FUSION_ERR_INVALID_ARG, kw
    assert call(dtype=2) == fz.FUSION_ERR_DTYPE
    for kw in (dict(workspace=None), dict(workspace=FAKE + 8), dict(workspace_bytes=1000)):
        assert call(**kw) == fz.FUSION_ERR_WORKSPACE, kw


def test_append_rejects_bad_arguments():
    for kw in (dict(in_=fz.ragged(5, 10, 100, FAKE)), dict(in_=fz.ragged(-1, 10, 100, FAKE)), dict(in_=fz.ragged(4, 0, 100, FAKE)),
               dict(in_=fz.ragged(4, 10, -1, FAKE)), dict(in_=fz.ragged(4, 10, 1 << 31, FAKE))):
        assert append(**kw) == fz.FUSION_ERR_SHAPE, kw
    for kw in (dict(k=None), dict(v=None), dict(lengths_out=None), dict(k=FAKE + 4), dict(v=FAKE + 8), dict(k_stride=-128),
               dict(v_stride=132), dict(in_=fz.ragged(4, 10, 100, None))):
        assert append(**kw) == fz.FUSION_ERR_INVALID_ARG, kw
    assert append(dtype=fz.FUSION_F32, k_stride=130) == fz.FUSION_ERR_INVALID_ARG


def test_attention_rejects_bad_arguments():
    for heads in (0, 1, 9, -2, fz.FUSION_CACHE_MAX_HEADS + 2):
        assert attention(heads=heads) == fz.FUSION_ERR_SHAPE, heads
        assert size(heads) == 0
    big = dict(max_batch=65535, max_pages=1 << 16)   # 2^16 sequences of 2^20 tokens
    assert attention(cache(**big), heads=2) == fz.FUSION_ERR_SHAPE and size(2, **big) == 0
    assert size(2, max_batch=1 << 15, max_pages=1 << 16, weights=None) > 0
    for kw in (dict(q=None), dict(out=None), dict(q=FAKE + 2), dict(out=FAKE + 8), dict(q_stride=-8), dict(q_stride=516),
               dict(scale=math.nan), dict(scale=math.inf), dict(window=-1), dict(sinks=-1)):
        assert attention(**kw) == fz.FUSION_ERR_INVALID_ARG, kw
    assert attention(workspace_bytes=size() - 1) == fz.FUSION_ERR_WORKSPACE
    assert attention(heads=16, workspace_bytes=size(8)) == fz.FUSION_ERR_WORKSPACE


def test_evict_rejects_bad_arguments():
    assert evict(cache(weights=None)) == fz.FUSION_ERR_INVALID_ARG
    for kw in (dict(budget=None), dict(lengths_out=None), dict(sinks=-1), dict(recent=-1), dict(keep_idx=FAKE, keep_stride=0)):
        assert evict(**kw) == fz.FUSION_ERR_INVALID_ARG, kw
    assert evict(page_table_out=FAKE + 64, max_pages_out=0) == fz.FUSION_ERR_SHAPE


def test_workspace_size():
    assert size() > 0 and size() % 256 == 0
    assert size(16) > size(8) > size(8, weights=None)
    assert size(max_pages=1000) > size()
    assert size(max_batch=0) > 0


def test_constants_and_status():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "fusion.h")).read()
    for name in ("FUSION_CACHE_MAX_BATCH", "FUSION_CACHE_MAX_PAGE_TOKENS", "FUSION_CACHE_MAX_HEAD_DIM", "FUSION_CACHE_MAX_HEADS",
                 "FUSION_DEV_BAD_CACHE"):
        assert f"#define {name} {getattr(fz, name)}" in text
    assert "cache" in fz.fusion_status_string(fz.FUSION_DEV_BAD_CACHE)


def test_runner_refuses_tensors_that_do_not_fit():
    rows = lambda t, n, h=2, d=8, dtype="f32": runner._rows_ptr(t, n, h, d, runner.TORCH_DTYPE[dtype], -1, "rows")   # noqa: E731
    t = torch.zeros(4, 16)
    assert rows(t, 4) == (t.data_ptr(), 16) and rows(t.view(4, 2, 8), 3)[1] == 16
    packed = torch.zeros(4, 48)
    assert rows(packed[:, 16:32], 4) == (packed.data_ptr() + 64, 48)
    assert rows(packed[:, 16:32].unflatten(1, (2, 8)), 4)[1] == 48
    for bad in (t[:3], t.double(), t.bfloat16(), torch.zeros(4, 8), torch.zeros(4, 32)[:, ::2], torch.zeros(4, 8, 2).transpose(1, 2),
                torch.zeros(64), torch.zeros(4, 2, 16)[:, :, :8], torch.tensor(0.0)):
        with pytest.raises(fz.FusionError):
            rows(bad, 4)
    for bad in (torch.zeros(4), torch.zeros(3, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)[::2],
                torch.zeros(4, 1, dtype=torch.int32)):
        with pytest.raises(fz.FusionError):
            runner._need(bad, torch.int32, -1, "lengths", 4)
    pool, per, table, n = torch.zeros(6, 2, 16, 8), torch.zeros(6, 16), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for bad in ((pool, pool[:5], table, n, None), (pool, pool, table.long(), n, None), (pool, pool, table, n[:2], None),
                (pool, pool, table, n, per[:5]), (pool, pool.bfloat16(), table, n, None), (pool, pool, table[0], n, None)):
        with pytest.raises(fz.FusionError):
            runner.cache_of("f32", *bad[:4], heads=4, sizes=bad[4])


# ---- the reference itself --------------------------------------------------------------------------------------------
def test_reference_eviction_against_enumeration():
    """The kept middle has the largest sum of weights, and of the sets with that sum the lexicographically smallest."""
    g = torch.Generator().manual_seed(1)
    for _ in range(60):
        n = int(torch.randint(0, 9, (1,), generator=g))
        w = (torch.randint(0, 4, (n,), generator=g) / 4).tolist()
        budget, sinks, recent = (int(torch.randint(lo, 9, (1,), generator=g)) for lo in (-1, 0, 0))
        m = min(max(budget, 0), n)
        s = min(sinks, m)
        r = min(recent, m - s)
        best = max(itertools.combinations(range(s, n - r), m - s - r), key=lambda c: (sum(w[j] for j in c), [-j for j in c]))
        assert ref.chosen(w, n, budget, sinks, recent) == [*range(s), *best, *range(n - r, n)]


def test_reference_attention_of_merged_tokens():
    """A token of size s weighs like s tokens of size 1, and one of size 0 like none."""
    c = ref.make("f32", [6], 1, 8, 4, sizes="whole", weights=True, seed=2)
    at = ref.places(c, 0, torch.arange(6))
    c["sizes"][at] = torch.tensor([1.0, 3.0, 0.0, 2.0, 1.0, 1.0])
    c["weights"][at] = 0.0
    rep = torch.tensor([0, 1, 1, 1, 3, 3, 4, 5])
    d = ref.make("f32", [8], 1, 8, 4, weights=True, seed=3)
    to = ref.places(d, 0, torch.arange(8))
    for name in ("k", "v"):
        d[name][to[0], :, to[1]] = c[name][at[0][rep], :, at[1][rep]]
    d["weights"][to] = 0.0
    q = torch.randn(1, 3, 8)
    a, _, wa, _ = ref.attention(c, q, "f32")
    b, _, wb, _ = ref.attention(d, q, "f32")
    assert torch.allclose(a, b, rtol=1e-12, atol=1e-14)
    assert torch.allclose(wa[at], torch.zeros(6, dtype=torch.float64).index_add_(0, rep, wb[to]), rtol=1e-12, atol=1e-14)
    assert abs(float(wb[to].sum()) - 3.0) < 1e-12     # the heads' probabilities


# ---- the sources -----------------------------------------------------------------------------------------------------
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_02612_gb300", "csrc")


def source(name):
    """A source without its comments."""
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


@pytest.mark.parametrize("name", ["cache.cuh", "cache_append.cu", "cache_attn.cu", "cache_attn_bf16.cu", "cache_evict.cu", "cache_rounds.cuh"])
def test_no_read_only_loads_in_kernels_that_start_early(name):
    """The kernels of the cache calls are resident while the kernel before them still runs, so nothing that they read is
    read-only for as long as they live, which the non-coherent path asks for."""
    text = source(name)
    assert len(text) > 1000, "the sources moved"
    found = re.findall(r"\bldg16\(|\b__ldg\(|\.nc\b|__restrict__", text)
    assert not found, found


def test_what_is_read_before_the_wait_is_read_past_the_l1_cache():
    """The weights' kernel looks its tokens up before its wait, which alone makes an SM forget older lines in its L1."""
    shared = source("cache.cuh")
    assert re.search(r"cache_entry\(const int \*p\) \{ return kEarly \? __ldcg\(p\) : \*p; \}", shared)
    for name, what in (("cache_page", "table"), ("cache_length", "lengths")):
        body = re.search(rf"\b{name}\(.*?\n}}\n", shared, re.S).group(0)
        assert f"cache_entry<kEarly>(&c.{what}[" in body and body.count(f"c.{what}[") == 1, body
    kernel = re.search(r"\bk_cache_weights\(.*?wait_for_previous\(\)", source("cache_attn.cu"), re.S).group(0)
    assert re.search(r"find_run<\w+, \w+, true>\(", kernel) and "cache_page<true>(" in kernel
    assert not re.search(r"c\.(table|lengths|weights|sizes)\[|p\.(logits|lse)\b|cache_(page|length)\(", kernel), kernel
    run = re.search(r"\bfind_run\(.*?\n}\n", source("cache_rounds.cuh"), re.S).group(0)
    assert not re.search(r"c\.(table|lengths)\[|\b(place_sequence|place_next|cache_page|cache_length)\(", run), run


# ---- arithmetic on the host ------------------------------------------------------------------------------------------
VISIBLE = r"""
#include <cstdio>
#include <cstdlib>
#include "cache.cuh"
int main(int argc, char **argv) {   // capacity window sinks length -> most, visible
    for (int k = 1; k + 3 < argc; k += 4) {
        fz::CacheAttnParams p{};
        p.c.capacity = atoi(argv[k]);
        fz::set_visible(p, atoi(argv[k + 1]), atoi(argv[k + 2]));
        printf("%d %d %d\n", p.most, fz::visible(p, atoi(argv[k + 3])), p.sinks);
    }
}
"""


def test_visible_tokens(tmp_path):
    """Windows and sinks of any size against capacities up to the largest, in whole numbers without bounds."""
    B = importlib.import_module("paper_2607_02612_gb300.build")
    (tmp_path / "v.cu").write_text(VISIBLE)
    subprocess.run([B._nvcc(), *B.ARCH, "-std=c++17", f"-I{B.INCLUDE}", f"-I{B.CSRC}", "-o", str(tmp_path / "v"), str(tmp_path / "v.cu")],
                   check=True, capture_output=True)
    cases = []
    for cap in (1, 2, 1024, (1 << 30) - 1, 1 << 30):
        some = sorted({0, 1, 2, 5, cap // 2, cap - 1, cap, cap + 1, (1 << 30) - 1, 1 << 30, (1 << 31) - 1})
        cases += [(cap, w, s, n) for w in some for s in some for n in {0, 1, 3, cap // 2, cap - 1, cap} if n <= cap]
    for k in range(0, len(cases), 1000):
        part = cases[k:k + 1000]
        out = subprocess.run([str(tmp_path / "v"), *[str(x) for c in part for x in c]], check=True, capture_output=True, text=True)
        for (cap, w, s, n), line in zip(part, out.stdout.splitlines(), strict=True):
            most, seen, sinks = map(int, line.split())
            want = min(n, w + s) if w else n
            assert seen == want and want <= most <= cap and 0 <= sinks <= cap, (cap, w, s, n, line)
            assert w == 0 or w >= cap or sinks >= min(s, n - w), (cap, w, s, n, line)   # (the places of those that are visible)


def test_rows_may_be_missing_where_there_are_none():
    for kw in (dict(k=None), dict(v=None)):
        assert append(**kw) == fz.FUSION_ERR_INVALID_ARG
        assert append(in_=fz.ragged(4, 10, 0, FAKE), workspace=None, **kw) == fz.FUSION_ERR_WORKSPACE   # (the next check)


def stub_cache(**kw):
    """What the runner's checks read of a cache, on the host; a call that passes them all reaches `call`."""
    c = dict(max_batch=3, heads=4, kv_heads=2, head_dim=8, torch_dtype=torch.float32, index=-1, device=torch.device("cpu"), code=fz.FUSION_F32,
             scale=1.0, _ws=FAKE, ws_bytes=1 << 20, c_struct=lambda: None, lengths=torch.zeros(3, dtype=torch.int32))
    c.update(kw)
    return types.SimpleNamespace(**c)


def test_runner_refuses_outputs_of_another_shape():
    c, q = stub_cache(max_batch=0), torch.zeros(0, 4, 8)
    good = torch.zeros(0, 4, 8)
    assert runner.Fusion.cache_attention(None, c, q, out=good) is good
    c, q = stub_cache(), torch.zeros(3, 4, 8)
    for shape in ((4, 3, 8), (8, 4, 3), (3, 8, 4), (2, 4, 8), (1, 12, 8), (96,), (3, 32), (3, 4, 8, 1), (2, 6, 8)):
        with pytest.raises(fz.FusionError):
            runner.Fusion.cache_attention(None, c, q, out=torch.zeros(shape))


def test_runner_refuses_rows_described_on_another_device():
    """A batch whose offsets, count or ids lie on another device than the cache (here: stand-ins that say so)."""
    elsewhere, here = types.SimpleNamespace(get_device=lambda: 1), types.SimpleNamespace(get_device=lambda: -1)
    t = torch.zeros(3, 16)
    for where in ("offsets", "batch", "ids"):
        rows = types.SimpleNamespace(max_batch=3, max_tokens=1, max_rows=3, offsets=here, batch=None, ids=None, ragged=lambda: None)
        setattr(rows, where, elsewhere)
        with pytest.raises(fz.FusionError):
            runner.Fusion.cache_append(None, stub_cache(), t, t, rows)


def test_runner_passes_numbers_of_tokens_of_any_size(monkeypatch):
    """Numbers beyond 32 bits mean all tokens (their low bits reached the call), negative ones are refused."""
    seen = []
    monkeypatch.setattr(runner, "_enqueue", lambda call, device, status, *args: seen.append(args))
    c = stub_cache(lib=types.SimpleNamespace(fusion_cache_attention=None, fusion_cache_evict=None))
    f = types.SimpleNamespace(status=None)
    q, budget, most = torch.zeros(3, 4, 8), torch.zeros(3, dtype=torch.int32), 2 ** 31 - 1
    for n, want in ((0, 0), (7, 7), (most, most), (1 << 31, most), ((1 << 32) + 5, most), (sys.maxsize, most), (1 << 70, most)):
        runner.Fusion.cache_attention(f, c, q, window=n, sinks=n)
        assert seen[-1][6:8] == (want, want)
        runner.Fusion.cache_evict(f, c, budget, sinks=n, recent=n)
        assert seen[-1][3:5] == (want, want)
    for n in (-1, -(1 << 32)):
        for kw in (dict(window=n), dict(sinks=n)):
            with pytest.raises(fz.FusionError):
                runner.Fusion.cache_attention(f, c, q, **kw)
        for kw in (dict(recent=n), dict(sinks=n)):
            with pytest.raises(fz.FusionError):
                runner.Fusion.cache_evict(f, c, budget, **kw)


def test_attention_refuses_scales_beyond_float32_in_base_2():
    """2.4e38 log2(e) is infinite in float32, and 0 times that no number."""
    for scale in (2.4e38, -2.4e38, 3.4e38):
        assert attention(scale=scale) == fz.FUSION_ERR_INVALID_ARG
    for scale in (2.3e38, -2.3e38, 0.0, 1e-45):
        assert attention(scale=scale, workspace=None) == fz.FUSION_ERR_WORKSPACE   # (the next check)


ROUNDS = r"""
#include <cstdio>
#include <cstdlib>
#include "cache_rounds.cuh"
int main(int argc, char **argv) {   // tokens warps -> fits
    for (int k = 1; k + 1 < argc; k += 2) printf("%d\n", (int)fz::rounds::counts_fit(atoll(argv[k]), atoll(argv[k + 1])));
    printf("%lld\n", fz::kCacheMaxHeadTokens);
}
"""


def test_rounds_are_counted_in_32_bits(tmp_path):
    """The bound that the kernels' rounds are held to, against the largest caches that the calls take, and the cache that the
    calls refuse just beyond it."""
    B = importlib.import_module("paper_2607_02612_gb300.build")
    (tmp_path / "r.cu").write_text(ROUNDS)
    subprocess.run([B._nvcc(), *B.ARCH, "-std=c++17", f"-I{B.INCLUDE}", f"-I{B.CSRC}", "-o", str(tmp_path / "r"), str(tmp_path / "r.cu")],
                   check=True, capture_output=True)
    sizes = [(tt, w) for tt in (1, 2, 4, 8, 16, 32) for w in (1, 4)]
    out = subprocess.run([str(tmp_path / "r"), *[str(x) for s in sizes for x in s]], check=True, capture_output=True, text=True)
    *fits, most = map(int, out.stdout.split())
    places = lambda heads: most // (fz.FUSION_CACHE_MAX_BATCH * heads)   # noqa: E731
    for (tt, w), ok in zip(sizes, fits, strict=True):
        worst = max(fz.FUSION_CACHE_MAX_BATCH * heads * -(-(128 if w == 1 else places(heads)) // (tt * w)) for heads in (1, 2, 64, 1024))
        assert not ok or worst < 1 << 32, (tt, w, worst)
    assert [s for s, ok in zip(sizes, fits) if ok] == [s for s in sizes if s[0] >= (2 if s[1] == 1 else 8)]   # (65535 * 1024 * 64 < 2^32)
    heads = 16
    cap = places(heads) // 16
    assert size(heads, max_batch=fz.FUSION_CACHE_MAX_BATCH, max_pages=cap, weights=None) > 0
    assert size(heads, max_batch=fz.FUSION_CACHE_MAX_BATCH, max_pages=cap + 1, weights=None) == 0


@pytest.mark.parametrize("off", [1, 2, 3, 6])
def test_misaligned_numbers_are_refused(off):
    """Pointers to 32-bit numbers, whose loads would fault."""
    bad = FAKE + off
    for call in (append, attention, evict):
        for kw in (dict(sizes=bad), dict(weights=bad), dict(page_table=bad), dict(lengths=bad)):
            assert call(cache(**kw)) == fz.FUSION_ERR_INVALID_ARG, kw
        assert call(dev_status=bad) == fz.FUSION_ERR_INVALID_ARG
    for kw in (dict(in_=fz.ragged(4, 10, 100, bad)), dict(in_=fz.ragged(4, 10, 100, FAKE, bad)), dict(in_=fz.ragged(4, 10, 100, FAKE, None, bad)),
               dict(sizes=bad), dict(scores=bad), dict(lengths_out=bad)):
        assert append(**kw) == fz.FUSION_ERR_INVALID_ARG, kw
    for kw in (dict(budget=bad), dict(page_table_out=bad, max_pages_out=4), dict(lengths_out=bad), dict(keep_idx=bad, keep_stride=8)):
        assert evict(**kw) == fz.FUSION_ERR_INVALID_ARG, kw
