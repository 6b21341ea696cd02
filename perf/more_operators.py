"""Position rotation on the way into the key-value cache, and the cache in 4 bits, on work of their whole range:
`Fusion.cache_append_rotated`, and `Fusion.cache_append`, `Fusion.cache_read`, `Fusion.cache_attention` and
`Fusion.cache_evict` on a `DevicePackedCache`; and the same in elementary torch operations.

A cache holds the keys and values of up to `batch` sequences in pages of `page` tokens, a size and an accumulated
attention weight per token, a page table and lengths.  Its pages lie in random order, as in a pool that has been in use.
In 4 bits a row of a head is held in groups of 16 dims: a scale of type e4m3 for each, the largest magnitude times 1/6
rounded, and the dims divided by it as e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign; to the nearest, ties to the even
code), two to a byte, the lower dim in the lower bits.  Kinds of cases:

  rotate   rows of a ragged batch go to the ends of their sequences, keys and queries rotated by their positions
  attend4  one new token per sequence attends to its cache in 4 bits: softmax(scale q.k + log size) v
  store4   rows go to a cache in 4 bits, rotated or not, and are read back as the values that it holds
  evict4   sequences in 4 bits keep their first and last tokens and the heaviest of the others, in other pages; the kept
           rows are read back
"""
import math

import torch

own = False   # True: the library's calls; False: the plain form

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # of e2m1, by code


def listed():
    return [
        # every step of a decoder: one token per sequence, positions ahead of the places since tokens were evicted
        dict(name="rotate_bf16_b256_token", kind="rotate", dtype="bf16", batch=256, shortest=1, longest=1, held=1000, ahead=500,
             heads=32, kv_heads=8, dim=128, turned=128, pairs="halves", page=16, sized=False, scored=False),
        # ViT-L/16 at 384 x 384 after pruning: tokens keep the positions that they had, sizes and scores with them
        dict(name="rotate_f32_b64_n577", kind="rotate", dtype="f32", batch=64, shortest=200, longest=577, held=0, ahead=300,
             heads=16, kv_heads=16, dim=64, turned=32, pairs="adjacent", page=16, sized=True, scored=True),
        # the compacted tokens of one image, DeiT-S heads: an interactive request, all latency
        dict(name="attend4_bf16_b1_n197", kind="attend4", dtype="bf16", batch=1, shortest=197, longest=197, heads=6,
             kv_heads=6, dim=64, page=16, window=0, sinks=0, sized=True, weighted=False),
        # a serving batch of ragged sequences with grouped heads, weights kept for a later eviction
        dict(name="attend4_bf16_b64_n4096", kind="attend4", dtype="bf16", batch=64, shortest=1, longest=4096, heads=32,
             kv_heads=8, dim=128, page=16, window=0, sinks=0, sized=False, weighted=True),
        # few very long sequences: the split over the cache's length
        dict(name="attend4_bf16_b4_n65537", kind="attend4", dtype="bf16", batch=4, shortest=60000, longest=65537, heads=32,
             kv_heads=8, dim=128, page=64, window=0, sinks=0, sized=False, weighted=False),
        # a sliding window with four sinks over long sequences: only the visible tokens are read
        dict(name="attend4_bf16_b48_window", kind="attend4", dtype="bf16", batch=48, shortest=200, longest=16384, heads=16,
             kv_heads=4, dim=64, page=32, window=1000, sinks=4, sized=False, weighted=True),
        # float32 queries, the reference setting: merged sizes, some tokens masked
        dict(name="attend4_f32_b16_n577", kind="attend4", dtype="f32", batch=16, shortest=300, longest=577, heads=16,
             kv_heads=16, dim=64, page=16, window=0, sinks=0, sized=True, weighted=True),
        # every step of a decoder over a cache in 4 bits
        dict(name="store4_bf16_b256_token", kind="store4", dtype="bf16", batch=256, shortest=1, longest=1, held=1000, ahead=500,
             heads=32, kv_heads=8, dim=128, turned=128, pairs="halves", page=16, sized=False, scored=False),
        # a compacted DeiT-S batch becomes the prefix of its sequences, sizes and scores with it, no rotation
        dict(name="store4_bf16_b256_n197", kind="store4", dtype="bf16", batch=256, shortest=100, longest=197, held=0, ahead=0,
             heads=6, kv_heads=6, dim=64, turned=0, pairs="halves", page=16, sized=True, scored=True),
        # one long prompt, half of the dims rotated, positions as places
        dict(name="store4_bf16_b1_n32768", kind="store4", dtype="bf16", batch=1, shortest=32768, longest=32768, held=0, ahead=0,
             heads=8, kv_heads=8, dim=128, turned=64, pairs="halves", page=64, sized=False, scored=False),
        # a small batch down to less than half
        dict(name="evict4_f32_b8_n577", kind="evict4", dtype="f32", batch=8, shortest=300, longest=577, budget=256,
             sinks=1, recent=16, kv_heads=6, dim=64, page=16, sized=True),
        # a serving batch of long sequences down to a fixed budget
        dict(name="evict4_bf16_b32_n8192", kind="evict4", dtype="bf16", batch=32, shortest=2048, longest=8192, budget=1500,
             sinks=4, recent=256, kv_heads=8, dim=128, page=16, sized=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "attend4", "attend4", "attend4", "store4", "store4", "evict4"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    kv_heads = rng.choice([1, 2, 3, 4, 6, 8, 16])
    dim = rng.choice([64, 64, 128, 128, 80, 96, 256] if kind == "rotate" else [64, 64, 128, 128, 32, 96, 256])
    batch = _log_int(rng, 1, 256)
    most = {"rotate": 8192, "attend4": 65537, "store4": 32768, "evict4": 16384}[kind]
    longest = _log_int(rng, 16 if kind == "evict4" else 1, most)
    if kind in ("rotate", "store4") and rng.random() < 0.15:
        longest = 1
    group = rng.choice([1, 1, 2, 4, 4, 7, 8, 16])
    part, adjacent, window = rng.random(), rng.random() < 0.4, rng.random() < 0.3
    share, sinks = rng.uniform(0.1, 1.05), rng.choice([0, 1, 4, 13])
    low = rng.choice([0.0, 0.5, 1.0])
    case = dict(kind=kind, dtype=dtype, batch=batch, kv_heads=kv_heads, dim=dim, page=rng.choice([8, 16, 16, 32, 64, 128]),
                sized=rng.random() < 0.5)
    held, ahead, scored = rng.choice([0, 0, 7, 333]), rng.choice([0, 1, 999]), rng.random() < 0.5
    unit = 32 if kind == "store4" else 16
    while True:   # no more work than the largest listed case
        case.update(longest=longest, shortest=longest if batch == 1 else max(1, int(longest * low)))
        if kind == "attend4":
            case.update(heads=kv_heads * group, window=max(1, int(longest * share / 2)) if window else 0, sinks=sinks,
                        weighted=scored)
        elif kind == "evict4":
            budget = max(1, int(longest * share))
            case.update(budget=budget, sinks=min(sinks, 4), recent=budget // 7)
        else:
            turned = dim if part < 0.5 else dim // 2 // unit * unit if part < 0.8 or kind == "rotate" else 0
            case.update(held=held, ahead=ahead, heads=kv_heads * min(group, 4), turned=turned or (unit if kind == "rotate" else 0),
                        pairs="adjacent" if adjacent else "halves", scored=scored)
        if work(case)["bytes"] < 300e6 or longest < 2:
            return case
        longest = longest * 3 // 4


def _lengths(case):
    """The lengths of a case's sequences, evenly spaced from shortest to longest."""
    b, lo, hi = case["batch"], case["shortest"], case["longest"]
    return [hi if b == 1 else lo + (hi - lo) * i // (b - 1) for i in range(b)]


def _visible(case):
    return [min(n, case["window"] + case["sinks"]) if case["window"] else n for n in _lengths(case)]


def _offsets(counts, dev):
    return torch.tensor([0, *counts], dtype=torch.int32, device=dev).cumsum(0).to(torch.int32)


def prepare(case, seed):
    dev, dt = torch.device("cuda"), DTYPES[case["dtype"]]
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    kind, batch, page, kv, dim = case["kind"], case["batch"], case["page"], case["kv_heads"], case["dim"]
    lens = _lengths(case)
    n = torch.tensor(lens, dtype=torch.int32, device=dev)[torch.randperm(batch, generator=g, device=dev)]
    held = case.get("held", 0)
    per = (held + case["longest"] + page - 1) // page          # pages of a sequence
    per_out = (min(case["budget"], case["longest"]) + page - 1) // page if kind == "evict4" else 0
    pages = batch * (per + per_out)
    perm = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    s = dict(case, table=perm[:batch * per].view(batch, per).contiguous())

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32).to(dt)

    def sizes_of(*shape):   # merged tokens: whole sizes; one in sixteen masked
        z = torch.randint(1, 5, shape, generator=g, device=dev).float()
        return z * (torch.rand(shape, generator=g, device=dev) > 1 / 16)

    filled = kind in ("attend4", "evict4")
    for name in ("k", "v"):
        if kind == "rotate":
            s[name] = torch.zeros((pages, kv, page, dim), device=dev, dtype=dt)
        elif filled:
            s[name], s[name + "_scales"] = _to4(normal(pages, kv, page, dim).float())
        else:
            s[name] = torch.zeros((pages, kv, page, dim // 2), device=dev, dtype=torch.uint8)
            s[name + "_scales"] = torch.zeros((pages, kv, page, _scale_bytes(dim)), device=dev, dtype=torch.uint8)
    tokens = (pages, page)
    s["sizes"] = (sizes_of(*tokens) if filled else torch.zeros(tokens, device=dev)) if case["sized"] else None
    s["lengths_out"] = torch.zeros((batch,), dtype=torch.int32, device=dev)
    if kind == "attend4":
        s["weights"] = torch.rand(tokens, generator=g, device=dev) if case["weighted"] else None
        s["lengths"] = n
        s["q"] = normal(batch, case["heads"], dim) * 2.0   # logits of a standard deviation of two
        s["scale"] = dim ** -0.5
    elif kind == "evict4":
        # accumulated weights: a few heavy tokens, many light ones
        s["weights"] = torch.rand(tokens, generator=g, device=dev).pow(4.0) * 8.0
        s["lengths"] = n
        s["table_out"] = perm[batch * per:].view(batch, per_out).contiguous()
        s["budgets"] = torch.full((batch,), case["budget"], dtype=torch.int32, device=dev)
        s["keep"] = torch.full((batch, min(case["budget"], case["longest"])), -1, dtype=torch.int32, device=dev)
        s["rows"] = sum(min(x, case["budget"]) for x in lens)
        s["offsets"] = _offsets([min(x, case["budget"]) for x in n.tolist()], dev)
        s["ids"] = None
    else:
        s["weights"] = torch.zeros(tokens, device=dev) if case["scored"] else None
        s["lengths"] = torch.full((batch,), held, dtype=torch.int32, device=dev)
        rows = s["rows"] = sum(lens)
        s["rows_k"], s["rows_v"], s["rows_q"] = normal(rows, kv * dim), normal(rows, kv * dim), normal(rows, case["heads"], dim)
        s["rows_size"] = sizes_of(rows) if case["sized"] else None
        s["rows_score"] = torch.rand((rows,), generator=g, device=dev).pow(4.0) * 8.0 if case["scored"] else None
        s["ids"] = torch.randperm(batch, generator=g, device=dev).to(torch.int32)
        s["offsets"] = _offsets(n.tolist(), dev)
        s["starts"] = s["lengths"]
        if case["turned"]:
            s["angles"] = _angles(held + case["longest"] + case["ahead"], case["turned"], dev)
            place = held + torch.arange(rows, device=dev) - s["offsets"].long()[_sample_of(s)]
            # ahead of their places by what was evicted or pruned before them: less for a sample's first rows
            more = torch.rand((rows,), generator=g, device=dev).mul(case["ahead"]).long().sort().values
            s["positions"] = (place + more).to(torch.int32) if case["ahead"] else None
    if own:
        _handles(s)
    return s


def _angles(positions, turned, dev):
    """cos and sin of position * 10000^(-2 i / turned), [positions, turned]: turned / 2 cosines, then as many sines."""
    i = torch.arange(turned // 2, dtype=torch.float64, device=dev)
    a = torch.arange(positions, dtype=torch.float64, device=dev)[:, None] * 10000.0 ** (-2.0 * i / turned)
    return torch.cat([a.cos(), a.sin()], dim=1).float()


def _handles(s):
    """What a program that calls the library keeps beside its tensors."""
    from paper_2607_02612_gb300 import runner
    s["fusion"] = runner.Fusion(s["batch"])
    heads = s.get("heads", s["kv_heads"])

    def cache(table, lengths):
        if s["kind"] == "rotate":
            return runner.cache_of(s["dtype"], s["k"], s["v"], table, lengths, sizes=s["sizes"], weights=s["weights"], heads=heads)
        return runner.packed_cache_of(s["dtype"], s["k"], s["v"], s["k_scales"], s["v_scales"], table, lengths, sizes=s["sizes"],
                                weights=s["weights"], heads=heads)

    s["cache"] = cache(s["table"], s["lengths"])
    if "offsets" in s:
        s["ragged"] = runner.RaggedRows(s["batch"], s["longest"], s["rows"], s["offsets"], ids=s["ids"])
        s["cache_after"] = cache(s.get("table_out", s["table"]), s["lengths_out"])
    if "angles" in s:
        s["rotation"] = runner.Rotation(s["angles"], s["pairs"])


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    f, kind = s["fusion"], s["kind"]
    if kind == "attend4":
        return {"out": f.cache_attention(s["cache"], s["q"], window=s["window"], sinks=s["sinks"]), "weights": s["weights"]}
    q = None
    if kind == "evict4":
        f.cache_evict(s["cache"], s["budgets"], sinks=s["sinks"], recent=s["recent"], page_table_out=s["table_out"],
                      lengths_out=s["lengths_out"], keep_idx=s["keep"])
    elif "rotation" in s:
        q = f.cache_append_rotated(s["cache"], s["rows_k"], s["rows_v"], s["rotation"], s["ragged"], positions=s["positions"],
                                   q=s["rows_q"], sizes=s["rows_size"], scores=s["rows_score"], lengths_out=s["lengths_out"])
    else:
        f.cache_append(s["cache"], s["rows_k"], s["rows_v"], s["ragged"], sizes=s["rows_size"], scores=s["rows_score"],
                       lengths_out=s["lengths_out"])
    if kind == "rotate":
        return _outputs(s, s["k"], s["v"], q)
    k, v = f.cache_read(s["cache_after"], s["ragged"], starts=s.get("starts"))
    return _outputs(s, k, v, q)


def _outputs(s, k, v, q):
    """Pools, or the rows that they hold; the rotated queries; per token sizes and weights; lengths, kept positions."""
    return {"k": k, "v": v, "q": q, "sizes": s["sizes"], "weights": s["weights"], "lengths_out": s["lengths_out"],
            "keep": s.get("keep")}


def _run_plain(s):
    kind = s["kind"]
    if kind == "attend4":
        return _attend4(s)
    q = None
    if kind == "evict4":
        _evict4(s)
    else:
        q = _append(s)
    if kind == "rotate":
        return _outputs(s, s["k"], s["v"], q)
    return _outputs(s, *_read4(s), q)


def _scale_bytes(dim):
    """Bytes of a row's scales: one for 16 dims, rounded up to whole words."""
    return (dim // 16 + 3) // 4 * 4


def _to4(x):
    """float32 [..., dim] in 4 bits: packed codes [..., dim / 2] and scales [..., _scale_bytes(dim)], both uint8."""
    a = x.unflatten(-1, (-1, 16))
    top = a.abs().amax(-1)
    scale = torch.where(torch.isfinite(top), (top * (1.0 / 6.0)).clamp(max=448.0), math.nan).to(torch.float8_e4m3fn)
    z = scale.float().unsqueeze(-1)
    code = torch.zeros(a.shape, dtype=torch.uint8, device=x.device)
    # the middle between two magnitudes times the scale is exact in 32 bits; a tie goes to the even code
    for border, even_below in ((0.25, True), (0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)):
        code += (a.abs() > z * border) if even_below else (a.abs() >= z * border)
    code = torch.where(z > 0, code + torch.signbit(a).to(torch.uint8) * 8, 0).flatten(-2)
    packed = code[..., 0::2] + code[..., 1::2] * 16
    return packed, torch.nn.functional.pad(scale.view(torch.uint8), (0, _scale_bytes(x.shape[-1]) - top.shape[-1]))


def _from4(packed, scales):
    """The float32 values of packed codes [..., dim / 2] and scales."""
    value = torch.tensor([*MAGNITUDES, *(-m for m in MAGNITUDES)], device=packed.device)
    pair = torch.stack([packed & 15, packed >> 4], dim=-1).int()
    v = value[pair].flatten(-2).unflatten(-1, (-1, 16))
    return (v * scales[..., :v.shape[-2]].contiguous().view(torch.float8_e4m3fn).float().unsqueeze(-1)).flatten(-2)


def _turn(x, c, z, pairs):
    """Rows x [rows, heads, dim] float32 with their first 2 c.shape[1] dims rotated by the angles of cosines c and sines z."""
    m = c.shape[1]
    c, z = c[:, None], z[:, None]
    out = x.clone()
    if pairs == "halves":
        a, b = x[..., :m], x[..., m:2 * m]
        out[..., :m], out[..., m:2 * m] = a * c - b * z, b * c + a * z
    else:
        a, b = x[..., 0:2 * m:2], x[..., 1:2 * m:2]
        out[..., 0:2 * m:2], out[..., 1:2 * m:2] = a * c - b * z, b * c + a * z
    return out


def _sample_of(s):
    """The sample of each row."""
    r = torch.arange(s["rows"], device=s["offsets"].device)
    return torch.searchsorted(s["offsets"][1:].long(), r, right=True)


def _slots(s, starts, table):
    """Sequence, page and place of each row of the batch, the rows of a sample from position `starts` of its sequence."""
    i = _sample_of(s)
    slot = s["ids"].long()[i] if s["ids"] is not None else i
    at = torch.arange(s["rows"], device=i.device) - s["offsets"].long()[i]
    pos = at + (starts.long()[i] if starts is not None else 0)
    return slot, pos, table.long()[slot, torch.div(pos, s["page"], rounding_mode="floor")], pos % s["page"]


def _append(s):
    slot, pos, pg, off = _slots(s, s["starts"], s["table"])
    shape = (s["rows"], s["kv_heads"], s["dim"])
    k, v, q = s["rows_k"].float().view(shape), s["rows_v"].float().view(shape), None
    if "angles" in s:
        w = s["angles"][pos if s["positions"] is None else s["positions"].long()]
        m = s["turned"] // 2
        k = _turn(k, w[:, :m], w[:, m:], s["pairs"])
        q = _turn(s["rows_q"].float(), w[:, :m], w[:, m:], s["pairs"]).to(s["rows_q"].dtype)
    for name, x in (("k", k), ("v", v)):
        if s["kind"] == "rotate":
            s[name][pg, :, off] = x.to(s[name].dtype)
        else:
            s[name][pg, :, off], s[name + "_scales"][pg, :, off] = _to4(x)
    if s["sizes"] is not None:
        s["sizes"][pg, off] = s["rows_size"]
    if s["weights"] is not None:
        s["weights"][pg, off] = s["rows_score"]
    s["lengths_out"].copy_(s["lengths"])
    s["lengths_out"].index_add_(0, s["ids"].long(), s["offsets"][1:] - s["offsets"][:-1])
    return q


def _read4(s):
    _, _, pg, off = _slots(s, s.get("starts"), s.get("table_out", s["table"]))
    return [_from4(s[name][pg, :, off], s[name + "_scales"][pg, :, off]).to(DTYPES[s["dtype"]]) for name in ("k", "v")]


def _place(table, pos, page):
    """Page and place in the page of positions [batch, m]."""
    at = torch.div(pos, page, rounding_mode="floor").clamp(max=table.shape[1] - 1)
    return table.long().gather(1, at), pos % page


def _attend4(s):
    batch, kv, dim, page, sinks, window = s["batch"], s["kv_heads"], s["dim"], s["page"], s["sinks"], s["window"]
    n = s["lengths"].long()[:, None]
    most = min(s["longest"], window + sinks) if window else s["longest"]
    pos = torch.arange(most, device=n.device)[None, :].expand(batch, most)
    if window:   # the sinks, then the window
        pos = torch.where(pos < sinks, pos, pos - sinks + (n - window).clamp(min=sinks))
    here = pos < n
    pg, off = _place(s["table"], torch.where(here, pos, 0), page)
    size = s["sizes"][pg, off] if s["sizes"] is not None else torch.ones_like(pos, dtype=torch.float32)
    here = here & (size > 0)
    kf = _from4(s["k"][pg, :, off], s["k_scales"][pg, :, off]).transpose(1, 2)     # [batch, kv, tokens, dim]
    q = s["q"].float().view(batch, kv, -1, dim)
    x = torch.matmul(q, kf.transpose(2, 3)) * s["scale"] + torch.log(size)[:, None, None, :]
    x = torch.where(here[:, None, None, :], x, -math.inf)
    x = torch.exp(x - x.amax(3, keepdim=True).clamp(min=-3.0e38))
    total = x.sum(3, keepdim=True)
    p = x / torch.where(total > 0, total, 1.0)
    vf = torch.where(here[:, :, None, None], _from4(s["v"][pg, :, off], s["v_scales"][pg, :, off]), 0.0).transpose(1, 2)
    out = torch.matmul(p, vf).reshape(batch, -1, dim).to(s["q"].dtype)
    if s["weights"] is not None:
        w = torch.where(here, p.sum((1, 2)), 0.0)
        s["weights"].index_put_((pg, off), w, accumulate=True)
    return {"out": out, "weights": s["weights"]}


def _evict4(s):
    batch, page, most, longest = s["batch"], s["page"], s["keep"].shape[1], s["longest"]
    n = s["lengths"].long()[:, None]
    m = torch.minimum(s["budgets"].long()[:, None].clamp(min=0), n)
    first = m.clamp(max=s["sinks"])
    last = (m - first).clamp(max=s["recent"])
    pos = torch.arange(longest, device=n.device)[None, :].expand(batch, longest)
    pg, off = _place(s["table"], torch.where(pos < n, pos, 0), page)
    w = s["weights"][pg, off]
    stay = (pos < first) | ((pos >= n - last) & (pos < n))
    w = torch.where(stay, math.inf, torch.where(pos < n, w, -math.inf))
    order = torch.sort(w, dim=1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(1, order, pos)
    keep = (rank < m) & (pos < n)
    to = torch.where(keep, keep.cumsum(1) - 1, most)
    src = torch.zeros((batch, most + 1), dtype=torch.long, device=n.device).scatter_(1, to, pos)[:, :most]
    at = torch.arange(most, device=n.device)[None, :].expand(batch, most)
    new = at < m
    spg, soff = _place(s["table"], src, page)
    dpg, doff = _place(s["table_out"], at, page)
    for name in ("k", "v", "k_scales", "v_scales"):
        t = s[name]
        t[dpg, :, doff] = torch.where(new[:, :, None, None], t[spg, :, soff], t[dpg, :, doff])
    for name in ("sizes", "weights"):
        t = s[name]
        if t is not None:
            t[dpg, doff] = torch.where(new, t[spg, soff], t[dpg, doff])
    s["keep"].copy_(torch.where(new, src, s["keep"].long()))
    s["lengths_out"].copy_(m[:, 0])


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    elements = 2 * case["kv_heads"] * case["dim"]              # of a token's keys and values
    row, row4 = elements * size, elements * 9 // 16            # in 4 bits: half a byte and a 16th
    kind, extra = case["kind"], 4 if case["sized"] else 0
    if kind == "attend4":
        seen = sum(_visible(case))
        token = row4 + extra + (8 if case["weighted"] else 0)
        return {"bytes": seen * token + seen // case["page"] * 4 + 2 * case["batch"] * case["heads"] * case["dim"] * size,
                "flops": 4.0 * seen * case["heads"] * case["dim"]}
    if kind == "evict4":
        kept = sum(min(n, case["budget"]) for n in _lengths(case))
        return {"bytes": 4 * sum(_lengths(case)) + kept * (2 * (row4 + extra + 4) + 4 + row4 + row), "flops": 0}
    rows = sum(_lengths(case))
    token = 2 * (extra + (4 if case["scored"] else 0)) + row
    if case["turned"]:
        token += 2 * case["heads"] * case["dim"] * size + (4 if case["ahead"] else 0)
    # cosines and sines: once for each position of the batch
    table = min(rows, case["longest"] + case["ahead"]) * case["turned"] * 4
    turns = 6.0 * rows * case["turned"] / 2 * (case["kv_heads"] + case["heads"])
    return {"bytes": rows * (token + (row if kind == "rotate" else 2 * row4 + row)) + table, "flops": turns}


def exact(case, seed):
    """run()'s outputs in 64 bits, sequence by sequence from the definitions."""
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    if case["kind"] == "attend4":
        return _exact_attend(s)
    if case["kind"] == "evict4":
        return _exact_evict(s)
    page, kv, dim, dev = s["page"], s["kv_heads"], s["dim"], s["lengths"].device
    offs, out_n = s["offsets"].tolist(), s["lengths"].tolist()
    k, v = s["rows_k"].double().view(-1, kv, dim), s["rows_v"].double().view(-1, kv, dim)
    q = s["rows_q"].double() if case["turned"] else None
    got = {name: None if s[name] is None else s[name].double() for name in ("sizes", "weights")}
    for name in ("k", "v"):
        got[name] = s[name].double() if case["kind"] == "rotate" else []
    for i, slot in enumerate(s["ids"].tolist()):
        a, b, n = offs[i], offs[i + 1], out_n[slot]
        p = torch.arange(n, n + b - a, device=dev)
        where = (s["table"][slot].long()[p // page], p % page)
        if case["turned"]:
            w = s["angles"].double()[p if s["positions"] is None else s["positions"][a:b].long()]
            k[a:b], q[a:b] = _exact_turn(k[a:b], w, case), _exact_turn(q[a:b], w, case)
        for name, x in (("k", k[a:b]), ("v", v[a:b])):
            if case["kind"] == "rotate":
                got[name][where[0], :, where[1]] = x
            else:
                got[name].append(_exact_near(x))
        if got["sizes"] is not None:
            got["sizes"][where] = s["rows_size"][a:b].double()
        if got["weights"] is not None:
            got["weights"][where] = s["rows_score"][a:b].double()
        out_n[slot] = n + b - a
    if case["kind"] == "store4":
        got["k"], got["v"] = torch.cat(got["k"]), torch.cat(got["v"])
    return dict(got, q=q, lengths_out=torch.tensor(out_n, dtype=torch.int32), keep=None)


def _exact_turn(x, w, case):
    """x as complex numbers times those of the angles."""
    m = case["turned"] // 2
    e = torch.complex(w[:, :m], w[:, m:])[:, None]
    flat = x[..., :2 * m]
    if case["pairs"] == "halves":
        y = torch.complex(flat[..., :m], flat[..., m:]) * e
        y = torch.cat([y.real, y.imag], dim=-1)
    else:
        y = torch.view_as_real(torch.view_as_complex(flat.unflatten(-1, (m, 2)).contiguous()) * e).flatten(-2)
    return torch.cat([y, x[..., 2 * m:]], dim=-1)


def _exact_near(x):
    """What the cache in 4 bits holds for x: every dim's nearest magnitude times the group's scale."""
    a = x.unflatten(-1, (-1, 16))
    want = a.abs().amax(-1, keepdim=True) / 6.0
    step = torch.exp2(torch.floor(torch.log2(want.clamp(min=2.0 ** -6))) - 3.0)   # of e4m3 numbers of this size
    scale = (torch.round(want / step) * step).clamp(max=448.0)
    y = torch.where(scale > 0, a.abs() / scale, 0.0).clamp(max=6.0)
    # magnitudes are whole halves up to 2, whole numbers up to 4, even ones up to 6
    unit = torch.where(y < 2.0, 0.5, torch.where(y < 4.0, 1.0, 2.0))
    return (torch.copysign(torch.round(y / unit) * unit, a) * scale).flatten(-2)


def _exact_rows(s, name, where, scales):
    """Rows of a pool in 4 bits as doubles, from its bits."""
    byte, sc = s[name][where[0], :, where[1]].long(), scales[where[0], :, where[1]].long()
    code = torch.stack([byte % 16, byte // 16], dim=-1).flatten(-2)
    e, m = code % 8 // 2, code % 2
    mag = torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * torch.exp2(e.double() - 1.0)) * torch.where(code >= 8, -1.0, 1.0)
    e, m = sc % 128 // 8, sc % 8
    scale = torch.where(e == 0, m * 2.0 ** -9, (1.0 + m / 8.0) * torch.exp2(e.double() - 7.0))
    return mag * scale[..., :mag.shape[-1] // 16].repeat_interleave(16, dim=-1)


def _exact_evict(s):
    page, dev = s["page"], s["lengths"].device
    sizes, weights = (t if t is None else t.double() for t in (s["sizes"], s["weights"]))
    keep, out_n, rows = s["keep"].cpu(), [], {"k": [], "v": []}
    for b, n in enumerate(s["lengths"].tolist()):
        m = min(max(s["budget"], 0), n)
        first = min(s["sinks"], m)
        last = min(s["recent"], m - first)
        p = torch.arange(n, device=dev)
        src = (s["table"][b].long()[p // page], p % page)
        mine = weights[src].tolist()
        middle = sorted(range(first, n - last), key=lambda j: (-mine[j], j))[:m - first - last]
        chosen = sorted([*range(first), *middle, *range(n - last, n)])
        keep[b, :m] = torch.tensor(chosen, dtype=torch.int32)
        c = torch.tensor(chosen, dtype=torch.long, device=dev)
        src = (src[0][c], src[1][c])
        dst = (s["table_out"][b].long()[p[:m] // page], p[:m] % page)
        for name in ("k", "v"):
            rows[name].append(_exact_rows(s, name, src, s[name + "_scales"]))
        for t in (sizes, weights):
            if t is not None:
                t[dst] = t[src]
        out_n.append(m)
    return {"k": torch.cat(rows["k"]), "v": torch.cat(rows["v"]), "q": None, "sizes": sizes, "weights": weights,
            "lengths_out": torch.tensor(out_n, dtype=torch.int32), "keep": keep}


def _exact_attend(s):
    page, kv, dim, heads = s["page"], s["kv_heads"], s["dim"], s["heads"]
    outs, weights = [], None if s["weights"] is None else s["weights"].double()
    for b, n in enumerate(s["lengths"].tolist()):
        p = torch.arange(n, device=s["k"].device)
        if s["window"]:
            p = p[(p < s["sinks"]) | (p >= n - s["window"])]
        at = (s["table"][b].long()[p // page], p % page)
        if s["sizes"] is not None:
            p = p[s["sizes"][at] > 0]
            at = (s["table"][b].long()[p // page], p % page)
        if not len(p):
            outs.append(torch.zeros((heads, dim), dtype=torch.float64, device=p.device))
            continue
        k, v = (_exact_rows(s, name, at, s[name + "_scales"]) for name in ("k", "v"))
        q = s["q"][b].double().view(kv, heads // kv, dim)
        x = torch.einsum("hgd,nhd->hgn", q, k) * s["scale"]
        if s["sizes"] is not None:
            x = x + torch.log(s["sizes"][at].double())
        e = torch.exp(x - x.max(2, keepdim=True).values)
        e = e / e.sum(2, keepdim=True)
        outs.append(torch.einsum("hgn,nhd->hgd", e, v).reshape(heads, dim))
        if weights is not None:
            weights[at] += e.sum((0, 1))
    return {"out": torch.stack(outs), "weights": weights}
