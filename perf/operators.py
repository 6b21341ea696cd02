"""The key-value cache operators on work of their whole range: `Fusion.cache_append`, `Fusion.cache_attention` and
`Fusion.cache_evict`, and the same in elementary torch operations.

A cache holds the keys and values of up to `batch` sequences in pages of `page` tokens: pools [pages, kv_heads, page,
dim], a size and an accumulated attention weight per token, a page table and lengths.  Its pages lie in random order,
as in a pool that has been in use.  Kinds of cases:

  attend  one new token per sequence attends to its cache: softmax(scale q.k + log size) v, the weights accumulated
  append  rows of a ragged batch go to the ends of their sequences
  evict   each sequence keeps its first and last tokens and the heaviest of the others, in other pages
  prompt  a long prompt is appended and evicted to its budget in place
"""
import math

import torch

own = False   # True: the library's calls; False: the plain form

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # the compacted tokens of one image, DeiT-S heads: an interactive request, all latency
        dict(name="attend_bf16_b1_n197", kind="attend", dtype="bf16", batch=1, shortest=197, longest=197, heads=6,
             kv_heads=6, dim=64, page=16, window=0, sinks=0, sized=True, weighted=False),
        # a serving batch of ragged sequences with grouped heads, weights kept for a later eviction
        dict(name="attend_bf16_b64_n4096", kind="attend", dtype="bf16", batch=64, shortest=1, longest=4096, heads=32,
             kv_heads=8, dim=128, page=16, window=0, sinks=0, sized=False, weighted=True),
        # few very long sequences: the split over the cache's length
        dict(name="attend_bf16_b4_n65537", kind="attend", dtype="bf16", batch=4, shortest=60000, longest=65537, heads=32,
             kv_heads=8, dim=128, page=64, window=0, sinks=0, sized=False, weighted=False),
        # a sliding window with four sinks over long sequences: only the visible tokens are read
        dict(name="attend_bf16_b48_window", kind="attend", dtype="bf16", batch=48, shortest=200, longest=16384, heads=16,
             kv_heads=4, dim=64, page=32, window=1000, sinks=4, sized=False, weighted=True),
        # float32, the reference setting: ViT-L/16 tokens at 384 x 384 with merged sizes, some tokens masked
        dict(name="attend_f32_b16_n577", kind="attend", dtype="f32", batch=16, shortest=300, longest=577, heads=16,
             kv_heads=16, dim=64, page=16, window=0, sinks=0, sized=True, weighted=True),
        # one key head for all query heads
        dict(name="attend_bf16_b8_mqa", kind="attend", dtype="bf16", batch=8, shortest=2000, longest=8192, heads=32,
             kv_heads=1, dim=128, page=128, window=0, sinks=0, sized=True, weighted=False),
        # one token per sequence, every step of a decoder
        dict(name="append_bf16_b256_token", kind="append", dtype="bf16", batch=256, shortest=1, longest=1, held=1000,
             kv_heads=8, dim=128, page=16, sized=False, scored=False),
        # a compacted DeiT-S batch becomes the prefix of its sequences, sizes and scores with it
        dict(name="append_bf16_b256_n197", kind="append", dtype="bf16", batch=256, shortest=100, longest=197, held=0,
             kv_heads=6, dim=64, page=16, sized=True, scored=True),
        # a small float32 batch down to less than half
        dict(name="evict_f32_b8_n577", kind="evict", dtype="f32", batch=8, shortest=300, longest=577, budget=256,
             sinks=1, recent=16, kv_heads=6, dim=64, page=16, sized=True),
        # a serving batch of long sequences down to a fixed budget
        dict(name="evict_bf16_b32_n8192", kind="evict", dtype="bf16", batch=32, shortest=2048, longest=8192, budget=4000,
             sinks=4, recent=256, kv_heads=8, dim=128, page=16, sized=False),
        # one long prompt, appended and halved in place
        dict(name="prompt_bf16_b1_n32768", kind="prompt", dtype="bf16", batch=1, shortest=32768, longest=32768,
             budget=16384, sinks=4, recent=1024, kv_heads=8, dim=128, page=64, sized=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "evict", "evict", "prompt"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    kv_heads = rng.choice([1, 2, 3, 4, 6, 8, 16])
    dim = rng.choice([64, 64, 128, 128, 80, 96, 256])
    case = dict(kind=kind, dtype=dtype)
    row = 2 * kv_heads * dim * (2 if dtype == "bf16" else 4)
    batch = 1 if kind == "prompt" else _log_int(rng, 1, 256)
    moved = {"attend": 900 << 20, "append": 400 << 20, "evict": 280 << 20, "prompt": 200 << 20}[kind]   # of keys and values
    most = max(64, min({"attend": 65537, "append": 1024, "evict": 16384, "prompt": 32768}[kind], moved // (row * batch)))
    longest = _log_int(rng, 1 if kind != "evict" else 16, most) if rng.random() < 0.9 or kind != "append" else 1
    shortest = rng.choice([1, max(1, longest // 2), longest]) if batch > 1 else longest
    case.update(batch=batch, shortest=shortest, longest=longest, kv_heads=kv_heads, dim=dim,
                page=rng.choice([8, 16, 16, 32, 64, 128]), sized=rng.random() < 0.5)
    if kind == "attend":
        group = rng.choice([1, 1, 2, 4, 4, 7, 8, 16])
        case.update(heads=kv_heads * group, window=_log_int(rng, 1, longest) if rng.random() < 0.3 else 0,
                    sinks=rng.choice([0, 1, 4, 13]), weighted=rng.random() < 0.5)
    elif kind == "append":
        case.update(held=rng.choice([0, 0, 7, 333]), scored=rng.random() < 0.5)
    else:
        budget = max(1, int(longest * rng.uniform(0.1, 1.05)))
        case.update(budget=budget, sinks=rng.choice([0, 1, 4]), recent=rng.randint(0, max(0, budget // 4)))
    return case


def _lengths(case):
    """The lengths of a case's sequences, evenly spaced from shortest to longest."""
    b, lo, hi = case["batch"], case["shortest"], case["longest"]
    return [hi if b == 1 else lo + (hi - lo) * i // (b - 1) for i in range(b)]


def _visible(case):
    return [min(n, case["window"] + case["sinks"]) if case["window"] else n for n in _lengths(case)]


def prepare(case, seed):
    dev, dt = torch.device("cuda"), DTYPES[case["dtype"]]
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    kind, batch, page, kv, dim = case["kind"], case["batch"], case["page"], case["kv_heads"], case["dim"]
    lens = _lengths(case)
    order = torch.randperm(batch, generator=g, device=dev)
    n = torch.tensor(lens, dtype=torch.int32, device=dev)[order]
    held = case.get("held", 0)
    per = (held + case["longest"] + page - 1) // page          # pages of a sequence
    per_out = (min(case["budget"], case["longest"]) + page - 1) // page if kind == "evict" else 0
    pages = batch * (per + per_out)
    perm = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    s = dict(case, table=perm[:batch * per].view(batch, per).contiguous())

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32).to(dt)

    def sizes_of(*shape):   # merged tokens: whole sizes; one in sixteen masked
        z = torch.randint(1, 5, shape, generator=g, device=dev).float()
        return z * (torch.rand(shape, generator=g, device=dev) > 1 / 16)

    filled = kind in ("attend", "evict")
    for name in ("k", "v"):
        s[name] = normal(pages, kv, page, dim) if filled else torch.zeros((pages, kv, page, dim), device=dev, dtype=dt)
    tokens = (pages, page)
    s["sizes"] = (sizes_of(*tokens) if filled else torch.zeros(tokens, device=dev)) if case["sized"] else None
    if kind == "attend":
        s["weights"] = torch.rand(tokens, generator=g, device=dev) if case["weighted"] else None
        s["lengths"] = n
        s["q"] = normal(batch, case["heads"], dim) * 2.0   # logits of a standard deviation of two
        s["scale"] = dim ** -0.5
    elif kind == "evict":
        # accumulated weights: a few heavy tokens, many light ones
        s["weights"] = torch.rand(tokens, generator=g, device=dev).pow(4.0) * 8.0
        s["lengths"] = n
        s["table_out"] = perm[batch * per:].view(batch, per_out).contiguous()
    else:
        s["weights"] = torch.zeros(tokens, device=dev) if kind == "prompt" or case["scored"] else None
        s["lengths"] = torch.full((batch,), held, dtype=torch.int32, device=dev)
        rows = sum(lens)
        s["rows_k"], s["rows_v"] = normal(rows, kv * dim), normal(rows, kv * dim)
        s["rows_size"] = sizes_of(rows) if case["sized"] else None
        s["rows_score"] = torch.rand((rows,), generator=g, device=dev).pow(4.0) * 8.0 if s["weights"] is not None else None
        s["ids"] = torch.randperm(batch, generator=g, device=dev).to(torch.int32)
        s["offsets"] = torch.cat([n.new_zeros(1), n.cumsum(0).to(torch.int32)])
    if kind in ("evict", "prompt"):
        s["budgets"] = torch.full((batch,), case["budget"], dtype=torch.int32, device=dev)
        s["keep"] = torch.full((batch, min(case["budget"], case["longest"])), -1, dtype=torch.int32, device=dev)
    s["lengths_out"] = torch.zeros((batch,), dtype=torch.int32, device=dev)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program that calls the library keeps beside its tensors."""
    from paper_2607_02612_gb300 import runner
    s["fusion"] = runner.Fusion(s["batch"])
    s["cache"] = runner.cache_of(s["dtype"], s["k"], s["v"], s["table"], s["lengths"], sizes=s["sizes"],
                                 weights=s["weights"], heads=s.get("heads", s["kv_heads"]))
    if "offsets" in s:
        s["rows"] = runner.RaggedRows(s["batch"], s["longest"], s["rows_k"].shape[0], s["offsets"], ids=s["ids"])
    if s["kind"] == "prompt":   # the cache with the prompt in it
        s["cache_full"] = runner.cache_of(s["dtype"], s["k"], s["v"], s["table"], s["lengths_out"], sizes=s["sizes"],
                                          weights=s["weights"], heads=s["kv_heads"])


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    f, kind = s["fusion"], s["kind"]
    if kind == "attend":
        out = f.cache_attention(s["cache"], s["q"], window=s["window"], sinks=s["sinks"])
        return {"out": out, "weights": s["weights"]}
    if kind in ("append", "prompt"):
        f.cache_append(s["cache"], s["rows_k"], s["rows_v"], s["rows"], sizes=s["rows_size"], scores=s["rows_score"],
                       lengths_out=s["lengths_out"])
    if kind == "evict":
        f.cache_evict(s["cache"], s["budgets"], sinks=s["sinks"], recent=s["recent"], page_table_out=s["table_out"],
                      lengths_out=s["lengths_out"], keep_idx=s["keep"])
    if kind == "prompt":
        f.cache_evict(s["cache_full"], s["budgets"], sinks=s["sinks"], recent=s["recent"], keep_idx=s["keep"])
    return _state_outputs(s)


def _state_outputs(s):
    names = ["k", "v", "sizes", "weights", "lengths_out"] + (["keep"] if "keep" in s else [])
    return {name: s[name] for name in names}


def _run_plain(s):
    if s["kind"] == "attend":
        return _attend(s)
    if s["kind"] in ("append", "prompt"):
        _append(s)
    if s["kind"] == "evict":
        _evict(s, s["lengths"], s["table_out"])
    if s["kind"] == "prompt":
        _evict(s, s["lengths_out"].clone(), s["table"])
    return _state_outputs(s)


def _place(table, pos, page):
    """Page and place in the page of positions [batch, m]."""
    at = torch.div(pos, page, rounding_mode="floor").clamp(max=table.shape[1] - 1)
    return table.long().gather(1, at), pos % page


def _attend(s):
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
    kf = s["k"][pg, :, off].float().transpose(1, 2)     # [batch, kv, tokens, dim]
    q = s["q"].float().view(batch, kv, -1, dim)
    x = torch.matmul(q, kf.transpose(2, 3)) * s["scale"] + torch.log(size)[:, None, None, :]
    x = torch.where(here[:, None, None, :], x, -math.inf)
    x = torch.exp(x - x.amax(3, keepdim=True).clamp(min=-3.0e38))
    total = x.sum(3, keepdim=True)
    p = x / torch.where(total > 0, total, 1.0)
    vf = torch.where(here[:, :, None, None], s["v"][pg, :, off].float(), 0.0).transpose(1, 2)
    out = torch.matmul(p, vf).reshape(batch, -1, dim).to(s["q"].dtype)
    if s["weights"] is not None:
        w = torch.where(here, p.sum((1, 2)), 0.0)
        s["weights"].index_put_((pg, off), w, accumulate=True)
    return {"out": out, "weights": s["weights"]}


def _append(s):
    rows = s["rows_k"].shape[0]
    r = torch.arange(rows, device=s["ids"].device)
    i = torch.searchsorted(s["offsets"][1:].long(), r, right=True)
    slot = s["ids"].long()[i]
    pos = s["lengths"].long()[slot] + r - s["offsets"].long()[i]
    pg = s["table"].long()[slot, torch.div(pos, s["page"], rounding_mode="floor")]
    off = pos % s["page"]
    shape = (rows, s["kv_heads"], s["dim"])
    s["k"][pg, :, off] = s["rows_k"].view(shape)
    s["v"][pg, :, off] = s["rows_v"].view(shape)
    if s["sizes"] is not None:
        s["sizes"][pg, off] = s["rows_size"]
    if s["weights"] is not None:
        s["weights"][pg, off] = s["rows_score"]
    new = s["offsets"][1:] - s["offsets"][:-1]
    s["lengths_out"].copy_(s["lengths"])
    s["lengths_out"].index_add_(0, s["ids"].long(), new)


def _evict(s, lengths, table_out):
    batch, page, most = s["batch"], s["page"], s["keep"].shape[1]
    longest = s["longest"]
    n = lengths.long()[:, None]
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
    dpg, doff = _place(table_out, at, page)
    for name in ("k", "v"):
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
    row = 2 * case["kv_heads"] * case["dim"] * size            # a token's keys and values
    kind, extra = case["kind"], 4 if case["sized"] else 0
    if kind == "attend":
        seen = sum(_visible(case))
        token = row + extra + (8 if case["weighted"] else 0)
        return {"bytes": seen * token + seen // case["page"] * 4 + 2 * case["batch"] * case["heads"] * case["dim"] * size,
                "flops": 4.0 * seen * case["heads"] * case["dim"]}
    rows = sum(_lengths(case))
    appended = 2 * rows * (row + extra + (4 if kind == "prompt" or case.get("scored") else 0))
    if kind == "append":
        return {"bytes": appended, "flops": 0}
    kept = sum(min(n, case["budget"]) for n in _lengths(case))
    evicted = 4 * rows + kept * (2 * (row + extra + 4) + 4)
    return {"bytes": evicted + (appended if kind == "prompt" else 0), "flops": 0}


def exact(case, seed):
    """run()'s outputs in 64 bits, sequence by sequence from the definitions."""
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    if case["kind"] == "attend":
        return _exact_attend(s)
    k, v = s["k"].double(), s["v"].double()
    sizes, weights = (t if t is None else t.double() for t in (s["sizes"], s["weights"]))
    page, kv, dim = s["page"], s["kv_heads"], s["dim"]
    n, out_n = s["lengths"].tolist(), s["lengths"].tolist()
    keep = s["keep"].cpu() if "keep" in s else None
    if "rows_k" in s:
        offs = s["offsets"].tolist()
        for i, slot in enumerate(s["ids"].tolist()):
            a, b = offs[i], offs[i + 1]
            p = torch.arange(n[slot], n[slot] + b - a, device=k.device)
            where = (s["table"][slot].long()[p // page], p % page)
            k[where[0], :, where[1]] = s["rows_k"][a:b].double().view(-1, kv, dim)
            v[where[0], :, where[1]] = s["rows_v"][a:b].double().view(-1, kv, dim)
            if sizes is not None:
                sizes[where] = s["rows_size"][a:b].double()
            if weights is not None:
                weights[where] = s["rows_score"][a:b].double()
            out_n[slot] = n[slot] + b - a
    if keep is not None:
        for b in range(case["batch"]):
            have = out_n[b]
            m = min(max(case["budget"], 0), have)
            first = min(case["sinks"], m)
            last = min(case["recent"], m - first)
            p = torch.arange(have, device=k.device)
            src = (s["table"][b].long()[p // page], p % page)
            mine = weights[src].tolist()
            middle = sorted(range(first, have - last), key=lambda j: (-mine[j], j))[:m - first - last]
            chosen = sorted([*range(first), *middle, *range(have - last, have)])
            keep[b, :m] = torch.tensor(chosen, dtype=torch.int32)
            c = torch.tensor(chosen, dtype=torch.long, device=k.device)
            dst = ((s["table_out"] if "table_out" in s else s["table"])[b].long()[p[:m] // page], p[:m] % page)
            for t in (k, v):
                t[dst[0], :, dst[1]] = t[src[0][c], :, src[1][c]]
            for t in (sizes, weights):
                if t is not None:
                    t[dst] = t[src[0][c], src[1][c]]
            out_n[b] = m
    got = {"k": k, "v": v, "sizes": sizes, "weights": weights, "lengths_out": torch.tensor(out_n, dtype=torch.int32)}
    if keep is not None:
        got["keep"] = keep
    return got


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
        q = s["q"][b].double().view(kv, heads // kv, dim)
        x = torch.einsum("hgd,nhd->hgn", q, s["k"][at[0], :, at[1]].double()) * s["scale"]
        if s["sizes"] is not None:
            x = x + torch.log(s["sizes"][at].double())
        e = torch.exp(x - x.max(2, keepdim=True).values)
        e = e / e.sum(2, keepdim=True)
        outs.append(torch.einsum("hgn,nhd->hgd", e, s["v"][at[0], :, at[1]].double()).reshape(heads, dim))
        if weights is not None:
            weights[at] += e.sum((0, 1))
    return {"out": torch.stack(outs), "weights": weights}
