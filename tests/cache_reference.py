"""The key-value cache calls in 64 bits on the host, sequence by sequence from their definitions (torch on the CPU), and
the caches that the tests build.  A cache here is a dict of host tensors: k, v [pages, kv_heads, page, dim] in the storage
type, sizes and weights [pages, page] float32 or None, table [batch, pages of a row] int32, lengths [batch] int32."""
import math

import torch

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def places(c, b, pos, table=None):
    """Page and place of positions of sequence b."""
    t = (c["table"] if table is None else table)[b].long()
    page = c["k"].shape[2]
    return t[pos // page], pos % page


def make(dtype, lengths, kv_heads, dim, page, *, room=0, sizes=None, weights=False, spare=3, seed=0, spread=1.0):
    """A cache of sequences of these lengths with room for `room` more tokens each, its pages in random order among `spare`
    more; everything that no sequence holds is NaN.  sizes: None, "whole" (1 to 4) or "masked" (some 0, NaN keys there)."""
    g = torch.Generator().manual_seed(seed)
    batch, longest = len(lengths), max(list(lengths) + [0])
    per = max(1, -(-(longest + room) // page))
    pages = batch * per + spare
    c = dict(table=torch.randperm(pages, generator=g)[:batch * per].view(batch, per).to(torch.int32),
             lengths=torch.tensor(lengths, dtype=torch.int32))
    for name in ("k", "v"):
        c[name] = torch.full((pages, kv_heads, page, dim), math.nan, dtype=TYPES[dtype])
    c["sizes"] = torch.full((pages, page), math.nan) if sizes else None
    c["weights"] = torch.full((pages, page), math.nan) if weights else None
    for b, n in enumerate(lengths):
        pos = torch.arange(n)
        pg, off = places(c, b, pos)
        k = torch.randn((n, kv_heads, dim), generator=g) * spread
        v = torch.randn((n, kv_heads, dim), generator=g)
        if sizes:
            z = torch.randint(1, 5, (n,), generator=g).float()
            if sizes == "masked":
                z[torch.rand(n, generator=g) < 0.3] = 0.0
                k[z == 0] = math.nan
                v[z == 0] = math.inf
            c["sizes"][pg, off] = z
        c["k"][pg, :, off] = k.to(TYPES[dtype])
        c["v"][pg, :, off] = v.to(TYPES[dtype])
        if weights:
            c["weights"][pg, off] = torch.rand(n, generator=g)
    return c


def copy(c):
    return {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in c.items()}


def append(c, k, v, offsets, ids=None, sizes=None, scores=None, count=None):
    """Appends in place to c; returns the new lengths."""
    new = c["lengths"].clone()
    for i in range(len(offsets) - 1 if count is None else count):
        t = i if ids is None else int(ids[i])
        a, e, at = int(offsets[i]), int(offsets[i + 1]), int(c["lengths"][t])
        pg, off = places(c, t, torch.arange(at, at + e - a))
        shape = (e - a, c["k"].shape[1], c["k"].shape[3])
        c["k"][pg, :, off] = k[a:e].reshape(shape)
        c["v"][pg, :, off] = v[a:e].reshape(shape)
        if c["sizes"] is not None:
            c["sizes"][pg, off] = sizes[a:e] if sizes is not None else torch.ones(e - a)
        if c["weights"] is not None:
            c["weights"][pg, off] = scores[a:e] if scores is not None else torch.zeros(e - a)
        new[t] = at + e - a
    return new


def visible(n, window, sinks):
    pos = torch.arange(n)
    return pos[(pos < sinks) | (pos >= n - window)] if window else pos


def attention(c, q, dtype, *, scale=None, window=0, sinks=0):
    """(out, tolerance, weights, tolerance): out [batch, heads, dim] and the accumulated weights in 64 bits.

    The tolerances count the roundings.  A logit (base e) is a float32 sum of `dim` products: off by at most
    (dim + 4) 2^-24 scale sum|q k| and a few steps of its own; so a probability is off by a factor 1 + d, d twice that,
    plus 2^-20 for the exponential.  Sums over n tokens in float32, at least four at a time, lose (n / 4 + 64) 2^-24 of the
    sum of magnitudes.  bf16 adds 2^-16 of sum p |v| (the probabilities, two bf16 terms, as operands) and 2^-8 of the output."""
    batch, heads, dim = q.shape
    kv = c["k"].shape[1]
    group = heads // kv
    scale = dim ** -0.5 if scale is None else scale
    out, tol = torch.zeros((batch, heads, dim), dtype=torch.float64), torch.zeros((batch, heads, dim), dtype=torch.float64)
    w = None if c["weights"] is None else c["weights"].double()
    wtol = None if w is None else torch.zeros_like(w)
    for b in range(batch):
        pos = visible(int(c["lengths"][b]), window, sinks)
        at = places(c, b, pos)
        if c["sizes"] is not None:
            pos = pos[c["sizes"][at] != 0]
            at = places(c, b, pos)
        n = len(pos)
        if n == 0:
            continue
        k = c["k"][at[0], :, at[1]].double().repeat_interleave(group, dim=1)   # [n, heads, dim]
        v = c["v"][at[0], :, at[1]].double().repeat_interleave(group, dim=1)
        x = torch.einsum("hd,nhd->hn", q[b].double(), k) * scale
        mag = torch.einsum("hd,nhd->hn", q[b].double().abs(), k.abs()) * abs(scale)
        if c["sizes"] is not None:
            x = x + torch.log(c["sizes"][at].double())
        p = torch.exp(x - x.max(1, keepdim=True).values)
        p = p / p.sum(1, keepdim=True)
        d = 2 * ((dim + 4) * 2.0 ** -24 * mag.max(1).values + 4 * 2.0 ** -24 * x.abs().max(1).values) + 2.0 ** -20
        d = torch.expm1(d) + (n / 4 + 64) * 2.0 ** -24
        out[b] = torch.einsum("hn,nhd->hd", p, v)
        a = torch.einsum("hn,nhd->hd", p, v.abs())
        tol[b] = 2 * d[:, None] * a + 2.0 ** -24 * out[b].abs() + 1e-37
        if dtype == "bf16":
            tol[b] += 2.0 ** -16 * a + 2.0 ** -8 * out[b].abs()
        if w is not None:
            w[at] += p.sum(0)
            wtol[at] = 2 * (d[:, None] * p).sum(0) + (heads + 1) * 2.0 ** -24 * w[at].abs()
    return out, tol, w, wtol


def chosen(weights, n, budget, sinks, recent):
    """Positions that a sequence of these weights keeps."""
    m = min(max(budget, 0), n)
    s = min(sinks, m)
    r = min(recent, m - s)
    middle = sorted(range(s, n - r), key=lambda j: (-weights[j], j))[:m - s - r]
    return sorted([*range(s), *middle, *range(n - r, n)])


def evict(c, budget, *, sinks=0, recent=0, table_out=None):
    """Evicts in place in c (or into table_out's pages); returns (new lengths, kept positions per sequence)."""
    new, keeps = [], []
    for b, n in enumerate(c["lengths"].tolist()):
        keep = chosen(c["weights"][places(c, b, torch.arange(n))].tolist(), n, int(budget[b]), sinks, recent)
        src = places(c, b, torch.tensor(keep, dtype=torch.long))
        dst = places(c, b, torch.arange(len(keep)), table_out)
        for name in ("k", "v"):
            c[name][dst[0], :, dst[1]] = c[name][src[0], :, src[1]]
        for name in ("sizes", "weights"):
            if c[name] is not None:
                c[name][dst] = c[name][src]
        new.append(len(keep))
        keeps.append(keep)
    return torch.tensor(new, dtype=torch.int32), keeps


def bits(t):
    """A tensor's bit patterns, for comparisons in which NaN equals itself."""
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)
