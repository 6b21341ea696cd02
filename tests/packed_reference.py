"""The key-value cache in 4 bits and the rotation of keys and queries, on the host from their definitions, and the caches that
the tests build.  A packed cache here is a dict like cache_reference's, with k and v [pages, kv_heads, page, dim / 2] and
k_scales and v_scales [pages, kv_heads, page, bytes], all uint8."""
import math

import torch

import cache_reference as ref

MAGNITUDES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
MIDDLES = (MAGNITUDES[1:] + MAGNITUDES[:-1]) / 2
NAN_SCALE, JUNK = 0x7F, 0xFF   # JUNK: in codes -6, in scales NaN


def scale_bytes(dim):
    return (dim // 16 + 3) // 4 * 4


def e4m3_value(byte):
    """The double that an e4m3 byte stands for."""
    b = byte.long()
    e, m = b % 128 // 8, (b % 8).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (1.0 + m / 8.0) * torch.exp2(e.double() - 7.0))
    v = torch.where(b % 128 == 127, math.nan, v)
    return torch.where(b >= 128, -v, v)


E4M3 = e4m3_value(torch.arange(127))   # finite ones >= 0, ascending: their bytes are their places


def e4m3_byte(x):
    """The byte of the e4m3 number nearest to x >= 0 (double; ties to the even byte), 448 at most."""
    hi = torch.searchsorted(E4M3, x).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = x - E4M3[lo], E4M3[hi] - x
    return torch.where(dl < dh, lo, torch.where(dh < dl, hi, torch.where(lo % 2 == 0, lo, hi))).to(torch.uint8)


def pack(x):
    """float32 rows [..., dim] -> packed codes and scales."""
    assert x.dtype == torch.float32
    a = x.unflatten(-1, (-1, 16))
    top = a.abs().amax(-1)
    fine = torch.isfinite(top)
    want = top * torch.tensor(1.0 / 6.0, dtype=torch.float32)   # rounded to float32, as the definition has it
    scale = torch.where(fine, e4m3_byte(torch.where(fine, want, 0.0).double().clamp(max=448.0)), NAN_SCALE)
    z = torch.where(fine, e4m3_value(scale), 0.0).unsqueeze(-1)
    y = torch.where(z > 0, a.double().abs(), 0.0)
    # exact: a middle has 3 significant bits, a scale 4, a dim 24
    code = sum(((y > z * mid) if i % 2 == 0 else (y >= z * mid)).to(torch.uint8) for i, mid in enumerate(MIDDLES.tolist()))
    code = torch.where(z > 0, code + torch.signbit(a).to(torch.uint8) * 8, 0).to(torch.uint8).flatten(-2)
    packed = code[..., 0::2] + code[..., 1::2] * 16
    return packed, torch.nn.functional.pad(scale.to(torch.uint8), (0, scale_bytes(x.shape[-1]) - scale.shape[-1]))


def unpack(packed, scales):
    """The doubles that packed codes and scales stand for."""
    code = torch.stack([packed & 15, packed >> 4], dim=-1).flatten(-2).long()
    v = MAGNITUDES[code % 8] * torch.where(code >= 8, -1.0, 1.0)
    dim = code.shape[-1]
    return v * e4m3_value(scales[..., :dim // 16]).repeat_interleave(16, dim=-1)


def turn(x, table, pos, pairs):
    """float32 rows x [rows, heads, dim] rotated by their positions, every product and sum rounded to float32."""
    assert x.dtype == torch.float32
    m = table.shape[1] // 2
    c, s = table[pos.long()][:, None, :m], table[pos.long()][:, None, m:]
    out = x.clone()
    at = (slice(0, m), slice(m, 2 * m)) if pairs == "halves" else (slice(0, 2 * m, 2), slice(1, 2 * m, 2))
    a, b = x[..., at[0]], x[..., at[1]]
    ac, bs, bc, as_ = a * c, b * s, b * c, a * s   # (one operation at a time: none is fused)
    out[..., at[0]] = ac - bs
    out[..., at[1]] = bc + as_
    return out


def make(lengths, kv_heads, dim, page, *, room=0, sizes=None, weights=False, spare=3, seed=0, spread=1.0):
    """A packed cache like cache_reference.make's: what no sequence holds, what lies behind the scales, and the keys and values
    of masked tokens are JUNK."""
    c = ref.make("f32", lengths, kv_heads, dim, page, room=room, sizes=sizes, weights=weights, spare=spare, seed=seed, spread=spread)
    full = {name: c[name] for name in ("k", "v")}
    shape = c["k"].shape[:3]
    for name in ("k", "v"):
        c[name] = torch.full((*shape, dim // 2), JUNK, dtype=torch.uint8)
        c[name + "_scales"] = torch.full((*shape, scale_bytes(dim)), JUNK, dtype=torch.uint8)
    for b, n in enumerate(lengths):
        pg, off = ref.places(dict(c, k=c["k"]), b, torch.arange(n))
        live = torch.ones(n, dtype=torch.bool) if c["sizes"] is None else c["sizes"][pg, off] != 0
        pg, off = pg[live], off[live]
        for name in ("k", "v"):
            codes, scales = pack(full[name][pg, :, off])
            c[name][pg, :, off] = codes
            c[name + "_scales"][pg, :, off, :dim // 16] = scales[..., :dim // 16]
    return c


def append(c, k, v, offsets, ids=None, sizes=None, scores=None, rows=slice(None)):
    """Appends float32 rows k and v [rows, kv_heads, dim] in place to c; returns the new lengths."""
    out = {"k": k, "v": v}
    new = c["lengths"].clone()
    for i in range(len(offsets) - 1):
        t = i if ids is None else int(ids[i])
        a, e, at = int(offsets[i]), int(offsets[i + 1]), int(c["lengths"][t])
        pg, off = ref.places(c, t, torch.arange(at, at + e - a))
        for name, x in out.items():
            c[name][pg, :, off], c[name + "_scales"][pg, :, off] = pack(x[a:e].contiguous())
        if c["sizes"] is not None:
            c["sizes"][pg, off] = sizes[a:e] if sizes is not None else torch.ones(e - a)
        if c["weights"] is not None:
            c["weights"][pg, off] = scores[a:e] if scores is not None else torch.zeros(e - a)
        new[t] = at + e - a
    return new


def attention(c, q, dtype, *, scale=None, window=0, sinks=0):
    """(out, tolerance, weights, tolerance): out [batch, heads, dim] and the accumulated weights in 64 bits.

    The tolerances count the roundings.  A query times a power of two enters as one float16, which holds bf16's 8 bits (dims
    below 2^-31 of the largest: off by 2^-39 of it), or as two for float32, off by 2^-11 2^-11.  A logit (base e) sums `dim`
    products in float32, whose sums the matrix instruction may cut off instead of rounding: (dim + 4) 2^-23 scale sum|q k|,
    and a few steps of its own; so a probability is off by a factor 1 + d, d twice that, plus 2^-20 for the exponential.  It
    enters the second product as a float16 (two), off by 2^-11 (2^-22) of itself or, below float16's normal numbers, by
    2^-25 where the sum of probabilities is at least 2^7.  Sums over n tokens in float32, four at a time at least, lose
    (n / 4 + 64) 2^-23 of the sum of magnitudes.  The output is rounded to bf16 by 2^-8 at most."""
    batch, heads, dim = q.shape
    kv = c["k"].shape[1]
    group = heads // kv
    scale = dim ** -0.5 if scale is None else scale
    out, tol = torch.zeros((batch, heads, dim), dtype=torch.float64), torch.zeros((batch, heads, dim), dtype=torch.float64)
    w = None if c["weights"] is None else c["weights"].double()
    wtol = None if w is None else torch.zeros_like(w)
    for b in range(batch):
        pos = ref.visible(int(c["lengths"][b]), window, sinks)
        at = ref.places(c, b, pos)
        if c["sizes"] is not None:
            pos = pos[c["sizes"][at] != 0]
            at = ref.places(c, b, pos)
        n = len(pos)
        if n == 0:
            continue
        k, v = (unpack(c[name][at[0], :, at[1]], c[name + "_scales"][at[0], :, at[1]]).repeat_interleave(group, dim=1) for name in ("k", "v"))
        qb = q[b].double()
        x = torch.einsum("hd,nhd->hn", qb, k) * scale
        mag = torch.einsum("hd,nhd->hn", qb.abs(), k.abs()) * abs(scale)
        small = torch.einsum("h,nhd->hn", qb.abs().amax(1), k.abs()) * abs(scale) * 2.0 ** -39
        if c["sizes"] is not None:
            x = x + torch.log(c["sizes"][at].double())
        p = torch.exp(x - x.max(1, keepdim=True).values)
        p = p / p.sum(1, keepdim=True)
        step = (dim + 4) * 2.0 ** -23 + (2.0 ** -22 if dtype == "f32" else 0.0)
        d = 2 * ((step * mag + small).max(1).values + 4 * 2.0 ** -24 * x.abs().max(1).values) + 2.0 ** -20
        d = torch.expm1(d) + (n / 4 + 64) * 2.0 ** -23
        out[b] = torch.einsum("hn,nhd->hd", p, v)
        a = torch.einsum("hn,nhd->hd", p, v.abs())
        tol[b] = (2 * d[:, None] + (2.0 ** -22 if dtype == "f32" else 2.0 ** -11)) * a + 2.0 ** -32 * v.abs().sum(0)
        tol[b] += 2.0 ** -24 * out[b].abs() + 1e-37
        if dtype == "bf16":
            tol[b] += 2.0 ** -8 * out[b].abs()
        if w is not None:
            w[at] += p.sum(0)
            wtol[at] = 2 * (d[:, None] * p).sum(0) + (heads + 1) * 2.0 ** -24 * w[at].abs()
    return out, tol, w, wtol


def evict(c, budget, *, sinks=0, recent=0, table_out=None):
    """Evicts in place in c (or into table_out's pages); returns (new lengths, kept positions per sequence)."""
    plain = {name: c[name].clone() for name in ("k_scales", "v_scales")}
    before = ref.copy(c)
    new, keeps = ref.evict(c, budget, sinks=sinks, recent=recent, table_out=table_out)
    for b, keep in enumerate(keeps):   # the scales as the codes
        src = ref.places(before, b, torch.tensor(keep, dtype=torch.long))
        dst = ref.places(before, b, torch.arange(len(keep)), table_out)
        for name, old in plain.items():
            c[name][dst[0], :, dst[1]] = old[src[0], :, src[1]]
    return new, keeps
