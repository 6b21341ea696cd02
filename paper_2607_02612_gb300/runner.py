"""Python-side plumbing around the C ABI: device buffers, output allocation,
stage chains and CUDA-graph capture.  torch provides memory and streams only;
every step of the computation runs in libfusion.so.
"""
from __future__ import annotations

from dataclasses import dataclass, field
from typing import Dict, List, Optional

import numpy as np
import torch

from . import _binding as fb

DTYPE_CODE = {"f32": fb.FUSION_F32, "bf16": fb.FUSION_BF16}
TORCH_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def tokens_to_torch(a: np.ndarray, dtype: str, device) -> torch.Tensor:
    """float32 array or bf16 bit patterns (uint16) -> device tensor of the storage dtype."""
    a = np.ascontiguousarray(a)
    if dtype == "bf16":
        return torch.from_numpy(a.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(a.astype(np.float32, copy=False)).to(device)


def tokens_to_numpy(t: torch.Tensor, dtype: str) -> np.ndarray:
    """Device tensor -> float32 array or bf16 bit patterns (uint16)."""
    if dtype == "bf16":
        return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
    return t.float().cpu().numpy()


@dataclass
class DeviceBatch:
    """A ragged token batch on the device plus the host-side bounds the C ABI needs."""
    dtype: str
    dim: int
    max_batch: int
    max_tokens: int
    max_rows: int
    x: torch.Tensor
    keys: torch.Tensor
    sizes: torch.Tensor
    scores: Optional[torch.Tensor]
    offsets: torch.Tensor
    batch: Optional[torch.Tensor] = None
    ids: Optional[torch.Tensor] = None

    @property
    def key_dim(self) -> int:
        return int(self.keys.shape[1])

    def ragged(self) -> fb.fusion_ragged:
        return fb.ragged(self.max_batch, self.max_tokens, self.max_rows, self.offsets, self.batch, self.ids)


def device_batch(dtype: str, offsets, x, keys, sizes, scores, ids=None, max_tokens=None,
                 device="cuda") -> DeviceBatch:
    offsets = np.asarray(offsets, np.int32)
    B = len(offsets) - 1
    xt = tokens_to_torch(x, dtype, device)
    kt = xt if keys is x else tokens_to_torch(keys, dtype, device)
    if max_tokens is None:
        max_tokens = int(np.max(np.diff(offsets))) if B > 0 else 1
    return DeviceBatch(
        dtype=dtype, dim=int(xt.shape[1]), max_batch=B, max_tokens=int(max_tokens), max_rows=int(xt.shape[0]),
        x=xt, keys=kt, sizes=torch.from_numpy(np.asarray(sizes, np.float32)).to(device),
        scores=None if scores is None else torch.from_numpy(np.asarray(scores, np.float32)).to(device),
        offsets=torch.from_numpy(offsets).to(device),
        ids=None if ids is None else torch.from_numpy(np.asarray(ids, np.int32)).to(device))


@dataclass(frozen=True)
class RaggedRows:
    """The samples that rows belong to, without the rows (a DeviceBatch describes its own in the same way)."""
    max_batch: int
    max_tokens: int
    max_rows: int
    offsets: torch.Tensor
    batch: Optional[torch.Tensor] = None
    ids: Optional[torch.Tensor] = None

    def __post_init__(self):
        index = self.offsets.get_device()
        _need(self.offsets, torch.int32, index, "offsets", self.max_batch + 1)
        _need(self.batch, torch.int32, index, "batch", 1)
        _need(self.ids, torch.int32, index, "ids", self.max_batch)
        object.__setattr__(self, "_c", fb.ragged(self.max_batch, self.max_tokens, self.max_rows, self.offsets, self.batch,
                                                 self.ids))

    def ragged(self) -> fb.fusion_ragged:
        return self._c


def _enqueue(call, device: int, status: torch.Tensor, *args) -> None:
    """A call of the C ABI on the device's current torch stream, the device made the current one (without a context
    object where it is already, which is 1.5 us of the host's time); the status word is its last argument but the stream."""
    if status.get_device() != device:
        raise fb.FusionError("the status word and the cache are on different devices")
    stream = torch._C._cuda_getCurrentRawStream(device)
    if torch._C._cuda_getDevice() == device:   # (a third of torch.cuda.current_device()'s time)
        rc = call(*args, status.data_ptr(), stream)
    else:
        with torch.cuda.device(device):
            rc = call(*args, status.data_ptr(), stream)
    if rc:
        fb.check(rc)


def _rows_ptr(t: torch.Tensor, rows: int, heads: int, head_dim: int, dtype: torch.dtype, device: int, what: str):
    """Address and row stride of `rows` rows, [rows, heads * dim] or [rows, heads, dim], any stride between rows and
    contiguous inside one; device: an index (-1: the host)."""
    shape, width = t.shape, heads * head_dim
    if t.is_contiguous() and (shape == (rows, heads, head_dim) or shape == (rows, width)):   # (the usual case, in half the time)
        ok, stride = True, width
    else:
        ok, stride = len(shape) in (2, 3) and shape[0] >= rows, width
        if ok and len(shape) == 2:
            ok = shape[1] == width and (width == 1 or t.stride(1) == 1)
        elif ok:
            ok = shape[1] == heads and shape[2] == head_dim and t.stride(2) == 1 and (heads == 1 or t.stride(1) == head_dim)
        if ok and shape[0] > 1:
            stride = t.stride(0)
    if not ok or t.dtype != dtype or t.get_device() != device:
        raise fb.FusionError(f"{what}: at least {rows} {dtype} rows of {heads} x {head_dim} elements on device {device}, "
                             "contiguous inside a row, expected")
    return t.data_ptr(), stride


def _need(t: Optional[torch.Tensor], dtype: torch.dtype, device: int, what: str, least: int = 0, dim: int = 1):
    """The address of t (None: None), a contiguous tensor of this type on this device, of `dim` dimensions and at least
    `least` elements."""
    if t is None:
        return None
    if t.dtype != dtype or t.get_device() != device or t.dim() != dim or t.numel() < least or not t.is_contiguous():
        raise fb.FusionError(f"{what}: a contiguous {dim}-dimensional {dtype} tensor of at least {least} elements on device "
                             f"{device} expected")
    return t.data_ptr()


def _tokens(n: int, what: str) -> int:
    """A number of tokens for the C ABI; one that its 32 bits do not hold is more than any cache has, and means all."""
    if n < 0:
        raise fb.FusionError(f"{what}: a number >= 0 expected")
    return n if n < 1 << 31 else (1 << 31) - 1


@dataclass
class DeviceCache:
    """A paged key-value cache on the device (fusion_cache) with the scratch of its calls, which also fixes the number
    of query heads.  The tensors are changed in place, not replaced.  Calls that may overlap on the device (on other streams,
    or in graphs that do) need a cache object each."""
    dtype: str
    heads: int
    k: torch.Tensor            # [num_pages, kv_heads, page_tokens, head_dim]
    v: torch.Tensor
    page_table: torch.Tensor   # [max_batch, max_pages] int32
    lengths: torch.Tensor      # [max_batch] int32
    sizes: Optional[torch.Tensor] = None     # [num_pages, page_tokens] float32
    weights: Optional[torch.Tensor] = None
    workspace: torch.Tensor = field(init=False)
    ws_bytes: int = field(init=False)

    def __post_init__(self):
        pages, kv_heads, page_tokens, dim = self.k.shape
        ok = self.k.dtype == self.v.dtype == TORCH_DTYPE[self.dtype] and self.v.shape == self.k.shape
        ok = ok and self.page_table.dim() == 2 and self.page_table.dtype == torch.int32
        ok = ok and self.lengths.shape == self.page_table.shape[:1] and self.lengths.dtype == torch.int32
        for t in (self.sizes, self.weights):
            ok = ok and (t is None or (t.shape == (pages, page_tokens) and t.dtype == torch.float32))
        ok = ok and all(t is None or t.device == self.k.device
                        for t in (self.v, self.page_table, self.lengths, self.sizes, self.weights))
        if not ok:
            raise fb.FusionError("cache tensors of the wrong shape, type or device")
        self.max_batch, self.max_pages = (int(n) for n in self.page_table.shape)
        self.kv_heads, self.page_tokens, self.head_dim = int(kv_heads), int(page_tokens), int(dim)
        if not self.k.is_cuda:
            raise fb.FusionError("device tensors expected")
        self._c = fb.cache(self.max_batch, self.max_pages, page_tokens, kv_heads, dim, pages, self.k, self.v, self.sizes,
                           self.weights, self.page_table, self.lengths)
        self.ws_bytes = fb.fusion_cache_workspace_size(self._c, self.heads)
        if self.ws_bytes == 0:
            raise fb.FusionError("cache shape or number of heads out of range")
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.k.device)
        self.workspace[:1 << 18].zero_()   # the counters; the rest need not be zero
        self.device, self.index = self.k.device, self.k.get_device()
        self.code, self.torch_dtype = DTYPE_CODE[self.dtype], TORCH_DTYPE[self.dtype]
        self.scale = self.head_dim ** -0.5
        self.lib = fb.load()
        self._ws = self.workspace.data_ptr()
        self._one = RaggedRows(self.max_batch, 1, self.max_batch,
                               torch.arange(self.max_batch + 1, dtype=torch.int32, device=self.device))

    def c_struct(self) -> fb.fusion_cache:
        return self._c

    def one_row_each(self) -> RaggedRows:
        """A row per sequence, in the sequences' order."""
        return self._one


def cache_of(dtype: str, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor, *, heads: int,
             sizes: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None) -> DeviceCache:
    """A cache over the caller's pools, page table and lengths."""
    return DeviceCache(dtype, int(heads), k, v, page_table, lengths, sizes, weights)


def device_cache(dtype: str, max_batch: int, max_tokens: int, heads: int, kv_heads: int, head_dim: int, *,
                 page_tokens: int = 16, sizes: bool = False, weights: bool = False, device="cuda") -> DeviceCache:
    """An empty cache with room for max_tokens tokens in each sequence, its pages laid out one sequence after another."""
    per = -(-max_tokens // page_tokens)
    pages = max(1, max_batch * per)
    pool = lambda: torch.zeros((pages, kv_heads, page_tokens, head_dim), dtype=TORCH_DTYPE[dtype], device=device)   # noqa: E731
    per_token = lambda on: torch.zeros((pages, page_tokens), dtype=torch.float32, device=device) if on else None   # noqa: E731
    table = torch.arange(max_batch * per, dtype=torch.int32, device=device).view(max_batch, per)
    return DeviceCache(dtype, heads, pool(), pool(), table, torch.zeros(max_batch, dtype=torch.int32, device=device),
                       per_token(sizes), per_token(weights))


@dataclass
class HeadTensors:
    gamma: torch.Tensor
    beta: torch.Tensor
    eps: float
    weight: torch.Tensor
    bias: torch.Tensor
    tau: float

    @property
    def classes(self) -> int:
        return int(self.weight.shape[0])

    def c_struct(self) -> fb.fusion_exit_head:
        return fb.exit_head(self.gamma, self.beta, self.eps, self.weight, self.bias, self.classes, self.tau)


def head_tensors(head, dtype: str, device="cuda") -> HeadTensors:
    return HeadTensors(tokens_to_torch(head.gamma, dtype, device), tokens_to_torch(head.beta, dtype, device),
                       float(head.eps), tokens_to_torch(head.weight, dtype, device),
                       torch.from_numpy(np.asarray(head.bias, np.float32)).to(device), float(head.tau))


@dataclass
class MlpHeadTensors:
    """An MLP exit head on the device (fusion_mlp_head)."""
    pool: int
    gamma: torch.Tensor
    beta: torch.Tensor
    eps: float
    w1: torch.Tensor
    b1: torch.Tensor
    w2: torch.Tensor
    b2: torch.Tensor
    tau: float

    @property
    def hidden(self) -> int:
        return int(self.w1.shape[0])

    @property
    def classes(self) -> int:
        return int(self.w2.shape[0])

    def c_struct(self) -> fb.fusion_mlp_head:
        return fb.mlp_head(self.pool, self.gamma, self.beta, self.eps, self.w1, self.b1, self.hidden, self.w2,
                           self.b2, self.classes, self.tau)


def mlp_head_tensors(head, dtype: str, device="cuda") -> MlpHeadTensors:
    f32 = lambda a: torch.from_numpy(np.asarray(a, np.float32)).to(device)   # noqa: E731
    return MlpHeadTensors(int(head.pool), tokens_to_torch(head.gamma, dtype, device),
                          tokens_to_torch(head.beta, dtype, device), float(head.eps),
                          tokens_to_torch(head.w1, dtype, device), f32(head.b1),
                          tokens_to_torch(head.w2, dtype, device), f32(head.b2), float(head.tau))


class Fusion:
    """Owns a zero-initialised workspace and a device status word; each method
    allocates its outputs and enqueues one C-ABI call on the current stream."""

    def __init__(self, max_batch: int, classes: int = 1, device="cuda"):
        self.device = torch.device(device)
        self.ws_bytes = fb.fusion_workspace_size(max_batch, classes)
        self.workspace = torch.zeros(self.ws_bytes, dtype=torch.uint8, device=self.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._mlp_ws: Optional[torch.Tensor] = None   # scratch of exit_check_mlp, sized at first use
        self.max_batch = max_batch
        self.classes = classes

    def _outputs(self, b: DeviceBatch, with_scores: bool) -> Dict[str, torch.Tensor]:
        dev = self.device
        return dict(
            x=torch.empty((b.max_rows, b.dim), dtype=TORCH_DTYPE[b.dtype], device=dev),
            sizes=torch.empty(b.max_rows, dtype=torch.float32, device=dev),
            scores=torch.empty(b.max_rows, dtype=torch.float32, device=dev) if with_scores else None,
            offsets=torch.zeros(b.max_batch + 1, dtype=torch.int32, device=dev),
            keep_idx=torch.full((b.max_rows,), -1, dtype=torch.int32, device=dev))

    def _exit_outputs(self, n: int, classes: int) -> Dict[str, torch.Tensor]:
        """Zeroed exit outputs out of one allocation (one fill on the device instead of three, and 10 us
        less of the host's time for each)."""
        k = n * classes
        z = torch.zeros(k + n + (n + 3) // 4, dtype=torch.float32, device=self.device)
        return dict(exit_mask=z[k + n:].view(torch.uint8)[:n], logits=z[:k].view(n, classes), max_prob=z[k:k + n])

    def merge(self, b: DeviceBatch, r: torch.Tensor, *, dst_map=True, a_match=True) -> Dict[str, torch.Tensor]:
        o = self._outputs(b, b.scores is not None)
        o["dst_map"] = torch.full((b.max_rows,), -1, dtype=torch.int32, device=self.device) if dst_map else None
        o["a_match"] = torch.full((b.max_rows,), -1, dtype=torch.int32, device=self.device) if a_match else None
        fb.check(fb.fusion_merge(DTYPE_CODE[b.dtype], b.ragged(), b.x, b.dim, b.keys, b.key_dim, b.sizes,
                                 b.scores, r, o["x"], o["sizes"], o["scores"], o["offsets"], o["keep_idx"],
                                 o["dst_map"], o["a_match"], self.workspace, self.ws_bytes, self.status))
        return o

    def merge_router(self, b: DeviceBatch, w: torch.Tensor, beta: float, tau_tgt: float, tau_ref: float,
                     out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
        """Merge counts r (by original id) from the router with profile scaling (Eq. 4-5)."""
        o = out if out is not None else dict(
            r=torch.zeros(b.max_batch, dtype=torch.int32, device=self.device),
            m=torch.zeros(b.max_batch, dtype=torch.float32, device=self.device))
        fb.check(fb.fusion_merge_router(DTYPE_CODE[b.dtype], b.ragged(), b.x, b.dim, w, beta, tau_tgt, tau_ref,
                                        o["r"], o["m"], self.status))
        return o

    def token_scores(self, b: DeviceBatch, w: torch.Tensor, bias: float,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Prune scores s = w . z + bias of every token row from a linear pruning router (Eq. 8)."""
        o = out if out is not None else torch.zeros(b.max_rows, dtype=torch.float32, device=self.device)
        fb.check(fb.fusion_token_scores(DTYPE_CODE[b.dtype], b.ragged(), b.x, b.dim, w, bias, o, self.status))
        return o

    def exit_check_mlp(self, b: DeviceBatch, head: "MlpHeadTensors") -> Dict[str, torch.Tensor]:
        """Exit check with an MLP exit head (SpatialPool or CLS-only), its own scratch."""
        o = self._exit_outputs(b.max_batch, head.classes)
        ws, nbytes = self.mlp_workspace(b, head)
        fb.check(fb.fusion_exit_check_mlp(DTYPE_CODE[b.dtype], b.ragged(), b.x, b.dim, b.sizes, head.c_struct(),
                                          o["exit_mask"], o["logits"], o["max_prob"], ws, nbytes, self.status))
        return o

    def mlp_workspace(self, b: DeviceBatch, head: "MlpHeadTensors"):
        """The zero-filled scratch of the MLP-head calls (it grows to the largest head seen;
        a Chain sizes it for all its stages before any graph capture)."""
        # the stage's size covers the exit check alone too (its layout starts with the same scratch)
        nbytes = fb.fusion_stage_mlp_workspace_size(b.max_batch, b.max_rows, b.dim, head.hidden, head.classes)
        if self._mlp_ws is None or self._mlp_ws.numel() < nbytes:
            self._mlp_ws = torch.zeros(nbytes, dtype=torch.uint8, device=self.device)
        return self._mlp_ws, nbytes

    def attention(self, b: DeviceBatch, qkv: torch.Tensor, heads: int, sizes: Optional[torch.Tensor] = None,
                  out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Size-aware attention of the batch's samples: qkv [max_rows, 3 * heads * 64] bf16, sizes
        [max_rows] (None: plain attention); returns [max_rows, heads * 64] bf16."""
        o = out if out is not None else torch.zeros((b.max_rows, heads * fb.FUSION_ATTN_HEAD_DIM),
                                                    dtype=torch.bfloat16, device=self.device)
        fb.check(fb.fusion_attention(DTYPE_CODE["bf16"], b.ragged(), qkv, heads, fb.FUSION_ATTN_HEAD_DIM, sizes, o,
                                     self.status))
        return o

    def cache_append(self, c: DeviceCache, k: torch.Tensor, v: torch.Tensor, rows=None, *,
                     sizes: Optional[torch.Tensor] = None, scores: Optional[torch.Tensor] = None,
                     lengths_out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Appends the rows of k and v ([rows, kv_heads * head_dim], any stride between rows) to the sequences that `rows`
        (a DeviceBatch or RaggedRows; None: one row per sequence) says; returns the new lengths (the cache's own, raised
        in place, unless lengths_out is given)."""
        o = lengths_out if lengths_out is not None else c.lengths
        if c.max_batch == 0:
            return o
        if rows is None:
            rows = c.one_row_each()
        elif any(t is not None and t.get_device() != c.index for t in (rows.offsets, rows.batch, rows.ids)):
            raise fb.FusionError(f"the rows' offsets, count and ids on the cache's device ({c.index}) expected")
        kp, ks = _rows_ptr(k, rows.max_rows, c.kv_heads, c.head_dim, c.torch_dtype, c.index, "keys")
        vp, vs = _rows_ptr(v, rows.max_rows, c.kv_heads, c.head_dim, c.torch_dtype, c.index, "values")
        zp = _need(sizes, torch.float32, c.index, "sizes", rows.max_rows)
        wp = _need(scores, torch.float32, c.index, "scores", rows.max_rows)
        op = _need(o, torch.int32, c.index, "lengths_out", c.max_batch)
        _enqueue(c.lib.fusion_cache_append, c.index, self.status, c.code, c.c_struct(), rows.ragged(), kp, ks, vp, vs, zp,
                 wp, op, c._ws, c.ws_bytes)
        return o

    def cache_attention(self, c: DeviceCache, q: torch.Tensor, *, scale: Optional[float] = None, window: int = 0,
                        sinks: int = 0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of one new token per sequence, q [max_batch, heads, head_dim] (any stride between sequences), over
        the visible tokens of its cache; accumulates the weights where the cache keeps them.  scale None:
        head_dim ** -0.5.  Returns [max_batch, heads, head_dim] (out, where it is given; rows behind the last sequence's stay)."""
        qp, qs = _rows_ptr(q, c.max_batch, c.heads, c.head_dim, c.torch_dtype, c.index, "queries")
        if out is None:
            out = torch.empty((c.max_batch, c.heads, c.head_dim), dtype=c.torch_dtype, device=c.device)
            op = out.data_ptr()
        else:
            op = _need(out, c.torch_dtype, c.index, "out", dim=3)
            if out.shape[0] < c.max_batch or out.shape[1] != c.heads or out.shape[2] != c.head_dim:
                raise fb.FusionError(f"out: [{c.max_batch}, {c.heads}, {c.head_dim}] expected")
        if c.max_batch == 0:
            return out
        _enqueue(c.lib.fusion_cache_attention, c.index, self.status, c.code, c.c_struct(), qp, qs, c.heads,
                 c.scale if scale is None else scale, _tokens(window, "window"), _tokens(sinks, "sinks"), op, c._ws, c.ws_bytes)
        return out

    def cache_evict(self, c: DeviceCache, budget: torch.Tensor, *, sinks: int = 0, recent: int = 0,
                    page_table_out: Optional[torch.Tensor] = None, lengths_out: Optional[torch.Tensor] = None,
                    keep_idx: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Prunes each sequence to budget[b] tokens by accumulated weight, in place or into other pages; keep_idx
        [max_batch, n] receives the kept positions.  Returns the new lengths (the cache's own unless lengths_out is given)."""
        o = lengths_out if lengths_out is not None else c.lengths
        if c.max_batch == 0:
            return o
        op = _need(o, torch.int32, c.index, "lengths_out", c.max_batch)
        bp = _need(budget, torch.int32, c.index, "budget", c.max_batch)
        tp = _need(page_table_out, torch.int32, c.index, "page_table_out", dim=2)
        kp = _need(keep_idx, torch.int32, c.index, "keep_idx", dim=2)
        for t, what in ((page_table_out, "page_table_out"), (keep_idx, "keep_idx")):
            if t is not None and t.shape[0] < c.max_batch:
                raise fb.FusionError(f"{what}: a row per sequence expected")
        _enqueue(c.lib.fusion_cache_evict, c.index, self.status, c.code, c.c_struct(), bp, _tokens(sinks, "sinks"),
                 _tokens(recent, "recent"), tp, page_table_out.shape[1] if tp is not None else 0, op, kp,
                 keep_idx.shape[1] if kp is not None else 0, c._ws, c.ws_bytes)
        return o

    def exit_check(self, b: DeviceBatch, head: HeadTensors) -> Dict[str, torch.Tensor]:
        o = self._exit_outputs(b.max_batch, head.classes)
        fb.check(fb.fusion_exit_check(DTYPE_CODE[b.dtype], b.ragged(), b.x, b.dim, head.c_struct(),
                                      o["exit_mask"], o["logits"], o["max_prob"], self.workspace, self.ws_bytes,
                                      self.status))
        return o

    def prune(self, b: DeviceBatch, rho: torch.Tensor) -> Dict[str, torch.Tensor]:
        o = self._outputs(b, True)
        fb.check(fb.fusion_prune(DTYPE_CODE[b.dtype], b.ragged(), b.x, b.dim, b.sizes, b.scores, rho, o["x"],
                                 o["sizes"], o["scores"], o["offsets"], o["keep_idx"], self.workspace,
                                 self.ws_bytes, self.status))
        return o

    def compact(self, b: DeviceBatch, exit_mask: torch.Tensor) -> Dict[str, torch.Tensor]:
        o = self._outputs(b, b.scores is not None)
        o["ids"] = torch.zeros(b.max_batch, dtype=torch.int32, device=self.device)
        o["batch"] = torch.zeros(1, dtype=torch.int32, device=self.device)
        fb.check(fb.fusion_compact(DTYPE_CODE[b.dtype], b.ragged(), b.x, b.dim, b.sizes, b.scores, exit_mask,
                                   o["x"], o["sizes"], o["scores"], o["offsets"], o["ids"], o["batch"],
                                   o["keep_idx"], self.workspace, self.ws_bytes, self.status))
        return o

    def stage(self, b: DeviceBatch, flags: int, r=None, rho=None, head: Optional[HeadTensors] = None,
              a_match: bool = False, out: Optional[Dict[str, torch.Tensor]] = None,
              mlp_head: Optional["MlpHeadTensors"] = None) -> Dict[str, torch.Tensor]:
        """One fused stage; the exit check uses `head` (linear) or `mlp_head` (an MLP exit head)."""
        o = out if out is not None else self.stage_outputs(b, flags, head, a_match, mlp_head=mlp_head)
        if mlp_head is not None:
            ws, nbytes = self.mlp_workspace(b, mlp_head)
            fb.check(fb.fusion_stage_mlp(
                DTYPE_CODE[b.dtype], flags, b.ragged(), b.x, b.dim, b.keys, b.key_dim, b.sizes, b.scores, r, rho,
                mlp_head.c_struct(), o["exit_mask"], o["logits"], o["max_prob"], o["x"], o["sizes"], o["scores"],
                o["offsets"], o["ids"], o["batch"], o["keep_idx"], o.get("a_match"), ws, nbytes, self.status))
            return o
        fb.check(fb.fusion_stage(
            DTYPE_CODE[b.dtype], flags, b.ragged(), b.x, b.dim, b.keys, b.key_dim, b.sizes, b.scores, r, rho,
            head.c_struct() if head is not None else None, o["exit_mask"], o["logits"], o["max_prob"], o["x"],
            o["sizes"], o["scores"], o["offsets"], o["ids"], o["batch"], o["keep_idx"], o.get("a_match"),
            self.workspace, self.ws_bytes, self.status))
        return o

    def stage_outputs(self, b: DeviceBatch, flags: int, head: Optional[HeadTensors], a_match: bool = False,
                      mlp_head: Optional["MlpHeadTensors"] = None):
        dev = self.device
        o = self._outputs(b, b.scores is not None)
        o["ids"] = torch.zeros(b.max_batch, dtype=torch.int32, device=dev)
        o["batch"] = torch.zeros(1, dtype=torch.int32, device=dev)
        has_exit = bool(flags & fb.FUSION_STAGE_EXIT)
        o["exit_mask"] = torch.zeros(b.max_batch, dtype=torch.uint8, device=dev) if has_exit else None
        classes = (mlp_head or head).classes if has_exit else 0
        o["logits"] = torch.zeros((b.max_batch, classes), dtype=torch.float32, device=dev) if has_exit else None
        o["max_prob"] = torch.zeros(b.max_batch, dtype=torch.float32, device=dev) if has_exit else None
        o["a_match"] = torch.full((b.max_rows,), -1, dtype=torch.int32, device=dev) if a_match else None
        return o


def output_batch(b: DeviceBatch, o: Dict[str, torch.Tensor]) -> DeviceBatch:
    """The batch a stage hands to the next block (keys alias the new tokens)."""
    return DeviceBatch(dtype=b.dtype, dim=b.dim, max_batch=b.max_batch, max_tokens=b.max_tokens,
                       max_rows=b.max_rows, x=o["x"], keys=o["x"], sizes=o["sizes"], scores=o["scores"],
                       offsets=o["offsets"], batch=o["batch"], ids=o["ids"])


@dataclass
class ChainStage:
    flags: int
    r: Optional[torch.Tensor] = None
    rho: Optional[torch.Tensor] = None
    head: Optional[HeadTensors] = None
    mlp_head: Optional[MlpHeadTensors] = None   # an MLP exit head in place of `head`


@dataclass
class Chain:
    """A schedule of stages over pre-allocated buffers; stage s+1 reads what stage s wrote.
    run() enqueues every stage on the current stream with no host synchronisation."""
    fusion: Fusion
    inp: DeviceBatch
    stages: List[ChainStage]
    outs: List[Dict[str, torch.Tensor]] = field(default_factory=list)
    batches: List[DeviceBatch] = field(default_factory=list)

    def __post_init__(self):
        b = self.inp
        for st in self.stages:
            o = self.fusion.stage_outputs(b, st.flags, st.head, mlp_head=st.mlp_head)
            if st.mlp_head is not None:
                self.fusion.mlp_workspace(b, st.mlp_head)   # sized before any capture
            self.outs.append(o)
            self.batches.append(b)
            b = output_batch(b, o)

    def run_stage(self, s: int, stream=None):
        st, b, o = self.stages[s], self.batches[s], self.outs[s]
        if st.mlp_head is not None:
            ws, nbytes = self.fusion.mlp_workspace(b, st.mlp_head)
            fb.check(fb.fusion_stage_mlp(
                DTYPE_CODE[b.dtype], st.flags, b.ragged(), b.x, b.dim, b.keys, b.key_dim, b.sizes, b.scores, st.r,
                st.rho, st.mlp_head.c_struct(), o["exit_mask"], o["logits"], o["max_prob"], o["x"], o["sizes"],
                o["scores"], o["offsets"], o["ids"], o["batch"], o["keep_idx"], None, ws, nbytes, self.fusion.status,
                stream))
            return
        fb.check(fb.fusion_stage(
            DTYPE_CODE[b.dtype], st.flags, b.ragged(), b.x, b.dim, b.keys, b.key_dim, b.sizes, b.scores, st.r,
            st.rho, st.head.c_struct() if st.head is not None else None, o["exit_mask"], o["logits"],
            o["max_prob"], o["x"], o["sizes"], o["scores"], o["offsets"], o["ids"], o["batch"], o["keep_idx"],
            None, self.fusion.workspace, self.fusion.ws_bytes, self.fusion.status, stream))

    def run(self, stream=None):
        for s in range(len(self.stages)):
            self.run_stage(s, stream)

    def capture(self) -> torch.cuda.CUDAGraph:
        """Capture the whole chain as one CUDA graph (run() once before, eagerly)."""
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            self.run()
        return g

    def host_results(self) -> "HostResults":
        """Pinned host buffers sized for this chain's results (see HostResults)."""
        return HostResults(self)

    def clone(self) -> "Chain":
        """The same schedule over its own input, output and scratch buffers (the stage
        parameters, read only, are shared); the inputs start as a copy of this chain's."""
        b = self.inp
        x = b.x.clone()
        keys = x if b.keys is b.x else b.keys.clone()
        cp = lambda t: None if t is None else t.clone()   # noqa: E731
        inp = DeviceBatch(dtype=b.dtype, dim=b.dim, max_batch=b.max_batch, max_tokens=b.max_tokens,
                          max_rows=b.max_rows, x=x, keys=keys, sizes=b.sizes.clone(), scores=cp(b.scores),
                          offsets=b.offsets.clone(), batch=cp(b.batch), ids=cp(b.ids))
        fus = Fusion(self.fusion.max_batch, self.fusion.classes, self.fusion.device)
        return Chain(fus, inp, list(self.stages))


class HostResults:
    """Pinned host copies of a chain's results: the survivors of the last stage (count,
    offsets, ids, sizes, token rows), every exit check's mask and max probability over the
    images entering it, and the device status word.

    fetch() runs on the current stream after the chain was enqueued: one asynchronous copy
    of the fixed-size parts (the count, the offsets bound, the exit outputs), one host wait,
    then copies of the survivors' exact extent and a second wait.  Returns host views
    (valid until the next fetch) and the number of bytes copied."""

    def __init__(self, chain: Chain):
        last = chain.outs[-1]
        self._last = last
        self._exits = [(o["exit_mask"], o["max_prob"]) for o in chain.outs if o["exit_mask"] is not None]
        # images entering each exit check (None: the whole input batch)
        self._exit_in = [b.batch for b, o in zip(chain.batches, chain.outs) if o["exit_mask"] is not None]
        self._exit_max = [b.max_batch for b, o in zip(chain.batches, chain.outs) if o["exit_mask"] is not None]
        pin = lambda t: torch.empty(t.shape, dtype=t.dtype).pin_memory()   # noqa: E731
        self.batch = pin(last["batch"])
        self.offsets = pin(last["offsets"])
        self.ids = pin(last["ids"])
        self.sizes = pin(last["sizes"])
        self.x = pin(last["x"])
        self.exits = [(pin(m), pin(p)) for m, p in self._exits]
        self.exit_in = [None if t is None else pin(t) for t in self._exit_in]
        self._status = chain.fusion.status
        self.status = pin(self._status)

    def fetch(self):
        self.fetch_fixed()
        torch.cuda.current_stream().synchronize()
        self.fetch_exact()
        torch.cuda.current_stream().synchronize()
        return self.result()

    def fetch_fixed(self):
        """Enqueue (current stream) the copies whose size the host knows: the survivor count,
        the offsets bound and the exit outputs."""
        last = self._last
        self.batch.copy_(last["batch"], non_blocking=True)
        self.offsets.copy_(last["offsets"], non_blocking=True)
        self.status.copy_(self._status, non_blocking=True)
        self._n = self.batch.numel() * 4 + self.offsets.numel() * 4 + 4
        for (hm, hp), (m, p), hc, c in zip(self.exits, self._exits, self.exit_in, self._exit_in):
            hm.copy_(m, non_blocking=True)
            hp.copy_(p, non_blocking=True)
            self._n += hm.numel() * hm.element_size() + hp.numel() * hp.element_size()
            if hc is not None:
                hc.copy_(c, non_blocking=True)
                self._n += 4

    def fetch_exact(self):
        """Enqueue (current stream) the survivors' rows; the fixed copies must have landed."""
        last = self._last
        self._nb = int(self.batch[0])
        self._rows = int(self.offsets[self._nb])
        for name, k in (("ids", self._nb), ("sizes", self._rows), ("x", self._rows)):
            h = getattr(self, name)
            h[:k].copy_(last[name][:k], non_blocking=True)
            self._n += h[:k].numel() * h.element_size()

    def result(self):
        nb, rows = self._nb, self._rows
        res = {"batch": nb, "offsets": self.offsets[:nb + 1], "ids": self.ids[:nb], "sizes": self.sizes[:rows],
               "x": self.x[:rows], "status": int(self.status[0]), "exits": []}
        for (hm, hp), hc, mx in zip(self.exits, self.exit_in, self._exit_max):
            n = mx if hc is None else int(hc[0])
            res["exits"].append((hm[:n], hp[:n]))
        return res, self._n


class Pipeline:
    """Back-to-back steps of one schedule with host inputs and host results, the copies
    overlapped with the computation: step k runs on slot k % 2 (a chain with its own
    buffers, replayed as a CUDA graph), its inputs are copied on one copy stream while step
    k - 1 computes, and its results come back on another.  The survivors' exact extent is
    known only once the host has read their count, so submit() of step k returns the results
    of step k - 1 (None for the first) and finish() those of the last step; host results stay
    valid until the next call.  Slots are not reused before their results are on the host."""

    def __init__(self, chain: Chain):
        self.chains = [chain, chain.clone()]
        self.graphs = []
        for ch in self.chains:
            ch.run()
            torch.cuda.synchronize()
            self.graphs.append(ch.capture())
        self.hr = [ch.host_results() for ch in self.chains]
        self.s_h2d, self.s_cmp, self.s_d2h = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.Stream()
        ev = lambda: [torch.cuda.Event(), torch.cuda.Event()]   # noqa: E731
        self.ev_h2d, self.ev_cmp, self.ev_cnt, self.ev_res = ev(), ev(), ev(), ev()
        self.k = 0
        self.pending: Optional[int] = None

    def _inputs(self, slot: int) -> Dict[str, torch.Tensor]:
        b = self.chains[slot].inp
        d = {"x": b.x.view(torch.int16) if b.dtype == "bf16" else b.x, "sizes": b.sizes, "offsets": b.offsets}
        if b.keys is not b.x:
            d["keys"] = b.keys.view(torch.int16) if b.dtype == "bf16" else b.keys
        if b.scores is not None:
            d["scores"] = b.scores
        return d

    def submit(self, host: Dict[str, torch.Tensor]):
        """host: pinned tensors named after the input fields (x as int16 bits for bf16)."""
        c = self.k % 2
        dst = self._inputs(c)
        with torch.cuda.stream(self.s_h2d):
            if self.k >= 2:
                self.s_h2d.wait_event(self.ev_cmp[c])   # the slot's previous replay read its inputs
            for name, t in host.items():
                dst[name].copy_(t, non_blocking=True)
            self.ev_h2d[c].record(self.s_h2d)
        with torch.cuda.stream(self.s_cmp):
            self.s_cmp.wait_event(self.ev_h2d[c])
            if self.k >= 2:
                self.s_cmp.wait_event(self.ev_res[c])   # the slot's previous results are on the host
            self.graphs[c].replay()
            self.ev_cmp[c].record(self.s_cmp)
        prev = self._complete()
        with torch.cuda.stream(self.s_d2h):
            self.s_d2h.wait_event(self.ev_cmp[c])
            self.hr[c].fetch_fixed()
            self.ev_cnt[c].record(self.s_d2h)
        self.pending = c
        self.k += 1
        return prev

    def _complete(self):
        p = self.pending
        if p is None:
            return None
        self.pending = None
        self.ev_cnt[p].synchronize()
        with torch.cuda.stream(self.s_d2h):
            self.hr[p].fetch_exact()
            self.ev_res[p].record(self.s_d2h)
        self.ev_res[p].synchronize()
        return self.hr[p].result()

    def finish(self):
        """Results of the last submitted step (None if there is none)."""
        return self._complete()

    def status(self) -> int:
        """OR of the slots' device status words (synchronises)."""
        torch.cuda.synchronize()
        return int(self.chains[0].fusion.status.item()) | int(self.chains[1].fusion.status.item())
