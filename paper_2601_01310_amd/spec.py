"""The operators of a speculative decode step around a paged KV cache, over
tensors: shapes, types and strides are checked here, the work runs in the
library's HIP kernels (``include/tg.h`` says what each computes).

Objects bind their tensors once, as :class:`tg.EwForward` does, so that a
decode loop's calls allocate nothing: new values go into the bound tensors in
place. A call runs on the tensors' device, whichever is current, on ``stream``
or on that device's current stream; who passes another stream than the tensors'
own orders it behind what filled them and keeps them until it is done. An object
has one workspace, one set of outputs and one argument block, so its calls follow
one another: one thread and one stream at a time (others behind an event), and an
object of its own for each that runs beside it. ::

    cache = KvCache.empty(n_layers=32, n_pages=4096, page_size=16, Hkv=8, D=128,
                          B=64, max_pages=64, device="cuda")
    cache.reserve(lengths, q_offsets, slots, status)
    attend = TreeAttention(cache, q, q_offsets, lengths, tree_mask)
    out = attend(layer=3)
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from . import tg

_DTYPES = {torch.bfloat16: tg.BF16, torch.float16: tg.F16}


def _want(t: Optional[torch.Tensor], name: str, dtype, shape=None, optional=False):
    """Checks one dense device tensor; None in ``shape`` is any size."""
    if t is None:
        if optional:
            return
        raise ValueError(f"{name} is required")
    if t.device.type != "cuda":
        raise ValueError(f"{name}: libtg takes device tensors only")
    if t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype}, {dtype} required")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and (t.dim() != len(shape) or any(
            n is not None and n != m for n, m in zip(shape, t.shape))):
        raise ValueError(f"{name} is {list(t.shape)}, {list(shape)} required")


def _rows(t: torch.Tensor, name: str, dtype, inner) -> int:
    """Checks [rows, *inner] with dense rows; returns the row stride (of one row,
    whose stride means nothing, one that is taken)."""
    if t.device.type != "cuda":
        raise ValueError(f"{name}: libtg takes device tensors only")
    if t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype}, {dtype} required")
    if t.dim() != 1 + len(inner) or tuple(t.shape[1:]) != tuple(inner):
        raise ValueError(f"{name} is {list(t.shape)}, [rows, {', '.join(map(str, inner))}] required")
    dense = 1
    for n, stride in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if n > 1 and stride != dense:
            raise ValueError(f"{name}: a row must be contiguous")
        dense *= n
    return t.stride(0) if t.shape[0] > 1 else -(-max(dense, t.stride(0)) // 8) * 8


_current_device = torch._C._cuda_getDevice
_current_stream = torch._C._cuda_getCurrentRawStream


def _run(call, device: int, stream, *args):
    """A call of the library with ``args`` and the stream. ``device``, the
    tensors', is made the current one for it: kernels start there, and a null
    stream is the current device's."""
    if stream is None:
        stream = _current_stream(device)
    elif not isinstance(stream, int):
        stream = stream.cuda_stream
    if _current_device() == device:
        status = call(*args, stream)
    else:
        with torch.cuda.device(device):
            status = call(*args, stream)
    if status != tg.TG_OK:
        raise tg.TgError(status, call.__name__)


def _int32(t: torch.Tensor, name: str, device: int, n: int, dim: int = 1) -> int:
    """Address of a dense int32 tensor on ``device`` with n elements (-1: any),
    checked in a few short calls: the page calls are a microsecond's work on
    the host otherwise."""
    if (t.dtype is torch.int32 and t.get_device() == device and t.dim() == dim
            and (n < 0 or t.numel() == n) and t.is_contiguous()):
        return t.data_ptr()
    _want(t, name, torch.int32, (None if n < 0 else n,) if dim == 1 else (None,) * dim)
    raise ValueError(f"{name} is {list(t.shape)} on {t.device}: not what the cache needs")


def _same_device(*tensors):
    devices = {t.device for t in tensors if t is not None}
    if len(devices) > 1:
        raise ValueError(f"tensors lie on several devices: {sorted(map(str, devices))}")


class KvCache:
    """Pages of K and V, [n_layers, n_pages, page_size, Hkv, D] (rows dense;
    layers and pages may be strided), the page table [B, max_pages] int32 (-1
    = no page), ``held`` [B] and ``refcount`` [n_pages] int32."""

    def __init__(self, k, v, page_table, held, refcount):
        if k.dtype not in _DTYPES:
            raise ValueError(f"k is {k.dtype}, bfloat16 or float16 required")
        if k.dim() != 5 or v.shape != k.shape or v.dtype != k.dtype or v.stride() != k.stride():
            raise ValueError("k and v must be [layers, pages, page_size, Hkv, D], alike in shape, "
                             "type and strides")
        layers, pages, size, Hkv, D = k.shape
        for n, stride, dense in ((size, k.stride(2), Hkv * D), (Hkv, k.stride(3), D),
                                 (D, k.stride(4), 1)):
            if n > 1 and stride != dense:
                raise ValueError("a page must be contiguous")
        if k.device.type != "cuda" or v.device.type != "cuda":
            raise ValueError("libtg takes device tensors only")
        _want(page_table, "page_table", torch.int32, (None, None))
        B, max_pages = page_table.shape
        _want(held, "held", torch.int32, (B,))
        _want(refcount, "refcount", torch.int32, (pages,))
        _same_device(k, v, page_table, held, refcount)
        self.k, self.v, self.page_table = k, v, page_table
        self.held, self.refcount = held, refcount
        a = self.args = tg.KvCacheArgs()
        a.dtype, a.n_layers, a.n_pages, a.page_size = _DTYPES[k.dtype], layers, pages, size
        a.Hkv, a.D, a.B, a.max_pages = Hkv, D, B, max_pages
        a.layer_stride = k.stride(0) if layers > 1 else 0
        a.page_stride = k.stride(1) if pages > 1 else size * Hkv * D
        a.k, a.v, a.page_table = k.data_ptr(), v.data_ptr(), page_table.data_ptr()
        a.held, a.refcount = held.data_ptr(), refcount.data_ptr()
        self._ref, self._device, self._lib = ctypes.byref(a), k.get_device(), tg.load()

    @classmethod
    def empty(cls, n_layers, n_pages, page_size, Hkv, D, B, max_pages, dtype=torch.bfloat16,
              device="cuda"):
        """A cache of its own: every page free, no request holds any. Pages
        start at zero."""
        k = torch.zeros((n_layers, n_pages, page_size, Hkv, D), dtype=dtype, device=device)
        ints = dict(dtype=torch.int32, device=device)
        return cls(k, torch.zeros_like(k), torch.full((B, max_pages), -1, **ints),
                   torch.zeros(B, **ints), torch.zeros(n_pages, **ints))

    def reserve(self, lengths, q_offsets, slots, status, stream=None):
        """Pages for the new rows, none of which others hold; fills ``slots`` [T]
        and ``status`` [B]."""
        B, d = self.args.B, self._device
        _run(self._lib.tg_kv_pages_reserve, d, stream, self._ref, _int32(lengths, "lengths", d, B),
             _int32(q_offsets, "q_offsets", d, B + 1), slots.shape[0],
             _int32(slots, "slots", d, -1), _int32(status, "status", d, B))

    def fork(self, lengths, src, dst, status, stream=None):
        """Requests ``dst`` become copies of ``src``; updates ``lengths``."""
        n, d = src.shape[0], self._device
        _run(self._lib.tg_kv_pages_fork, d, stream, self._ref,
             _int32(lengths, "lengths", d, self.args.B), _int32(src, "src", d, n),
             _int32(dst, "dst", d, n), n, _int32(status, "status", d, n))

    def trim(self, keep, stream=None):
        """Gives back the pages past ``keep`` [B] tokens of each request."""
        _run(self._lib.tg_kv_pages_trim, self._device, stream, self._ref,
             _int32(keep, "keep", self._device, self.args.B))

    def compact(self, path, n_keep, lengths, new_lengths, stream=None):
        """Moves the kept rows of every layer together (``path`` [B, max_path]
        and ``n_keep`` [B] as :class:`VerifyTree` returns them)."""
        B, d, most = self.args.B, self._device, path.shape[-1]
        _run(self._lib.tg_kv_compact, d, stream, self._ref, _int32(path, "path", d, B * most, 2),
             most, _int32(n_keep, "n_keep", d, B), _int32(lengths, "lengths", d, B),
             _int32(new_lengths, "new_lengths", d, B))


class QkNormRope:
    """Norms, rotation and cache rows of ``qkv`` [T, Hq + 2 Hkv, D]; returns the
    queries [T, Hq, D] (``q_out``, or a tensor of its own). ``cos_sin``
    [max_pos, rot] float32; ``rot`` 0 and no table: no rotation; no weights: no
    norms."""

    def __init__(self, cache: KvCache, qkv, Hq, positions, slots, cos_sin=None, q_weight=None,
                 k_weight=None, q_out=None, eps=1e-6, interleaved=False):
        c, dtype = cache.args, cache.k.dtype
        stride = _rows(qkv, "qkv", dtype, (Hq + 2 * c.Hkv, c.D))
        T = qkv.shape[0]
        if q_out is None:
            q_out = torch.empty((T, Hq, c.D), dtype=dtype, device=qkv.device)
        q_stride = _rows(q_out, "q_out", dtype, (Hq, c.D))
        if q_out.shape[0] != T:
            raise ValueError(f"q_out has {q_out.shape[0]} rows, {T} required")
        _want(slots, "slots", torch.int32, (T,))
        rot = 0 if cos_sin is None else cos_sin.shape[-1]
        _want(cos_sin, "cos_sin", torch.float32, (None, None), optional=True)
        _want(positions, "positions", torch.int32, (T,), optional=rot == 0)
        _want(q_weight, "q_weight", dtype, (c.D,), optional=True)
        _want(k_weight, "k_weight", dtype, (c.D,), optional=True)
        _same_device(cache.k, qkv, q_out, slots, cos_sin, positions, q_weight, k_weight)
        self._keep = (cache, qkv, positions, slots, cos_sin, q_weight, k_weight)
        self.q_out = q_out
        a = self.args = tg.QkArgs()
        a.cache, a.T, a.Hq, a.rot = c, T, Hq, rot
        a.interleaved, a.eps = int(interleaved), eps
        a.max_pos = 0 if cos_sin is None else cos_sin.shape[0]
        a.qkv_stride, a.q_out_stride = stride, q_stride
        for name, t in dict(qkv=qkv, q_weight=q_weight, k_weight=k_weight, cos_sin=cos_sin,
                            positions=positions, slots=slots, q_out=q_out).items():
            setattr(a, name, None if t is None else t.data_ptr())
        self._ref, self._device = ctypes.byref(a), qkv.get_device()
        self._call = tg.load().tg_qk_norm_rope

    def __call__(self, layer=0, stream=None):
        self.args.layer = layer
        _run(self._call, self._device, stream, self._ref)
        return self.q_out


def _mask(tree_mask, T) -> int:
    """Words per row of a [T, W] int64 mask; 0 for none."""
    if tree_mask is None:
        return 0
    _want(tree_mask, "tree_mask", torch.int64, (T, None))
    return tree_mask.shape[1]


class TreeAttention:
    """Attention of ``q`` [T, Hq, D] over the cache; returns ``out`` (a tensor
    of its own if not given). ``tree_mask`` [T, W] int64 (the bits of tg.h's
    uint64 words) or None for chains; ``max_nodes`` bounds a request's rows. By
    default T does, and the kernel is chosen for the mean, T / B: give it where
    some requests have many more rows than others."""

    def __init__(self, cache: KvCache, q, q_offsets, lengths, tree_mask=None, scale=None,
                 max_nodes=None, out=None):
        c, dtype = cache.args, cache.k.dtype
        T, Hq = q.shape[0], q.shape[1]
        stride = _rows(q, "q", dtype, (Hq, c.D))
        if out is None:
            out = torch.empty((T, Hq, c.D), dtype=dtype, device=q.device)
        out_stride = _rows(out, "out", dtype, (Hq, c.D))
        if out.shape[0] != T:
            raise ValueError(f"out has {out.shape[0]} rows, {T} required")
        _want(q_offsets, "q_offsets", torch.int32, (c.B + 1,))
        _want(lengths, "lengths", torch.int32, (c.B,))
        words = _mask(tree_mask, T)
        _same_device(cache.k, q, out, q_offsets, lengths, tree_mask)
        a = self.args = tg.TreeAttnArgs()
        if max_nodes is None:
            max_nodes = max(1, min(T, tg.MAX_NODES, 64 * words if words else tg.MAX_NODES))
            a.typical_nodes = -(-T // max(1, c.B))
        self._keep = (cache, q, q_offsets, lengths, tree_mask)
        self.out = out
        a.cache, a.T, a.Hq, a.max_nodes, a.mask_words = c, T, Hq, max_nodes, words
        a.scale = 1.0 / math.sqrt(c.D) if scale is None else scale
        a.q_stride, a.out_stride = stride, out_stride
        for name, t in dict(q=q, q_offsets=q_offsets, lengths=lengths, tree_mask=tree_mask,
                            out=out).items():
            setattr(a, name, None if t is None else t.data_ptr())
        self.ws_bytes = tg.tg_tree_attention_workspace(a)
        if self.ws_bytes == 0:
            raise tg.TgError(tg.load().tg_tree_attention(ctypes.byref(a), None, 0, None),
                             "workspace")
        self.ws = tg.workspace(self.ws_bytes, q.device)
        self._ref, self._device, self._ws = ctypes.byref(a), q.get_device(), self.ws.data_ptr()
        self._call = tg.load().tg_tree_attention

    def __call__(self, layer=0, stream=None):
        self.args.layer = layer
        _run(self._call, self._device, stream, self._ref, self._ws, self.ws_bytes)
        return self.out


class VerifyTree:
    """Which drafted tokens stay. ``target_probs`` (and ``draft_probs``) [T, V]
    float32 with dense rows, ``tokens`` [T] int32, ``u_accept`` [T] and
    ``u_next`` [B] float32 in [0, 1). ``status`` [B] int32: that of
    :meth:`KvCache.reserve`, whose refused requests keep nothing (without it, give
    only requests that have got their pages). Returns (tokens_out [B, max_path], path
    [B, max_path], n_out [B]) int32."""

    def __init__(self, target_probs, tokens, u_accept, u_next, q_offsets, tree_mask=None,
                 max_path=None, max_nodes=None, draft_probs=None, status=None):
        T, V = target_probs.shape
        B = u_next.shape[0]
        stride = _rows(target_probs, "target_probs", torch.float32, (V,))
        draft_stride = 0
        if draft_probs is not None:
            draft_stride = _rows(draft_probs, "draft_probs", torch.float32, (V,))
            if draft_probs.shape[0] != T:
                raise ValueError(f"draft_probs has {draft_probs.shape[0]} rows, {T} required")
        _want(tokens, "tokens", torch.int32, (T,))
        _want(u_accept, "u_accept", torch.float32, (T,))
        _want(u_next, "u_next", torch.float32, (B,))
        _want(q_offsets, "q_offsets", torch.int32, (B + 1,))
        _want(status, "status", torch.int32, (B,), optional=True)
        words = _mask(tree_mask, T)
        _same_device(target_probs, draft_probs, tokens, u_accept, u_next, q_offsets, tree_mask,
                     status)
        if max_nodes is None:
            max_nodes = max(1, min(T, tg.MAX_NODES, 64 * words if words else tg.MAX_NODES))
        max_path = max_nodes if max_path is None else max_path
        ints = dict(dtype=torch.int32, device=target_probs.device)
        self.tokens_out = torch.empty((B, max_path), **ints)
        self.path = torch.empty((B, max_path), **ints)
        self.n_out = torch.empty((B,), **ints)
        self._keep = (target_probs, draft_probs, tokens, u_accept, u_next, q_offsets, tree_mask,
                      status)
        a = self.args = tg.VerifyArgs()
        a.B, a.T, a.V, a.max_path, a.max_nodes, a.mask_words = B, T, V, max_path, max_nodes, words
        a.target_stride, a.draft_stride = stride, draft_stride
        for name, t in dict(target_probs=target_probs, draft_probs=draft_probs, tokens=tokens,
                            u_accept=u_accept, u_next=u_next, q_offsets=q_offsets,
                            tree_mask=tree_mask, tokens_out=self.tokens_out, path=self.path,
                            n_out=self.n_out, status=status).items():
            setattr(a, name, None if t is None else t.data_ptr())
        self.ws_bytes = tg.tg_verify_tree_workspace(a)
        if self.ws_bytes == 0:
            raise tg.TgError(tg.load().tg_verify_tree(ctypes.byref(a), None, 0, None), "workspace")
        self.ws = tg.workspace(self.ws_bytes, target_probs.device)
        self._ref, self._device = ctypes.byref(a), target_probs.get_device()
        self._ws, self._call = self.ws.data_ptr(), tg.load().tg_verify_tree

    def __call__(self, stream=None):
        _run(self._call, self._device, stream, self._ref, self._ws, self.ws_bytes)
        return self.tokens_out, self.path, self.n_out
