"""Python binding of the 8-bit paged KV cache (griffin_paged_* in
include/griffin_verify.h): checks and argument marshalling only.

Both calls run on the caller's current stream (or `stream`), take the
sequences' state from device tensors, and synchronise nothing, so that they
can be captured into a graph.
"""

from __future__ import annotations

import struct
from typing import NamedTuple, Optional, Sequence

import torch

from . import _native as N

_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_E4M3 = torch.float8_e4m3fn
# the C structs griffin_append and griffin_attention, field by field
_APPEND = struct.Struct("@4P4i5PP3qP3qd7i0q").pack
_ATTENTION = struct.Struct("@4P4i5PP3qP3qP3qP3qf9i0q").pack


class PagedPool(NamedTuple):
    """One layer's pages: k e4m3 [pages][Hkv][page / 32][dh / 16][32][16],
    v e4m3 [pages][Hkv][page / 32][dh][32], and their tiles' exponents
    k_exp, v_exp int8 [pages][Hkv][page / 32]."""
    k: torch.Tensor
    v: torch.Tensor
    k_exp: torch.Tensor
    v_exp: torch.Tensor


def paged_pool(n_pages: int, n_kv_heads: int, head_dim: int, page: int = 64, device="cuda",
               layers: Optional[int] = None) -> PagedPool:
    """An empty pool of one layer; layers: of that many, as a leading dimension
    of its tensors (what a paged TreeVerifier takes; layer_pool gives one)."""
    if n_pages < 1 or n_kv_heads < 1 or head_dim not in (64, 128) or page < 32 or page % 32:
        raise ValueError("a pool needs pages and heads, head_dim 64 or 128 and pages of a multiple of 32 slots")
    tiles = (() if layers is None else (layers,)) + (n_pages, n_kv_heads, page // 32)
    byte = lambda *s: torch.zeros(tiles + s, dtype=torch.uint8, device=device).view(_E4M3)  # noqa: E731
    exps = lambda: torch.full(tiles, -110, dtype=torch.int8, device=device)  # noqa: E731
    return PagedPool(byte(head_dim // 16, 32, 16), byte(head_dim, 32), exps(), exps())


def layer_pool(pool: Sequence[torch.Tensor], layer: int) -> PagedPool:
    """One layer of a pool of several."""
    return PagedPool(*(t[layer] for t in pool))


def paged_read(pool: Sequence[torch.Tensor], table: torch.Tensor, n: int):
    """The first n cached slots of one sequence (table: its pages) as float32
    (k, v), each [Hkv, n, dh]."""
    k, v, ke, ve = pool
    pages = table[: -(-n // (k.shape[2] * 32))].long()
    if n < 0 or table.dim() != 1 or len(pages) * k.shape[2] * 32 < n:
        raise ValueError(f"the table does not hold {n} slots")
    if len(pages) and not 0 <= int(pages.min()) <= int(pages.max()) < k.shape[0]:
        raise ValueError("a page is not in the pool")
    fk = torch.ldexp(k[pages].float(), ke[pages].int()[..., None, None, None])  # [p, Hkv, t, dh/16, 32, 16]
    fv = torch.ldexp(v[pages].float(), ve[pages].int()[..., None, None])        # [p, Hkv, t, dh, 32]
    fk = fk.permute(1, 0, 2, 4, 3, 5).reshape(k.shape[1], -1, v.shape[3])
    fv = fv.permute(1, 0, 2, 4, 3).reshape(k.shape[1], -1, v.shape[3])
    return fk[:, :n], fv[:, :n]


def _pool_fields(pool):
    """Pointers and sizes of a pool; (fields, heads, head_dim, device's index)."""
    k, v, ke, ve = pool
    if k.dim() != 6 or k.dtype is not _E4M3 or v.dtype is not _E4M3 or ke.dtype is not torch.int8 or \
            ve.dtype is not torch.int8:
        raise ValueError("a pool is (k, v, k_exp, v_exp) as paged_pool lays them out")
    n, heads, tpp, chunks, slots, dims = k.shape
    dh, tiles = chunks * 16, (n, heads, tpp)
    if slots != 32 or dims != 16 or v.shape != (n, heads, tpp, dh, 32) or ke.shape != tiles or ve.shape != tiles or not (
            k.is_contiguous() and v.is_contiguous() and ke.is_contiguous() and ve.is_contiguous()):
        raise ValueError("a pool's tensors must be contiguous and of the same pages, heads and head_dim")
    dev = k.get_device()
    if dev < 0 or v.get_device() != dev or ke.get_device() != dev or ve.get_device() != dev:
        raise ValueError("a pool lies on one CUDA device")
    return (k.data_ptr(), v.data_ptr(), ke.data_ptr(), ve.data_ptr(), n, tpp * 32, heads, dh), heads, dh, dev


def _ints(t: Optional[torch.Tensor], what: str, dev, shape, dtype=torch.int32) -> int:
    """Address of an optional contiguous integer tensor."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{dev}")
    return t.data_ptr()


def _table(table: torch.Tensor, lengths: torch.Tensor, dev):
    if table.dtype is not torch.int32 or table.dim() != 2 or table.get_device() != dev:
        raise ValueError(f"table must be an int32 [batch, pages] tensor on cuda:{dev}")
    b, cols = table.shape
    stride, unit = table.stride()
    if unit != 1:
        raise ValueError("table: a sequence's pages must be contiguous")
    # the stride of a single row is not used (and may be anything)
    return b, cols, stride if b > 1 else cols, _ints(lengths, "lengths", dev, (b,))


def _rows(t: torch.Tensor, what: str, dev, dtype, shape):
    """Address and strides of rows [batch, rows, heads, dh]."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        raise ValueError(f"{what} must be a {dtype} tensor of shape {tuple(shape)} on cuda:{dev}")
    seq, row, head, unit = t.stride()
    if unit != 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    return t.data_ptr(), seq, row, head


def _on(stream, call, pool, *tensors, **named):
    """call(pool, *tensors, **named) with `stream`, ordered after the caller's,
    current.  The allocator learns of it: no tensor's memory is used again
    before the stream's work with it has ended."""
    if stream.device != pool[0].device:
        raise ValueError("the stream must be one of the pool's device")
    here = torch.cuda.current_stream(stream.device)
    stream.wait_stream(here)
    with torch.cuda.stream(stream):
        out = call(pool, *tensors, **named)
    for t in (*pool, *tensors, *named.values()):
        if isinstance(t, torch.Tensor):
            t.record_stream(stream)
    if out is not None and named.get("out") is None:
        out.record_stream(here)
    return out


def _call(fn, dev, *args):
    """A library call with the device's current stream as its last argument."""
    if torch._C._cuda_getDevice() != dev:
        with torch.cuda.device(dev):
            rc = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    else:
        rc = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    if rc != N.GRIFFIN_OK:
        raise N.GriffinError(rc, fn.__name__)


def paged_append(pool: Sequence[torch.Tensor], table: torch.Tensor, lengths: torch.Tensor, k: torch.Tensor,
                 v: torch.Tensor, *, counts: Optional[torch.Tensor] = None, path: Optional[torch.Tensor] = None,
                 rope_base: Optional[float] = None, status: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> None:
    """Append rows of k, v [batch, rows, Hkv, dh] (bf16, fp16 or fp32; any
    strides, the last dimension contiguous) to the cache.

    table int32 [batch, pages]; lengths int32 [batch], the slots cached before
    (not changed); counts int32 [batch], the sequences' new rows (None: all);
    path int32 [batch, n], the source row of each new one (None: in order);
    rope_base: rotate the keys by their slot's angle on the way (None: they are
    rotated already); status: an int32 tensor of one element that collects
    GRIFFIN_PAGED_* bits of what the device found out of range."""
    if stream is not None:
        return _on(stream, paged_append, pool, table, lengths, k, v, counts=counts, path=path, rope_base=rope_base,
                   status=status)
    fields, heads, dh, dev = _pool_fields(pool)
    b, cols, stride, lens = _table(table, lengths, dev)
    dtype = k.dtype
    if dtype not in _DTYPES or k.dim() != 4:
        raise ValueError("k must be a bf16, fp16 or fp32 tensor [batch, rows, heads, head_dim]")
    rows = k.shape[1]
    if rope_base is not None and not rope_base > 0:
        raise ValueError("rope_base must be positive")
    shape = (b, rows, heads, dh)
    new, path_at = rows, 0
    if path is not None:
        if path.dim() != 2:
            raise ValueError("path must be an int32 [batch, n] tensor")
        new = path.shape[1]
        path_at = _ints(path, "path", dev, (b, new))
    args = _APPEND(*fields, table.data_ptr(), lens, _ints(counts, "counts", dev, (b,)), path_at,
                   _ints(status, "status", dev, (1,)), *_rows(k, "k", dev, dtype, shape), *_rows(v, "v", dev, dtype, shape),
                   rope_base or 0.0, stride, cols, new, b, rows, new, _DTYPES[dtype])
    if rows and new:
        _call(N.lib.griffin_paged_append, dev, args)


def paged_attention(pool: Sequence[torch.Tensor], table: torch.Tensor, lengths: torch.Tensor, q: torch.Tensor,
                    k: torch.Tensor, v: torch.Tensor, *, anc: Optional[torch.Tensor] = None,
                    counts: Optional[torch.Tensor] = None, window: int = 0, sinks: int = 0,
                    scale: Optional[float] = None, max_length: Optional[int] = None,
                    out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Attention of up to 64 nodes per sequence over the cached slots and the
    nodes of their own root path; returns `out` [batch, nodes, Hq, dh].

    q [batch, nodes, Hq, dh] and the nodes' own k, v [batch, nodes, Hkv, dh]
    (bf16, fp16 or fp32 alike; q and k rotated; any strides, the last dimension
    contiguous); anc int64 [batch, nodes], bit j of a node set where it sees
    node j (tree_prepare's masks; None: a chain); counts int32 [batch], the
    sequences' nodes (None: all); window > 0: only what stands less than that
    many positions before a node, and the first `sinks` positions; scale None:
    1 / sqrt(dh); max_length: a bound of lengths (None: what the table holds);
    out: rows of absent nodes are left as they were (None: new, they are zero);
    status: as for paged_append."""
    if stream is not None:
        return _on(stream, paged_attention, pool, table, lengths, q, k, v, anc=anc, counts=counts, window=window,
                   sinks=sinks, scale=scale, max_length=max_length, out=out, status=status)
    fields, heads, dh, dev = _pool_fields(pool)
    b, cols, stride, lens = _table(table, lengths, dev)
    dtype = q.dtype
    if dtype not in _DTYPES or q.dim() != 4:
        raise ValueError("q must be a bf16, fp16 or fp32 tensor [batch, nodes, heads, head_dim]")
    nodes, hq = q.shape[1:3]
    shape, kv = (b, nodes, hq, dh), (b, nodes, heads, dh)
    if out is None:
        make = torch.empty if counts is None else torch.zeros
        out = make(shape, dtype=dtype, device=dev)
    args = _ATTENTION(*fields, table.data_ptr(), lens, _ints(counts, "counts", dev, (b,)),
                      _ints(anc, "anc", dev, (b, nodes), torch.int64), _ints(status, "status", dev, (1,)),
                      *_rows(q, "q", dev, dtype, shape), *_rows(k, "k", dev, dtype, kv), *_rows(v, "v", dev, dtype, kv),
                      *_rows(out, "out", dev, dtype, shape), dh ** -0.5 if scale is None else scale, stride, cols,
                      -1 if max_length is None else max_length, b, nodes, hq, _DTYPES[dtype], window, sinks)
    need = N.lib.griffin_paged_attention_workspace(args)
    if need:
        work = torch.empty(need, dtype=torch.uint8, device=dev)
        _call(N.lib.griffin_paged_attention, dev, args, work.data_ptr(), need)
    else:
        _call(N.lib.griffin_paged_attention, dev, args, None, 0)
    return out
