"""ctypes binding of the paged 4-bit KV cache of libmars (argument marshalling only).

One decode cycle of a speculative-decoding program, with ``c`` a :class:`KVCache`::

    kv_cache.resize(c, extra)                               # room for the next tree's nodes
    for each layer:
        kv_cache.append(c, layer, k, v)                     # [B, N, kv_heads, d] of the draft nodes
        o = kv_cache.tree_attention(q, c, layer, parent, out=o, status=st, workspace=ws)    # [B, N, q_heads, d]
    out = mars.lmhead_verify(...)                           # or mars.verify_tree on logits
    kv_cache.commit(c, out["path_nodes"], out["accept_len"])

Every call is asynchronous on the current stream of the cache's device; per-sequence problems are
reported in the status tensors (``STATUS``), host-detectable ones raise :class:`mars.MarsError`.
"""
from __future__ import annotations

import ctypes

import torch

from . import mars
from .mars import MarsError, _check, lib

FP16 = 2
MAX_SEQS = 8192
STATUS = {0: "ok", 1: "bad tree", 3: "timeout", 5: "no room", 7: "out of pages", 8: "bad path", 9: "bad fork"}

_DTYPES = {torch.bfloat16: mars.BF16, torch.float32: mars.FP32, torch.float16: FP16}


class _CacheStruct(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("pages", "scales", "block_table", "seq_len", "seq_pages", "page_refs",
                                                "free_bits")]
                + [(n, ctypes.c_int) for n in ("layers", "num_pages", "kv_heads", "head_dim", "page_size", "seqs",
                                               "table_width")])


class KVCache:
    """The device tensors of one cache (see mars_kv.h) and the descriptor that points at them.

    pages uint8 [layers, num_pages, kv_heads, page bytes], scales float32 [layers, 2, kv_heads],
    block_table int32 [seqs, table_width], seq_len / seq_pages int32 [seqs], page_refs int32
    [num_pages], free_bits int32 [(num_pages + 31) // 32], all contiguous on one device.  The tensors
    may be read at any time; seq_len may be set by the program, the page tables belong to the calls.
    """

    def __init__(self, pages, scales, block_table, seq_len, seq_pages, page_refs, free_bits, head_dim: int,
                 page_size: int):
        layers, num_pages, kv_heads, page_bytes = pages.shape
        seqs, width = block_table.shape
        want = (("pages", pages, torch.uint8, (layers, num_pages, kv_heads, page_size * head_dim * 9 // 8)),
                ("scales", scales, torch.float32, (layers, 2, kv_heads)),
                ("block_table", block_table, torch.int32, (seqs, width)), ("seq_len", seq_len, torch.int32, (seqs,)),
                ("seq_pages", seq_pages, torch.int32, (seqs,)), ("page_refs", page_refs, torch.int32, (num_pages,)),
                ("free_bits", free_bits, torch.int32, ((num_pages + 31) // 32,)))
        for name, t, dtype, shape in want:
            if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.device != pages.device:
                raise MarsError(f"{name} must be a contiguous {dtype} tensor {list(shape)} on {pages.device}, got "
                                f"{t.dtype} {list(t.shape)} on {t.device}")
        if not pages.is_cuda:
            raise MarsError("the cache must live in device memory")
        if lib().mars_kv_pool_bytes(layers, num_pages, kv_heads, head_dim, page_size) == 0 or seqs > MAX_SEQS:
            raise MarsError("unsupported sizes")
        self.pages, self.scales, self.block_table, self.seq_len = pages, scales, block_table, seq_len
        self.seq_pages, self.page_refs, self.free_bits = seq_pages, page_refs, free_bits
        self.layers, self.num_pages, self.kv_heads, self.head_dim = layers, num_pages, kv_heads, head_dim
        self.page_size, self.seqs, self.table_width, self.device = page_size, seqs, width, pages.device
        self._struct = _CacheStruct(pages.data_ptr(), scales.data_ptr(), block_table.data_ptr(), seq_len.data_ptr(),
                                    seq_pages.data_ptr(), page_refs.data_ptr(), free_bits.data_ptr(), layers, num_pages,
                                    kv_heads, head_dim, page_size, seqs, width)
        self._ref = ctypes.byref(self._struct)
        self._index = pages.get_device()

    @classmethod
    def empty(cls, layers: int, num_pages: int, kv_heads: int, head_dim: int, page_size: int, seqs: int,
              table_width: int, device, scales=None) -> "KVCache":
        """A cache without sequences: every page free.  `scales` float [layers, 2, kv_heads] (default 1)."""
        z = dict(dtype=torch.int32, device=device)
        bits = torch.full(((num_pages + 31) // 32,), -1, **z)
        if num_pages % 32:
            bits[-1] = (1 << (num_pages % 32)) - 1
        if scales is None:
            scales = torch.ones((layers, 2, kv_heads), dtype=torch.float32, device=device)
        scales = torch.as_tensor(scales, dtype=torch.float32, device=device).contiguous()
        if not bool(((scales > 0) & torch.isfinite(scales)).all()):
            raise MarsError("scales must be positive and finite")
        return cls(torch.zeros((layers, num_pages, kv_heads, page_size * head_dim * 9 // 8), dtype=torch.uint8,
                               device=device), scales, torch.full((seqs, table_width), -1, **z),
                   torch.zeros((seqs,), **z), torch.zeros((seqs,), **z), torch.zeros((num_pages,), **z), bits, head_dim,
                   page_size)


# The calls below run a few times per layer and decode step, so their host time counts: attributes are
# read once, devices compared by index, the stream taken as a raw handle.

def _call(fn, cache: KVCache, *args) -> None:
    """fn(descriptor, *args, stream) with the cache's device current; raises on a refusal."""
    idx = cache._index
    stream = torch._C._cuda_getCurrentRawStream(idx)
    if torch._C._cuda_getDevice() == idx:
        code = fn(cache._ref, *args, stream)
    else:
        with torch.cuda.device(idx):
            code = fn(cache._ref, *args, stream)
    if code:
        _check(code, fn.__name__)


def _i32(t, n: int, index: int, name: str):
    """Device pointer of an int32 tensor of n entries, None for None."""
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.get_device() != index or t.numel() != n or not t.is_contiguous():
        raise MarsError(f"{name} must be a contiguous int32 tensor of {n} entries on the cache's device")
    return t.data_ptr()


def _rows(t, heads: int, d: int, index: int, name: str):
    """[B, N, heads, d] with unit inner stride and rows b*N + i at one stride: (pointer, row, head)."""
    shape = t.shape
    if len(shape) != 4 or shape[2] != heads or shape[3] != d or t.get_device() != index or t.dtype not in _DTYPES:
        raise MarsError(f"{name} must be [B, N, {heads}, {d}] of bfloat16, float16 or float32 on the cache's device")
    sb, sn, sh, sd = t.stride()
    if shape[1] == 1:
        sn = sb if shape[0] > 1 else heads * d
    elif shape[0] > 1 and sb != shape[1] * sn:
        sd = 0
    if sd != 1:
        raise MarsError(f"{name}: rows b*N + i must lie at one stride, with unit inner stride")
    return t.data_ptr(), sn, sh if heads > 1 else d


def resize(cache: KVCache, extra: torch.Tensor, status: torch.Tensor | None = None) -> torch.Tensor | None:
    """mars_kv_resize: pages for seq_len[b] + extra[b] tokens of every sequence (0 trims, -1 releases,
    below: leave).  Returns `status` (int32 [seqs]) as it was given."""
    dev = cache._index
    _call(lib().mars_kv_resize, cache, _i32(extra, cache.seqs, dev, "extra"), _i32(status, cache.seqs, dev, "status"))
    return status


def append(cache: KVCache, layer: int, k: torch.Tensor, v: torch.Tensor, count: torch.Tensor | None = None,
           status: torch.Tensor | None = None) -> None:
    """mars_kv_append: rows k, v [B, N, kv_heads, head_dim] to positions seq_len[b] + i."""
    dev = cache._index
    kp, kr, kh = _rows(k, cache.kv_heads, cache.head_dim, dev, "k")
    vp, vr, vh = _rows(v, cache.kv_heads, cache.head_dim, dev, "v")
    if k.shape != v.shape or k.dtype is not v.dtype:
        raise MarsError("k and v must have the same shape and dtype")
    B, N = k.shape[:2]
    _call(lib().mars_kv_append, cache, layer, kp, kr, kh, vp, vr, vh, _DTYPES[k.dtype], B, N,
          _i32(count, B, dev, "count"), _i32(status, B, dev, "status"))


def attention_workspace_bytes(B: int, N: int, q_heads: int, kv_heads: int, head_dim: int) -> int:
    return int(lib().mars_tree_attention_workspace_bytes(B, N, q_heads, kv_heads, head_dim))


def attention_workspace(q: torch.Tensor, cache: KVCache) -> torch.Tensor:
    """A zeroed workspace for tree_attention calls with q of this shape; such a workspace serves any
    number of calls that do not overlap."""
    need = attention_workspace_bytes(q.shape[0], q.shape[1], q.shape[2], cache.kv_heads, cache.head_dim)
    if need == 0:
        raise MarsError("unsupported sizes")
    return torch.zeros((need,), dtype=torch.uint8, device=cache.device)


def tree_attention(q: torch.Tensor, cache: KVCache, layer: int, parent: torch.Tensor | None = None,
                   count: torch.Tensor | None = None, scale: float | None = None, out: torch.Tensor | None = None,
                   status: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """mars_tree_attention: q [B, N, q_heads, head_dim] over the cache; parent int32 [B, N], [N] or None
    (chains).  `workspace` comes from ``attention_workspace`` and is used by these calls only; without
    one, a call allocates and clears its own.  Rows without a result (behind `count`, absent nodes, sequences
    whose `status` is not 0) keep what `out` holds, and are zero in an output that the call allocates.  A
    sequence whose status is 3 (timeout) has NaN in the rows that were not computed."""
    dev, H = cache._index, cache.kv_heads
    if q.dim() != 4 or q.shape[2] % H:
        raise MarsError("q must be [B, N, q_heads, head_dim] with q_heads a multiple of kv_heads")
    B, N, Hq, d = q.shape
    qp, qr, qh = _rows(q, Hq, cache.head_dim, dev, "q")
    if out is None:
        out = torch.zeros((B, N, Hq, d), dtype=q.dtype, device=cache.device)
    op, orow, oh = _rows(out, Hq, cache.head_dim, dev, "out")
    if out.dtype is not q.dtype or out.shape != q.shape:
        raise MarsError("out must have the shape and dtype of q")
    flags, pp = 0, None
    if parent is not None:
        shared = parent.dim() == 1
        flags = mars.SHARED_PARENT if shared else 0
        pp = _i32(parent, N if shared else B * N, dev, "parent")
    if workspace is None:
        need = attention_workspace_bytes(B, N, Hq, H, d)
        if need == 0:
            raise MarsError("unsupported sizes")
        workspace = torch.empty((need,), dtype=torch.uint8, device=cache.device)
    else:
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise MarsError("workspace must be a contiguous tensor on the cache's device")
        flags |= mars.COUNTERS_ZERO
    _call(lib().mars_tree_attention, cache, layer, qp, qr, qh, _DTYPES[q.dtype], Hq, B, N, pp,
          _i32(count, B, dev, "count"), d ** -0.5 if scale is None else scale, flags, op, orow, oh,
          _i32(status, B, dev, "status"), workspace.data_ptr(), workspace.nbytes)
    return out


def commit(cache: KVCache, path_nodes: torch.Tensor | None, accept_len: torch.Tensor,
           new_len: torch.Tensor | None = None, status: torch.Tensor | None = None) -> torch.Tensor:
    """mars_kv_commit with the path_nodes [B, W] and accept_len [B] of a verification (path_nodes None:
    chains).  `new_len` int32 [B] receives the lengths, by default cache.seq_len itself."""
    dev = cache._index
    B = accept_len.numel()
    W = 0
    if path_nodes is not None:
        if path_nodes.dim() != 2 or path_nodes.shape[0] != B:
            raise MarsError("path_nodes must be [B, W]")
        W = path_nodes.shape[1]
    if new_len is None or new_len is cache.seq_len:
        new_len = cache.seq_len
        lp = new_len.data_ptr()
    else:
        lp = _i32(new_len, B, dev, "new_len")
    _call(lib().mars_kv_commit, cache, _i32(path_nodes, B * W, dev, "path_nodes"), W,
          _i32(accept_len, B, dev, "accept_len"), B, lp, _i32(status, B, dev, "status"))
    return new_len


def fork(cache: KVCache, src: torch.Tensor, dst: torch.Tensor, status: torch.Tensor | None = None) -> torch.Tensor:
    """mars_kv_fork: sequence dst[p] becomes a copy of src[p]; returns the pairs' status."""
    dev = cache._index
    n = src.numel()
    if status is None:
        status = torch.empty((n,), dtype=torch.int32, device=cache.device)
    _call(lib().mars_kv_fork, cache, _i32(src, n, dev, "src"), _i32(dst, n, dev, "dst"), n, _i32(status, n, dev, "status"))
    return status


def gather(cache: KVCache, layer0: int, layers: int, start: torch.Tensor | None, count: torch.Tensor | None,
           rows: int | None = None, dtype=torch.bfloat16, out=None):
    """mars_kv_gather: (k, v), each [layers, B, rows, kv_heads, head_dim], of positions start[b] ..
    start[b] + count[b] - 1; `out` = such a pair to write into (its dtype is used)."""
    dev = cache._index
    B = start.numel() if start is not None else count.numel() if count is not None else cache.seqs
    if out is None:
        if rows is None:
            raise MarsError("gather needs `rows` or `out`")
        shape = (layers, B, rows, cache.kv_heads, cache.head_dim)
        out = (torch.zeros(shape, dtype=dtype, device=cache.device), torch.zeros(shape, dtype=dtype, device=cache.device))
    k, v = out
    shape = k.shape
    if len(shape) != 5 or shape != v.shape or shape[0] != layers or shape[1] != B or shape[3] != cache.kv_heads \
            or shape[4] != cache.head_dim or k.dtype is not v.dtype or k.dtype not in _DTYPES \
            or not (k.is_contiguous() and v.is_contiguous()) or k.get_device() != dev or v.get_device() != dev:
        raise MarsError("out must be two contiguous [layers, B, rows, kv_heads, head_dim] tensors of one dtype")
    _call(lib().mars_kv_gather, cache, layer0, layers, B, _i32(start, B, dev, "start"), _i32(count, B, dev, "count"),
          shape[2], k.data_ptr(), v.data_ptr(), _DTYPES[k.dtype])
    return k, v
