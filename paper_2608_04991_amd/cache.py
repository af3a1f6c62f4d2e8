"""Python binding of include/rac_cache.h: the paged key-value cache and the
attention of drafted trees.  Re-exported by the package.

    cfg = CacheConfig(layers=1, kv_heads=8, head_dim=128, page_tokens=32, pages=4096, seqs=64, max_pages=512)
    pool = torch.zeros(rac_cache_pool_bytes(cfg), dtype=torch.uint8, device="cuda")
    table, lengths, refs = rac_cache_new(cfg)
    tree = TreeConfig(q_heads=32, rows=q.shape[0], max_rows=64, max_draft=64)
    ws = torch.empty(rac_tree_attention_workspace(cfg, tree), dtype=torch.uint8, device="cuda")
    rac_tree_attention(cfg, tree, 0, pool, table, lengths, q, start, k, v, out, ws, mask=mask)
    rac_cache_commit(cfg, pool, table, lengths, refs, k[None], v[None], start, committed, ws2, path=path)

As in the rest of the package every step runs in HIP kernels; PyTorch supplies
device memory and the stream.
"""
from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass, fields

import paper_2608_04991_amd as _rac

__all__ = [
    "RAC_CACHE_BF16", "RAC_CACHE_FP16", "RAC_CACHE_FP8", "CacheConfig", "TreeConfig", "rac_cache_pool_bytes",
    "rac_cache_new", "rac_tree_attention_workspace", "rac_tree_attention", "rac_cache_fork",
    "rac_cache_commit_workspace", "rac_cache_commit", "rac_cache_copy", "rac_predictor_tree_workspace",
    "rac_predictor_tree_step", "EvictConfig", "rac_tree_weights_workspace", "rac_tree_weights",
    "rac_cache_weights_commit", "rac_cache_evict_workspace", "rac_cache_evict",
]

RAC_CACHE_BF16 = 0
RAC_CACHE_FP16 = 1
RAC_CACHE_FP8 = 2


class _CacheConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("layers", "kv_heads", "head_dim", "page_tokens", "pages", "seqs",
                                              "max_pages", "type")] + \
               [("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float)]


class _TreeConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("q_heads", "rows", "max_rows", "max_draft", "window")] + \
               [("scale", ctypes.c_float)]


class _TreeTensors(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "v", "q_start", "draft_start", "mask", "out", "lse")] + \
               [(n, ctypes.c_int64) for n in ("q_stride", "kv_stride", "out_stride")] + \
               [(n, ctypes.c_int32) for n in ("draft_rows", "mask_words")]


class _EvictConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("sets", "first", "recent")]


class _Kept:
    """A configuration that keeps what its fields fix: the library's struct, a
    reference to it, sizes.  A copy or a pickle has the fields alone."""

    def __getstate__(self) -> dict:
        return {f.name: getattr(self, f.name) for f in fields(self)}


@dataclass(frozen=True)
class CacheConfig(_Kept):
    layers: int
    kv_heads: int
    head_dim: int
    page_tokens: int
    pages: int
    seqs: int
    max_pages: int
    type: int = RAC_CACHE_BF16
    k_scale: float = 1.0
    v_scale: float = 1.0

    def _c(self) -> _CacheConfig:
        return self._struct

    # (made once a configuration: the small calls are bound by the host, and the
    # library reads the struct during the call only)
    @functools.cached_property
    def _struct(self) -> _CacheConfig:
        return _CacheConfig(self.layers, self.kv_heads, self.head_dim, self.page_tokens, self.pages, self.seqs,
                            self.max_pages, self.type, self.k_scale, self.v_scale)

    @functools.cached_property
    def _ref(self):
        return ctypes.byref(self._struct)

    @functools.cached_property
    def _pool_bytes(self) -> int:
        return int(_rac.library().rac_cache_pool_bytes(self._ref))

    @functools.cached_property
    def _commit_bytes(self) -> int:
        return int(_rac.library().rac_cache_commit_workspace(self._ref))


@dataclass(frozen=True)
class TreeConfig(_Kept):
    q_heads: int
    rows: int
    max_rows: int
    max_draft: int
    window: int = 0
    scale: float = 0.0

    def _c(self) -> _TreeConfig:
        return self._struct

    @functools.cached_property
    def _struct(self) -> _TreeConfig:
        return _TreeConfig(self.q_heads, self.rows, self.max_rows, self.max_draft, self.window, self.scale)

    @functools.cached_property
    def _ref(self):
        return ctypes.byref(self._struct)


@dataclass(frozen=True)
class EvictConfig(_Kept):
    sets: int = 1
    first: int = 0
    recent: int = 0

    def _c(self) -> _EvictConfig:
        return self._struct

    @functools.cached_property
    def _struct(self) -> _EvictConfig:
        return _EvictConfig(self.sets, self.first, self.recent)

    @functools.cached_property
    def _ref(self):
        return ctypes.byref(self._struct)


def declare(L) -> None:
    """The argument types of the library's cache functions."""
    cp, tp, vp, i32, i64 = (ctypes.POINTER(_CacheConfig), ctypes.POINTER(_TreeConfig), ctypes.c_void_p,
                            ctypes.c_int32, ctypes.c_int64)
    ep = ctypes.POINTER(_EvictConfig)
    sz = ctypes.c_size_t
    for name, args, res in (
            ("rac_cache_pool_bytes", [cp], sz),
            ("rac_tree_attention_workspace", [cp, tp], sz),
            ("rac_tree_attention", [cp, tp, i32, vp, vp, vp, ctypes.POINTER(_TreeTensors), vp, sz, vp], ctypes.c_int),
            ("rac_cache_fork", [cp, vp, vp, vp, vp, vp, vp, vp], ctypes.c_int),
            ("rac_cache_commit_workspace", [cp], sz),
            ("rac_cache_commit", [cp, vp, vp, vp, vp, vp, vp, i64, i64, i32, vp, vp, i32, vp, vp, sz, vp],
             ctypes.c_int),
            ("rac_cache_copy", [cp, vp, vp, vp, vp, i32, vp], ctypes.c_int),
            ("rac_tree_weights_workspace", [cp, tp], sz),
            ("rac_tree_weights", [cp, tp, i32, i32, vp, vp, vp, ctypes.POINTER(_TreeTensors), vp, vp, vp, sz, vp],
             ctypes.c_int),
            ("rac_cache_weights_commit", [cp, i32, vp, vp, vp, vp, i32, vp, i32, vp, vp], ctypes.c_int),
            ("rac_cache_evict_workspace", [cp, ep], sz),
            ("rac_cache_evict", [cp, ep, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
            ("rac_predictor_tree_workspace", [ctypes.POINTER(_rac._PredConfig), cp, tp], sz),
            ("rac_predictor_tree_step", [ctypes.POINTER(_rac._PredConfig), cp, tp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32,
                                         vp, vp, vp, i32, vp, vp, sz, vp], ctypes.c_int)):
        f = getattr(L, name)
        f.argtypes = args
        f.restype = res


def _pool(cfg: CacheConfig, pool, what: str = "pool"):
    """Address of a pool tensor of any element type, checked by its bytes."""
    if pool is None or isinstance(pool, int):
        return pool
    size = pool.element_size()
    return _rac._dev(pool, what, size, -(-cfg._pool_bytes // size))


def _rows(t, what: str, rows: int, heads: int, dim: int):
    """(address, elements between rows, rows) of a 16-bit [rows][heads][dim]
    tensor whose heads lie together; its rows may be apart."""
    try:
        n, h, d = t.shape
        row, head, one = t.stride()
        if n <= 1:
            row = heads * dim
        if h == heads and d == dim and n >= rows and one == 1 and (head == dim or h == 1) and row >= heads * dim \
                and t.is_cuda and t.element_size() == 2:
            return t.data_ptr(), row, n
    except (AttributeError, ValueError, TypeError):
        if t is None or isinstance(t, int):
            return t, heads * dim, rows
    raise ValueError(f"{what}: expected a GPU tensor of 2-byte elements, [{rows}][{heads}][{dim}], heads and channels "
                     "contiguous")


def _drafts(t, what: str, rows: int, heads: int, dim: int):
    """_rows of drafted keys or values.  How many there are comes from the tensor,
    so an address is not enough."""
    if isinstance(t, int):
        raise ValueError(f"{what}: expected a GPU tensor, not an address: its rows are counted")
    return _rows(t, what, rows, heads, dim)


def _words(mask) -> int:
    """Words of a mask's row, 0 without a mask."""
    if isinstance(mask, int):
        raise ValueError("mask: expected a GPU tensor, not an address: the words of its rows are counted")
    return 0 if mask is None else int(mask.shape[-1])


def rac_cache_pool_bytes(cfg: CacheConfig) -> int:
    return cfg._pool_bytes


def rac_cache_new(cfg: CacheConfig, device: str = "cuda"):
    """(table, lengths, refs) of an empty cache."""
    import torch
    return (torch.full((cfg.seqs, cfg.max_pages), -1, dtype=torch.int32, device=device),
            torch.zeros(cfg.seqs, dtype=torch.int32, device=device),
            torch.zeros(cfg.pages, dtype=torch.int32, device=device))


def rac_tree_attention_workspace(cfg: CacheConfig, tree: TreeConfig) -> int:
    # (both are immutable: the size of the last pair stays with the tree)
    last = tree.__dict__.get("_workspace")
    if last is None or last[0] is not cfg:
        last = cfg, int(_rac.library().rac_tree_attention_workspace(cfg._ref, tree._ref))
        tree.__dict__["_workspace"] = last
    return last[1]


def rac_tree_attention(cfg: CacheConfig, tree: TreeConfig, layer: int, pool, table, lengths, q, q_start, k, v, out,
                       workspace, *, draft_start=None, mask=None, lse=None, stream=None) -> None:
    """Attention of query rows q (16-bit [rows][q_heads][head_dim]) over the
    committed tokens in the pool and the drafted ones k, v ([draft_rows]
    [kv_heads][head_dim], or None).  q_start, draft_start: int32 [seqs + 1];
    mask: int64 [rows][words], the drafted tokens each row sees; lse: fp32
    [rows][q_heads].  Rows of q, k, v and out may be apart (views of a larger
    tensor); k and v by the same distance."""
    dev = _rac._dev
    R, Q, H, D, S = tree.rows, tree.q_heads, cfg.kv_heads, cfg.head_dim, cfg.seqs
    qp, qs, _ = _rows(q, "q", R, Q, D)
    op, os_, _ = _rows(out, "out", R, Q, D)
    kp, ks, drafted = _drafts(k, "k", 0, H, D)
    vp, vs, _ = _drafts(v, "v", drafted, H, D)
    if ks != vs and drafted > 1 and v is not None:
        raise ValueError("k and v: expected the same distance between rows")
    words = _words(mask)
    t = _TreeTensors(qp, kp, vp, dev(q_start, "q_start", 4, S + 1), dev(draft_start, "draft_start", 4, S + 1),
                     dev(mask, "mask", 8, R * words), op, dev(lse, "lse", 4, R * Q), qs, ks, os_, drafted, words)
    need = rac_tree_attention_workspace(cfg, tree)
    status = _rac.library().rac_tree_attention(
        cfg._ref, tree._ref, layer, _pool(cfg, pool), dev(table, "table", 4, S * cfg.max_pages),
        dev(lengths, "lengths", 4, S), ctypes.byref(t), dev(workspace, "workspace", 1, need), need, _rac._stream(stream))
    if status:
        _rac._check(status, "rac_tree_attention")


def rac_cache_fork(cfg: CacheConfig, parents, table, lengths, refs, keep_from=None, keep_to=None, stream=None) -> None:
    """Sequence d becomes a view of positions [keep_from[d], keep_to[d]) of what
    sequence parents[d] held (int32 [seqs] each): fork, reorder, roll back, bound
    and free sequences, in place."""
    dev, S = _rac._dev, cfg.seqs
    _rac._check(_rac.library().rac_cache_fork(
        cfg._ref, dev(parents, "parents", 4, S), dev(keep_from, "keep_from", 4, S),
        dev(keep_to, "keep_to", 4, S), dev(table, "table", 4, S * cfg.max_pages), dev(lengths, "lengths", 4, S),
        dev(refs, "refs", 4, cfg.pages), _rac._stream(stream)), "rac_cache_fork")


def rac_cache_commit_workspace(cfg: CacheConfig) -> int:
    return cfg._commit_bytes


def _layers(t, what: str, cfg: CacheConfig):
    """(address, elements between rows, between layers, rows) of a 16-bit
    [layers][rows][kv_heads][head_dim] tensor."""
    H, D = cfg.kv_heads, cfg.head_dim
    try:
        layers, rows, heads, dim = t.shape
        layer, row, head, one = t.stride()
        if layers == cfg.layers and heads == H and dim == D and t.is_cuda and t.element_size() == 2:
            if t.numel() == 0:
                return t.data_ptr(), H * D, 0, rows
            if rows == 1:
                row = H * D
            if one == 1 and (head == D or H == 1) and row >= H * D:
                return t.data_ptr(), row, layer if layers > 1 else 0, rows
    except (AttributeError, ValueError, TypeError):
        pass
    raise ValueError(f"{what}: expected a GPU tensor of 2-byte elements, [{cfg.layers}][rows][{H}][{D}], heads and "
                     "channels contiguous")


def rac_cache_commit(cfg: CacheConfig, pool, table, lengths, refs, k, v, draft_start, committed, workspace, *,
                     path=None, max_path: int | None = None, stream=None) -> None:
    """Appends the accepted drafted tokens of every sequence to it, in all
    layers: k, v 16-bit [layers][rows][kv_heads][head_dim], draft_start int32
    [seqs + 1], path int32 [seqs][max_path] (None: all rows of a sequence, at
    most max_path); committed int32 [seqs] receives the tokens appended."""
    dev, S = _rac._dev, cfg.seqs
    kp, row, layer, rows = _layers(k, "k", cfg)
    vp, vrow, vlayer, vrows = _layers(v, "v", cfg)
    if vrows != rows or vrow != row or vlayer != layer:
        raise ValueError("k and v: expected the same rows, apart by the same distances")
    if max_path is None:
        if isinstance(path, int):
            raise ValueError("path: an address needs max_path beside it")
        max_path = rows if path is None else int(path.shape[-1])
    elif S > 1 and path is not None and not isinstance(path, int) and path.dim() > 1 and path.shape[-1] != max_path:
        raise ValueError(f"path: its rows have {path.shape[-1]} entries, but max_path is {max_path}")
    _rac._check(_rac.library().rac_cache_commit(
        cfg._ref, _pool(cfg, pool), dev(table, "table", 4, S * cfg.max_pages),
        dev(lengths, "lengths", 4, S), dev(refs, "refs", 4, cfg.pages), kp, vp, row, layer, rows,
        dev(draft_start, "draft_start", 4, S + 1), dev(path, "path", 4, S * int(max_path)), int(max_path),
        dev(committed, "committed", 4, S), dev(workspace, "workspace", 1, cfg._commit_bytes), cfg._commit_bytes,
        _rac._stream(stream)), "rac_cache_commit")


def rac_cache_copy(cfg: CacheConfig, src_pool, src, dst_pool, dst, n: int | None = None, stream=None) -> None:
    """Copies page src[i] of src_pool to page dst[i] of dst_pool (int32 arrays)."""
    count = int(n) if n is not None else int(src.numel())
    _rac._check(_rac.library().rac_cache_copy(
        cfg._ref, _pool(cfg, src_pool, "src_pool"), _rac._dev(src, "src", 4, count),
        _pool(cfg, dst_pool, "dst_pool"), _rac._dev(dst, "dst", 4, count), count, _rac._stream(stream)),
        "rac_cache_copy")


def _sums(cfg: CacheConfig, weight, what: str = "weight") -> int:
    """Sets of a tensor of sums, [seqs][sets][positions]."""
    try:
        seqs, sets, positions = weight.shape
    except (AttributeError, ValueError):
        raise ValueError(f"{what}: expected a GPU tensor, [{cfg.seqs}][sets][{cfg.max_pages * cfg.page_tokens}]") from None
    if seqs != cfg.seqs or positions != cfg.max_pages * cfg.page_tokens or sets not in (1, cfg.layers * cfg.kv_heads):
        raise ValueError(f"{what}: expected [{cfg.seqs}][1 or {cfg.layers * cfg.kv_heads}]"
                         f"[{cfg.max_pages * cfg.page_tokens}], got {list(weight.shape)}")
    return sets


def _draft_sums(draft_weight, sets: int, rows: int):
    """Address of the drafted tokens' sums, [sets][rows]."""
    if draft_weight is not None and tuple(getattr(draft_weight, "shape", ())) != (sets, rows):
        raise ValueError(f"draft_weight: expected a GPU tensor, [{sets}][{rows}]")
    return _rac._dev(draft_weight, "draft_weight", 4, sets * rows)


def rac_tree_weights_workspace(cfg: CacheConfig, tree: TreeConfig) -> int:
    # (as that of the attention)
    last = tree.__dict__.get("_weights_workspace")
    if last is None or last[0] is not cfg:
        last = cfg, int(_rac.library().rac_tree_weights_workspace(cfg._ref, tree._ref))
        tree.__dict__["_weights_workspace"] = last
    return last[1]


def rac_tree_weights(cfg: CacheConfig, tree: TreeConfig, layer: int, pool, table, lengths, q, q_start, k, lse, weight,
                     workspace, *, draft_weight=None, draft_start=None, mask=None, stream=None) -> None:
    """Adds the attention weight that the call of rac_tree_attention with the same
    arguments gives to the committed tokens to weight (fp32 [seqs][sets][positions],
    sets 1 or layers * kv_heads) and to the drafted ones to draft_weight (fp32
    [sets][draft_rows]).  lse: fp32 [rows][q_heads], from that call."""
    dev = _rac._dev
    R, Q, H, D, S = tree.rows, tree.q_heads, cfg.kv_heads, cfg.head_dim, cfg.seqs
    sets = _sums(cfg, weight)
    qp, qs, _ = _rows(q, "q", R, Q, D)
    kp, ks, drafted = _drafts(k, "k", 0, H, D)
    words = _words(mask)
    t = _TreeTensors(qp, kp, None, dev(q_start, "q_start", 4, S + 1), dev(draft_start, "draft_start", 4, S + 1),
                     dev(mask, "mask", 8, R * words), None, dev(lse, "lse", 4, R * Q), qs, ks, Q * D, drafted, words)
    need = rac_tree_weights_workspace(cfg, tree)
    status = _rac.library().rac_tree_weights(
        cfg._ref, tree._ref, layer, sets, _pool(cfg, pool), dev(table, "table", 4, S * cfg.max_pages),
        dev(lengths, "lengths", 4, S), ctypes.byref(t), dev(weight, "weight", 4, 0),
        _draft_sums(draft_weight, sets, drafted), dev(workspace, "workspace", 1, need), need, _rac._stream(stream))
    if status:
        _rac._check(status, "rac_tree_weights")


def rac_cache_weights_commit(cfg: CacheConfig, lengths, committed, draft_start, draft_weight, weight, *, path=None,
                             max_path: int | None = None, draft_rows: int | None = None, stream=None) -> None:
    """After rac_cache_commit: the sums of the appended tokens in weight become those
    of the rows they came from in draft_weight (None: zeros; then draft_rows says how
    many rows there were)."""
    dev, S, sets = _rac._dev, cfg.seqs, _sums(cfg, weight)
    if draft_rows is None:
        draft_rows = 0 if draft_weight is None else int(draft_weight.shape[-1])
    if max_path is None:
        if isinstance(path, int):
            raise ValueError("path: an address needs max_path beside it")
        max_path = draft_rows if path is None else int(path.shape[-1])
    elif S > 1 and path is not None and not isinstance(path, int) and path.dim() > 1 and path.shape[-1] != max_path:
        raise ValueError(f"path: its rows have {path.shape[-1]} entries, but max_path is {max_path}")
    _rac._check(_rac.library().rac_cache_weights_commit(
        cfg._ref, sets, dev(lengths, "lengths", 4, S), dev(committed, "committed", 4, S),
        dev(draft_start, "draft_start", 4, S + 1), dev(path, "path", 4, S * int(max_path)), int(max_path),
        _draft_sums(draft_weight, sets, draft_rows), int(draft_rows), dev(weight, "weight", 4, 0), _rac._stream(stream)),
        "rac_cache_weights_commit")


def rac_cache_evict_workspace(cfg: CacheConfig, evict: EvictConfig) -> int:
    last = evict.__dict__.get("_workspace")
    if last is None or last[0] is not cfg:
        last = cfg, int(_rac.library().rac_cache_evict_workspace(cfg._ref, evict._ref))
        evict.__dict__["_workspace"] = last
    return last[1]


def rac_cache_evict(cfg: CacheConfig, evict: EvictConfig, pool, table, lengths, refs, weight, keep, evicted, workspace, *,
                    source=None, stream=None) -> None:
    """Cuts every sequence s to keep[s] tokens (int32 [seqs], negative: not asked): the
    first and last ones of `evict` and those of the largest weight (fp32 [seqs][sets]
    [positions]).  evicted: int32 [seqs], tokens let go, -1 for want of pages; source:
    int32, as weight, former positions."""
    dev, S = _rac._dev, cfg.seqs
    if _sums(cfg, weight) != evict.sets:
        raise ValueError(f"weight: expected {evict.sets} sets, got {weight.shape[1]}")
    need = rac_cache_evict_workspace(cfg, evict)
    status = _rac.library().rac_cache_evict(
        cfg._ref, evict._ref, _pool(cfg, pool), dev(table, "table", 4, S * cfg.max_pages), dev(lengths, "lengths", 4, S),
        dev(refs, "refs", 4, cfg.pages), dev(weight, "weight", 4, 0), dev(keep, "keep", 4, S),
        dev(evicted, "evicted", 4, S), dev(source, "source", 4, weight.numel()), dev(workspace, "workspace", 1, need), need,
        _rac._stream(stream))
    if status:
        _rac._check(status, "rac_cache_evict")


def rac_predictor_tree_workspace(cfg, cache: CacheConfig, tree: TreeConfig) -> int:
    return int(_rac.library().rac_predictor_tree_workspace(ctypes.byref(cfg._c()), cache._ref, tree._ref))


def rac_predictor_tree_step(cfg, cache: CacheConfig, tree: TreeConfig, weights, pool, table, lengths, q_start,
                            draft_start, slot, pos, h_prev, draft_k, draft_v, ref_out, workspace, *, mask=None,
                            stream=None) -> None:
    """One predictor step over drafted trees (cfg: PredictorConfig): row r's
    input h_prev[r] (bf16 [rows][hidden]) at position pos[r] stores its key and
    value in row slot[r] of draft_k and draft_v (bf16 [draft_rows][heads][64]) and
    predicts ref_out[r]."""
    dev, R, S, need = _rac._dev, tree.rows, cache.seqs, rac_predictor_tree_workspace(cfg, cache, tree)
    kp, ks, drafted = _drafts(draft_k, "draft_k", 0, cfg.heads, 64)
    vp, vs, _ = _drafts(draft_v, "draft_v", drafted, cfg.heads, 64)
    if drafted > 1 and (ks != cfg.model or vs != cfg.model):
        raise ValueError("draft_k and draft_v: expected contiguous rows")
    words = _words(mask)
    _rac._check(_rac.library().rac_predictor_tree_step(
        ctypes.byref(cfg._c()), cache._ref, tree._ref, dev(weights, "weights", 1, 0), _pool(cache, pool),
        dev(table, "table", 4, S * cache.max_pages), dev(lengths, "lengths", 4, S), dev(q_start, "q_start", 4, S + 1),
        dev(draft_start, "draft_start", 4, S + 1), dev(slot, "slot", 4, R), dev(pos, "pos", 4, R),
        dev(mask, "mask", 8, R * words), words, dev(h_prev, "h_prev", 2, R * cfg.hidden), kp, vp, drafted,
        dev(ref_out, "ref_out", 2, R * cfg.hidden), dev(workspace, "workspace", 1, need), need, _rac._stream(stream)),
        "rac_predictor_tree_step")
