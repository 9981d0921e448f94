"""Binding of the cache's operators (include/fairserve_cache.h): a cache held in 4 bits, and
the pages that the requests of a cache share; on torch's current stream.

Argument marshalling only, in the manner of ``engine``: descriptors (KVCache4, CacheLayers,
PagePool) check their tensors once and keep them alive, calls raise the status word `err`
and do not clear it.  Attention with sinks over the 16-bit cache is fs_paged_attention's
argument ``sinks``.
"""
from __future__ import annotations

import ctypes as C

from . import engine
from .engine import (FS_BF16, FS_F16, KVCache, Rope, Step, _bounded, _done, _lib, _new, _on,
                     _one_device, _rows, _there, _torch, _vector, _want, _want_32, _workspace,
                     cleared_err_word)

EXPORTED_CACHE = ("fs_attention_sinks_workspace", "fs_paged_attention_sinks", "fs_rope_append4",
                  "fs_cache4_rows", "fs_attention4_workspace", "fs_paged_attention4",
                  "fs_pages_free", "fs_pages_workspace", "fs_pages_fork", "fs_pages_compact",
                  "fs_pages_copy", "fs_pages_copy4")


class fs_kv_cache4(C.Structure):
    _fields_ = [("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("page_size", C.c_int32),
                ("n_pages", C.c_int64), ("k", C.c_void_p), ("v", C.c_void_p),
                ("page_stride", C.c_int64), ("head_stride", C.c_int64),
                ("token_stride", C.c_int64), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("scale_page_stride", C.c_int64), ("scale_head_stride", C.c_int64),
                ("scale_token_stride", C.c_int64), ("table", C.c_void_p),
                ("table_stride", C.c_int64)]


class fs_pages(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_rows", C.c_int32),
                ("width", C.c_int32), ("refs", C.c_void_p), ("table", C.c_void_p),
                ("held", C.c_void_p), ("table_stride", C.c_int64)]


def signatures():
    P, I32, I64, SZ, F = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
    return {
        "fs_attention_sinks_workspace": ([P, P, I32, I32, I32], SZ),
        "fs_paged_attention_sinks": ([P, P, I32, F, I32, I32, P, I64, P, I64, P, P, SZ, P, P], I32),
        "fs_rope_append4": ([P, P, P, I32, I32, P, I64, P, I64, P, I64, P, I64, P, P], I32),
        "fs_cache4_rows": ([P, P, I32, P, I64, P, I64, P, P], I32),
        "fs_attention4_workspace": ([P, P, I32, I32, I32], SZ),
        "fs_paged_attention4": ([P, P, I32, I32, F, I32, I32, P, I64, P, I64, P, P, SZ, P, P], I32),
        "fs_pages_free": ([P, I32, P, P, P], I32),
        "fs_pages_workspace": ([P, I32], SZ),
        "fs_pages_fork": ([P, I32, P, P, P, P, P, P, P, SZ, P, P], I32),
        "fs_pages_compact": ([P, P, P, I64, P, P, P, P, SZ, P, P], I32),
        "fs_pages_copy": ([P, I32, I32, P, P, P, P, P], I32),
        "fs_pages_copy4": ([P, I32, I32, P, P, P, P, P], I32),
    }


def _row_type(dtype):
    torch = _torch()
    if dtype == torch.bfloat16:
        return FS_BF16
    if dtype == torch.float16:
        return FS_F16
    raise TypeError(f"dtype {dtype} is not supported (bfloat16, float16)")


class KVCache4:
    """A paged cache in 4 bits: codes k, v uint8 [pages][kv_heads][page_size][head_dim / 2] and
    scale bytes k_scale, v_scale uint8 [pages][kv_heads][page_size][head_dim / 32] (any strides
    with the last dimension packed; k and v, and their scales, alike), table as in KVCache."""

    def __init__(self, k, v, k_scale, v_scale, table):
        torch = _torch()
        u8 = torch.uint8
        _want(k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and
              k.dtype == v.dtype == u8, "k and v: uint8, four dimensions, alike in shape and strides")
        n, h, page, half = k.shape
        _want(half % 16 == 0, "k, v: head_dim a multiple of 32")
        _want(k_scale.shape == v_scale.shape == (n, h, page, half // 16) and
              k_scale.stride() == v_scale.stride() and k_scale.dtype == v_scale.dtype == u8,
              "k_scale and v_scale: uint8 [pages][kv_heads][page_size][head_dim / 32], alike in strides")
        _want((half <= 1 or k.stride(3) == 1) and (half <= 16 or k_scale.stride(3) == 1),
              "k, v and their scales: the last dimension is not packed")
        _want(table.dim() == 2 and table.dtype == torch.int32 and
              (table.shape[1] <= 1 or table.stride(1) == 1), "table: int32 [n][width]")
        _want_32("k, v", *k.shape[1:])
        self.k, self.v, self.k_scale, self.v_scale, self.table = k, v, k_scale, v_scale, table
        self.gpu = _one_device(k, v, k_scale, v_scale, table)
        self.n_kv_heads, self.head_dim = h, 2 * half
        self.n_seqs, self.most_kv = table.shape[0], table.shape[1] * page
        self.s = fs_kv_cache4(h, 2 * half, page, n, k.data_ptr(), v.data_ptr(), *k.stride()[:3],
                              k_scale.data_ptr(), v_scale.data_ptr(), *k_scale.stride()[:3],
                              table.data_ptr(), KVCache._table_stride(table))
        self.ref = C.addressof(self.s)

    check = KVCache.check


class CacheLayers:
    """The caches of a model's layers, alike in all but their addresses (KVCache or KVCache4),
    for copies of pages in all of them at once."""

    def __init__(self, caches):
        caches = list(caches)
        _want(len(caches) > 0, "caches: at least one")
        kind = type(caches[0])
        _want(kind in (KVCache, KVCache4) and all(type(c) is kind for c in caches),
              "caches: all KVCache or all KVCache4")
        _want(len({c.gpu for c in caches}) == 1, "caches: one GPU")
        self.caches, self.gpu, self.n = caches, caches[0].gpu, len(caches)
        self.four = kind is KVCache4
        self.s = (type(caches[0].s) * self.n)(*(c.s for c in caches))
        self.ref = C.addressof(self.s)


class PagePool:
    """The pages of a cache: refs int32 [pages] (how many rows hold a page), the page table
    int32 [rows][width] and held int32 [rows] (the pages each row holds)."""

    def __init__(self, refs, table, held, page_size):
        torch = _torch()
        _want(table.dim() == 2 and table.dtype == torch.int32 and
              (table.shape[1] <= 1 or table.stride(1) == 1), "table: int32 [rows][width]")
        _want_32("refs, table", refs.shape[0], *table.shape)
        rp = _vector(refs, torch.int32, refs.shape[0], "refs")
        _want(held.shape[0] == table.shape[0], "held: a value for every row of the table")
        self.refs, self.table, self.held = refs, table, held
        self.gpu = _one_device(refs, table, held)
        self.n_pages, self.n_rows, self.width = refs.shape[0], table.shape[0], table.shape[1]
        self.s = fs_pages(self.n_pages, int(page_size), self.n_rows, self.width, rp,
                          table.data_ptr(), _vector(held, torch.int32, self.n_rows, "held"),
                          KVCache._table_stride(table))
        self.ref = C.addressof(self.s)
        self._bytes = {}

    def workspace(self, n):
        """Bytes of workspace that a fork of n rows (0: a compaction) takes."""
        need = self._bytes.get(n)
        if need is None:
            need = self._bytes[n] = _lib().fs_pages_workspace(self.ref, n)
        return need


def fs_rope_append4(step: Step, cache: KVCache4, rope: Rope, q, k, v, q_out=None, err=None,
                    check=True):
    """fs_rope_append into a cache of 4 bits; returns the turned q (q_out, which may be q)."""
    T, HK, D, gpu, dtype = step.rows, cache.n_kv_heads, cache.head_dim, step.gpu, k.dtype
    if v.dtype != dtype or (q is not None and q.dtype != dtype):
        raise ValueError("q, k, v: one dtype")
    code = _row_type(dtype)
    cache.check(step, "fs_rope_append4")
    if rope.rows is not None and rope.rows < T:
        raise ValueError("pos: a position for every row")
    if cache.gpu != gpu or rope.gpu != gpu:
        raise ValueError("cache, rope and step: one GPU")
    _on(gpu, q, k, v, q_out, err)
    if gpu != engine._current_gpu():
        return _there(gpu, fs_rope_append4, step, cache, rope, q, k, v, q_out, err, check)
    kp, ks = _rows(k, "k", (T, HK, D))
    vp, vs = _rows(v, "v", (T, HK, D))
    H, qp, qs, op, os_ = 0, None, 0, None, 0
    if q is not None:
        H = q.shape[1]
        if H >= 1 << 31:
            raise ValueError("q: beyond 32 bits")
        qp, qs = _rows(q, "q", (T, H, D))
        if q_out is None:
            q_out = _torch().empty_like(q)  # packed, whatever q's row stride
            op, os_ = q_out.data_ptr(), H * D
        else:
            _want(q_out.dtype == dtype, "q_out: the dtype of q")
            op, os_ = _rows(q_out, "q_out", (T, H, D))
    if err is None:
        err = cleared_err_word(k.device)
    code = _lib().fs_rope_append4(step.ref, cache.ref, rope.ref, code, H, qp, qs, kp, ks, vp, vs,
                                  op, os_, err.data_ptr(), engine._raw_stream(gpu))
    if code or check:
        _done(code, "fs_rope_append4", err, check)
    return q_out


def fs_cache4_rows(step: Step, cache: KVCache4, dtype=None, k=None, v=None, err=None, check=True):
    """What the cache holds at the step's rows: (k, v) [rows][kv_heads][head_dim] of dtype (made
    where not given; bfloat16 unless k, v or dtype say otherwise)."""
    torch = _torch()
    T, HK, D, gpu = step.rows, cache.n_kv_heads, cache.head_dim, step.gpu
    if dtype is None:
        dtype = k.dtype if k is not None else v.dtype if v is not None else torch.bfloat16
    code = _row_type(dtype)
    if (k is not None and k.dtype != dtype) or (v is not None and v.dtype != dtype):
        raise ValueError("k, v: the dtype asked for")
    cache.check(step, "fs_cache4_rows")
    if cache.gpu != gpu:
        raise ValueError("cache and step: one GPU")
    _on(gpu, step.q_off, k, v, err)
    if gpu != engine._current_gpu():
        return _there(gpu, fs_cache4_rows, step, cache, dtype, k, v, err, check)
    if k is None:
        k = torch.empty_strided((T, HK, D), (HK * D, D, 1), dtype=dtype, device=cache.k.device)
        kp, ks = k.data_ptr(), HK * D
    else:
        kp, ks = _rows(k, "k", (T, HK, D))
    if v is None:
        v = torch.empty_strided((T, HK, D), (HK * D, D, 1), dtype=dtype, device=cache.k.device)
        vp, vs = v.data_ptr(), HK * D
    else:
        vp, vs = _rows(v, "v", (T, HK, D))
    if err is None:
        err = cleared_err_word(cache.k.device)
    code = _lib().fs_cache4_rows(step.ref, cache.ref, code, kp, ks, vp, vs, err.data_ptr(),
                                 engine._raw_stream(gpu))
    if code or check:
        _done(code, "fs_cache4_rows", err, check)
    return k, v


def fs_paged_attention4(step: Step, cache: KVCache4, q, scale, window=0, sinks=0, out=None,
                        lse=None, want_lse=False, ws=None, err=None, check=True):
    """fs_paged_attention over a cache of 4 bits; returns out, or (out, lse) when the
    log-sum-exp [rows][heads] is wanted."""
    shape, gpu = q.shape, step.gpu
    T, H, D = shape
    code = _row_type(q.dtype)
    if D != cache.head_dim:
        raise ValueError("q: the cache's head_dim")
    cache.check(step, "fs_paged_attention4")
    if cache.gpu != gpu:
        raise ValueError("cache and step: one GPU")
    _on(gpu, q, out, lse, ws, err)
    if gpu != engine._current_gpu():
        return _there(gpu, fs_paged_attention4, step, cache, q, scale, window, sinks, out, lse,
                      want_lse, ws, err, check)
    qp, qs = _rows(q, "q", (step.rows, H, D))
    if out is None:
        out = _torch().empty_like(q)  # packed, whatever q's row stride
        op, os_ = out.data_ptr(), H * D
    else:
        _want(out.dtype == q.dtype, "out: the dtype of q")
        op, os_ = _rows(out, "out", (T, H, D))
    lp = None
    if lse is not None:
        _want(lse.dtype == _torch().float32 and lse.is_contiguous() and lse.numel() == T * H,
              "lse: packed float32 [rows][heads]")
        lp = lse.data_ptr()
    elif want_lse:
        lse = _new((T, H), _torch().float32, q.device)
        lp = lse.data_ptr()
    if err is None:
        err = cleared_err_word(q.device)
    L = _lib()
    window, sinks = _bounded(window), _bounded(sinks)
    ws, wp, wn = _workspace(ws, L.fs_attention4_workspace(step.ref, cache.ref, H, window, sinks), q)
    code = L.fs_paged_attention4(step.ref, cache.ref, code, H, scale, window, sinks, qp, qs, op, os_,
                                 lp, wp, wn, err.data_ptr(), engine._raw_stream(gpu))
    if code or check:
        _done(code, "fs_paged_attention4", err, check)
    return out if lse is None else (out, lse)


_i32 = None


def _ids(t, n, name):
    """A contiguous int32 vector of n values."""
    global _i32
    if _i32 is None:
        _i32 = _torch().int32
    if t.dtype is not _i32 or t.dim() != 1 or t.size(0) != n or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous int32 vector of {n} values")
    return t.data_ptr()


def fs_pages_free(pool: PagePool, rows, err=None, check=True):
    """Lets go of all pages of the table's rows `rows` (int32 on the device)."""
    gpu = pool.gpu
    _on(gpu, rows, err)
    if gpu != engine._current_gpu():
        return _there(gpu, fs_pages_free, pool, rows, err, check)
    n = rows.size(0)
    _want_32("rows", n)
    rp = _ids(rows, n, "rows")
    if err is None:
        err = cleared_err_word(rows.device)
    code = _lib().fs_pages_free(pool.ref, n, rp, err.data_ptr(), engine._raw_stream(gpu))
    if code or check:
        _done(code, "fs_pages_free", err, check)


def fs_pages_fork(pool: PagePool, parent, child, shared, room, src=None, dst=None, ws=None,
                  err=None, check=True):
    """Gives each row child[i] the first shared[i] tokens of row parent[i] (-1: none) and room
    for room[i] tokens; returns (src, dst) [n] for fs_pages_copy (-1: no page to copy)."""
    torch = _torch()
    gpu = pool.gpu
    _on(gpu, parent, child, shared, room, src, dst, ws, err)
    if gpu != engine._current_gpu():
        return _there(gpu, fs_pages_fork, pool, parent, child, shared, room, src, dst, ws, err, check)
    n = child.size(0)
    _want_32("child", n)
    pp, cp = _ids(parent, n, "parent"), _ids(child, n, "child")
    sp, mp = _ids(shared, n, "shared"), _ids(room, n, "room")
    if src is None:
        src = torch.empty_like(child)
        srcp = src.data_ptr()
    else:
        srcp = _ids(src, n, "src")
    if dst is None:
        dst = torch.empty_like(child)
        dstp = dst.data_ptr()
    else:
        dstp = _ids(dst, n, "dst")
    if err is None:
        err = cleared_err_word(child.device)
    L = _lib()
    ws, wp, wn = _workspace(ws, pool.workspace(n), child)
    code = L.fs_pages_fork(pool.ref, n, pp, cp, sp, mp, srcp, dstp, wp, wn, err.data_ptr(),
                           engine._raw_stream(gpu))
    if code or check:
        _done(code, "fs_pages_fork", err, check)
    return src, dst


def fs_pages_compact(pool: PagePool, refs_out=None, table_out=None, src=None, dst=None, count=None,
                     ws=None, err=None, check=True):
    """Moves the pages in use to the lowest ids: refs and table get the new ids, in place unless
    refs_out and table_out are given; returns (src, dst, count) for fs_pages_copy."""
    torch = _torch()
    gpu, n = pool.gpu, pool.n_pages // 2
    _on(gpu, refs_out, table_out, src, dst, count, ws, err)
    if gpu != engine._current_gpu():
        return _there(gpu, fs_pages_compact, pool, refs_out, table_out, src, dst, count, ws, err, check)
    rp = pool.s.refs if refs_out is None else _ids(refs_out, pool.n_pages, "refs_out")
    if table_out is None:
        tp, stride = pool.s.table, pool.s.table_stride
    else:
        _want(table_out.dtype == torch.int32 and table_out.shape == pool.table.shape and
              (pool.width <= 1 or table_out.stride(1) == 1), "table_out: like the table")
        tp, stride = table_out.data_ptr(), KVCache._table_stride(table_out)
    like = pool.refs
    src = like.new_empty(n) if src is None else src
    dst = like.new_empty(n) if dst is None else dst
    count = like.new_empty(1) if count is None else count
    sp, dp, cp = _ids(src, n, "src"), _ids(dst, n, "dst"), _ids(count, 1, "count")
    if err is None:
        err = cleared_err_word(like.device)
    L = _lib()
    ws, wp, wn = _workspace(ws, pool.workspace(0), like)
    code = L.fs_pages_compact(pool.ref, rp, tp, stride, sp, dp, cp, wp, wn,
                              err.data_ptr(), engine._raw_stream(gpu))
    if code or check:
        _done(code, "fs_pages_compact", err, check)
    return src, dst, count


def fs_pages_copy(caches, src, dst, count=None, err=None, check=True):
    """Copies page src[i] to page dst[i] (-1, -1: none; i < count where it is given) in a
    KVCache, a KVCache4 or the CacheLayers of several."""
    layers = caches if isinstance(caches, CacheLayers) else CacheLayers([caches])
    gpu = layers.gpu
    _on(gpu, src, dst, count, err)
    if gpu != engine._current_gpu():
        return _there(gpu, fs_pages_copy, layers, src, dst, count, err, check)
    n = src.size(0)
    _want_32("src", n)
    sp, dp = _ids(src, n, "src"), _ids(dst, n, "dst")
    cp = None if count is None else _ids(count, 1, "count")
    if err is None:
        err = cleared_err_word(src.device)
    L = _lib()
    copy = L.fs_pages_copy4 if layers.four else L.fs_pages_copy
    code = copy(layers.ref, layers.n, n, sp, dp, cp, err.data_ptr(), engine._raw_stream(gpu))
    if code or check:
        _done(code, "fs_pages_copy", err, check)

