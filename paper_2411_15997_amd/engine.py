"""Binding of the engine-step operators (include/fairserve_engine.h): descriptors over the
caller's tensors and the calls, on torch's current stream.

Argument marshalling only.  A descriptor (Step, KVCache, Adapters, Rope, Sampling) checks
its tensors once and keeps them alive; a serving loop makes it once and calls with it.
The calls raise the status word `err` and do not clear it: pass one cleared word
(cleared_err_word, fs_clear_status) to every call of a step with check=False and look at
it once with sync_check.  Without `err` a call takes a cleared word of its own.
"""
from __future__ import annotations

import ctypes as C

import numpy as np

FS_BF16, FS_F16, FS_F32 = 0, 1, 2
FS_ROPE_PLAIN, FS_ROPE_LINEAR, FS_ROPE_BASE, FS_ROPE_PARTS = 0, 1, 2, 3
FS_E_ARG = 1
ALIGN = 256

EXPORTED_ENGINE = ("fs_clear_status", "fs_adapter_workspace", "fs_adapter_linear",
                   "fs_rope_frequencies", "fs_rope_append", "fs_attention_workspace",
                   "fs_paged_attention", "fs_sample_workspace", "fs_sample")


class fs_step(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("q_off_h", C.c_void_p), ("q_off", C.c_void_p),
                ("kv_len", C.c_void_p), ("max_kv", C.c_int32)]


class fs_kv_cache(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("page_size", C.c_int32), ("n_pages", C.c_int64), ("k", C.c_void_p),
                ("v", C.c_void_p), ("page_stride", C.c_int64), ("head_stride", C.c_int64),
                ("token_stride", C.c_int64), ("table", C.c_void_p), ("table_stride", C.c_int64)]


class fs_adapters(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("in_features", C.c_int32), ("out_features", C.c_int32),
                ("n_adapters", C.c_int32), ("max_rank", C.c_int32), ("a", C.c_void_p),
                ("b", C.c_void_p), ("rank", C.c_void_p), ("scale", C.c_void_p),
                ("adapter", C.c_void_p)]


class fs_rope(C.Structure):
    _fields_ = [("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("inv_freq", C.c_void_p),
                ("factor", C.c_float), ("pos", C.c_void_p)]


class fs_sampling(C.Structure):
    _fields_ = [("temperature", C.c_void_p), ("top_k", C.c_void_p), ("top_p", C.c_void_p),
                ("min_p", C.c_void_p)]


def signatures():
    P, I32, I64, SZ, F, D = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float, C.c_double
    S = K = A = R = G = P  # the descriptors' addresses
    return {
        "fs_clear_status": ([P, P], I32),
        "fs_adapter_workspace": ([S, A], SZ),
        "fs_adapter_linear": ([S, A, P, I64, P, P, I64, P, SZ, P, P], I32),
        "fs_rope_frequencies": ([I32, D, I32, D, I32, D, D, P, P], I32),
        "fs_rope_append": ([S, K, R, I32, P, I64, P, I64, P, I64, P, I64, P, P], I32),
        "fs_attention_workspace": ([S, K, I32, I32], SZ),
        "fs_paged_attention": ([S, K, I32, F, I32, P, I64, P, I64, P, P, SZ, P, P], I32),
        "fs_sample_workspace": ([I32, I32, I32], SZ),
        "fs_sample": ([I32, I32, I32, P, I64, G, P, P, P, P, P, SZ, P, P], I32),
    }


_fns = None


def _lib():
    """The loaded library's entry points (looked up once)."""
    global _fns
    if _fns is None:
        from . import _lib as load
        _fns = load()
    return _fns


_torch_mod = None


def _torch():
    global _torch_mod
    if _torch_mod is None:
        import torch
        _torch_mod = torch
    return _torch_mod


def _fail(code, where):
    from . import FairServeError
    raise FairServeError(code, where)


def _dtype_code(t):
    torch = _torch()
    d = t.dtype
    code = FS_BF16 if d == torch.bfloat16 else FS_F16 if d == torch.float16 else \
        FS_F32 if d == torch.float32 else None
    if code is None:
        raise TypeError(f"dtype {t.dtype} is not supported (bfloat16, float16, float32)")
    return code


def _want(cond, what):
    if not cond:
        raise ValueError(what)


def _want_32(what, *sizes):
    """Sizes that the library takes as int32 (ctypes would cut larger ones down to 32 bits)."""
    _want(all(-1 << 31 <= n < 1 << 31 for n in sizes), f"{what}: beyond 32 bits")


def _raw_stream(gpu):
    """The current stream of the GPU of that index; itself looked up once."""
    global _raw_stream
    _raw_stream = _torch()._C._cuda_getCurrentRawStream
    return _raw_stream(gpu)


def _current_gpu():
    """The index of the current GPU; itself looked up once."""
    global _current_gpu
    _current_gpu = _torch()._C._cuda_getDevice
    return _current_gpu()


def _there(gpu, call, *args):
    """The call with its tensors' GPU current.  (The handle of a default stream names no GPU:
    kernels would go to the current one.)"""
    with _torch().cuda.device(gpu):
        return call(*args)


def _one_device(*tensors):
    """The index of the device of the tensors given (None among them is left out)."""
    devices = {t.device for t in tensors if t is not None}
    _want(len(devices) == 1, f"tensors on one device, not on {sorted(map(str, devices))}")
    return devices.pop().index


def _on(index, *tensors):
    """The tensors given are on the GPU of that index (what the host could not read the GPU
    would fault on)."""
    if index is None:
        raise ValueError("every tensor of a call on one GPU")
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError("every tensor of a call on one GPU")


def _vector(t, dtype, n, name):
    """A contiguous device vector of `n` values of `dtype`, or None."""
    if t is None:
        return None
    if t.dtype != dtype or t.dim() != 1 or t.shape[0] < n or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} vector of {n} values")
    return t.data_ptr()


def _rows(t, name, shape):
    """Pointer and row stride of a tensor of rows whose inner dimensions are packed."""
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, wanted {shape}")
    st = t.stride()
    inner = shape[-1]
    if st[-1] != 1 and inner != 1 or len(st) == 3 and st[1] != inner and shape[1] != 1:
        raise ValueError(f"{name}: inner dimensions are not packed")
    if shape[0] > 1:
        return t.data_ptr(), st[0]
    return t.data_ptr(), (inner if len(st) == 2 else inner * shape[1])


def _new(shape, dtype, device):
    """A packed tensor (two dimensions); empty_strided is torch's cheapest way to one."""
    return _torch().empty_strided(shape, (shape[1], 1), dtype=dtype, device=device)


def _workspace(ws, need, like):
    if need == 0:
        return None, None, 0
    if ws is None:
        ws = _torch().empty(need, dtype=_torch().uint8, device=like.device)
    elif not ws.is_contiguous():
        raise ValueError("ws: packed (its size is that of its values)")
    return ws, ws.data_ptr(), ws.numel() * ws.element_size()


def cleared_err_word(device="cuda"):
    return _torch().zeros(1, dtype=_torch().int32, device=device)


def fs_clear_status(err):
    gpu = err.get_device()
    _on(None if gpu < 0 else gpu, err)
    if gpu != _current_gpu():
        return _there(gpu, fs_clear_status, err)
    code = _lib().fs_clear_status(err.data_ptr(), _raw_stream(gpu))
    if code:
        _fail(code, "fs_clear_status")


def _done(code, where, err, check):
    if code:
        _fail(code, where)
    if check:
        from . import sync_check
        sync_check(err, where)


class Step:
    """The requests of one engine step: q_off (host sequence and its int32 device copy,
    made when not given; one that is given has to hold the same values, they are not
    compared), kv_len [n] int32 on the device and the host bound max_kv."""

    def __init__(self, q_off_h, q_off=None, kv_len=None, max_kv=0, device="cuda"):
        torch = _torch()
        # a copy: the grids and the outputs' sizes are taken from it at every call
        given = np.asarray(q_off_h)
        self.q_off_h = given.astype(np.int32)  # astype copies
        _want((self.q_off_h == given).all(), "q_off: beyond 32 bits")
        n = self.q_off_h.shape[0] - 1
        _want(n >= 0, "q_off: at least one value")
        self.n, self.rows = n, int(self.q_off_h[-1])
        self.q_off = torch.from_numpy(self.q_off_h.copy()).to(device) if q_off is None else q_off
        self.kv_len, self.max_kv = kv_len, int(max_kv)
        _want_32("max_kv", self.max_kv)
        self.gpu = _one_device(self.q_off, kv_len)
        self.s = fs_step(n, self.q_off_h.ctypes.data,
                         _vector(self.q_off, torch.int32, n + 1, "q_off"),
                         _vector(kv_len, torch.int32, n, "kv_len"), self.max_kv)
        self.ref = C.addressof(self.s)


class KVCache:
    """A paged cache: k and v [pages][kv_heads][page_size][head_dim] (any strides with the
    last dimension packed; k and v alike), table [n][width] int32 of page ids (rows may be
    further apart than their width; a step's max_kv keeps to the width)."""

    def __init__(self, k, v, table):
        torch = _torch()
        _want(k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and
              k.dtype == v.dtype, "k and v: four dimensions, alike in shape, strides and dtype")
        _want(k.shape[3] == 1 or k.stride(3) == 1, "k, v: the last dimension is not packed")
        _want(table.dim() == 2 and table.dtype == torch.int32 and
              (table.shape[1] <= 1 or table.stride(1) == 1), "table: int32 [n][width]")
        _want_32("k, v", *k.shape[1:])
        self.k, self.v, self.table, self.gpu = k, v, table, _one_device(k, v, table)
        self.n_kv_heads, self.head_dim, self.dtype = k.shape[1], k.shape[3], k.dtype
        self.n_seqs, self.most_kv = table.shape[0], table.shape[1] * k.shape[2]
        self.s = fs_kv_cache(_dtype_code(k), k.shape[1], k.shape[3], k.shape[2], k.shape[0],
                             k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2),
                             table.data_ptr(), self._table_stride(table))
        self.ref = C.addressof(self.s)

    @staticmethod
    def _table_stride(table):
        if table.shape[0] > 1:
            _want(table.stride(0) >= table.shape[1], "table: rows overlap")
            return table.stride(0)
        return table.shape[1]

    def check(self, step, where):
        """A page id for every token that a request of the step may hold (the library knows
        how far apart the table's rows are, not their width)."""
        if self.n_seqs < step.n:
            raise ValueError("table: a row for every request")
        if step.max_kv > self.most_kv and step.n > 0:
            _fail(FS_E_ARG, where)


class Adapters:
    """Low-rank adapters: a [n][max_rank][K], b [n][N][max_rank] (packed), adapter [n_seqs]
    int32 (-1: none), rank [n] int32 and scale [n] float (each may be None)."""

    def __init__(self, a, b, adapter, rank=None, scale=None):
        torch = _torch()
        _want(a.dim() == 3 and b.dim() == 3 and a.is_contiguous() and b.is_contiguous() and
              a.dtype == b.dtype and a.shape[0] == b.shape[0] and a.shape[1] == b.shape[2],
              "a [n][max_rank][K] and b [n][N][max_rank]: packed, of one dtype")
        n, r, k = a.shape
        _want_32("a, b", n, r, k, b.shape[1])
        self.keep = (a, b, adapter, rank, scale)
        self.gpu = _one_device(*self.keep)
        self.dtype, self.K, self.N, self.n_seqs = a.dtype, k, b.shape[1], adapter.shape[0]
        self.s = fs_adapters(_dtype_code(a), k, b.shape[1], n, r, a.data_ptr(), b.data_ptr(),
                             _vector(rank, torch.int32, n, "rank"),
                             _vector(scale, torch.float32, n, "scale"),
                             _vector(adapter, torch.int32, 0, "adapter"))
        self.ref = C.addressof(self.s)


class Rope:
    """Rotary positions: inv_freq [rotary_dim / 2] float on the device, the pair layout, the
    factor of long-context scaling and, when not the cache positions, pos [rows] int32."""

    def __init__(self, inv_freq, interleaved=False, factor=1.0, pos=None):
        torch = _torch()
        self.rows = None if pos is None else pos.shape[0]
        self.inv_freq, self.pos, self.gpu = inv_freq, pos, _one_device(inv_freq, pos)
        n = inv_freq.shape[0]
        _want_32("inv_freq", 2 * n)
        self.s = fs_rope(2 * n, int(bool(interleaved)), _vector(inv_freq, torch.float32, n, "inv_freq"),
                         float(factor), _vector(pos, torch.int32, 0, "pos"))
        self.ref = C.addressof(self.s)


class Sampling:
    """Per-row sampling settings on the device (each may be None)."""

    def __init__(self, temperature=None, top_k=None, top_p=None, min_p=None):
        torch = _torch()
        self.keep = (temperature, top_k, top_p, min_p)
        self.rows = min((t.shape[0] for t in self.keep if t is not None), default=None)
        self.gpu = _one_device(*self.keep) if self.rows is not None else None
        self.s = fs_sampling(_vector(temperature, torch.float32, 0, "temperature"),
                             _vector(top_k, torch.int32, 0, "top_k"),
                             _vector(top_p, torch.float32, 0, "top_p"),
                             _vector(min_p, torch.float32, 0, "min_p"))
        self.ref = C.addressof(self.s)


def fs_adapter_linear(step: Step, adapters: Adapters, x, w, y=None, ws=None, err=None, check=True):
    """y = x w^T plus every request's adapter; x [rows][K], w [N][K], returns y [rows][N]."""
    K, N, dtype, gpu, T = adapters.K, adapters.N, adapters.dtype, step.gpu, step.rows
    xp, xs = _rows(x, "x", (T, K))
    if w.shape != (N, K) or not w.is_contiguous():
        raise ValueError("w: packed [N][K]")
    if x.dtype != dtype or w.dtype != dtype:
        raise ValueError("x, w and adapters: one dtype")
    if adapters.n_seqs < step.n:
        raise ValueError("adapter: an id for every request")
    if adapters.gpu != gpu:
        raise ValueError("adapters and step: one GPU")
    _on(gpu, x, w, y, ws, err)
    if gpu != _current_gpu():
        return _there(gpu, fs_adapter_linear, step, adapters, x, w, y, ws, err, check)
    if y is None:
        y = _new((T, N), dtype, x.device)
        yp, ys = y.data_ptr(), N
    else:
        _want(y.dtype == dtype, "y: the dtype of x")
        yp, ys = _rows(y, "y", (T, N))
    if err is None:
        err = cleared_err_word(x.device)
    L = _lib()
    ws, wp, wn = _workspace(ws, L.fs_adapter_workspace(step.ref, adapters.ref), x)
    code = L.fs_adapter_linear(step.ref, adapters.ref, xp, xs, w.data_ptr(), yp, ys, wp, wn,
                               err.data_ptr(), _raw_stream(gpu))
    if code or check:
        _done(code, "fs_adapter_linear", err, check)
    return y


def fs_rope_frequencies(rotary_dim, theta0=10000.0, scaling=FS_ROPE_PLAIN, scale=1.0,
                        original_len=4096, beta_fast=32.0, beta_slow=1.0):
    """Host helper: (inv_freq [rotary_dim / 2] float32, factor)."""
    f = np.zeros(max(1, rotary_dim // 2), np.float32)
    m = np.zeros(1, np.float32)
    code = _lib().fs_rope_frequencies(int(rotary_dim), float(theta0), int(scaling), float(scale),
                                      int(original_len), float(beta_fast), float(beta_slow),
                                      f.ctypes.data, m.ctypes.data)
    if code:
        _fail(code, "fs_rope_frequencies")
    return f[:rotary_dim // 2], float(m[0])


def fs_rope_append(step: Step, cache: KVCache, rope: Rope, q, k, v, q_out=None, err=None,
                   check=True):
    """Turns q [rows][heads][dim] and k, appends k and v [rows][kv_heads][dim] to the cache;
    returns the turned q (q_out, which may be q itself)."""
    T, HK, D, dtype, gpu = step.rows, cache.n_kv_heads, cache.head_dim, cache.dtype, step.gpu
    if k.dtype != dtype or v.dtype != dtype or (q is not None and q.dtype != dtype):
        raise ValueError("q, k, v: the cache's dtype")
    cache.check(step, "fs_rope_append")
    if rope.rows is not None and rope.rows < T:
        raise ValueError("pos: a position for every row")
    if cache.gpu != gpu or rope.gpu != gpu:
        raise ValueError("cache, rope and step: one GPU")
    _on(gpu, q, k, v, q_out, err)
    if gpu != _current_gpu():
        return _there(gpu, fs_rope_append, step, cache, rope, q, k, v, q_out, err, check)
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
            _want(q_out.dtype == q.dtype, "q_out: the dtype of q")
            op, os_ = _rows(q_out, "q_out", (T, H, D))
    if err is None:
        err = cleared_err_word(k.device)
    code = _lib().fs_rope_append(step.ref, cache.ref, rope.ref, H, qp, qs, kp, ks, vp, vs, op, os_,
                                 err.data_ptr(), _raw_stream(gpu))
    if code or check:
        _done(code, "fs_rope_append", err, check)
    return q_out


def fs_paged_attention(step: Step, cache: KVCache, q, scale, window=0, out=None, lse=None,
                       want_lse=False, ws=None, err=None, check=True):
    """Attention of q [rows][heads][dim] over the cache; returns out, or (out, lse) when the
    log-sum-exp [rows][heads] is wanted."""
    shape, gpu = q.shape, step.gpu
    T, H, D = shape
    if q.dtype != cache.dtype or D != cache.head_dim:
        raise ValueError("q: the cache's dtype and head_dim")
    cache.check(step, "fs_paged_attention")
    if cache.gpu != gpu:
        raise ValueError("cache and step: one GPU")
    _on(gpu, q, out, lse, ws, err)
    if gpu != _current_gpu():
        return _there(gpu, fs_paged_attention, step, cache, q, scale, window, out, lse, want_lse, ws,
                      err, check)
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
    window = max(-1, min(int(window), 0x7fffffff))  # one beyond every length is none
    ws, wp, wn = _workspace(ws, L.fs_attention_workspace(step.ref, cache.ref, H, window), q)
    code = L.fs_paged_attention(step.ref, cache.ref, H, scale, window, qp, qs, op, os_, lp, wp, wn,
                                err.data_ptr(), _raw_stream(gpu))
    if code or check:
        _done(code, "fs_paged_attention", err, check)
    return out if lse is None else (out, lse)


def fs_sample(logits, u, sampling: Sampling, token=None, logprob=None, kept=None, ws=None,
              err=None, check=True):
    """The next token of each row of logits [rows][vocab] for the random numbers u [rows];
    returns (token int32, logprob float32, kept int32), each [rows]."""
    torch = _torch()
    n, V = logits.shape
    if n >= 1 << 31 or V >= 1 << 31:
        raise ValueError("logits: beyond 32 bits")
    stride = logits.stride()
    _want(n <= 1 or stride[0] >= V, "logits: rows overlap")
    _want(V == 1 or stride[1] == 1, "logits: rows are not packed")
    _want(sampling.rows is None or sampling.rows >= n, "sampling: a setting for every row")
    up = _vector(u, torch.float32, n, "u")
    dev = logits.device
    _on(dev.index, u, token, logprob, kept, ws, err)
    _want(sampling.gpu is None or sampling.gpu == dev.index, "logits and sampling: one GPU")
    if dev.index != _current_gpu():
        return _there(dev.index, fs_sample, logits, u, sampling, token, logprob, kept, ws, err, check)
    like = u if u.shape[0] == n else u[:n]

    def output(t, dtype, name):
        if t is None:
            t = torch.empty_like(like, dtype=dtype)
            return t, t.data_ptr()
        return t, _vector(t, dtype, n, name)

    token, tp = output(token, torch.int32, "token")
    logprob, lp = output(logprob, torch.float32, "logprob")
    kept, kp = output(kept, torch.int32, "kept")
    err = cleared_err_word(dev) if err is None else err
    code = _dtype_code(logits)
    L = _lib()
    ws, wp, wn = _workspace(ws, L.fs_sample_workspace(code, n, V), logits)
    _done(L.fs_sample(code, n, V, logits.data_ptr(), stride[0] if n > 1 else V,
                      sampling.ref, up, tp, lp, kp, wp, wn, err.data_ptr(), _raw_stream(dev.index)),
          "fs_sample", err, check)
    return token, logprob, kept
