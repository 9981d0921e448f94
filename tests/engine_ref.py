"""The engine step's operators in 64 bits, row by row (the oracle of test_gpu_engine.py),
with the error bounds that the 16-bit results are held to."""
import math

import numpy as np
import torch

U16 = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # unit roundoffs
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -24}          # f16 goes subnormal below 2^-14
E32 = 2.0 ** -24
ONE = 1 << 40


def linear(x, w, a, b, q_off, adapter, rank=None, scale=None):
    """(y, bound) in float64: y = x w^T + scale (x a^T) b^T with the row's adapter.  The
    bound: one rounding to 16 bits, fp32 sums of K + 2 R terms, and the two-part h (its
    second part is rounded to u of a remainder of at most u of h)."""
    u, tiny = U16[x.dtype], TINY[x.dtype]
    X, W = x.double().cpu(), w.double().cpu()
    y, mag = X @ W.t(), X.abs() @ W.abs().t()
    extra = torch.zeros_like(y)
    for s in range(len(q_off) - 1):
        ad = int(adapter[s])
        if ad < 0:
            continue
        r = int(rank[ad]) if rank is not None else a.shape[1]
        c = float(scale[ad]) if scale is not None else 1.0
        A, B = a[ad, :r].double().cpu(), b[ad, :, :r].double().cpu()
        rows = slice(q_off[s], q_off[s + 1])
        y[rows] += c * ((X[rows] @ A.t()) @ B.t())
        mag[rows] += abs(c) * ((X[rows].abs() @ A.abs().t()) @ B.abs().t())
        extra[rows] += tiny * B.abs().sum(1)[None]
    terms = x.shape[1] + 2 * a.shape[1] + 8
    return y, u * y.abs() + (terms * E32 + 4 * u * u) * mag + extra + tiny


def positions(q_off, kv_len):
    return [[kv - (q1 - q0) + i for i in range(q1 - q0)]
            for q0, q1, kv in zip(q_off, q_off[1:], kv_len)]


def rope_rows(x, pos, inv_freq, rotary, interleaved, factor):
    """(turned rows, bound) of x [n][heads][dim] at positions pos [n], float64."""
    u, tiny = U16[x.dtype], TINY[x.dtype]
    X = x.double().cpu().numpy()
    th = np.asarray(pos, np.float64)[:, None] * inv_freq.double().cpu().numpy()[None]
    c, s = np.cos(th)[:, None] * factor, np.sin(th)[:, None] * factor
    half = rotary // 2
    i0 = np.arange(half) * (2 if interleaved else 1)
    i1 = i0 + (1 if interleaved else half)
    y = X.copy()
    y[..., i0] = X[..., i0] * c - X[..., i1] * s
    y[..., i1] = X[..., i1] * c + X[..., i0] * s
    mag = np.zeros_like(X)
    mag[..., i0] = mag[..., i1] = (np.abs(X[..., i0]) + np.abs(X[..., i1])) * abs(factor)
    # the reduced angle, sin, cos, the factor and the sum: eight fp32 roundings of at most
    # pi times 2^-24 each
    return y, u * np.abs(y) + 32 * E32 * mag + tiny


def kv_rows(cache, table_row, n, page, head):
    """The first n cached rows of one request and head, in float64."""
    j = np.arange(n)
    ids = np.asarray(table_row)[j // page]
    return cache[ids, head, j % page].double().cpu()


def attention(q, k_cache, v_cache, table, q_off, kv_len, scale, window):
    """(out, bound, lse, lse bound) in float64.  The bound: one rounding of the result and
    one of each probability, scores with fp32 sums of dim terms (their error moves a
    probability by as much), fp32 sums over the keys, and 2^-20 for the exponentials."""
    u, tiny = U16[q.dtype], TINY[q.dtype]
    T, H, D = q.shape
    HK, page = k_cache.shape[1], k_cache.shape[2]
    grp = H // HK
    out = torch.zeros(T, H, D, dtype=torch.float64)
    tol = torch.zeros_like(out)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64)
    ltol = torch.zeros(T, H, dtype=torch.float64)
    Q = q.double().cpu()
    tab = table.cpu().numpy()
    for s, pos in enumerate(positions(q_off, kv_len)):
        if not pos or kv_len[s] == 0:
            continue
        for m in range(HK):
            K = kv_rows(k_cache, tab[s], kv_len[s], page, m)
            V = kv_rows(v_cache, tab[s], kv_len[s], page, m)
            for i, p in enumerate(pos):
                lo = max(0, p - window + 1) if window else 0
                if p < 0 or lo > p:
                    continue
                t = q_off[s] + i
                qq = Q[t, m * grp:(m + 1) * grp]
                sc = scale * qq @ K[lo:p + 1].t()
                prob = torch.softmax(sc, -1)
                o = prob @ V[lo:p + 1]
                ds = (D + 4) * E32 * abs(scale) * (qq.abs() @ K[lo:p + 1].abs().t()).amax(-1)
                rel = 2 * ds + (p + 1 - lo + 8) * E32 + 2.0 ** -20
                out[t, m * grp:(m + 1) * grp] = o
                tol[t, m * grp:(m + 1) * grp] = u * o.abs() + tiny + \
                    (u + rel)[:, None] * (prob @ V[lo:p + 1].abs())
                lse[t, m * grp:(m + 1) * grp] = torch.logsumexp(sc, -1)
                ltol[t, m * grp:(m + 1) * grp] = rel + 2 * E32 * lse[t, m * grp:(m + 1) * grp].abs()
    return out, tol, lse, ltol


def sample_row(x, u, t, k, p, m):
    """(token, logprob, kept) of one row, in Python integers.  x: float32 numpy."""
    x = np.where(np.isnan(x), -np.inf, x).astype(np.float64)
    order = np.argsort(-x, kind="stable")          # larger first, equal ones by id
    if x[order[0]] == -np.inf:
        return -1, -math.inf, 0
    if t == 0:
        return int(order[0]), 0.0, 1
    best = x[order[0]]
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        y = (best - x[order]) * (1.4426950408889634 / np.float64(np.float32(t)))
        y = np.where(x[order] == best, 0.0, y)
        w = [int(v) for v in np.floor(np.exp2(-y) * ONE)]
    n = len(w)
    if 0 < k < n:
        w[k:] = [0] * (n - k)
    if p < 1:
        total = sum(w)
        limit = max(1, math.ceil(float(np.float32(p)) * float(total)))
        run = 0
        for i in range(n):
            if run >= limit:
                w[i:] = [0] * (n - i)
                break
            run += w[i]
    least = math.ceil(float(np.float32(m)) * ONE)
    w = [v if v >= least else 0 for v in w]
    by_id = [0] * n
    for i, v in zip(order, w):
        by_id[i] = v
    total = sum(by_id)
    goal = min(math.floor(float(np.float32(u)) * float(total)), total - 1)
    run = 0
    for i, v in enumerate(by_id):
        run += v
        if run > goal:
            return i, math.log(v / total), sum(1 for z in by_id if z)
    raise AssertionError
