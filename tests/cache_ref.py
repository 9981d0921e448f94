"""The cache's operators in 64 bits and in Python integers (the oracle of the cache tests):
the 4-bit format, attention with a window and sinks, a pool of pages."""
import math

import numpy as np
import torch

import engine_ref as ref

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TOP = {torch.bfloat16: 252, torch.float16: 140}


def quantise(x, top):
    """(codes 0..15 [..., dim], bytes [..., dim / 32]) of x [..., dim], values of fp32."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    fine = np.isfinite(g).all(-1)
    g = np.where(fine[..., None], g, 0.0)
    most = np.abs(g).max(-1)
    E = np.floor(np.log2(np.maximum(most, 1e-300))) - 4
    for _ in range(3):                      # the least E with most <= 7 * 2^E
        E = np.where(most > 7 * 2.0 ** E, E + 1, E)
    E = np.clip(E, 1 - 127, top - 127)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])     # of two equally near ones the even code
    off = np.abs(np.abs(g)[..., None] / 2.0 ** E[..., None, None] - LEVELS[order])
    code = order[off.argmin(-1)] | np.signbit(g) << 3
    byte = np.where(fine, E + 127, 255).astype(np.uint8)
    return code.astype(np.uint8).reshape(x.shape), byte


def pack(code):
    return torch.from_numpy(code[..., 0::2] | code[..., 1::2] << 4)


def values(codes, scales, top):
    """float64 of packed codes [..., dim / 2] and scale bytes [..., dim / 32] (uint8 tensors)."""
    c = codes.cpu().numpy()
    both = np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], -1)
    b = scales.cpu().numpy().astype(np.int64)
    unit = np.where(b > top, np.nan, 2.0 ** (np.maximum(b, 1) - 127.0))
    x = LEVELS[both & 7] * np.where(both & 8, -1.0, 1.0)
    return torch.from_numpy((x.reshape(*b.shape, 32) * unit[..., None]).reshape(both.shape))


def seen(p, kv, window, sinks):
    """The cached tokens that a row at position p sees."""
    lo = max(0, p - window + 1) if window else 0
    return [j for j in range(min(sinks, lo))] + list(range(lo, min(p + 1, kv)))


def attention(q, k, v, table, q_off, kv_len, scale, window, sinks):
    """engine_ref.attention with sinks; k and v [pages][kv_heads][page][dim] in any type."""
    u, tiny = ref.U16[q.dtype], ref.TINY[q.dtype]
    T, H, D = q.shape
    HK, page = k.shape[1], k.shape[2]
    grp = H // HK
    out = torch.zeros(T, H, D, dtype=torch.float64)
    tol = torch.zeros_like(out)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64)
    ltol = torch.zeros(T, H, dtype=torch.float64)
    Q, tab = q.double().cpu(), table.cpu().numpy()
    for s, pos in enumerate(ref.positions(q_off, kv_len)):
        if not pos or kv_len[s] == 0:
            continue
        for m in range(HK):
            K = ref.kv_rows(k, tab[s], kv_len[s], page, m)
            V = ref.kv_rows(v, tab[s], kv_len[s], page, m)
            for i, p in enumerate(pos):
                at = seen(p, kv_len[s], window, sinks) if p >= 0 else []
                if not at:
                    continue
                t = q_off[s] + i
                qq, kk, vv = Q[t, m * grp:(m + 1) * grp], K[at], V[at]
                sc = scale * qq @ kk.t()
                prob = torch.softmax(sc, -1)
                o = prob @ vv
                ds = (D + 4) * ref.E32 * abs(scale) * (qq.abs() @ kk.abs().t()).amax(-1)
                rel = 2 * ds + (len(at) + 8) * ref.E32 + 2.0 ** -20
                out[t, m * grp:(m + 1) * grp] = o
                tol[t, m * grp:(m + 1) * grp] = u * o.abs() + tiny + \
                    (u + rel)[:, None] * (prob @ vv.abs())
                lse[t, m * grp:(m + 1) * grp] = torch.logsumexp(sc, -1)
                ltol[t, m * grp:(m + 1) * grp] = rel + 2 * ref.E32 * lse[t, m * grp:(m + 1) * grp].abs()
    return out, tol, lse, ltol


class Pool:
    """A pool of pages in Python lists."""

    def __init__(self, n_pages, page, rows, width):
        self.page, self.width = page, width
        self.refs = [0] * n_pages
        self.table = [[0] * width for _ in range(rows)]
        self.held = [0] * rows

    def free(self, rows):
        for r in rows:
            for p in self.table[r][:self.held[r]]:
                self.refs[p] -= 1
            self.held[r] = 0

    def fork(self, parent, child, shared, room):
        """(src, dst); asks for sound arguments."""
        free = [p for p, n in enumerate(self.refs) if n == 0]
        src, dst, rows = [], [], []
        for p, c, s, r in zip(parent, child, shared, room):
            full, pages = s // self.page, -(-r // self.page)
            new, free = free[:pages - full], free[pages - full:]
            rows.append((c, (self.table[p][:full] if full else []) + new))
            part = s % self.page > 0
            src.append(self.table[p][full] if part else -1)
            dst.append(new[0] if part else -1)
        for c, ids in rows:
            self.table[c][:len(ids)] = ids
            self.held[c] = len(ids)
            for p in ids:
                self.refs[p] += 1
        return src, dst

    def compact(self):
        live = [p for p, n in enumerate(self.refs) if n]
        L = len(live)
        src = [p for p in live if p >= L]
        dst = [p for p in range(L) if not self.refs[p]]
        place = dict(zip(src, dst))
        for a, b in place.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        for row, n in zip(self.table, self.held):
            row[:n] = [place.get(p, p) for p in row[:n]]
        return src, dst
