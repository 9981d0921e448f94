"""cache_ref.attention for calls of many heads: the same result and bounds, a request's rows and
heads at once."""
import math

import numpy as np
import torch

import engine_ref as ref


def attention(q, k, v, table, q_off, kv_len, scale, window, sinks):
    u, tiny = ref.U16[q.dtype], ref.TINY[q.dtype]
    T, H, D = q.shape
    HK, page = k.shape[1], k.shape[2]
    grp = H // HK
    out, tol = (torch.zeros(T, H, D, dtype=torch.float64) for _ in range(2))
    lse = torch.full((T, H), -math.inf, dtype=torch.float64)
    ltol = torch.zeros(T, H, dtype=torch.float64)
    tab = table.cpu().numpy()
    for s, (a, b, kv) in enumerate(zip(q_off, q_off[1:], kv_len)):
        n = b - a
        if n == 0 or kv == 0:
            continue
        j = np.arange(kv)
        K, V = (x[tab[s][j // page], :, j % page].double().cpu().transpose(0, 1) for x in (k, v))
        j, p = torch.arange(kv)[None], (kv - n + torch.arange(n))[:, None]
        see = (j <= p) & ((j > p - window) | (j < sinks) if window else torch.ones_like(j, dtype=torch.bool))
        count = see.sum(-1)
        # rows of one key/value head: [heads][tokens * group]
        Q = q[a:b].double().cpu().view(n, HK, grp, D).permute(1, 0, 2, 3).reshape(HK, n * grp, D)
        hide = ~see.repeat_interleave(grp, 0)
        sc = (scale * (Q @ K.transpose(1, 2).contiguous())).masked_fill(hide, -math.inf)
        prob = torch.softmax(sc, -1).masked_fill(hide, 0.0)
        size = (Q.abs() @ K.abs().transpose(1, 2).contiguous()).masked_fill(hide, 0.0).amax(-1)
        ds = (D + 4) * ref.E32 * abs(scale) * size
        rel = 2 * ds + (count.repeat_interleave(grp) + 8) * ref.E32 + 2.0 ** -20
        o, top = prob @ V, torch.logsumexp(sc, -1)
        some = (count > 0).repeat_interleave(grp)
        bound = (u * o.abs() + tiny + (u + rel)[..., None] * (prob @ V.abs())) * some[:, None]
        lbound = torch.where(some, rel + 2 * ref.E32 * top.abs(), torch.zeros_like(rel))

        def back(x):
            return x.view(HK, n, grp, *x.shape[2:]).transpose(0, 1).reshape(n, H, *x.shape[2:])
        out[a:b], tol[a:b], lse[a:b], ltol[a:b] = back(o), back(bound), back(top), back(lbound)
    return out, tol, lse, ltol
