"""Timed cases of the cache's operators: the append to a cache held in 4 bits, attention over
that cache, attention with a window whose first tokens stay visible, and the pages of a
cache (freed, forked, copied, compacted).

run() computes a case either in plain torch operations (`own` false) or through the
package's public entry points.  Request counts, step sizes and app counts follow the
repository's workloads (steps of 4,096 and 16,384 tokens, 8 to 32 apps, 8 to 256 users);
widths are generic.

A cache in 4 bits holds groups of 32 neighbouring values of a head: a byte b for the power
of two 2^(b - 127), the least one of which the group's largest value is at most 7 times, and
for each value a code of sign, two bits of exponent and one of fraction (0, 0.5, 1, 1.5, 2,
3, 4, 6), the nearest one (ties to the even code), low half of a byte first.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TOP_BYTE = {"bf16": 252, "f16": 140}         # the largest power of two whose codes stay in range


# ----------------------------------------------------------------- cases

def _cache(name, op, dtype, seqs, chunk, most_kv, heads, kv_heads, dim, page, **more):
    c = {"name": name, "op": op, "dtype": dtype, "seqs": seqs, "chunk": chunk, "most_kv": most_kv,
         "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page}
    c.update(more)
    return c


def _pages(name, op, dtype, seqs, most, page, kv_heads, dim, layers, **more):
    c = {"name": name, "op": op, "dtype": dtype, "seqs": seqs, "most": most, "page": page,
         "kv_heads": kv_heads, "dim": dim, "layers": layers}
    c.update(more)
    return c


def listed():
    return [
        # eight users' single tokens
        _cache("append4_decode", "append4", "bf16", 8, 1, 2000, 32, 8, 128, 16, rotary=128,
               interleaved=False),
        # a 16,384-token step of prompts, half of each head turned
        _cache("append4_step", "append4", "f16", 11, 2048, 16384, 32, 8, 128, 16, rotary=64,
               interleaved=True),
        # four short answers under way: latency
        _cache("attn4_decode_small", "attention4", "bf16", 4, 1, 500, 32, 8, 128, 16, window=0,
               sinks=0),
        # 128 running requests with contexts up to a 16,384-token step
        _cache("attn4_decode_batch", "attention4", "bf16", 128, 1, 16384, 32, 8, 128, 16, window=0,
               sinks=0),
        # one answer over one long document
        _cache("attn4_decode_long", "attention4", "f16", 1, 1, 200001, 32, 4, 128, 32, window=0,
               sinks=0),
        # the next 4,096 tokens of one long prompt
        _cache("attn4_chunk", "attention4", "bf16", 1, 4096, 32768, 32, 8, 128, 16, window=0,
               sinks=0),
        # 64 running requests that keep their newest 1,000 tokens and the first four
        _cache("sinks_decode", "sinks", "bf16", 64, 1, 16384, 32, 8, 128, 16, window=1000, sinks=4),
        # chunks of prompts and single tokens together, head_dim 64
        _cache("sinks_mixed", "sinks", "f16", 24, 1024, 8192, 16, 16, 64, 16, window=2000, sinks=20),
        # eight finished calls make room for eight of the same two apps
        _pages("fork_small", "fork", "bf16", 8, 600, 16, 8, 128, 1, apps=2, shared=300),
        # 256 calls of 8 apps begin with their apps' system prompts, a cache of four layers
        _pages("fork_batch", "fork", "bf16", 256, 2000, 32, 4, 64, 4, apps=8, shared=1200),
        # a pool of eight users, half of its pages free
        _pages("compact_small", "compact", "f16", 8, 1000, 16, 4, 64, 1, live=0.5),
        # a pool of 200 requests of up to 4,096 tokens, two thirds live
        _pages("compact_large", "compact", "bf16", 200, 4096, 16, 8, 128, 1, live=0.67),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed kinds; sizes over their whole ranges, odd ones among them."""
    op = rng.choice(("append4", "attention4", "attention4", "sinks", "fork", "compact"))
    dtype = rng.choice(("bf16", "f16"))
    page = rng.choice((8, 16, 32, 64))
    if op in ("fork", "compact"):
        most = _log_int(rng, 20, 4096)
        seqs = _log_int(rng, 1, max(1, min(256, 400000 // most)))
        kv_heads, dim = rng.choice((1, 2, 4, 8)), rng.choice((64, 128))
        layers = rng.randint(1, max(1, min(4, 600000000 // (seqs * (most + page) * kv_heads * dim * 4))))
        if op == "fork":
            return _pages("", op, dtype, seqs, most, page, kv_heads, dim, layers,
                          apps=rng.randint(1, 32), shared=rng.randint(0, most))
        return _pages("", op, dtype, seqs, most, page, kv_heads, dim, layers,
                      live=rng.uniform(0.05, 0.95))
    dim = rng.choice((64, 128, 128))
    kv_heads = rng.choice((1, 2, 4, 8, 16))
    heads = min(kv_heads * rng.choice((1, 2, 3, 4, 7, 8)), 64) // kv_heads * kv_heads
    if op == "append4":
        chunk = 1 if rng.random() < 0.4 else _log_int(rng, 2, 2048)
        seqs = _log_int(rng, 1, 256 if chunk == 1 else max(2, 16384 // chunk))
        return _cache("", op, dtype, seqs, chunk, max(chunk, _log_int(rng, 64, 16384)), heads,
                      kv_heads, dim, page, rotary=rng.choice((dim, dim // 2, 24)),
                      interleaved=rng.random() < 0.5)
    window, sinks = rng.choice(((0, 0), (0, 0), (700, 0), (1000, 4))) if op == "attention4" else \
        (_log_int(rng, 1, 4000), rng.choice((1, 4, 5, 16, 100)))
    if rng.random() < 0.5:                     # single tokens
        most = _log_int(rng, 16, 100000)
        seqs = _log_int(rng, 1, max(1, min(256, 800000 // most)))
        return _cache("", op, dtype, seqs, 1, most, heads, kv_heads, dim, page, window=window,
                      sinks=sinks)
    chunk = _log_int(rng, 2, 3000)
    most = max(chunk, _log_int(rng, chunk, 16384))
    seqs = max(1, min(32, int(4e7 / (chunk * most)), 200000 // most))
    return _cache("", op, dtype, _log_int(rng, 1, max(1, seqs)), chunk, most, heads, kv_heads, dim,
                  page, window=window, sinks=sinks)


# ----------------------------------------------------------------- inputs

def _shape_rng(case):
    """The shape of a case is the same for every seed."""
    import random
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lengths(case):
    """Rows and cached tokens of each request of an engine step."""
    rng = _shape_rng(case)
    chunk, most, seqs = case["chunk"], case["most_kv"], case["seqs"]
    if chunk == 1:
        q = [1] * seqs
    elif seqs == 1:
        q = [chunk]
    else:                                      # mostly chunks, some requests already decode
        q = [chunk] + [1 if rng.random() < 0.25 else rng.randint(1, chunk) for _ in range(seqs - 1)]
    kv = [most] + [_log_int(rng, 1, most) for _ in range(seqs - 1)]
    kv = [max(a, b) for a, b in zip(q, kv)]
    return q, kv


def _prompts(case):
    """Of a fork: the apps' prompts in tokens, and each call's app, shared tokens and room."""
    rng = _shape_rng(case)
    prompt = [rng.randint(0, case["shared"]) + 1 for _ in range(case["apps"])]
    prompt[0] = case["shared"] + 1
    app = [rng.randrange(case["apps"]) for _ in range(case["seqs"])]
    shared = [prompt[a] if rng.random() < 0.8 else rng.randint(0, prompt[a]) for a in app]
    room = [max(s, rng.randint(1, case["most"])) for s in shared]
    return prompt, app, shared, room


def _held(case):
    """Of a pool to be compacted: the pages of each request, and of the pool."""
    rng = _shape_rng(case)
    held = [-(-_log_int(rng, 1, case["most"]) // case["page"]) for _ in range(case["seqs"])]
    return held, max(int(sum(held) / case["live"]), sum(held) + 1)


def _quantise(x, top):
    """(codes two to a byte, scale bytes) of float32 x [..., dim]."""
    g = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(g.abs().amax(-1))
    byte = torch.where(m > 0.875, e - 2, e - 3).add_(127).clamp_(1, top)
    y = torch.ldexp(g.abs(), 127 - byte[..., None])
    code = torch.zeros_like(y, dtype=torch.uint8)
    # halfway between two levels the even code: the lower one of 0.25, 1.25, 2.5 and 5
    for i, (a, b) in enumerate(zip(LEVELS, LEVELS[1:])):
        code += (y > (a + b) / 2) if i % 2 == 0 else (y >= (a + b) / 2)
    code |= (g < 0).to(torch.uint8) << 3
    code = code.flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, byte.to(torch.uint8)


def _values(code, byte):
    """float32 values of codes [..., dim / 2] and scale bytes [..., dim / 32]."""
    levels = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=code.device)
    both = torch.stack((code & 15, code >> 4), -1).flatten(-2).int()
    power = torch.exp2(byte.float() - 127)
    return (levels[both].unflatten(-1, (-1, 32)) * power[..., None]).flatten(-2)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    dev = "cuda"
    st = {"case": case, "op": case["op"]}
    dt = TYPES[case["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device=dev).normal_(0, 1, generator=g)

    if own:
        import paper_2411_15997_amd as fs
        st["err"] = fs.cleared_err_word(dev)
    if case["op"] in ("fork", "compact"):
        return _prepare_pages(st, case, g, normal)

    q_len, kv_len = _lengths(case)
    st["q_len"], st["rows"] = q_len, sum(q_len)
    off = [0]
    for n in q_len:
        off.append(off[-1] + n)
    st["q_off"] = torch.tensor(off, dtype=torch.int32, device=dev)
    st["kv_len"] = torch.tensor(kv_len, dtype=torch.int32, device=dev)
    st["seq_of_row"] = torch.repeat_interleave(torch.arange(len(q_len), device=dev),
                                               torch.tensor(q_len, device=dev))

    # a paged cache: every request's pages somewhere among the others'
    page, hk, d, h = case["page"], case["kv_heads"], case["dim"], case["heads"]
    need = [-(-x // page) for x in kv_len]
    width, total = max(need), sum(need)
    perm = torch.randperm(total, device=dev, generator=g).to(torch.int32)
    col = torch.arange(width, device=dev)
    first = torch.tensor([sum(need[:i]) for i in range(len(need))], device=dev)
    have = col[None] < torch.tensor(need, device=dev)[:, None]
    st["table"] = torch.where(have, perm[(first[:, None] + col).clamp(max=total - 1)],
                              torch.zeros_like(perm[:1]))
    # some channels of the keys are larger than others, as rotary heads have them
    st["channel"] = torch.exp(0.5 * torch.randn(hk, d, device=dev, generator=g)).to(dt)
    k = normal(total, hk, page, d) * st["channel"][:, None]
    v = normal(total, hk, page, d)
    if case["op"] == "sinks":
        st["k"], st["v"] = k, v
    else:
        top = TOP_BYTE[case["dtype"]]
        st["k"], st["k_scale"] = _quantise(k.float(), top)
        st["v"], st["v_scale"] = _quantise(v.float(), top)
    if own:
        st["step"] = fs.Step(off, st["q_off"], st["kv_len"], max_kv=max(kv_len))
        st["cache"] = fs.KVCache(k, v, st["table"]) if case["op"] == "sinks" else \
            fs.KVCache4(st["k"], st["v"], st["k_scale"], st["v_scale"], st["table"])
    if case["op"] != "append4":
        st["q"] = normal(st["rows"], h, d)
        st["scale"] = d ** -0.5
        return st
    st["qkv"] = normal(st["rows"], h + 2 * hk, d)          # one joint projection's output
    st["qkv"][:, h:h + hk] *= st["channel"]
    rot = case["rotary"]
    st["inv_freq"] = torch.tensor([10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)],
                                  dtype=torch.float32, device=dev)
    if own:
        st["rope"] = fs.Rope(st["inv_freq"], case["interleaved"])
    return st


def _prepare_pages(st, case, g, normal):
    dev, page = "cuda", case["page"]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    if case["op"] == "fork":
        prompt, app, shared, room = _prompts(case)
        # the calls that finish held what those that begin will hold, in pages of their own
        held = [-(-x // page) for x in prompt] + [-(-x // page) for x in room]
        pages = sum(held) + 16
        st["parent"], st["shared"], st["room"] = i32(app), i32(shared), i32(room)
        st["child"] = torch.arange(len(prompt), len(held), dtype=torch.int32, device=dev)
    else:
        held, pages = _held(case)
    st["pages"] = pages
    perm = torch.randperm(pages, device=dev, generator=g).to(torch.int32)
    col = torch.arange(max(held), device=dev)
    have = col[None] < i32(held)[:, None]
    first = torch.tensor([sum(held[:i]) for i in range(len(held))], device=dev)
    table = perm[(first[:, None] + col).clamp(max=pages - 1)]
    if case["op"] == "fork":            # whole pages of the prompts are the apps' own
        full = (st["shared"] // page)[:, None]
        table[len(prompt):] = torch.where(col[None] < full, table[st["parent"].long()],
                                          table[len(prompt):])
    st["table"] = torch.where(have, table, torch.zeros_like(table))
    st["refs"] = torch.bincount(st["table"][have].long(), minlength=pages).to(torch.int32)
    st["held"] = i32(held)
    n = case["layers"]
    shape = (pages, case["kv_heads"], page, case["dim"])
    st["k"], st["v"] = [normal(*shape) for _ in range(n)], [normal(*shape) for _ in range(n)]
    if case["op"] == "compact":
        st["table_out"], st["refs_out"] = torch.zeros_like(st["table"]), torch.zeros_like(st["refs"])
    if own:
        import paper_2411_15997_amd as fs
        st["pool"] = fs.PagePool(st["refs"], st["table"], st["held"], page)
        st["caches"] = fs.CacheLayers([fs.KVCache(k, v, st["table"])
                                       for k, v in zip(st["k"], st["v"])])
    return st


# ----------------------------------------------------------------- one pass

def run(st):
    if own:
        return _own(st)
    return {"append4": _plain_append, "attention4": _plain_attention, "sinks": _plain_attention,
            "fork": _plain_fork, "compact": _plain_compact}[st["op"]](st)


def _own(st):
    import paper_2411_15997_amd as fs
    op, err, c = st["op"], st["err"], st["case"]
    if op == "append4":
        h, hk, qkv = c["heads"], c["kv_heads"], st["qkv"]
        q = fs.fs_rope_append4(st["step"], st["cache"], st["rope"], qkv[:, :h], qkv[:, h:h + hk],
                               qkv[:, h + hk:], err=err, check=False)
        k, v = fs.fs_cache4_rows(st["step"], st["cache"], qkv.dtype, err=err, check=False)
        return {"q": q, "k": k, "v": v}
    if op == "attention4":
        out, lse = fs.fs_paged_attention4(st["step"], st["cache"], st["q"], st["scale"],
                                          window=c["window"], sinks=c["sinks"], want_lse=True,
                                          err=err, check=False)
        return {"out": out, "lse": lse}
    if op == "sinks":
        out, lse = fs.fs_paged_attention(st["step"], st["cache"], st["q"], st["scale"],
                                         window=c["window"], sinks=c["sinks"], want_lse=True,
                                         err=err, check=False)
        return {"out": out, "lse": lse}
    if op == "fork":
        fs.fs_pages_free(st["pool"], st["child"], err=err, check=False)
        src, dst = fs.fs_pages_fork(st["pool"], st["parent"], st["child"], st["shared"], st["room"],
                                    err=err, check=False)
        fs.fs_pages_copy(st["caches"], src, dst, err=err, check=False)
        return {"refs": st["refs"], "table": st["table"], "held": st["held"], "src": src, "dst": dst,
                "k": st["k"], "v": st["v"]}
    src, dst, count = fs.fs_pages_compact(st["pool"], refs_out=st["refs_out"],
                                          table_out=st["table_out"], err=err, check=False)
    fs.fs_pages_copy(st["caches"], src, dst, count, err=err, check=False)
    return {"refs": st["refs_out"], "table": st["table_out"], "src": src, "dst": dst, "count": count,
            "k": st["k"], "v": st["v"]}


def _positions(st):
    """Position of every row: the last rows of a request are its newest tokens."""
    s = st["seq_of_row"]
    n = (st["q_off"][1:] - st["q_off"][:-1])[s]
    i = torch.arange(st["rows"], device=s.device) - st["q_off"][s]
    return (st["kv_len"][s] - n + i).long()


def _turn(x, cos, sin, rotary, interleaved):
    a, b = (x[..., 0:rotary:2], x[..., 1:rotary:2]) if interleaved else \
        (x[..., :rotary // 2], x[..., rotary // 2:rotary])
    p, q = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((p, q), -1).flatten(-2) if interleaved else torch.cat((p, q), -1)
    return torch.cat((turned, x[..., rotary:]), -1)


def _plain_append(st):
    c = st["case"]
    h, hk, page, dt = c["heads"], c["kv_heads"], c["page"], st["qkv"].dtype
    pos = _positions(st)
    # in 64 bits: the angle grows with the position, and a key's code must not hang on an
    # error of 32 bits where the key is next to the border of two codes
    theta = pos.double()[:, None] * st["inv_freq"].double()[None]
    cos, sin = theta.cos()[:, None], theta.sin()[:, None]
    q = _turn(st["qkv"][:, :h].float(), cos.float(), sin.float(), c["rotary"], c["interleaved"])
    k = _turn(st["qkv"][:, h:h + hk].double(), cos, sin, c["rotary"], c["interleaved"]).float()
    at, slot = st["table"][st["seq_of_row"], pos // page].long(), pos % page
    top = TOP_BYTE[c["dtype"]]
    st["k"][at, :, slot], st["k_scale"][at, :, slot] = _quantise(k, top)
    st["v"][at, :, slot], st["v_scale"][at, :, slot] = _quantise(st["qkv"][:, h + hk:].float(), top)
    return {"q": q.to(dt), "k": _values(st["k"][at, :, slot], st["k_scale"][at, :, slot]).to(dt),
            "v": _values(st["v"][at, :, slot], st["v_scale"][at, :, slot]).to(dt)}


def _plain_attention(st):
    c = st["case"]
    h, hk, d, page = c["heads"], c["kv_heads"], c["dim"], c["page"]
    grp, dev = h // hk, st["q"].device
    seqs, most_q, most_kv = c["seqs"], max(st["q_len"]), c["most_kv"]
    j = torch.arange(most_kv, device=dev)
    at = st["table"][:, j // page].long()
    live = (j[None] < st["kv_len"][:, None])[:, None, :, None]
    zero = torch.zeros((), device=dev)

    def rows_of(name):             # [seqs * kv_heads][most_kv][d]
        x = st[name][at, :, j % page]
        x = _values(x, st[name + "_scale"][at, :, j % page]) if st["op"] == "attention4" else x
        x = x.permute(0, 2, 1, 3).float()
        return torch.where(live, x, zero).reshape(seqs * hk, most_kv, d)

    k, v = rows_of("k"), rows_of("v")
    n = st["q_off"][1:] - st["q_off"][:-1]
    s = st["seq_of_row"]
    i = (torch.arange(st["rows"], device=dev) - st["q_off"][s]).long()
    q = torch.zeros(seqs, most_q, h, d, device=dev)
    q[s, i] = st["q"].float()
    q = q.view(seqs, most_q, hk, grp, d).permute(0, 2, 1, 3, 4).reshape(seqs * hk, most_q * grp, d)
    score = torch.bmm(q, k.transpose(1, 2).contiguous()).view(seqs, hk, most_q, grp, most_kv)
    score *= st["scale"]
    pos = (st["kv_len"] - n)[:, None] + torch.arange(most_q, device=dev)[None]
    see = j[None, None] <= pos[:, :, None]
    if c["window"]:
        see &= (j[None, None] > pos[:, :, None] - c["window"]) | (j < c["sinks"])
    score.masked_fill_(~see[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), zero, top)
    score -= top
    score.exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.bmm(score.view(seqs * hk, most_q * grp, most_kv), v)
    out = out.view(seqs, hk, most_q, grp, d) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + total.log())[..., 0]
    out = out.permute(0, 2, 1, 3, 4).reshape(seqs, most_q, h, d)[s, i]
    lse = lse.permute(0, 2, 1, 3).reshape(seqs, most_q, h)[s, i]
    return {"out": out.to(st["q"].dtype), "lse": lse}


def _plain_copy(st, src, dst):
    go = src >= 0
    src, dst = src[go].long(), dst[go].long()
    for x in st["k"] + st["v"]:
        x[dst] = x[src]


def _places(flag, ids, n):
    """[n]: the ids whose flag is set, in order, then -1."""
    out = torch.full((n + 1,), -1, dtype=torch.int32, device=ids.device)
    out.scatter_(0, torch.where(flag, torch.cumsum(flag, 0) - 1, n).clamp(max=n), ids)
    return out[:n]


def _plain_fork(st):
    page, table, refs, held = st["case"]["page"], st["table"], st["refs"], st["held"]
    parent, child = st["parent"].long(), st["child"].long()
    col = torch.arange(table.shape[1], device=table.device)[None]
    one = torch.ones((), dtype=torch.int32, device=table.device)
    # the finished calls' pages
    gone = (col < held[child][:, None]).int().flatten()
    refs.index_add_(0, table[child].flatten(), -gone)
    # whole pages of the prompt are shared, a begun one is copied, the rest is new
    full, part = st["shared"] // page, st["shared"] % page > 0
    pages = (st["room"] + page - 1) // page
    new = pages - full
    first = torch.cumsum(new, 0) - new
    ids = torch.arange(st["pages"], dtype=torch.int32, device=table.device)
    free = _places(refs == 0, ids, st["pages"])
    got = free[(first[:, None] + col - full[:, None]).clamp(0, st["pages"] - 1)]
    rows = torch.where(col < full[:, None], table[parent], got)
    rows = torch.where(col < pages[:, None], rows, table[child])
    src = torch.where(part, table[parent].gather(1, full[:, None].long())[:, 0], -one)
    dst = torch.where(part, free[first.clamp(max=st["pages"] - 1)], -one)
    table[child] = rows
    held[child] = pages
    refs.index_add_(0, rows.flatten().clamp(min=0), (col < pages[:, None]).int().flatten())
    _plain_copy(st, src, dst)
    return {"refs": refs, "table": table, "held": held, "src": src, "dst": dst, "k": st["k"],
            "v": st["v"]}


def _plain_compact(st):
    refs, table, n = st["refs"], st["table"], st["pages"]
    ids = torch.arange(n, dtype=torch.int32, device=refs.device)
    live = refs > 0
    most = live.sum()
    src = _places(live & (ids >= most), ids, n // 2)
    dst = _places(~live & (ids < most), ids, n // 2)
    dst = torch.where(src >= 0, dst, src)
    count = (src >= 0).sum().int()[None]
    place = ids.clone()
    go = src >= 0
    place[src[go].long()] = dst[go]
    st["refs_out"].zero_()
    st["refs_out"][place[live].long()] = refs[live]
    col = torch.arange(table.shape[1], device=table.device)[None]
    st["table_out"].copy_(torch.where(col < st["held"][:, None], place[table.long()], st["table_out"]))
    _plain_copy(st, src, dst)
    return {"refs": st["refs_out"], "table": st["table_out"], "src": src, "dst": dst, "count": count,
            "k": st["k"], "v": st["v"]}


# ----------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"] in ("fork", "compact"):
        page_bytes = 2 * 2 * case["kv_heads"] * case["page"] * case["dim"] * case["layers"]
        if case["op"] == "fork":
            prompt, _, shared, room = _prompts(case)
            held = sum(-(-x // case["page"]) for x in room)
            pages = held + sum(-(-x // case["page"]) for x in prompt) + 16
            copies = sum(s % case["page"] > 0 for s in shared)
            return {"bytes": 2 * copies * page_bytes + 4 * (pages + 4 * held + 8 * case["seqs"]),
                    "flops": 0}
        held, pages = _held(case)
        moves = sum(held) * (pages - sum(held)) // pages       # of pages anywhere in the pool
        return {"bytes": 2 * moves * page_bytes + 4 * (2 * pages + 2 * sum(held) + 4 * moves),
                "flops": 0}
    q, kv = _lengths(case)
    t = sum(q)
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "append4":        # the appended rows are read back in 16 bits
        row4 = 2 * hk * (d // 2 + d // 32)
        return {"bytes": 2 * t * (2 * h + 2 * hk) * d + t * row4 + t * row4 + 2 * t * 2 * hk * d,
                "flops": 3 * t * (h + hk) * case["rotary"]}
    win, sinks = case["window"], case["sinks"]
    read, pairs = 0, 0
    for a, b in zip(q, kv):
        for i in range(a):
            p = b - a + i
            lo = max(0, p - win + 1) if win else 0
            pairs += p + 1 - lo + min(sinks, lo)
        lo = max(0, b - a - win + 1) if win else 0
        read += b - lo + min(sinks, lo)
    row = d * 2 if case["op"] == "sinks" else d // 2 + d // 32
    return {"bytes": 2 * read * hk * row + 2 * 2 * t * h * d + 4 * t * h, "flops": 4 * d * h * pairs}


# ----------------------------------------------------------------- in 64 bits

def exact(case, seed):
    if case["op"] in ("fork", "compact"):
        return None                    # whole numbers and copies
    st = prepare(case, seed)
    q_len, kv_len = _lengths(case)
    off = [0]
    for n in q_len:
        off.append(off[-1] + n)
    if case["op"] == "append4":
        return _exact_append(st, case, q_len, kv_len, off)
    return _exact_attention(st, case, q_len, kv_len, off)


def _nearest(x, top):
    """The values that float64 x [..., dim] has in 4 bits."""
    g = x.unflatten(-1, (-1, 32))
    most = g.abs().amax(-1, keepdim=True)
    power = torch.floor(torch.log2(most.clamp(min=1e-300))) - 3
    power = torch.where(most > 7 * torch.exp2(power), power + 1, power)
    power = torch.where(most > 7 * torch.exp2(power), power + 1, power)
    unit = torch.exp2(power.clamp(-126, top - 127))
    # even codes first, so that they win where two are equally near
    order = torch.tensor([LEVELS[i] for i in (0, 2, 4, 6, 1, 3, 5, 7)], dtype=torch.float64,
                         device=x.device)
    off = ((g.abs() / unit)[..., None] - order).abs()
    best, level = off[..., 0], torch.zeros_like(g)
    for i in range(1, 8):
        nearer = off[..., i] < best
        best, level = torch.where(nearer, off[..., i], best), torch.where(nearer, order[i], level)
    return (torch.sign(g) * level * unit).flatten(-2)


def _exact_append(st, case, q_len, kv_len, off):
    h, hk, rot = case["heads"], case["kv_heads"], case["rotary"]
    half = rot // 2
    first = torch.arange(half, device="cuda") * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else half)
    f = st["inv_freq"].double()
    top = TOP_BYTE[case["dtype"]]
    q_out = torch.empty(off[-1], h, case["dim"], dtype=torch.float64, device="cuda")
    k_out = torch.empty(off[-1], hk, case["dim"], dtype=torch.float64, device="cuda")
    v_out = torch.empty_like(k_out)
    for s, (n, kv) in enumerate(zip(q_len, kv_len)):
        rows = slice(off[s], off[s + 1])
        x = st["qkv"][rows].double()
        p = torch.arange(kv - n, kv, device="cuda")
        z = torch.polar(torch.ones(n, half, dtype=torch.float64, device="cuda"), p.double()[:, None] * f)
        turned = torch.complex(x[:, :h + hk, first], x[:, :h + hk, second]) * z[:, None]
        y = x.clone()
        y[:, :h + hk, first] = turned.real
        y[:, :h + hk, second] = turned.imag
        q_out[rows] = y[:, :h]
        k_out[rows] = _nearest(y[:, h:h + hk].float().double(), top)
        v_out[rows] = _nearest(y[:, h + hk:], top)
    return {"q": q_out, "k": k_out, "v": v_out}


def _exact_attention(st, case, q_len, kv_len, off):
    h, hk, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    win, sinks, grp = case["window"], case["sinks"], h // hk
    out = torch.empty(off[-1], h, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(off[-1], h, dtype=torch.float64, device="cuda")
    value = [(-1) ** (i >> 3) * (0.5 * (i & 1) if i & 6 == 0 else (1 + 0.5 * (i & 1)) * 2.0 ** ((i >> 1 & 3) - 1))
             for i in range(16)]
    value = torch.tensor(value, dtype=torch.float64, device="cuda")

    def rows_of(name, at, m, slot, kv):
        x = st[name][at, m, slot]
        if case["op"] == "sinks":
            return x.double()
        y = torch.empty(kv, d, dtype=torch.float64, device="cuda")
        y[:, 0::2], y[:, 1::2] = value[(x % 16).long()], value[(x // 16).long()]
        unit = torch.pow(2.0, st[name + "_scale"][at, m, slot].double() - 127)
        return y * torch.repeat_interleave(unit, 32, dim=1)

    for s, (n, kv) in enumerate(zip(q_len, kv_len)):
        j = torch.arange(kv, device="cuda")
        at = st["table"][s].long()[j // page]
        p = torch.arange(kv - n, kv, device="cuda")
        see = (j[None] <= p[:, None]) & ((j[None] > p[:, None] - win) | (j < sinks) if win else True)
        for m in range(hk):
            k, v = rows_of("k", at, m, j % page, kv), rows_of("v", at, m, j % page, kv)
            for i in range(m * grp, (m + 1) * grp):
                q = st["q"][off[s]:off[s + 1], i].double()
                score = (q @ k.t().contiguous()) * float(st["scale"])
                score = score.masked_fill(~see, -math.inf)
                out[off[s]:off[s + 1], i] = torch.softmax(score, -1) @ v
                lse[off[s]:off[s + 1], i] = torch.logsumexp(score, -1)
    return {"out": out, "lse": lse}
