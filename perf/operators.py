"""Timed cases of the engine step's operators: a projection with every request's low-rank
adapter beside it, rotary positions with the append to the paged KV cache, attention of
the step's tokens over that cache, and the choice of the next token.

run() computes a case either in plain torch operations (`own` false) or through the
package's public entry points.  Request counts, step sizes and adapter counts follow the
repository's workloads (steps of 4,096 and 16,384 tokens, 8 to 32 apps, 8 to 256 users);
widths and vocabularies are generic.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
LOG2E = 1.4426950408889634
ONE = 1 << 40                  # weight of the largest logit


# ----------------------------------------------------------------- cases

def _linear(name, dtype, seqs, tokens, k, n, adapters, rank, none=0.0):
    return {"name": name, "op": "linear", "dtype": dtype, "seqs": seqs, "tokens": tokens, "k": k,
            "n": n, "adapters": adapters, "rank": rank, "none": none}


def _cache(name, op, dtype, seqs, chunk, most_kv, heads, kv_heads, dim, page, **more):
    c = {"name": name, "op": op, "dtype": dtype, "seqs": seqs, "chunk": chunk, "most_kv": most_kv,
         "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page}
    c.update(more)
    return c


def _sample(name, dtype, rows, vocab, mode):
    return {"name": name, "op": "sample", "dtype": dtype, "rows": rows, "vocab": vocab,
            "mode": mode}


def listed():
    return [
        # one decoded token for each of 64 running requests of 8 apps, joint q, k, v projection
        _linear("linear_decode", "bf16", 64, 64, 4096, 6144, 8, 16),
        # a 4,096-token step's share of chunks, odd lengths, some requests without an adapter
        _linear("linear_ragged", "f16", 13, 1999, 2048, 2560, 32, 32, none=0.25),
        # a whole 16,384-token step of prompts
        _linear("linear_step", "bf16", 24, 16384, 4096, 4096, 16, 16),
        # eight users' single tokens
        _cache("rope_decode", "rope", "bf16", 8, 1, 2000, 32, 8, 128, 16, rotary=128,
               interleaved=False, scaling="plain"),
        # a 16,384-token step, half of each head turned, long-context scaling
        _cache("rope_step", "rope", "f16", 11, 2048, 16384, 32, 8, 128, 16, rotary=64,
               interleaved=True, scaling="parts"),
        # four short answers under way: latency
        _cache("attn_decode_small", "attention", "bf16", 4, 1, 500, 32, 8, 128, 16, window=0),
        # 64 running requests with contexts up to a 16,384-token step
        _cache("attn_decode_batch", "attention", "bf16", 64, 1, 16384, 32, 8, 128, 16, window=0),
        # one answer over one long document
        _cache("attn_decode_long", "attention", "f16", 1, 1, 200001, 32, 4, 128, 32, window=0),
        # chunks of prompts and single tokens together, a sliding window
        _cache("attn_mixed", "attention", "bf16", 24, 1024, 8192, 16, 16, 64, 16, window=3000),
        # the next 4,096 tokens of one long prompt
        _cache("attn_chunk_long", "attention", "bf16", 1, 4096, 32768, 32, 8, 128, 16, window=0),
        # one user's token, small vocabulary, top-k and top-p
        _sample("sample_one", "f32", 1, 32000, "all"),
        # a full batch over a large vocabulary, each row with settings of its own
        _sample("sample_batch", "bf16", 256, 131072, "mixed"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed kinds; sizes over their whole ranges, odd ones among them."""
    op = rng.choice(("linear", "rope", "attention", "attention", "sample"))
    dtype = rng.choice(("bf16", "f16"))
    if op == "linear":
        seqs = _log_int(rng, 1, 256)
        tokens = seqs if rng.random() < 0.5 else _log_int(rng, seqs, 12000)
        return _linear("", dtype, seqs, max(tokens, seqs), 8 * _log_int(rng, 64, 640),
                       8 * _log_int(rng, 32, 800), rng.randint(1, 32), rng.choice((8, 16, 24, 32, 64)),
                       none=rng.choice((0.0, 0.3)))
    if op == "sample":
        return _sample("", rng.choice(("bf16", "f16", "f32")), _log_int(rng, 1, 256),
                       _log_int(rng, 1000, 131072), rng.choice(("all", "mixed", "p", "k", "free")))
    dim = rng.choice((64, 128, 128))
    kv_heads = rng.choice((1, 2, 4, 8, 16))
    heads = kv_heads * rng.choice((1, 2, 3, 4, 7, 8))
    page = rng.choice((8, 16, 32, 64))
    if op == "rope":
        chunk = 1 if rng.random() < 0.4 else _log_int(rng, 2, 2048)
        seqs = _log_int(rng, 1, 256 if chunk == 1 else max(2, 16384 // chunk))
        return _cache("", op, dtype, seqs, chunk, max(chunk, _log_int(rng, 64, 16384)),
                      min(heads, 64), kv_heads, dim, page, rotary=rng.choice((dim, dim // 2, 24)),
                      interleaved=rng.random() < 0.5,
                      scaling=rng.choice(("plain", "linear", "base", "parts")))
    heads = min(heads, 64) // kv_heads * kv_heads
    window = rng.choice((0, 0, 0, 1000))
    if rng.random() < 0.5:                     # single tokens
        most = _log_int(rng, 16, 100000)
        seqs = _log_int(rng, 1, max(1, min(256, 800000 // most)))
        return _cache("", op, dtype, seqs, 1, most, heads, kv_heads, dim, page, window=window)
    chunk = _log_int(rng, 2, 3000)
    most = max(chunk, _log_int(rng, chunk, 16384))
    seqs = max(1, min(32, int(4e7 / (chunk * most)), 200000 // most))
    return _cache("", op, dtype, _log_int(rng, 1, max(1, seqs)), chunk, most, heads, kv_heads, dim,
                  page, window=window)


# ----------------------------------------------------------------- inputs

def _even_parts(rng, total, parts):
    """`parts` lengths of at least one that sum to `total`, uneven."""
    cut = sorted(rng.sample(range(1, total), parts - 1)) if parts > 1 else []
    edge = [0] + cut + [total]
    return [b - a for a, b in zip(edge, edge[1:])]


def _lengths(case):
    """Rows and cached tokens of each request: the shape of a case, the same for every seed."""
    import random
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    if case["op"] == "linear":
        q = _even_parts(rng, case["tokens"], case["seqs"])
        return q, q
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


def _frequencies(rotary, scaling):
    """Rotary frequencies (base 10,000; scaled 8 times beyond 4,096 tokens) and the factor."""
    half = rotary // 2
    f = [10000.0 ** (-2.0 * i / rotary) for i in range(half)]
    s = 8.0
    if scaling == "linear":
        return [x / s for x in f], 1.0
    if scaling == "base":
        base = 10000.0 * s ** (rotary / (rotary - 2.0))
        return [base ** (-2.0 * i / rotary) for i in range(half)], 1.0
    if scaling == "parts":
        out = []
        for x in f:
            turns = 4096 * x / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / (32.0 - 1.0)))
            out.append(x / s * (1 - keep) + x * keep)
        return out, 0.1 * math.log(s) + 1.0
    return f, 1.0


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    dev = "cuda"
    st = {"case": case, "op": case["op"]}
    dt = TYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return torch.empty(shape, dtype=dtype, device=dev).normal_(0, std, generator=g)

    def uniform(n, lo, hi):
        return torch.rand(n, device=dev, generator=g) * (hi - lo) + lo

    if case["op"] == "sample":
        rows, vocab, mode = case["rows"], case["vocab"], case["mode"]
        st["logits"] = normal(rows, vocab, std=2.5)
        st["u"] = torch.rand(rows, device=dev, generator=g)
        t, p, m = uniform(rows, 0.5, 1.3), uniform(rows, 0.5, 0.99), uniform(rows, 0.0, 0.2)
        k = torch.randint(1, 200, (rows,), device=dev, generator=g, dtype=torch.int32)
        if mode == "mixed":        # every fourth row: greedy, top-p alone, top-k with top-p, min-p
            kind = torch.arange(rows, device=dev) % 4
            t = torch.where(kind == 0, torch.zeros_like(t), t)
            p = torch.where((kind == 0) | (kind == 3), torch.ones_like(p), p)
            k = torch.where(kind == 2, k, torch.zeros_like(k))
            m = torch.where(kind == 3, m, torch.zeros_like(m))
        st["temperature"] = t
        st["top_k"] = k if mode in ("all", "mixed", "k") else None
        st["top_p"] = p if mode in ("all", "mixed", "p") else None
        st["min_p"] = m if mode in ("all", "mixed") else None
        if own:
            import paper_2411_15997_amd as fs
            st["err"] = fs.cleared_err_word(dev)
            st["params"] = fs.Sampling(st["temperature"], st["top_k"], st["top_p"], st["min_p"])
        return st

    q_len, kv_len = _lengths(case)
    st["q_len"], st["rows"] = q_len, sum(q_len)
    off = [0]
    for n in q_len:
        off.append(off[-1] + n)
    st["q_off"] = torch.tensor(off, dtype=torch.int32, device=dev)
    st["kv_len"] = torch.tensor(kv_len, dtype=torch.int32, device=dev)
    st["seq_of_row"] = torch.repeat_interleave(torch.arange(len(q_len), device=dev),
                                               torch.tensor(q_len, device=dev))
    if own:
        import paper_2411_15997_amd as fs
        st["err"] = fs.cleared_err_word(dev)
        st["step"] = fs.Step(off, st["q_off"], st["kv_len"], max_kv=max(kv_len))

    if case["op"] == "linear":
        k, n, na, r = case["k"], case["n"], case["adapters"], case["rank"]
        st["x"] = normal(st["rows"], k)
        st["w"] = normal(n, k, std=k ** -0.5)
        st["a"] = normal(na, r, k, std=k ** -0.5)
        st["b"] = normal(na, n, r, std=0.5 * r ** -0.5)
        st["scale"] = uniform(na, 0.5, 2.0)
        st["rank"] = torch.randint(max(1, r // 2), r + 1, (na,), device=dev, generator=g,
                                   dtype=torch.int32)
        ad = torch.randint(0, na, (len(q_len),), device=dev, generator=g, dtype=torch.int32)
        skip = torch.rand(len(q_len), device=dev, generator=g) < case["none"]
        st["adapter"] = torch.where(skip, torch.full_like(ad, -1), ad)
        if own:
            st["adapters"] = fs.Adapters(st["a"], st["b"], st["adapter"], st["rank"], st["scale"])
        return st

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
    st["k_cache"] = normal(total, hk, page, d)
    st["v_cache"] = normal(total, hk, page, d)
    if own:
        st["cache"] = fs.KVCache(st["k_cache"], st["v_cache"], st["table"])
    if case["op"] == "attention":
        st["q"] = normal(st["rows"], h, d)
        st["scale"] = d ** -0.5
        return st
    f, factor = _frequencies(case["rotary"], case["scaling"])
    st["qkv"] = normal(st["rows"], h + 2 * hk, d)          # one joint projection's output
    st["inv_freq"] = torch.tensor(f, dtype=torch.float32, device=dev)
    st["factor"] = factor
    if own:
        st["rope"] = fs.Rope(st["inv_freq"], case["interleaved"], factor)
    return st


# ----------------------------------------------------------------- one pass

def run(st):
    op = st["op"]
    if own:
        return _own(st)
    return {"linear": _plain_linear, "rope": _plain_rope, "attention": _plain_attention,
            "sample": _plain_sample}[op](st)


def _own(st):
    import paper_2411_15997_amd as fs
    op, err = st["op"], st["err"]
    if op == "linear":
        return {"y": fs.fs_adapter_linear(st["step"], st["adapters"], st["x"], st["w"], err=err,
                                          check=False)}
    if op == "rope":
        c = st["case"]
        h, hk = c["heads"], c["kv_heads"]
        qkv = st["qkv"]
        q = fs.fs_rope_append(st["step"], st["cache"], st["rope"], qkv[:, :h], qkv[:, h:h + hk],
                              qkv[:, h + hk:], err=err, check=False)
        return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"]}
    if op == "attention":
        out, lse = fs.fs_paged_attention(st["step"], st["cache"], st["q"], st["scale"],
                                         window=st["case"]["window"], want_lse=True, err=err,
                                         check=False)
        return {"out": out, "lse": lse}
    token, logprob, kept = fs.fs_sample(st["logits"], st["u"], st["params"], err=err, check=False)
    return {"token": token, "logprob": logprob, "kept": kept}


def _plain_linear(st):
    c = st["case"]
    x, w = st["x"].float(), st["w"].float()
    y = x @ w.t()
    na, r = c["adapters"], c["rank"]
    # every adapter's products for every row, the row's own picked by a mask
    row_ad = st["adapter"][st["seq_of_row"]]
    on = torch.arange(r, device=x.device)[None] < st["rank"][:, None]
    a = torch.where(on[:, :, None], st["a"].float(), torch.zeros((), device=x.device))
    b = torch.where(on[:, None, :], st["b"].float(), torch.zeros((), device=x.device))
    h = (x @ a.reshape(na * r, -1).t()).view(-1, na, r) * st["scale"][None, :, None]
    mine = row_ad[:, None] == torch.arange(na, device=x.device)[None]
    h = torch.where(mine[:, :, None], h, torch.zeros((), device=x.device))
    y += h.reshape(-1, na * r) @ b.permute(0, 2, 1).reshape(na * r, -1)
    return {"y": y.to(st["x"].dtype)}


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


def _plain_rope(st):
    c = st["case"]
    h, hk, page = c["heads"], c["kv_heads"], c["page"]
    pos = _positions(st)
    # the angle grows with the position: its product is taken in 64 bits, the rest in 32
    theta = pos.double()[:, None] * st["inv_freq"].double()[None]
    cos = (theta.cos() * st["factor"]).float()[:, None]
    sin = (theta.sin() * st["factor"]).float()[:, None]
    x = st["qkv"].float()
    dt = st["qkv"].dtype
    turned = _turn(x[:, :h + hk], cos, sin, c["rotary"], c["interleaved"]).to(dt)
    at = st["table"][st["seq_of_row"], pos // page].long()
    st["k_cache"][at, :, pos % page] = turned[:, h:]
    st["v_cache"][at, :, pos % page] = st["qkv"][:, h + hk:]
    return {"q": turned[:, :h].contiguous(), "k_cache": st["k_cache"], "v_cache": st["v_cache"]}


def _plain_attention(st):
    c = st["case"]
    h, hk, d, page = c["heads"], c["kv_heads"], c["dim"], c["page"]
    grp, dev = h // hk, st["q"].device
    seqs, most_q, most_kv = c["seqs"], max(st["q_len"]), c["most_kv"]
    j = torch.arange(most_kv, device=dev)
    at = st["table"][:, j // page].long()
    live = (j[None] < st["kv_len"][:, None])[:, None, :, None]
    zero = torch.zeros((), device=dev)

    def rows_of(cache):            # [seqs * kv_heads][most_kv][d]
        x = cache[at, :, j % page].permute(0, 2, 1, 3).float()
        return torch.where(live, x, zero).reshape(seqs * hk, most_kv, d)

    k, v = rows_of(st["k_cache"]), rows_of(st["v_cache"])
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
        see &= j[None, None] > pos[:, :, None] - c["window"]
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


def _plain_sample(st):
    """The weights are whole numbers (2^40 for the largest logit), so that sums are exact."""
    x = st["logits"].float()
    rows, vocab = x.shape
    dev = x.device
    zero = torch.zeros((), dtype=torch.int64, device=dev)
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    t = st["temperature"].double()[:, None]
    greedy = t == 0
    val, ids = torch.sort(x, dim=1, descending=True, stable=True)
    best = val[:, :1].double()
    y = (best - val.double()) * (LOG2E / torch.where(greedy, torch.ones_like(t), t))
    y = torch.where(val == val[:, :1], torch.zeros_like(y), y)
    w = torch.floor(torch.exp2(-y) * ONE).long()
    place = torch.arange(vocab, device=dev)[None]
    if st["top_k"] is not None:
        k = st["top_k"][:, None]
        w = torch.where((k <= 0) | (place < k), w, zero)
    if st["top_p"] is not None:
        p = st["top_p"].double()[:, None]
        before = torch.cumsum(w, 1) - w
        limit = torch.ceil(p * w.sum(1, keepdim=True).double()).long().clamp(min=1)
        w = torch.where((p >= 1) | (before < limit), w, zero)
    if st["min_p"] is not None:
        w = torch.where(w >= torch.ceil(st["min_p"].double() * ONE).long()[:, None], w, zero)
    w = torch.where(greedy & (place > 0), zero, w)
    by_id = torch.zeros_like(w).scatter_(1, ids, w)
    total = by_id.sum(1)
    goal = torch.minimum(torch.floor(st["u"].double() * total.double()).long(), total - 1)
    token = (torch.cumsum(by_id, 1) <= goal[:, None]).sum(1)
    mine = by_id.gather(1, token[:, None])[:, 0]
    logprob = (mine.double() / total.double()).log().float()
    return {"token": token.int(), "logprob": logprob, "kept": (w > 0).sum(1).int()}


# ----------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * size + case["rows"] * 32, "flops": 0}
    q, kv = _lengths(case)
    t = sum(q)
    if case["op"] == "linear":
        k, n, r = case["k"], case["n"], case["rank"]
        used = min(case["adapters"], case["seqs"])
        return {"bytes": size * (t * k + n * k + t * n + used * r * (k + n)),
                "flops": 2 * t * n * k + 2 * t * r * (k + n) * (1 - case["none"])}
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "rope":
        return {"bytes": 2 * t * (h + 2 * hk) * d * size, "flops": 3 * t * (h + hk) * case["rotary"]}
    win = case["window"]
    read, pairs = 0, 0
    for a, b in zip(q, kv):
        lo = max(0, b - a - win + 1) if win else 0
        read += b - lo
        first, last = b - a + 1, b                    # visible keys of the first and last row
        if win:
            full = max(0, min(a, last - win + 1)) if last >= win else 0
            short = a - full
            pairs += full * win + (first + first + short - 1) * short // 2
        else:
            pairs += (first + last) * a // 2
    return {"bytes": size * (2 * read * hk * d + 2 * t * h * d) + 4 * t * h,
            "flops": 4 * d * h * pairs}


# ----------------------------------------------------------------- in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "sample":
        return _exact_sample(st)
    q_len, kv_len = _lengths(case)
    off = [0]
    for n in q_len:
        off.append(off[-1] + n)
    if op == "linear":
        y = torch.empty(off[-1], case["n"], dtype=torch.float64, device="cuda")
        w = st["w"].double().t().contiguous()
        for s in range(len(q_len)):
            x = st["x"][off[s]:off[s + 1]].double()
            y[off[s]:off[s + 1]] = x @ w
            a = int(st["adapter"][s])
            if a >= 0:
                r = int(st["rank"][a])
                h = x @ st["a"][a, :r].double().t()
                y[off[s]:off[s + 1]] += float(st["scale"][a]) * (h @ st["b"][a, :, :r].double().t())
        return {"y": y}
    if op == "rope":
        return _exact_rope(st, case, q_len, kv_len, off)
    return _exact_attention(st, case, q_len, kv_len, off)


def _exact_rope(st, case, q_len, kv_len, off):
    h, hk, page, rot = case["heads"], case["kv_heads"], case["page"], case["rotary"]
    half = rot // 2
    first = torch.arange(half, device="cuda") * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else half)
    f = st["inv_freq"].double()
    q_out = torch.empty(off[-1], h, case["dim"], dtype=torch.float64, device="cuda")
    kc, vc = st["k_cache"].double(), st["v_cache"].double()
    for s, (n, kv) in enumerate(zip(q_len, kv_len)):
        x = st["qkv"][off[s]:off[s + 1]].double()
        p = torch.arange(kv - n, kv, device="cuda")
        z = torch.polar(torch.full((n, half), float(st["factor"]), dtype=torch.float64, device="cuda"),
                        p.double()[:, None] * f)
        turned = torch.complex(x[:, :h + hk, first], x[:, :h + hk, second]) * z[:, None]
        y = x.clone()
        y[:, :h + hk, first] = turned.real
        y[:, :h + hk, second] = turned.imag
        q_out[off[s]:off[s + 1]] = y[:, :h]
        at = st["table"][s].long()[p // page]
        kc[at, :, p % page] = y[:, h:h + hk]
        vc[at, :, p % page] = y[:, h + hk:]
    return {"q": q_out, "k_cache": kc, "v_cache": vc}


def _exact_attention(st, case, q_len, kv_len, off):
    h, hk, d, page, win = case["heads"], case["kv_heads"], case["dim"], case["page"], case["window"]
    grp = h // hk
    out = torch.empty(off[-1], h, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(off[-1], h, dtype=torch.float64, device="cuda")
    for s, (n, kv) in enumerate(zip(q_len, kv_len)):
        j = torch.arange(kv, device="cuda")
        at = st["table"][s].long()[j // page]
        p = torch.arange(kv - n, kv, device="cuda")
        see = (j[None] <= p[:, None]) & ((j[None] > p[:, None] - win) if win else True)
        for m in range(hk):
            k, v = (st[x][at, m, j % page].double() for x in ("k_cache", "v_cache"))
            for i in range(m * grp, (m + 1) * grp):
                q = st["q"][off[s]:off[s + 1], i].double()
                score = (q @ k.t().contiguous()) * float(st["scale"])
                score = score.masked_fill(~see, -math.inf)
                out[off[s]:off[s + 1], i] = torch.softmax(score, -1) @ v
                lse[off[s]:off[s + 1], i] = torch.logsumexp(score, -1)
    return {"out": out, "lse": lse}


def _exact_sample(st):
    """From real-valued probabilities; a token is a matter of the whole-number weights."""
    logits = st["logits"].double().cpu()
    rows = logits.shape[0]
    value = lambda name, i, other: other if st[name] is None else float(st[name][i])  # noqa: E731
    logprob = torch.empty(rows, dtype=torch.float64)
    for i in range(rows):
        t, k = value("temperature", i, 1.0), int(value("top_k", i, 0))
        if t == 0:
            logprob[i] = 0.0
            continue
        x, ids = torch.sort(logits[i], descending=True, stable=True)
        prob = torch.softmax(x / t, 0)
        if 0 < k < x.numel():
            prob[k:] = 0
        prob = prob / prob.sum()
        p = value("top_p", i, 1.0)
        if p < 1:
            prob[(torch.cumsum(prob, 0) - prob) >= p] = 0
        prob[prob < prob[0] * value("min_p", i, 0.0)] = 0
        prob = prob / prob.sum()
        by_id = torch.zeros_like(prob).scatter_(0, ids, prob)
        token = int((torch.cumsum(by_id, 0) <= float(st["u"][i])).sum().clamp(max=x.numel() - 1))
        logprob[i] = by_id[token].log()
    return {"token": None, "logprob": logprob, "kept": None}
