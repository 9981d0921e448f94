"""Runs the schedule of the literal engine (FS_ENGINE_LITERAL) through a small decoder.

The scheduler decides which calls an engine step prefills and which running calls decode
one more token; this example is the engine that does it, with the package's operators:

  per layer   fs_adapter_linear (q, k, v; every app has its own adapter), fs_rope_append,
              fs_paged_attention, fs_adapter_linear (output), two plain projections
              (with --cache4 fs_rope_append4 and fs_paged_attention4 on a cache in 4 bits)
  at the end  fs_adapter_linear (logits), fs_sample
  per step    fs_pages_fork and fs_pages_copy for the calls that begin, fs_pages_free for
              those that end, fs_pages_compact and fs_pages_copy from time to time

Weights and token ids are random; lengths, apps, admissions and the KV capacity are the
trace's.  A call is prefilled in its admission step and holds its pages until it has
L_O output tokens, as the engine model says.  With --system N the calls of an app begin
with the same N tokens, which are prefilled once and whose whole pages they share.

    python examples/engine_steps.py [--requests N] [--layers L] [--users U] [--cache4]
                                    [--system N] [--window N --sinks N]
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2411_15997_amd as fs  # noqa: E402
import tracegen as tg  # noqa: E402

PAGE = 16


def schedule(requests, users=8, step_ms=250.0, cap_tokens=8192):
    """A two-app trace through the literal engine: (trace, outputs on the host, capacity)."""
    wl = tg.scaled(tg.WORKLOADS["c1_small"], records=requests, users=users)
    tr = tg.generate(wl)
    dt = fs.DeviceTrace(tr)
    coef, per_rep = fs.workload_weights(wl, tr)
    w, keep = fs.make_weights(dt, coef, None, per_rep)
    lim = fs.make_limits(wl.window_us, wl.t_user, wl.t_app)
    eng = fs.make_engine(int(step_ms * 1000), cap_tokens, cap_tokens, literal=True)
    out = fs.Outputs(dt)
    ws, _, _ = fs.run_trace_buffers(dt)
    fs.fs_run_trace(dt, w, lim, eng, out, ws)
    return tr, out.host(), cap_tokens


class Decoder:
    """Random weights of a small decoder with an adapter for each app on its attention
    projections, and its paged caches (16 bits or, with cache4, 4 bits a value); attention over
    all cached tokens, or over a window and the first `sinks`."""

    def __init__(self, apps, pages, layers=2, width=512, heads=8, kv_heads=2, dim=64, vocab=2048,
                 rank=16, seed=0, dtype=torch.bfloat16, device="cuda", cache4=False, window=0,
                 sinks=0):
        g = torch.Generator(device).manual_seed(seed)

        def normal(*shape, std):
            return torch.empty(shape, dtype=dtype, device=device).normal_(0, std, generator=g)

        def cache():
            if not cache4:
                return [normal(pages, kv_heads, PAGE, dim, std=1.0) for _ in range(2)]
            return [torch.zeros(pages, kv_heads, PAGE, n, dtype=torch.uint8, device=device)
                    for n in (dim // 2, dim // 2, dim // 32, dim // 32)]

        self.cache4, self.window, self.sinks = cache4, window, sinks
        self.heads, self.kv_heads, self.dim, self.width, self.vocab = heads, kv_heads, dim, width, vocab
        qkv, hd = (heads + 2 * kv_heads) * dim, heads * dim
        self.embed = normal(vocab, width, std=1.0)
        self.head = normal(vocab, width, std=width ** -0.5)
        self.layers = [dict(
            qkv=normal(qkv, width, std=width ** -0.5), out=normal(width, hd, std=hd ** -0.5),
            up=normal(4 * width, width, std=width ** -0.5),
            down=normal(width, 4 * width, std=0.5 * width ** -0.5),
            a_qkv=normal(apps, rank, width, std=width ** -0.5), b_qkv=normal(apps, qkv, rank, std=0.1),
            a_out=normal(apps, rank, hd, std=hd ** -0.5), b_out=normal(apps, width, rank, std=0.1),
            cache=cache()) for _ in range(layers)]
        freq, factor = fs.fs_rope_frequencies(dim, 10000.0)
        self.rope = fs.Rope(torch.from_numpy(freq).to(device), False, factor)
        self.scale = dim ** -0.5
        self.dtype, self.device = dtype, device

    @staticmethod
    def norm(x):
        f = x.float()
        return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def caches(self, table):
        """Each layer's cache under a page table."""
        kind = fs.KVCache4 if self.cache4 else fs.KVCache
        return [kind(*L["cache"], table) for L in self.layers]

    def step(self, ids, q_off, kv_len, table, app, u, sampling, err):
        """One engine step: token ids of its rows, where each request's rows begin, its cached
        length with them, its pages and its app -> each request's next token, its logits."""
        dev = self.device
        step = fs.Step(q_off, kv_len=torch.tensor(kv_len, dtype=torch.int32, device=dev),
                       max_kv=max(kv_len), device=dev)
        table = torch.as_tensor(table).to(dev)
        app = torch.tensor(app, dtype=torch.int32, device=dev)
        h, hk, T = self.heads, self.kv_heads, step.rows
        x = self.embed[torch.tensor(ids, device=dev)]

        def linear(x, w, a=None, b=None):
            if a is None:               # the shared projection alone
                a, b = x.new_empty(0, 8, w.shape[1]), x.new_empty(0, w.shape[0], 8)
            return fs.fs_adapter_linear(step, fs.Adapters(a, b, app), x, w, err=err, check=False)

        append = fs.fs_rope_append4 if self.cache4 else fs.fs_rope_append
        attend = fs.fs_paged_attention4 if self.cache4 else fs.fs_paged_attention
        for L, cache in zip(self.layers, self.caches(table)):
            qkv = linear(self.norm(x), L["qkv"], L["a_qkv"], L["b_qkv"]).view(T, h + 2 * hk, self.dim)
            q = append(step, cache, self.rope, qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:], err=err,
                       check=False)
            o = attend(step, cache, q, self.scale, window=self.window, sinks=self.sinks, err=err,
                       check=False)
            x = x + linear(o.view(T, -1), L["out"], L["a_out"], L["b_out"])
            x = x + linear(torch.nn.functional.silu(linear(self.norm(x), L["up"])), L["down"])
        last = torch.tensor(q_off[1:], device=dev) - 1
        n = len(kv_len)
        rows = fs.Step(list(range(n + 1)), device=dev)          # one row a request
        none = fs.Adapters(x.new_empty(0, 8, self.width), x.new_empty(0, self.vocab, 8), app)
        logits = fs.fs_adapter_linear(rows, none, self.norm(x[last]), self.head, err=err, check=False)
        token, _, _ = fs.fs_sample(logits, u, sampling, err=err, check=False)
        return token, logits


class Pages:
    """Rows of a page table and the pages behind them, of all layers' caches at once."""

    def __init__(self, model, pages, rows, width):
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=model.device)  # noqa: E731
        self.pool = fs.PagePool(i32(pages), i32(rows, width), i32(rows), PAGE)
        self.layers = fs.CacheLayers(model.caches(self.pool.table))
        self.device = model.device

    def ids(self, x):
        return torch.tensor(x, dtype=torch.int32, device=self.device)

    def begin(self, forks, err):
        """forks: (parent row or -1, row, shared tokens, room in tokens) each."""
        src, dst = fs.fs_pages_fork(self.pool, *(self.ids(list(x)) for x in zip(*forks)), err=err,
                                    check=False)
        fs.fs_pages_copy(self.layers, src, dst, err=err, check=False)

    def end(self, rows, err):
        fs.fs_pages_free(self.pool, self.ids(rows), err=err, check=False)

    def compact(self, err):
        src, dst, count = fs.fs_pages_compact(self.pool, err=err, check=False)
        fs.fs_pages_copy(self.layers, src, dst, count, err=err, check=False)


def play(requests=120, layers=2, users=8, seed=0, greedy=False, system=0, cache4=False, window=0,
         sinks=0, compact_every=50):
    """Plays the schedule; returns what was generated and how the cache was used."""
    tr, h, cap = schedule(requests, users)
    n = tr.n
    status, admit = h["status"][:n], h["admit_step"][:n]
    len_in = np.asarray(tr.len_in, np.int64) + (0 if tr.len_sys is None else tr.len_sys)
    prompt = np.maximum(len_in, 1).astype(int)
    answer = np.maximum(np.asarray(tr.len_out), 1).astype(int)
    size = len_in + np.asarray(tr.len_out)
    admitted = np.nonzero(status == 0)[0]
    apps = tr.n_apps
    pages = max(2 * cap, 2 * int(size.max(initial=1))) // PAGE + 2 * len(admitted) + 1 + \
        apps * (-(-system // PAGE))
    model = Decoder(apps, pages, layers, seed=seed, cache4=cache4, window=window, sinks=sinks)
    rng = np.random.default_rng(seed)
    most = max(system, int((prompt + answer).max(initial=1)))
    store = Pages(model, pages, apps + len(admitted), -(-most // PAGE))
    slots = list(range(apps, apps + len(admitted)))[::-1]
    running, done = [], {}
    by_step = {}
    for g in admitted:
        by_step.setdefault(int(admit[g]), []).append(int(g))
    err = fs.cleared_err_word()

    def step(rows, new, kv, app, u, sampling):
        q_off = [0] + list(np.cumsum([len(x) for x in new]))
        table = store.pool.table[store.ids(rows).long()]
        return model.step([t for x in new for t in x], q_off, kv, table, app, u, sampling, err)[0]

    # the apps' prompts, prefilled once
    shared = [rng.integers(0, model.vocab, system).tolist() for _ in range(apps)]
    if system:
        store.begin([(-1, a, 0, system) for a in range(apps)], err)
        step(range(apps), shared, [system] * apps, list(range(apps)), torch.zeros(apps, device="cuda"),
             fs.Sampling())
    stats = dict(steps=0, rows=0, most_tokens=0, most_running=0, most_pages=0)
    torch.cuda.synchronize()
    began = time.perf_counter()
    last_step = max((int(admit[g]) + answer[g] for g in admitted), default=0)
    for s in range(last_step):
        forks = []
        for g in by_step.get(s, []):           # prefilled in this step
            # (the last token of a prompt is always the call's own: its logits are wanted)
            common = min(system, int(prompt[g]) - 1)
            app = int(tr.app[g])
            own = rng.integers(0, model.vocab, prompt[g] - common).tolist()
            row = slots.pop()
            forks.append((app if common else -1, row, common, int(prompt[g] + answer[g])))
            running.append(dict(g=g, ids=shared[app][:common] + own, new=own, row=row, app=app, out=[]))
        if not running:
            continue
        if forks:
            store.begin(forks, err)
        kv = [len(r["ids"]) for r in running]
        u = torch.from_numpy(rng.random(len(running), np.float32)).cuda()
        top_p = torch.full((len(running),), 0.9, device="cuda")
        temp = torch.full((len(running),), 0.0 if greedy else 0.8, device="cuda")
        token = step([r["row"] for r in running], [r["new"] for r in running], kv,
                     [r["app"] for r in running], u, fs.Sampling(temperature=temp, top_p=top_p))
        stats["steps"] += 1
        stats["rows"] += sum(len(r["new"]) for r in running)
        stats["most_running"] = max(stats["most_running"], len(running))
        stats["most_tokens"] = max(stats["most_tokens"], int(sum(size[r["g"]] for r in running)))
        for r, t in zip(running, token.tolist()):
            r["out"].append(t)
            r["ids"], r["new"] = r["ids"] + [t], [t]
        ended = [r for r in running if len(r["out"]) == answer[r["g"]]]
        if ended:
            stats["most_pages"] = max(stats["most_pages"], int((store.pool.refs > 0).sum()))
            store.end([r["row"] for r in ended], err)
        for r in ended:
            running.remove(r)
            slots.append(r["row"])
            done[r["g"]] = r
        if compact_every and s % compact_every == compact_every - 1:
            store.compact(err)
    fs.sync_check(err, "engine steps")
    stats.update(seconds=time.perf_counter() - began, tokens=sum(len(r["out"]) for r in done.values()),
                 admitted=len(admitted), requests=n, cap=cap, largest=int(size.max(initial=0)),
                 held=int((store.pool.refs > 0).sum()), pages=pages)
    return model, tr, done, stats


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--requests", type=int, default=120)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--users", type=int, default=8)
    ap.add_argument("--cache4", action="store_true", help="a cache of 4 bits a value")
    ap.add_argument("--system", type=int, default=0, help="tokens that an app's calls begin with")
    ap.add_argument("--window", type=int, default=0, help="newest tokens that attention sees (0: all)")
    ap.add_argument("--sinks", type=int, default=0, help="first tokens that it sees beside them")
    a = ap.parse_args()
    _, _, done, s = play(a.requests, a.layers, a.users, system=a.system, cache4=a.cache4,
                         window=a.window, sinks=a.sinks)
    print(f"{s['requests']} requests, {s['admitted']} admitted; {s['steps']} engine steps, {s['rows']} "
          f"token rows, {s['tokens']} tokens generated; at most {s['most_running']} calls and "
          f"{s['most_tokens']} of {s['cap']} KV tokens at once; {s['seconds']:.2f} s, "
          f"{1e3 * s['seconds'] / max(1, s['steps']):.2f} ms a step")


if __name__ == "__main__":
    main()
