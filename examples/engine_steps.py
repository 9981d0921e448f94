"""Runs the schedule of the literal engine (FS_ENGINE_LITERAL) through a small decoder.

The scheduler decides which calls an engine step prefills and which running calls decode
one more token; this example is the engine that does it, with the package's operators:

  per layer   fs_adapter_linear (q, k, v; every app has its own adapter), fs_rope_append,
              fs_paged_attention, fs_adapter_linear (output), two plain projections
  at the end  fs_adapter_linear (logits), fs_sample

Weights and token ids are random; lengths, apps, admissions and the KV capacity are the
trace's.  A call is prefilled in its admission step and holds its pages until it has
L_O output tokens, as the engine model says.

    python examples/engine_steps.py [--requests N] [--layers L] [--users U]
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
    projections, and its paged caches."""

    def __init__(self, apps, pages, layers=2, width=512, heads=8, kv_heads=2, dim=64, vocab=2048,
                 rank=16, seed=0, dtype=torch.bfloat16, device="cuda"):
        g = torch.Generator(device).manual_seed(seed)

        def normal(*shape, std):
            return torch.empty(shape, dtype=dtype, device=device).normal_(0, std, generator=g)

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
            k=normal(pages, kv_heads, PAGE, dim, std=1.0), v=normal(pages, kv_heads, PAGE, dim, std=1.0))
            for _ in range(layers)]
        freq, factor = fs.fs_rope_frequencies(dim, 10000.0)
        self.rope = fs.Rope(torch.from_numpy(freq).to(device), False, factor)
        self.scale = dim ** -0.5
        self.dtype, self.device = dtype, device

    @staticmethod
    def norm(x):
        f = x.float()
        return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def step(self, ids, q_off, kv_len, table, app, u, sampling, err):
        """One engine step: token ids of its rows, where each request's rows begin, its cached
        length with them, its pages and its app -> each request's next token, its logits."""
        dev = self.device
        step = fs.Step(q_off, kv_len=torch.tensor(kv_len, dtype=torch.int32, device=dev),
                       max_kv=max(kv_len), device=dev)
        table = torch.from_numpy(table).to(dev)
        app = torch.tensor(app, dtype=torch.int32, device=dev)
        h, hk, T = self.heads, self.kv_heads, step.rows
        x = self.embed[torch.tensor(ids, device=dev)]

        def linear(x, w, a=None, b=None):
            if a is None:               # the shared projection alone
                a, b = x.new_empty(0, 8, w.shape[1]), x.new_empty(0, w.shape[0], 8)
            return fs.fs_adapter_linear(step, fs.Adapters(a, b, app), x, w, err=err, check=False)

        for L in self.layers:
            cache = fs.KVCache(L["k"], L["v"], table)
            qkv = linear(self.norm(x), L["qkv"], L["a_qkv"], L["b_qkv"]).view(T, h + 2 * hk, self.dim)
            q = fs.fs_rope_append(step, cache, self.rope, qkv[:, :h], qkv[:, h:h + hk],
                                  qkv[:, h + hk:], err=err, check=False)
            o = fs.fs_paged_attention(step, cache, q, self.scale, err=err, check=False)
            x = x + linear(o.view(T, -1), L["out"], L["a_out"], L["b_out"])
            x = x + linear(torch.nn.functional.silu(linear(self.norm(x), L["up"])), L["down"])
        last = torch.tensor(q_off[1:], device=dev) - 1
        n = len(kv_len)
        rows = fs.Step(list(range(n + 1)), device=dev)          # one row a request
        none = fs.Adapters(x.new_empty(0, 8, self.width), x.new_empty(0, self.vocab, 8), app)
        logits = fs.fs_adapter_linear(rows, none, self.norm(x[last]), self.head, err=err, check=False)
        token, _, _ = fs.fs_sample(logits, u, sampling, err=err, check=False)
        return token, logits


def play(requests=120, layers=2, users=8, seed=0, greedy=False):
    """Plays the schedule; returns what was generated and how the cache was used."""
    tr, h, cap = schedule(requests, users)
    n = tr.n
    status, admit = h["status"][:n], h["admit_step"][:n]
    len_in = np.asarray(tr.len_in, np.int64) + (0 if tr.len_sys is None else tr.len_sys)
    prompt = np.maximum(len_in, 1).astype(int)
    answer = np.maximum(np.asarray(tr.len_out), 1).astype(int)
    size = len_in + np.asarray(tr.len_out)
    admitted = np.nonzero(status == 0)[0]
    pages = max(2 * cap, 2 * int(size.max(initial=1))) // PAGE + 2 * len(admitted) + 1
    model = Decoder(tr.n_apps, pages, layers, seed=seed)
    rng = np.random.default_rng(seed)
    free, running, done = list(range(pages))[::-1], [], {}
    by_step = {}
    for g in admitted:
        by_step.setdefault(int(admit[g]), []).append(int(g))
    err = fs.cleared_err_word()
    stats = dict(steps=0, rows=0, most_tokens=0, most_running=0)
    torch.cuda.synchronize()
    began = time.perf_counter()
    last_step = max((int(admit[g]) + answer[g] for g in admitted), default=0)
    for s in range(last_step):
        for g in by_step.get(s, []):           # prefilled in this step
            ids = rng.integers(0, model.vocab, prompt[g]).tolist()
            need = -(-(prompt[g] + answer[g]) // PAGE)
            running.append(dict(g=g, ids=ids, new=ids, pages=[free.pop() for _ in range(need)], out=[]))
        if not running:
            continue
        q_off = [0] + list(np.cumsum([len(r["new"]) for r in running]))
        kv = [len(r["ids"]) for r in running]
        table = np.zeros((len(running), max(len(r["pages"]) for r in running)), np.int32)
        for i, r in enumerate(running):
            table[i, :len(r["pages"])] = r["pages"]
        u = torch.from_numpy(rng.random(len(running), np.float32)).cuda()
        top_p = torch.full((len(running),), 0.9, device="cuda")
        temp = torch.full((len(running),), 0.0 if greedy else 0.8, device="cuda")
        token, _ = model.step([t for r in running for t in r["new"]], q_off, kv, table,
                              [int(tr.app[r["g"]]) for r in running], u,
                              fs.Sampling(temperature=temp, top_p=top_p), err)
        stats["steps"] += 1
        stats["rows"] += q_off[-1]
        stats["most_running"] = max(stats["most_running"], len(running))
        stats["most_tokens"] = max(stats["most_tokens"], int(sum(size[r["g"]] for r in running)))
        for r, t in zip(running, token.tolist()):
            r["out"].append(t)
            r["ids"], r["new"] = r["ids"] + [t], [t]
        for r in [r for r in running if len(r["out"]) == answer[r["g"]]]:
            running.remove(r)
            free.extend(r["pages"])
            done[r["g"]] = r
    fs.sync_check(err, "engine steps")
    stats.update(seconds=time.perf_counter() - began, tokens=sum(len(r["out"]) for r in done.values()),
                 admitted=len(admitted), requests=n, cap=cap, largest=int(size.max(initial=0)))
    return model, tr, done, stats


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--requests", type=int, default=120)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--users", type=int, default=8)
    a = ap.parse_args()
    _, _, done, s = play(a.requests, a.layers, a.users)
    print(f"{s['requests']} requests, {s['admitted']} admitted; {s['steps']} engine steps, {s['rows']} "
          f"token rows, {s['tokens']} tokens generated; at most {s['most_running']} calls and "
          f"{s['most_tokens']} of {s['cap']} KV tokens at once; {s['seconds']:.2f} s, "
          f"{1e3 * s['seconds'] / max(1, s['steps']):.2f} ms a step")


if __name__ == "__main__":
    main()
