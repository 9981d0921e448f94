"""The cache's operators together, as an engine uses them: prompts forked from their apps',
chunks and single tokens appended and attended to, calls that end, pages moved together; and
the example that does so."""
import math
import random

import pytest
import torch

import cache_ref as cref
import engine_ref as ref
import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_engine import BF, HF, gen, normal, within
from test_gpu_engine_steps import example

pytestmark = pytest.mark.gpu
PAGE, H, HK, D, VOCAB = 8, 4, 2, 64, 50


class Layer:
    """A layer whose queries, keys and values hang on the token alone."""

    def __init__(self, seed, dtype, four, pages, table):
        g = gen(seed)
        self.rows = normal(g, VOCAB, H + 2 * HK, D, dtype=dtype)
        if four:
            t = [torch.zeros(pages, HK, PAGE, n, dtype=torch.uint8, device="cuda")
                 for n in (D // 2, D // 2, D // 32, D // 32)]
            self.cache = fs.KVCache4(*t, table)
        else:
            t = [torch.zeros(pages, HK, PAGE, D, dtype=dtype, device="cuda") for _ in range(2)]
            self.cache = fs.KVCache(*t, table)


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
@pytest.mark.parametrize("four,dtype", [(False, BF), (True, BF), (True, HF)])
def test_an_engines_steps(four, dtype, window, sinks):
    """Every step's attention is the oracle's over the calls' own token lists, whatever pages
    they share and wherever these have been moved."""
    rng = random.Random(7)
    pages, rows, width, apps = 120, 14, 12, 2
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
    pool = fs.PagePool(torch.zeros(pages, dtype=torch.int32, device="cuda"), table,
                       torch.zeros(rows, dtype=torch.int32, device="cuda"), PAGE)
    layers = [Layer(s, dtype, four, pages, table) for s in (1, 2)]
    every = fs.CacheLayers([L.cache for L in layers])
    freq, factor = fs.fs_rope_frequencies(D, 10000.0)
    inv = torch.from_numpy(freq)
    rope, err = fs.Rope(inv.cuda(), False, factor), fs.cleared_err_word()
    scale, top = D ** -0.5, cref.TOP[dtype]
    append = fs.fs_rope_append4 if four else fs.fs_rope_append
    attend = fs.fs_paged_attention4 if four else fs.fs_paged_attention

    def rows_of(L, ids):
        """(turned queries, keys, values) of a call's tokens in 64 bits, as the cache has them."""
        x = L.rows[ids]
        y, _ = ref.rope_rows(x[:, :H + HK], list(range(len(ids))), inv, D, False, factor)
        y = torch.from_numpy(y)
        q, k, v = y[:, :H].to(dtype), y[:, H:], x[:, H + HK:]
        if not four:
            return q, k.to(dtype).double(), v.double()
        out = []
        for t in (k.float(), v.float()):
            code, byte = cref.quantise(t.numpy(), top)
            out.append(cref.values(cref.pack(code), torch.from_numpy(byte), top))
        return q, *out

    def engine_step(calls):
        """calls: (row, all token ids, new ones among them)."""
        q_off, kv = [0], [len(ids) for _, ids, _ in calls]
        for _, _, n in calls:
            q_off.append(q_off[-1] + n)
        step = fs.Step(q_off, kv_len=i32(kv), max_kv=max(kv))
        mine = table[i32([r for r, _, _ in calls]).long()]
        new = torch.tensor([t for _, ids, n in calls for t in ids[len(ids) - n:]])
        for L in layers:
            x = L.rows[new].cuda()
            kind = type(L.cache)
            cache = kind(*((L.cache.k, L.cache.v, L.cache.k_scale, L.cache.v_scale) if four else
                           (L.cache.k, L.cache.v)), mine)
            q = append(step, cache, rope, x[:, :H], x[:, H:H + HK], x[:, H + HK:], err=err, check=False)
            o, lse = attend(step, cache, q, scale, window=window, sinks=sinks, want_lse=True, err=err,
                            check=False)
            for i, (_, ids, n) in enumerate(calls):
                _, k, v = rows_of(L, ids)
                at = slice(q_off[i], q_off[i + 1])
                # (queries as the kernel has turned and rounded them; the oracle's cache holds the
                # call alone, one page for all)
                kk, vv = (t.transpose(0, 1)[None] for t in (k, v))
                # The kernel turns 16-bit keys in fp32: next to a border one's rounding may be the
                # other one, 2 u of it; eight of a key's 64 elements at most, each of the largest size.
                want, tol, wl, ltol = cref.attention(q[at].cpu(), kk, vv, torch.zeros(1, 1, dtype=torch.int32),
                                                     [0, n], [len(ids)], scale, window, sinks)
                if not four:
                    u = ref.U16[dtype]
                    ds = 2 * u * scale * float(q[at].double().abs().amax()) * float(k.abs().amax()) * D ** 0.5
                    tol, ltol = tol + 2 * ds * float(v.abs().amax()), ltol + ds
                within(o[at], want, tol, f"out of call {i}")
                within(lse[at], wl, ltol, f"lse of call {i}")

    prompts = [[rng.randrange(VOCAB) for _ in range(n)] for n in (21, 40)]
    fs.fs_pages_fork(pool, i32([-1, -1]), i32([0, 1]), i32([0, 0]), i32([21, 40]), err=err, check=False)
    engine_step([(a, prompts[a], len(prompts[a])) for a in range(apps)])
    free_rows, running = list(range(apps, rows)), []
    for turn in range(9):
        forks, new = [], []
        for _ in range(rng.randint(0, 3)):
            if not free_rows:
                break
            a = rng.randrange(apps)
            shared = rng.choice((len(prompts[a]), rng.randint(0, len(prompts[a]))))
            ids = prompts[a][:shared] + [rng.randrange(VOCAB) for _ in range(rng.randint(1, 20))]
            row = free_rows.pop()
            forks.append((a, row, shared, len(ids) + 12))
            new.append([row, ids, len(ids) - shared, 12])
        if forks:
            src, dst = fs.fs_pages_fork(pool, *(i32(list(x)) for x in zip(*forks)), err=err, check=False)
            fs.fs_pages_copy(every, src, dst, err=err, check=False)
        for c in running:                       # the others decode one token
            c[1].append(rng.randrange(VOCAB))
            c[2] = 1
        running += new
        if running:
            engine_step([(r, ids, n) for r, ids, n, _ in running])
        for c in running:
            c[3] -= 1
        ended = [c for c in running if c[3] == 0 or rng.random() < 0.15]
        running = [c for c in running if c not in ended]
        if ended:
            fs.fs_pages_free(pool, i32([c[0] for c in ended]), err=err, check=False)
            free_rows += [c[0] for c in ended]
        if turn % 3 == 2:
            src, dst, count = fs.fs_pages_compact(pool, err=err, check=False)
            fs.fs_pages_copy(every, src, dst, count, err=err, check=False)
            live = int((pool.refs > 0).sum())
            assert bool((pool.refs[:live] > 0).all()) and int(pool.refs[live:].sum()) == 0
    assert int(err) == 0
    fs.fs_pages_free(pool, i32([c[0] for c in running] + [0, 1]))
    assert int(pool.refs.sum()) == 0 and int(pool.held.sum()) == 0


@pytest.mark.parametrize("kw", [dict(system=40), dict(cache4=True), dict(cache4=True, system=100, window=64, sinks=4),
                                dict(window=100, sinks=8, compact_every=3)])
def test_the_example_with_the_caches_operators(kw):
    ex = example()
    model, tr, done, s = ex.play(requests=30, layers=2, **kw)
    say("engine steps", kw, s)
    assert len(done) == s["admitted"] > 0
    for g, r in done.items():
        assert len(r["out"]) == max(int(tr.len_out[g]), 1)
        assert all(0 <= t < model.vocab for t in r["out"])
    # all calls have ended: what is held are the apps' prompts
    assert s["held"] == tr.n_apps * math.ceil(kw.get("system", 0) / ex.PAGE)


@pytest.mark.parametrize("cache4", [False, True])
def test_compaction_changes_no_token(cache4):
    """Pages moved every third step, or never: bit by bit the same logits, so the same tokens."""
    ex = example()
    outs = [{g: r["out"] for g, r in ex.play(requests=30, layers=2, system=30, cache4=cache4,
                                             compact_every=n)[2].items()} for n in (0, 3)]
    assert outs[0] == outs[1]
