"""The 16-bit cache through the operators of its pages, value by value: what an engine's calls hold
after forks, appends, copies and compaction, and attention held to the bound of the keys as the
cache has them."""
import random

import pytest
import torch

import cache_ref as cref
import engine_ref as ref
import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_cache_steps import D, H, HK, PAGE, VOCAB, Layer
from test_gpu_engine import BF, HF, within

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def held_rows(cache, table_row, n):
    """(k, v) [n][kv_heads][dim] that a call of n tokens holds, through its row of the table."""
    j = torch.arange(n)
    ids = table_row.cpu()[j // PAGE].long()
    return cache.k.cpu()[ids, :, j % PAGE], cache.v.cpu()[ids, :, j % PAGE]


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_what_calls_hold_and_what_attention_makes_of_it(dtype, window, sinks):
    say("values of calls", dtype, window, sinks)
    rng = random.Random(11)
    pages, rows, width = 110, 12, 12
    table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
    pool = fs.PagePool(i32([0] * pages), table, i32([0] * rows), PAGE)
    layers = [Layer(s, dtype, False, pages, table) for s in (3, 4)]
    every = fs.CacheLayers([L.cache for L in layers])
    freq, factor = fs.fs_rope_frequencies(D, 10000.0)
    inv, err, scale = torch.from_numpy(freq), fs.cleared_err_word(), D ** -0.5
    rope = fs.Rope(inv.cuda(), False, factor)

    def engine_step(calls):
        """calls: (row, all token ids, new ones among them)."""
        q_off, kv = [0], [len(ids) for _, ids, _ in calls]
        for _, _, n in calls:
            q_off.append(q_off[-1] + n)
        step = fs.Step(q_off, kv_len=i32(kv), max_kv=max(kv))
        mine = table[i32([r for r, _, _ in calls]).long()]
        new = torch.tensor([t for _, ids, n in calls for t in ids[len(ids) - n:]])
        for L in layers:
            x, cache = L.rows[new].cuda(), fs.KVCache(L.cache.k, L.cache.v, mine)
            q = fs.fs_rope_append(step, cache, rope, x[:, :H], x[:, H:H + HK], x[:, H + HK:], err=err,
                                  check=False)
            o, lse = fs.fs_paged_attention(step, cache, q, scale, window, want_lse=True, err=err,
                                           check=False, sinks=sinks)
            for i, (_, ids, n) in enumerate(calls):
                k, v = held_rows(cache, mine[i], len(ids))
                # keys turned and rounded to the type, values as they were given
                y, bound = ref.rope_rows(L.rows[ids][:, H:H + HK], list(range(len(ids))), inv, D, False, factor)
                within(k, y, bound, f"keys of call {i}")
                assert torch.equal(v, L.rows[ids][:, H + HK:]), f"values of call {i}"
                # (the oracle's cache holds the call alone, one page for all)
                at = slice(q_off[i], q_off[i + 1])
                want, tol, wl, ltol = cref.attention(
                    q[at].cpu(), *(t.double().transpose(0, 1)[None] for t in (k, v)),
                    torch.zeros(1, 1, dtype=torch.int32), [0, n], [len(ids)], scale, window, sinks)
                within(o[at], want, tol, f"out of call {i}")
                within(lse[at], wl, ltol, f"lse of call {i}")

    prompts = [[rng.randrange(VOCAB) for _ in range(n)] for n in (19, 37)]
    fs.fs_pages_fork(pool, i32([-1, -1]), i32([0, 1]), i32([0, 0]), i32([19, 37]), err=err, check=False)
    engine_step([(a, prompts[a], len(prompts[a])) for a in (0, 1)])
    free_rows, running = list(range(2, rows)), []
    for turn in range(6):
        forks, new = [], []
        for _ in range(min(2, len(free_rows))):
            a = rng.randrange(2)
            shared = rng.choice((len(prompts[a]), rng.randint(0, len(prompts[a]))))
            ids = prompts[a][:shared] + [rng.randrange(VOCAB) for _ in range(rng.randint(1, 18))]
            row = free_rows.pop()
            forks.append((a, row, shared, len(ids) + 8))
            new.append([row, ids, len(ids) - shared, 8])
        if forks:
            src, dst = fs.fs_pages_fork(pool, *(i32(list(x)) for x in zip(*forks)), err=err, check=False)
            fs.fs_pages_copy(every, src, dst, err=err, check=False)
        for c in running:
            c[1].append(rng.randrange(VOCAB))
            c[2] = 1
        running += new
        engine_step([(r, ids, n) for r, ids, n, _ in running])
        for c in running:
            c[3] -= 1
        ended = [c for c in running if c[3] == 0 or rng.random() < 0.25]
        running = [c for c in running if c not in ended]
        if ended:
            fs.fs_pages_free(pool, i32([c[0] for c in ended]), err=err, check=False)
            free_rows += [c[0] for c in ended]
        if turn % 2:
            src, dst, count = fs.fs_pages_compact(pool, err=err, check=False)
            fs.fs_pages_copy(every, src, dst, count, err=err, check=False)
    assert int(err) == 0
