"""The pages of a cache against a pool in Python lists (cache_ref.Pool): rows let go, forks,
compaction, copies in caches of either kind and any strides, what is refused, graphs."""
import random

import numpy as np
import pytest
import torch

import cache_ref as cref
import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_engine import BF, HF, gen, normal

pytestmark = pytest.mark.gpu
E = fs.FairServeError


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def on_gpu(pool, pad=2):
    """A PagePool with the state of a cache_ref.Pool (the table's rows `pad` further apart)."""
    table = torch.full((len(pool.table), pool.width + pad), -7, dtype=torch.int32)
    table[:, :pool.width] = torch.tensor(pool.table, dtype=torch.int32)
    return fs.PagePool(i32(pool.refs), table.cuda()[:, :pool.width], i32(pool.held), pool.page)


def same(p, pool):
    assert p.refs.tolist() == pool.refs
    assert p.held.tolist() == pool.held
    assert p.table.tolist() == pool.table             # entries beyond held included


def random_pool(rng, n_pages, page, rows, width, use):
    """Rows that hold pages of their own, scattered, and share some prefixes."""
    pool = cref.Pool(n_pages, page, rows, width)
    ids = list(range(n_pages))
    rng.shuffle(ids)
    ids = ids[:int(use * n_pages)]
    pool.table = [[rng.randrange(n_pages) for _ in range(width)] for _ in range(rows)]
    for r in range(rows):
        n = min(rng.randint(0, width), len(ids))
        mine = [ids.pop() for _ in range(n)]
        if r and rng.random() < 0.4:
            other = rng.randrange(r)
            k = rng.randint(0, pool.held[other])
            mine = (pool.table[other][:k] + mine)[:width]
        pool.table[r][:len(mine)] = mine
        pool.held[r] = len(mine)
        for p in mine:
            pool.refs[p] += 1
    return pool


POOLS = [
    # pages, page size, rows, width, share in use
    (1, 16, 1, 1, 1.0),
    (7, 1, 3, 4, 0.5),
    (100, 16, 9, 13, 0.4),
    (2048, 8, 40, 30, 0.5),
    (2049, 4096, 65, 31, 0.3),
    (5000, 32, 300, 20, 0.6),
    (70001, 16, 50, 1300, 0.4),
    (3000, 8, 9000, 2, 0.5),                  # more rows than claims fit beside each other
    (2000, 8, 31, 1100, 0.9),                 # few pages and rows, wide ones
]


@pytest.mark.parametrize("n_pages,page,rows,width,use", POOLS)
def test_steps_of_a_pool(n_pages, page, rows, width, use):
    """Rows let go, forks (shared prefixes, whole and begun pages, no parent, no room) and
    compaction in turn, as the pool in lists."""
    say("pool", n_pages, page, rows, width, use)
    rng = random.Random(n_pages)
    pool = random_pool(rng, n_pages, page, rows, width, use)
    p = on_gpu(pool)
    for turn in range(4):
        gone = [r for r in range(rows) if rng.random() < 0.3]
        # a row named twice is let go once
        fs.fs_pages_free(p, i32(gone + gone[:1]) if gone else i32([]))
        pool.free(gone)
        same(p, pool)
        empty = [r for r in range(rows) if pool.held[r] == 0]
        rng.shuffle(empty)
        left = sum(n == 0 for n in pool.refs)
        forks = []
        for c in empty[:rng.randint(0, len(empty))]:
            par = rng.choice([-1] + [r for r in range(rows) if pool.held[r]])
            sh = rng.randint(0, pool.held[par] * page) if par >= 0 else 0
            if rng.random() < 0.3:
                sh -= sh % page
            room = rng.randint(sh, width * page)
            new = -(-room // page) - sh // page
            if new <= left:
                left -= new
                forks.append((par, c, sh, room))
        par, c, sh, room = ([f[i] for f in forks] for i in range(4))
        src, dst = fs.fs_pages_fork(p, i32(par), i32(c), i32(sh), i32(room))
        want = pool.fork(par, c, sh, room)
        assert (src.tolist(), dst.tolist()) == want
        same(p, pool)
        if turn % 2:
            src, dst, count = fs.fs_pages_compact(p)
            s, d = pool.compact()
            n = int(count)
            assert n == len(s) and src[:n].tolist() == s and dst[:n].tolist() == d
            assert bool((src[n:] == -1).all()) and bool((dst[n:] == -1).all())
            same(p, pool)


def test_compaction_into_other_arrays():
    rng = random.Random(3)
    pool = random_pool(rng, 3000, 16, 30, 40, 0.4)
    p = on_gpu(pool)
    refs, table = torch.full_like(p.refs, 99), torch.full((30, 50), 77, dtype=torch.int32).cuda()[:, :40]
    before = p.refs.clone(), p.table.clone()
    src, dst, count = fs.fs_pages_compact(p, refs_out=refs, table_out=table)
    assert torch.equal(before[0], p.refs) and torch.equal(before[1], p.table)
    s, d = pool.compact()
    assert src[:int(count)].tolist() == s and dst[:int(count)].tolist() == d
    assert refs.tolist() == pool.refs
    for r in range(30):
        n = pool.held[r]
        assert table[r, :n].tolist() == pool.table[r][:n] and bool((table[r, n:] == 77).all())


def test_a_page_kept_by_the_caller_moves_and_stays():
    pool = cref.Pool(10, 4, 2, 3)
    pool.refs[8] = 1                              # of no row
    pool.table[1][:2], pool.held[1] = [9, 1], 2
    pool.refs[9] = pool.refs[1] = 1
    p = on_gpu(pool)
    src, dst, count = fs.fs_pages_compact(p)
    assert int(count) == 2 and src[:2].tolist() == [8, 9] and dst[:2].tolist() == [0, 2]
    pool.compact()
    same(p, pool)
    fs.fs_pages_free(p, i32([1]))
    assert p.refs.tolist() == [1] + [0] * 9


def test_unsound_forks_get_nothing_and_the_others_theirs():
    pool = cref.Pool(40, 8, 8, 5)
    pool.fork([-1, -1], [0, 1], [0, 0], [40, 20])
    p = on_gpu(pool)
    bad = [(-2, 2, 0, 8), (8, 2, 0, 8), (0, 8, 0, 8), (0, -1, 0, 8), (0, 1, 0, 8),   # rows, a child that holds
           (0, 2, -1, 8), (0, 2, 9, 8), (0, 2, 0, 41), (1, 2, 25, 30), (-1, 2, 1, 8),  # lengths
           (3, 2, 1, 8), (0, 2, 0, 2 ** 31 - 1)]                                     # a parent without pages
    good = [(0, 3, 17, 30), (1, 4, 16, 16), (-1, 5, 0, 0), (-1, 6, 0, 9)]
    forks = [good[0]] + bad[:6] + [good[1]] + bad[6:] + good[2:] + [(0, 3, 8, 8)]      # row 3 again
    par, c, sh, room = ([f[i] for f in forks] for i in range(4))
    err = fs.cleared_err_word()
    src, dst = fs.fs_pages_fork(p, i32(par), i32(c), i32(sh), i32(room), err=err, check=False)
    assert int(err) == fs.FS_E_RANGE
    s, d = pool.fork(*([f[i] for f in good] for i in range(4)))
    same(p, pool)
    mine = [i for i, f in enumerate(forks) if f in good]
    assert [src[i].item() for i in mine] == s and [dst[i].item() for i in mine] == d
    rest = [i for i in range(len(forks)) if i not in mine]
    assert all(src[i].item() == dst[i].item() == -1 for i in rest)


def test_too_few_free_pages_give_nothing():
    pool = cref.Pool(20, 4, 6, 20)
    pool.fork([-1], [0], [0], [30])
    p = on_gpu(pool)
    for n in (13, 20):
        with pytest.raises(E) as e:
            fs.fs_pages_fork(p, i32([-1, 0]), i32([1, 2]), i32([0, 6]), i32([4 * n - 28, 30]))
        assert e.value.code == fs.FS_E_OVERFLOW
        same(p, pool)
    src, dst = fs.fs_pages_fork(p, i32([-1, 0]), i32([1, 2]), i32([0, 6]), i32([20, 30]))
    assert pool.fork([-1, 0], [1, 2], [0, 6], [20, 30]) == (src.tolist(), dst.tolist())
    same(p, pool)
    # many forks whose needs pass 32 bits together
    wide = fs.PagePool(i32([0] * 8), torch.zeros(300, 1 << 16, dtype=torch.int32).cuda(), i32([0] * 300), 4096)
    n = 300
    with pytest.raises(E) as e:
        fs.fs_pages_fork(wide, i32([-1] * n), i32(list(range(n))), i32([0] * n), i32([1 << 28] * n))
    assert e.value.code == fs.FS_E_OVERFLOW and int(wide.refs.sum()) == 0 and int(wide.held.sum()) == 0


def test_bad_ids_among_the_held_are_errors_not_addresses():
    def fresh():
        pool = cref.Pool(30, 4, 4, 6)
        pool.fork([-1, -1], [0, 1], [0, 0], [20, 8])
        pool.table[0][2] = 30
        pool.table[1][1] = -1
        return on_gpu(pool)
    p = fresh()
    with pytest.raises(E) as e:
        fs.fs_pages_free(p, i32([0, 1]))
    assert e.value.code == fs.FS_E_RANGE and int(p.held.sum()) == 0
    p = fresh()
    with pytest.raises(E) as e:
        fs.fs_pages_fork(p, i32([0]), i32([2]), i32([12]), i32([12]))
    assert e.value.code == fs.FS_E_RANGE and p.held.tolist() == [5, 2, 0, 0]
    p = fresh()
    with pytest.raises(E) as e:
        fs.fs_pages_compact(p)
    assert e.value.code == fs.FS_E_RANGE
    for rows in ([4], [-1], [1 << 30]):
        with pytest.raises(E) as e:
            fs.fs_pages_free(fresh(), i32(rows))
        assert e.value.code == fs.FS_E_RANGE
    for held in ([7, 0, 0, 0], [-1, 0, 0, 0]):
        p = fresh()
        p.held.copy_(i32(held))
        with pytest.raises(E) as e:
            fs.fs_pages_free(p, i32([0]))
        assert e.value.code == fs.FS_E_RANGE
        p.held.copy_(i32(held))
        with pytest.raises(E) as e:
            fs.fs_pages_compact(p)
        assert e.value.code == fs.FS_E_RANGE
    # a free page that is held: its count stays 0
    p = fresh()
    p.refs[p.table[0, 0].item()] = 0
    with pytest.raises(E) as e:
        fs.fs_pages_free(p, i32([0]))
    assert e.value.code == fs.FS_E_RANGE and int(p.refs.min()) == 0


# ----------------------------------------------------------------- copies

def caches(g, kind, n_pages, HK, page, D, layers, layout):
    """(CacheLayers, its tensors) with strides of the layout's kind."""
    def make(per, dtype):
        shape = {"heads": (n_pages, HK, page, per), "tokens": (n_pages, page, HK, per),
                 "padded": (n_pages, HK, page + 1, per + 16),
                 "joint": (n_pages, HK, page, 2, per)}[layout]
        x = torch.randint(0, 256, shape, generator=g, dtype=torch.uint8)
        x = (x if dtype == torch.uint8 else x.to(dtype)).cuda()
        return {"heads": lambda: x, "tokens": lambda: x.permute(0, 2, 1, 3),
                "padded": lambda: x[:, :, :page, :per], "joint": lambda: x.select(3, 1)}[layout]()
    table = torch.zeros(1, 1, dtype=torch.int32).cuda()
    out, all_t = [], []
    for _ in range(layers):
        if kind == 4:
            t = [make(D // 2, torch.uint8), make(D // 2, torch.uint8), make(D // 32, torch.uint8),
                 make(D // 32, torch.uint8)]
            out.append(fs.KVCache4(*t, table))
        else:
            t = [make(D, kind), make(D, kind)]
            out.append(fs.KVCache(*t, table))
        all_t += t
    return fs.CacheLayers(out), all_t


@pytest.mark.parametrize("layout", ["heads", "tokens", "padded", "joint"])
@pytest.mark.parametrize("kind,HK,page,D,layers", [
    (BF, 2, 16, 128, 1), (HF, 1, 1, 64, 3), (BF, 3, 64, 256, 2), (BF, 1, 2, 8, 50), (4, 2, 16, 128, 1),
    (4, 1, 1, 32, 2), (4, 3, 32, 96, 49), (4, 1, 4, 64, 97)])
def test_copies_of_pages(kind, HK, page, D, layers, layout):
    say("copy", kind, HK, page, D, layers, layout)
    g = gen(layers + D)
    n_pages = 23
    L, tensors = caches(g, kind, n_pages, HK, page, D, layers, layout)
    src, dst = [3, -1, 0, 22, 3, 7], [5, -1, 1, 2, 21, 20]
    want = []
    for t in tensors:
        w = t.clone()
        for a, b in zip(src, dst):
            if a >= 0:
                w[b] = t[a]
        want.append(w)
    fs.fs_pages_copy(L, i32(src), i32(dst))
    for t, w in zip(tensors, want):
        assert torch.equal(t, w)
    # a count on the device; more than there are is all
    for count in (0, 2, 100, -3):
        s2, d2 = i32([4, 9, 10]), i32([11, 12, 13])
        fs.fs_pages_copy(L, s2, d2, i32([count]))
        for t, w in zip(tensors, want):
            for a, b in list(zip((4, 9, 10), (11, 12, 13)))[:max(0, min(count, 3))]:
                w[b] = w[a]
            assert torch.equal(t, w)


def test_copies_refuse_bad_pages():
    g = gen(1)
    for kind in (BF, 4):
        L, tensors = caches(g, kind, 8, 1, 4, 64, 2, "heads")
        before = [t.clone() for t in tensors]
        for a, b in ((8, 1), (1, 8), (-2, 1), (1, -1), (-1, 1), (1 << 30, 1 << 30)):
            with pytest.raises(E) as e:
                fs.fs_pages_copy(L, i32([a]), i32([b]))
            assert e.value.code == fs.FS_E_RANGE
        for t, w in zip(tensors, before):
            assert torch.equal(t, w)


def test_copies_beyond_32_bits():
    big = torch.empty(3 * 1_300_000_000 + 4096, dtype=BF, device="cuda")
    k = big.as_strided((4, 1, 16, 64), (1_300_000_000, 1024, 64, 1))
    k.copy_(normal(gen(2), 4, 1, 16, 64).cuda())
    cache = fs.KVCache(k, k, torch.zeros(1, 1, dtype=torch.int32).cuda())
    last = k[3].clone()
    fs.fs_pages_copy(cache, i32([3]), i32([1]))
    assert torch.equal(k[1], last) and torch.equal(k[3], last)


def test_pages_in_a_graph():
    """A step's pages (calls that end, calls that begin, the begun pages' copies, compaction)
    captured once and replayed while the device data change."""
    rng = random.Random(9)
    pool = random_pool(rng, 400, 8, 20, 12, 0.5)
    p = on_gpu(pool)
    L, tensors = caches(gen(5), BF, 400, 2, 8, 64, 2, "heads")
    mirror = [t.cpu().clone() for t in tensors]
    err = fs.cleared_err_word()
    gone, par, child, sh, room = i32([0, 0]), i32([0, 0]), i32([0, 0]), i32([0, 0]), i32([0, 0])
    src, dst = torch.empty_like(child), torch.empty_like(child)
    csrc, cdst, count = i32([0] * 200), i32([0] * 200), i32([0])
    need = fs._lib().fs_pages_workspace(p.ref, 2)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step():
        fs.fs_pages_free(p, gone, err=err, check=False)
        fs.fs_pages_fork(p, par, child, sh, room, src=src, dst=dst, ws=ws, err=err, check=False)
        fs.fs_pages_copy(L, src, dst, err=err, check=False)
        fs.fs_pages_compact(p, src=csrc, dst=cdst, count=count, ws=ws, err=err, check=False)
        fs.fs_pages_copy(L, csrc, cdst, count, err=err, check=False)

    def copy(s, d):
        for t in mirror:
            old = t.clone()
            for a, b in zip(s, d):
                if a >= 0:
                    t[b] = old[a]

    graph = None
    for turn in range(5):
        full = [r for r in range(20) if pool.held[r] > 1]
        g2 = rng.sample(full, 2)
        parents = rng.sample([r for r in full if r not in g2], 2)
        shared = [rng.randint(0, pool.held[r] * 8) for r in parents]
        rooms = [rng.randint(s, 96) for s in shared]
        for t, v in ((gone, g2), (par, parents), (child, g2), (sh, shared), (room, rooms)):
            t.copy_(i32(v))
        if graph is None:                          # (a first eager step)
            step()
            torch.cuda.synchronize()
            if turn == 0:
                saved = [t.clone() for t in (p.refs, p.table, p.held, *tensors)]
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    step()
                for t, s in zip((p.refs, p.table, p.held, *tensors), saved):
                    t.copy_(s)
        else:
            graph.replay()
        torch.cuda.synchronize()
        pool.free(g2)
        copy(*pool.fork(parents, g2, shared, rooms))
        copy(*pool.compact())
        assert int(err) == 0
        same(p, pool)
        used = [q for q, n in enumerate(pool.refs) if n]
        for t, m in zip(tensors, mirror):
            assert torch.equal(t.cpu()[used], m[used])
