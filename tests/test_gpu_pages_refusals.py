"""What the calls of a pool of pages do at their limits, and what they refuse beside what they do
not: rows named more often than a launch has work-groups, a page id out of range or a free page
among the shared pages of some forks, a free page held by a row that is renumbered."""
import pytest
import torch

import cache_ref as cref
import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_pages import i32, on_gpu

pytestmark = pytest.mark.gpu


def alike(p, pool):
    """test_gpu_pages.same for large pools (a difference is not spelled out)."""
    for got, want in ((p.refs, pool.refs), (p.held, pool.held), (p.table, pool.table)):
        want = torch.tensor(want, dtype=torch.int32)
        bad = (got.cpu() != want).nonzero()
        assert bad.numel() == 0, (len(bad), bad[0].tolist())


@pytest.mark.parametrize("n", [65536, (1 << 24) + 5])
def test_rows_are_let_go_once_however_often_they_are_named(n):
    """More names than a launch has work-groups of."""
    say("rows named", n)
    pool = cref.Pool(3000, 4, 1000, 3)
    for r in range(1000):
        pool.table[r], pool.held[r] = [r, 1000 + r, 2999], 3
        for q in pool.table[r]:
            pool.refs[q] += 1
    p = on_gpu(pool)
    rows = torch.arange(n, dtype=torch.int32, device="cuda") % 997
    rows[-1] = 999
    fs.fs_pages_free(p, rows)
    pool.free(list(range(997)) + [999])
    alike(p, pool)


# pages, rows, forks asked for: one work-group that finishes the rows too, one that leaves them
# to others, more forks than it looks at, pools of many pages
SIZES = [(60, 40, 5), (2000, 200, 100), (2048, 1300, 1200), (2049, 40, 5), (9000, 600, 400)]


def a_pool(n_pages, rows, n):
    """A pool of pages of 8 tokens, five a row at most, whose rows 0 and 1 hold four pages each
    and keep no page of id 0; row 0 is sound.  (pool, forks): half of the forks share three and a
    half pages of row 0, the others of row 1, whose third page a caller breaks; as many pages are
    free as the sound half takes."""
    pool = cref.Pool(n_pages, 8, rows, 5)
    pool.fork([-1, -1, -1], [rows - 1, 0, 1], [0, 0, 0], [8, 32, 32])
    forks = [(i % 2, 2 + i, 28, 33) for i in range(n)]       # three shared, two new, one to copy
    want = 2 * ((n + 1) // 2)
    for p in [p for p, r in enumerate(pool.refs) if r == 0][want:]:
        pool.refs[p] = 1                                      # (the caller's)
    assert sum(r == 0 for r in pool.refs) == want
    return pool, forks


def fork_all(p, forks):
    err = fs.cleared_err_word()
    src, dst = fs.fs_pages_fork(p, *(i32(list(x)) for x in zip(*forks)), err=err, check=False)
    return src.tolist(), dst.tolist(), int(err)


@pytest.mark.parametrize("bad", [-1, "n_pages", 1 << 30])
@pytest.mark.parametrize("n_pages,rows,n", SIZES)
def test_a_page_out_of_range_refuses_its_own_forks_alone(n_pages, rows, n, bad):
    """The others get the lowest free pages in the order of their indices, and the pages suffice
    without those that the refused ones would have taken."""
    say("bad shared page", n_pages, rows, n, bad)
    pool, forks = a_pool(n_pages, rows, n)
    pool.table[1][2] = n_pages if bad == "n_pages" else bad
    p = on_gpu(pool)
    src, dst, err = fork_all(p, forks)
    assert err == fs.FS_E_RANGE
    s, d = pool.fork(*zip(*forks[0::2]))
    alike(p, pool)
    assert src[0::2] == s and dst[0::2] == d
    assert set(src[1::2]) == set(dst[1::2]) == {-1}


def test_a_bad_page_behind_the_shared_ones_refuses_nothing():
    pool, forks = a_pool(60, 40, 5)
    pool.table[1][3], forks = 60, [(0, 2, 28, 33), (1, 3, 24, 33)]
    p = on_gpu(pool)
    src, dst, err = fork_all(p, forks)
    assert err == 0 and (src, dst) == pool.fork(*zip(*forks))
    alike(p, pool)


@pytest.mark.parametrize("n_pages,rows,n", SIZES)
def test_a_free_page_among_the_shared_refuses_its_own_forks_alone(n_pages, rows, n):
    """A page that no row is counted for may be given out as a new one: to share it as well would
    make two rows write it."""
    say("free shared page", n_pages, rows, n)
    pool, forks = a_pool(n_pages, rows, n)
    lost = pool.table[1][2]
    pool.refs[lost] = 0                    # (free now, and the lowest)
    p = on_gpu(pool)
    src, dst, err = fork_all(p, forks)
    assert err == fs.FS_E_RANGE
    s, d = pool.fork(*zip(*forks[0::2]))
    alike(p, pool)
    assert src[0::2] == s and dst[0::2] == d and d[0] == lost
    assert set(src[1::2]) == set(dst[1::2]) == {-1}


@pytest.mark.parametrize("other", [False, True])
@pytest.mark.parametrize("n_pages,rows,width", [(40, 3, 6), (2000, 50, 6), (3000, 3, 6), (3000, 9, 1500)])
def test_compaction_refuses_a_held_page_that_is_free(n_pages, rows, width, other):
    """Below L as from there on: FS_E_RANGE, and the entry keeps its id; the other entries and the
    counts are renumbered."""
    say("held but free", n_pages, rows, width, other)
    # row 0 holds the pool's last pages, row 1 its first ones; L = 8
    for low, at in ((True, 2), (False, 2), (True, 0), (False, 3)):
        pool = cref.Pool(n_pages, 4, rows, width)
        pool.table[0][:5] = range(n_pages - 5, n_pages)
        pool.table[1][:4] = range(4)
        pool.held[:2] = [5, 4]
        for q in pool.table[0][:5] + pool.table[1][:4]:
            pool.refs[q] = 1
        row = 1 if low else 0
        lost = pool.table[row][at]
        pool.refs[lost] = 0
        p = on_gpu(pool)
        out = dict(refs_out=torch.full_like(p.refs, 9), table_out=p.table.clone()) if other else {}
        err = fs.cleared_err_word()
        src, dst, count = fs.fs_pages_compact(p, err=err, check=False, **out)
        assert int(err) == fs.FS_E_RANGE, (low, at)
        s, d = pool.compact()
        pool.table[row][at] = lost
        n = int(count)
        assert (src[:n].tolist(), dst[:n].tolist()) == (s, d)
        refs, table = (out["refs_out"], out["table_out"]) if other else (p.refs, p.table)
        assert refs.tolist() == pool.refs and table.tolist() == pool.table, (low, at)
