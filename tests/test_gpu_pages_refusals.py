"""What the calls of a pool of pages do at their limits, and what they refuse beside what they do
not: rows named more often than a launch has work-groups."""
import pytest
import torch

import cache_ref as cref
import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_pages import on_gpu

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
