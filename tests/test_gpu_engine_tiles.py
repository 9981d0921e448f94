"""Every tile and wave count of the adapters' two products against the 64-bit oracle: steps
whose products take tiles of 256 by 256, and first products of more than 512 row tiles."""
import pytest
import torch

import engine_ref as ref
import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_engine import BF, HF, gen, normal, offsets, within

pytestmark = pytest.mark.gpu


def check(lens, K, N, n, R, dtype, seed):
    g = gen(seed)
    q_off = offsets(lens)
    x, w = normal(g, q_off[-1], K, dtype=dtype), normal(g, N, K, dtype=dtype, std=K ** -0.5)
    a, b = normal(g, n, R, K, dtype=dtype, std=K ** -0.5), normal(g, n, N, R, dtype=dtype)
    rank = torch.randint(1, R + 1, (n,), generator=g, dtype=torch.int32)
    for i in range(n):                                     # what lies beyond a rank is not used
        a[i, int(rank[i]):] = float("inf")
        b[i, :, int(rank[i]):] = float("nan")
    scale = torch.rand(n, generator=g) * 3 - 1
    adapter = torch.randint(-1, n, (len(lens),), generator=g, dtype=torch.int32)
    adapter[0] = 0
    want, bound = ref.linear(x, w, a, b, q_off, adapter, rank, scale)
    ad = fs.Adapters(*[t.cuda() for t in (a, b, adapter, rank, scale)])
    y = torch.full((q_off[-1], N), float("nan"), dtype=dtype, device="cuda")
    fs.fs_adapter_linear(fs.Step(q_off), ad, x.cuda(), w.cuda(), y=y)
    within(y, want, bound, "y")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,K,N,n,R", [
    ([2000, 1, 900, 1, 498], 200, 3592, 3, 16),       # one adapter a wave's rows, and several
    ([1] * 300 + [3000], 136, 3600, 5, 40),
    ([3585], 72, 3336, 1, 128),                       # the last tile of one row
])
def test_tiles_of_256_by_256(lens, K, N, n, R, dtype):
    say("tiles of 256", lens[-3:], K, N, n, R, dtype)
    assert ((sum(lens) + 255) // 256) * ((N + 255) // 256) >= 192
    check(lens, K, N, n, R, dtype, 31)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("R", [8, 24, 40, 72, 128])
@pytest.mark.parametrize("lens", [[4000, 17, 1, 4200], [3] * 600])
def test_first_products_of_many_row_tiles(lens, R, dtype):
    """Four waves a work-group, for each count of 16-column tiles of h."""
    say("many row tiles", lens[:3], R, dtype)
    assert sum(lens) // 16 + len(lens) > 512
    check(lens, 264, 72, 4, R, dtype, R)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("R", [8, 24, 72, 128])
@pytest.mark.parametrize("K", [8, 64, 1096])
def test_first_products_of_few_row_tiles(K, R, dtype):
    """The other wave counts, with K shorter than the waves' shares and longer."""
    say("few row tiles", K, R, dtype)
    check([5, 16, 1, 33], K, 72, 3, R, dtype, K + R)
