"""What the engine step's kernels refuse of device data: the status word is raised and nothing
is read or written through it."""
import pytest
import torch

import paper_2411_15997_amd as fs
from test_gpu_engine import BF, gen, make_cache, normal, offsets, on_gpu

pytestmark = pytest.mark.gpu


def length_step(lens, kv, max_kv):
    return fs.Step(offsets(lens), kv_len=torch.tensor(kv, dtype=torch.int32).cuda(), max_kv=max_kv)


@pytest.mark.parametrize("lens,kv", [([1], [10]), ([3, 2], [4, 1 << 30]), ([2, 1], [-1, 9])])
def test_nothing_is_appended_for_a_length_out_of_range(lens, kv):
    """The other requests' tokens are; the request's own cached ones stay."""
    g = gen(8)
    k, v, table = make_cache(g, [9] * len(lens), 2, 64, 4, BF, garbage=1.0)
    cache = on_gpu(k, v, table)
    before_k, before_v = cache.k.clone(), cache.v.clone()
    T = sum(lens)
    kn, vn = normal(g, T, 2, 64).cuda(), normal(g, T, 2, 64).cuda()
    rope = fs.Rope(torch.ones(32).cuda())
    with pytest.raises(fs.FairServeError) as e:
        fs.fs_rope_append(length_step(lens, kv, 9), cache, rope, None, kn, vn)
    assert e.value.code == fs.FS_E_RANGE
    q_off = offsets(lens)
    for s, n in enumerate(kv):
        mine = table[s][:3].long()
        if not 0 <= n <= 9:
            assert torch.equal(cache.k[mine], before_k[mine]) and torch.equal(cache.v[mine], before_v[mine])
        else:
            for i in range(lens[s]):
                p = n - lens[s] + i
                assert torch.equal(cache.v[int(table[s, p // 4]), :, p % 4], vn[q_off[s] + i])
