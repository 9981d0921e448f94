"""Attention over both caches where its work is split in ways that small calls do not reach: more
than 256 requests times key/value heads (few rows whole where the card is full without splits)."""
import pytest
import torch

import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_engine import BF, HF, gen, make_cache, normal, on_gpu, step_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("n,most", [(64, 1000), (40, 1024), (33, 513)])
def test_sinks_that_do_not_count_change_no_bit_of_many_requests(n, most, dtype, D):
    """No window, or one beyond every length, over more than 256 request and head pairs whose
    longest are split: bit by bit fs_paged_attention without sinks."""
    say("sinks that do not count", n, most, dtype, D)
    g = gen(n + most)
    kv = [most, 0, 1, most - 1] + [int(x) for x in torch.randint(0, most + 1, (n - 4,), generator=g)]
    k, v, table = make_cache(g, kv, 8, D, 16, dtype)
    q = normal(g, n, 16, D, dtype=dtype).cuda()
    step, cache = step_of([1] * n, kv), on_gpu(k, v, table)
    plain, lse = fs.fs_paged_attention(step, cache, q, D ** -0.5, want_lse=True)
    for window, sinks in ((0, 4), (0, 2 ** 31 - 1), (most, 1), (2 ** 31 - 1, 7)):
        o, l = fs.fs_paged_attention(step, cache, q, D ** -0.5, window, want_lse=True, sinks=sinks)
        assert torch.equal(o, plain) and torch.equal(l, lse), (window, sinks)
