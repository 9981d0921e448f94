"""Attention of chunks whose keys are split over work-groups, against the 64-bit oracle: the
join finds each row's own request, whatever else its wave holds.  What the call has to write
(out, lse, its partial results) is filled with NaN before, so that a value that nobody wrote
shows."""
import math

import pytest
import torch

import engine_ref as ref
import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_engine import BF, HF, gen, make_cache, normal, offsets, on_gpu, step_of, within

pytestmark = pytest.mark.gpu

SPLIT = [
    # rows, cached lengths, heads, kv heads, dim, window
    ([101, 99], [9000, 3000], 14, 2, 64, 0),
    ([1, 300], [50, 5000], 14, 2, 64, 0),                        # a single token before a chunk
    ([1] * 40 + [201], list(range(3, 43)) + [6000], 7, 1, 128, 0),  # more requests than lanes of a row
    ([33, 40], [3000, 500], 14, 2, 64, 0),                       # a long context before a short one
    ([33, 40], [500, 3000], 14, 2, 64, 0),                       # and after it
    ([65, 65], [2500, 1100], 1, 1, 128, 0),
    ([65, 65], [1100, 2500], 7, 7, 128, 0),
    ([101] * 40, [150 + 71 * i for i in range(40)], 1, 1, 64, 0),
    ([101] * 40, [150 + 71 * i for i in range(40)], 1, 1, 128, 0),
    ([130, 0, 77, 1], [4000, 9, 2000, 1900], 3, 1, 128, 1500),   # windows of more than a split
    ([300, 1, 2], [2600, 2600, 2], 2, 2, 64, 0),                 # the last wave is not full
    ([70, 90], [60, 2100], 5, 5, 64, 0),                         # padding rows ahead
    ([96, 200], [1500, 2048], 8, 2, 128, 0),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,H,HK,D,window", SPLIT)
def test_split_chunks_are_joined_for_their_own_request(lens, kv, H, HK, D, window, dtype):
    say("split chunks", lens[-3:], kv[-3:], H, HK, D, window, dtype)
    g = gen(H * 1000 + D + len(lens))
    q_off = offsets(lens)
    T = q_off[-1]
    k, v, table = make_cache(g, kv, HK, D, 16, dtype)
    q = normal(g, T, H, D, dtype=dtype, std=1.5)
    scale = D ** -0.5
    want, tol, lse, ltol = ref.attention(q, k, v, table, q_off, kv, scale, window)
    step, cache = step_of(lens, kv), on_gpu(k, v, table)
    need = fs._lib().fs_attention_workspace(step.ref, cache.ref, H, window)
    assert need > 0
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")       # NaN, as floats
    out = torch.full((T, H, D), math.nan, dtype=dtype, device="cuda")
    got = torch.full((T, H), math.nan, device="cuda")
    fs.fs_paged_attention(step, cache, q.cuda(), scale, window, out=out, lse=got, ws=ws)
    within(out, want, tol, "out")
    empty = torch.isinf(lse)
    assert bool((got.cpu()[empty] == -math.inf).all())
    within(got.cpu()[~empty], lse[~empty], ltol[~empty], "lse")
