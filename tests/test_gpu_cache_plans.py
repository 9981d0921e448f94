"""Attention over both caches where its work is split in ways that small calls do not reach: more
than 256 requests times key/value heads (few rows whole where the card is full without splits),
and chunks of so many heads that 256 rows share a tile of keys."""
import math

import pytest
import torch

import cache_ref as cref
import cache_wide_ref as wide
import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_cache4 import both_values, make_cache4, on_gpu4
from test_gpu_engine import BF, HF, gen, make_cache, normal, offsets, on_gpu, step_of, within

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


def check(o, l, q, k, v, table, q_off, kv, scale, window, sinks):
    want, tol, lse, ltol = wide.attention(q, k, v, table, q_off, kv, scale, window, sinks)
    within(o, want, tol, "out")
    empty = torch.isinf(lse)
    assert bool((l.cpu()[empty] == -math.inf).all())
    within(l.cpu()[~empty], lse[~empty], ltol[~empty], "lse")


# ----------------------------------------------------------------- few rows of many requests

def ragged(g, n, most):
    edges = [most, 0, 1, most - 1, 511, 512, 513, 2]
    return edges + [int(x) for x in torch.randint(0, most + 1, (n - len(edges),), generator=g)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sinks,split", [(122, False), (123, False), (124, True)])
def test_windows_with_sinks_of_many_requests_whole_and_split(sinks, split, D, dtype):
    """40 requests of 8 key/value heads: 1,023 and 1,024 keys whole, 1,025 in splits."""
    say("sinks of many requests", sinks, D, dtype)
    g, n, window = gen(sinks + D), 40, 900
    kv = ragged(g, n, 1500)
    k, v, table = make_cache(g, kv, 8, D, 16, dtype)
    q, scale = normal(g, n, 16, D, dtype=dtype, std=2.0), D ** -0.5
    step, cache = step_of([1] * n, kv), on_gpu(k, v, table)
    assert (fs._lib().fs_attention_sinks_workspace(step.ref, cache.ref, 16, window, sinks) > 0) == split
    o, l = fs.fs_paged_attention(step, cache, q.cuda(), scale, window, want_lse=True, sinks=sinks)
    check(o, l, q, k, v, table, offsets([1] * n), kv, scale, window, sinks)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,most,window,sinks,split", [
    (40, 1663, 0, 0, False), (40, 1664, 0, 0, False), (40, 1665, 0, 0, True),
    (40, 1800, 1500, 163, False), (40, 1800, 1500, 164, True),
    (64, 2048, 0, 0, False), (64, 2049, 0, 0, True), (33, 1552, 0, 0, False), (33, 1553, 0, 0, True)])
def test_cache4_of_many_requests_whole_and_split(n, most, window, sinks, split, D, dtype):
    """Up to 1,024 keys and two for each request and head, 2,048 at most, whole."""
    say("4 bits of many requests", n, most, window, sinks, D, dtype)
    g = gen(most + D + n)
    kv = ragged(g, n, most)
    c = make_cache4(g, kv, 8, D, 16, dtype)
    k, v = both_values(c, dtype)
    q, scale = normal(g, n, 16, D, dtype=dtype, std=2.0), 0.7 * D ** -0.5
    step, cache = step_of([1] * n, kv), on_gpu4(*c)
    assert (fs._lib().fs_attention4_workspace(step.ref, cache.ref, 16, window, sinks) > 0) == split
    o, l = fs.fs_paged_attention4(step, cache, q.cuda(), scale, window, sinks, want_lse=True)
    check(o, l, q, k, v, c[4], offsets([1] * n), kv, scale, window, sinks)


# ----------------------------------------------------------------- chunks of 256 rows a work-group

def of_256_rows(lens, H, HK):
    """Chunks take 256 rows a work-group where no request has few rows and that still makes one
    for every compute unit."""
    G = H // HK
    return all(n == 0 or n * G > 64 for n in lens) and (sum(lens) * G // 256 + len(lens)) * HK >= 256


CHUNKS = [
    # rows, cached lengths, heads, kv heads: three tiles and padding ahead, two splits, shared heads
    ([300, 257, 70], [300, 700, 64], 64, 64),
    ([300], [1500], 128, 128),
    ([261, 0, 77], [500, 9, 333], 256, 64),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 9)])
@pytest.mark.parametrize("lens,kv,H,HK", CHUNKS)
def test_cache4_chunks_of_256_rows(lens, kv, H, HK, window, sinks, dtype):
    say("4 bits, 256 rows", lens, kv, H, HK, window, sinks, dtype)
    assert of_256_rows(lens, H, HK)
    g, q_off = gen(H + window), offsets(lens)
    c = make_cache4(g, kv, HK, 128, 16, dtype)
    k, v = both_values(c, dtype)
    q, scale = normal(g, q_off[-1], H, 128, dtype=dtype, std=2.0), -0.06
    o, l = fs.fs_paged_attention4(step_of(lens, kv), on_gpu4(*c), q.cuda(), scale, window, sinks, want_lse=True)
    check(o, l, q, k, v, c[4], q_off, kv, scale, window, sinks)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,H,HK,window,sinks", [(*c, w, s) for c in CHUNKS for w, s in ((150, 9), (20, 400))] +
                         [([300], [2500], 128, 128, 2000, 30)])
def test_chunks_of_256_rows_with_sinks(lens, kv, H, HK, window, sinks, dtype):
    say("sinks, 256 rows", lens, kv, H, HK, window, sinks, dtype)
    assert of_256_rows(lens, H, HK)
    g, q_off = gen(H + window), offsets(lens)
    k, v, table = make_cache(g, kv, HK, 128, 16, dtype)
    q, scale = normal(g, q_off[-1], H, 128, dtype=dtype, std=2.0), 0.09
    o, l = fs.fs_paged_attention(step_of(lens, kv), on_gpu(k, v, table), q.cuda(), scale, window,
                                 want_lse=True, sinks=sinks)
    check(o, l, q, k, v, table, q_off, kv, scale, window, sinks)


@pytest.mark.parametrize("large", [1.0, 256.0, 2.0 ** 100])
def test_queries_of_256_rows_keep_what_lies_far_below_their_largest_value(large):
    """The largest value of each group meets keys of 0, so the scores are the others'."""
    g, lens, kv, HK = gen(128), [80], [150], 256
    assert of_256_rows(lens, HK, HK)
    c = make_cache4(g, kv, HK, 128, 16, BF)
    c[0][..., ::16] &= 0xf0             # value 0 of each group of 32 is a zero
    q = normal(g, 80, HK, 128, dtype=BF) * torch.exp2(-(torch.arange(128) % 23).float()).to(BF)
    q[..., ::32] = large
    k, v = both_values(c, BF)
    # (|q| |k| has the zeros' terms as zeros too)
    _, _, lse, ltol = wide.attention(q, k, v, c[4], [0, 80], kv, 1.0, 0, 0)
    _, l = fs.fs_paged_attention4(step_of(lens, kv), on_gpu4(*c), q.cuda(), 1.0, want_lse=True)
    within(l, lse, ltol, "lse")


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,H,HK", CHUNKS)
def test_broken_groups_of_chunks_of_256_rows(lens, kv, H, HK, dtype, window, sinks):
    """A key's group that counts as NaN, a value's, and a query that is NaN reach the rows that see
    them, or its own; all others are bit by bit as without them."""
    say("broken, 256 rows", lens, kv, H, HK, dtype, window, sinks)
    assert of_256_rows(lens, H, HK)
    g, q_off, grp = gen(H), offsets(lens), H // HK
    c = list(make_cache4(g, kv, HK, 128, 16, dtype))
    q = normal(g, q_off[-1], H, 128, dtype=dtype)
    step, scale = step_of(lens, kv), 0.09
    plain, lplain = fs.fs_paged_attention4(step, on_gpu4(*c), q.cuda(), scale, window, sinks, want_lse=True)
    assert bool(torch.isfinite(plain).all())
    last = len(lens) - 1
    bad_k = [(last, kv[last] - 30, HK - 1, 1), (0, 2, 3, 0)]
    bad_v = [(0, kv[0] - 40, 0, 3), (0, 100, HK - 2, 1)]
    c[2], c[3] = c[2].clone(), c[3].clone()
    for (s, j, m, grpno), x in [(b, c[3]) for b in bad_v] + [(b, c[2]) for b in bad_k]:
        x[int(c[4][s, j // 16]), m, j % 16, grpno] = cref.TOP[dtype] + 1
    t_nan, h_nan = 40, H - 1
    q[t_nan, h_nan, 77] = math.nan
    out, lse = fs.fs_paged_attention4(step, on_gpu4(*c), q.cuda(), scale, window, sinks, want_lse=True)
    # what is NaN: whole rows by a key, columns by a value
    nan = torch.zeros(q_off[-1], H, 128, dtype=torch.bool)
    lnan = torch.zeros(q_off[-1], H, dtype=torch.bool)
    for s, j, m, grpno, value in [(*b, True) for b in bad_v] + [(*b, False) for b in bad_k]:
        p = kv[s] - lens[s] + torch.arange(lens[s])
        see = (j <= p) & ((j > p - window) | (j < sinks) if window else torch.ones_like(p, dtype=torch.bool))
        rows = q_off[s] + see.nonzero()[:, 0]
        for h in range(m * grp, (m + 1) * grp):
            if value:
                nan[rows, h, 32 * grpno:32 * grpno + 32] = True
            else:
                nan[rows, h], lnan[rows, h] = True, True
    nan[t_nan, h_nan], lnan[t_nan, h_nan] = True, True
    out, lse, plain, lplain = out.cpu(), lse.cpu(), plain.cpu(), lplain.cpu()
    assert torch.equal(out.isnan(), nan) and torch.equal(lse.isnan(), lnan)
    assert torch.equal(out[~nan], plain[~nan]) and torch.equal(lse[~lnan], lplain[~lnan])


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("at", ["sink", "behind", "newest"])
def test_values_that_are_not_finite_under_chunks_of_256_rows_with_sinks(at, dtype):
    say("not finite, 256 rows", at, dtype)
    lens, kv, H, window, sinks = [300, 257, 70], [300, 700, 90], 64, 20, 5
    assert of_256_rows(lens, H, H)
    g, q_off = gen(9), offsets(lens)
    k, v, table = make_cache(g, kv, H, 128, 16, dtype)
    q, scale = normal(g, q_off[-1], H, 128, dtype=dtype), 0.09
    j = {"sink": 3, "behind": kv[1] - lens[1] - window + 2, "newest": kv[1] - 1}[at]
    bad = v.clone()
    bad[int(table[1, j // 16]), 5, j % 16, 7] = math.nan
    bad[int(table[1, j // 16]), 5, j % 16, 90] = -math.inf
    o, l = fs.fs_paged_attention(step_of(lens, kv), on_gpu(k, bad, table), q.cuda(), scale, window,
                                 want_lse=True, sinks=sinks)
    want, tol, lse, ltol = wide.attention(q, k, v, table, q_off, kv, scale, window, sinks)
    p = kv[1] - lens[1] + torch.arange(lens[1])
    see = (j <= p) & ((j > p - window) | (j < sinks))
    nan = torch.zeros(q_off[-1], H, 128, dtype=torch.bool)
    rows = q_off[1] + see.nonzero()[:, 0]
    nan[rows, 5, 7] = nan[rows, 5, 90] = True
    o = o.cpu()
    assert torch.equal(~torch.isfinite(o), nan)
    within(o[~nan], want[~nan], tol[~nan], "out")
    within(l, lse, ltol, "lse")
