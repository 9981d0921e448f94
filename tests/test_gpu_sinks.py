"""Attention with a window whose first tokens stay visible, over the 16-bit cache, against the
oracle in cache_ref.py: few rows and chunks, whole and split, sinks beside, across and beyond
the window, pages of every size, values that are not finite."""
import math

import pytest
import torch

import cache_ref as cref
import engine_ref as ref
import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_engine import BF, HF, gen, make_cache, normal, offsets, on_gpu, step_of, within

pytestmark = pytest.mark.gpu

CASES = [
    # rows, cached lengths, heads, kv heads, dim, page, window, sinks
    ([1], [1], 1, 1, 64, 16, 5, 4),
    ([1, 1, 1], [40, 16, 333], 8, 2, 128, 16, 20, 4),
    ([1] * 5, [0, 1, 64, 65, 1000], 32, 8, 128, 16, 64, 17),
    ([1, 1], [5000, 70], 7, 1, 128, 32, 1500, 100),
    ([1, 1, 1], [700, 3, 129], 16, 16, 64, 8, 1, 1),
    ([1], [40001], 8, 1, 64, 64, 30000, 5000),            # split, sinks of several pages
    ([1, 1], [3000, 1500], 2, 1, 64, 1, 700, 600),        # more pages than are listed at once
    ([1, 1], [3000, 1500], 2, 1, 128, 1, 900, 511),
    ([1], [5000], 2, 1, 128, 1, 900, 1300),
    ([3, 0, 1, 20], [30, 9, 50, 60], 6, 2, 64, 16, 7, 3),
    ([40, 130], [40, 400], 8, 2, 128, 16, 33, 5),
    ([65, 2, 1], [1000, 2, 600], 3, 3, 128, 4, 7, 64),
    ([200], [900], 8, 8, 64, 16, 100, 33),
    ([70, 5, 9], [64, 2, 9], 4, 1, 128, 1, 3, 2),         # padding rows ahead
    ([17, 33], [517, 33], 14, 2, 64, 128, 50, 65),
    ([5, 1, 2], [3000, 3000, 2500], 12, 4, 128, 16, 1000, 30),
    ([257], [1771], 5, 1, 128, 16, 1200, 150),            # a chunk over split keys
    ([261, 0, 77], [500, 9, 333], 64, 16, 128, 16, 150, 400),
    ([100, 1, 1], [3000, 2000, 50], 4, 2, 64, 16, 2500, 1),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,H,HK,D,page,window,sinks", CASES)
def test_sinks(lens, kv, H, HK, D, page, window, sinks, dtype):
    say("sinks", lens[:6], kv[:6], H, HK, D, page, window, sinks, dtype)
    g = gen(H * 1000 + D + len(lens))
    q_off = offsets(lens)
    T = q_off[-1]
    k, v, table = make_cache(g, kv, HK, D, page, dtype, token_major=page == 16)
    wide = normal(g, T, H + 2, D, dtype=dtype, std=2.0)
    q, scale = wide[:, 1:1 + H], 1.3 * D ** -0.5
    want, tol, lse, ltol = cref.attention(q, k, v, table, q_off, kv, scale, window, sinks)
    out = torch.full((T, H + 1, D), 9.0, dtype=dtype, device="cuda")
    step, cache, qd = step_of(lens, kv), on_gpu(k, v, table), wide.cuda()[:, 1:1 + H]
    o, l = fs.fs_paged_attention(step, cache, qd, scale, window, out=out[:, :H], want_lse=True, sinks=sinks)
    within(o, want, tol, "out")
    empty = torch.isinf(lse)
    assert bool((l.cpu()[empty] == -math.inf).all())
    within(l.cpu()[~empty], lse[~empty], ltol[~empty], "lse")
    assert bool((out[:, H:] == 9).all())
    assert torch.equal(fs.fs_paged_attention(step, cache, qd, scale, window, sinks=sinks), o)


@pytest.mark.parametrize("lens,kv", [([1, 1], [3000, 0]), ([90, 70, 3], [200, 140, 3])])
def test_sinks_that_change_nothing(lens, kv):
    """None, no window, and a window beyond every length: bit by bit as without sinks."""
    g = gen(17)
    k, v, table = make_cache(g, kv, 2, 64, 16, HF)
    q = normal(g, sum(lens), 6, 64, dtype=HF).cuda()
    step, cache = step_of(lens, kv), on_gpu(k, v, table)
    plain = fs.fs_paged_attention(step, cache, q, 0.2)
    for window, sinks in ((0, 5), (0, 2 ** 31 - 1), (2 ** 31 - 1, 7), (max(kv), 4), (1 << 40, 1 << 40)):
        assert torch.equal(fs.fs_paged_attention(step, cache, q, 0.2, window=window, sinks=sinks), plain)
    windowed = fs.fs_paged_attention(step, cache, q, 0.2, window=9)
    assert torch.equal(fs.fs_paged_attention(step, cache, q, 0.2, window=9, sinks=0), windowed)
    # sinks beyond every length: all tokens are seen
    want, tol, _, _ = ref.attention(q, k, v, table, offsets(lens), kv, 0.2, 0)
    for sinks in (max(kv), 2 ** 31 - 1):
        within(fs.fs_paged_attention(step, cache, q, 0.2, window=9, sinks=sinks), want, tol, "out")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,H,HK,D", [([3, 2], [300, 90], 8, 2, 128), ([40, 30], [200, 333], 6, 2, 128),
                                            ([90, 80], [1500, 4000], 3, 1, 64),
                                            ([90, 1, 2], [1500, 3000, 90], 6, 2, 64)])
@pytest.mark.parametrize("where", ["sink", "behind", "newest"])
def test_values_that_are_not_finite_stay_with_the_rows_that_see_them(lens, kv, H, HK, D, dtype, where):
    say("not finite", lens, kv, H, HK, D, dtype, where)
    g = gen(D + H)
    q_off, window, sinks = offsets(lens), 20, 5
    k, v, table = make_cache(g, kv, HK, D, 16, dtype)
    q = normal(g, q_off[-1], H, D, dtype=dtype)
    step, scale = step_of(lens, kv), D ** -0.5
    at = {"sink": 3, "behind": kv[0] - lens[0] - window + 2, "newest": kv[0] - 1}[where]
    assert where != "behind" or sinks <= at < kv[0] - window
    want, tol, lse, ltol = cref.attention(q, k, v, table, q_off, kv, scale, window, sinks)
    bad = v.clone()
    bad[int(table[0, at // 16]), 0, at % 16, 7] = math.nan
    bad[int(table[0, at // 16]), 0, at % 16, 9] = math.inf
    out, l = fs.fs_paged_attention(step, on_gpu(k, bad, table), q.cuda(), scale, window, want_lse=True,
                                   sinks=sinks)
    out = out.cpu()
    within(l, lse, ltol, "lse")
    for s, pos in enumerate(ref.positions(q_off, kv)):
        for i, p in enumerate(pos):
            t = q_off[s] + i
            for h in range(H):
                nan = torch.zeros(D, dtype=torch.bool)
                if s == 0 and h // (H // HK) == 0 and at in cref.seen(p, kv[s], window, sinks):
                    nan[[7, 9]] = True
                assert torch.equal(~torch.isfinite(out[t, h]), nan), (t, h)
                within(out[t, h][~nan], want[t, h][~nan], tol[t, h][~nan], f"out {t} {h}")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 4)])
@pytest.mark.parametrize("n", [3, 40])
def test_a_score_of_inf_keeps_the_rows_sum_inf_while_its_neighbours_sums_grow(n, window, sinks, dtype):
    """lse is inf for a row that sees a score of inf, also when later keys move the references of
    the rows beside it, whose own results stay theirs."""
    kv, D, scale = 400, 64, 0.25
    k = torch.zeros(kv, D)
    k[:, 1] = torch.arange(kv) // 8      # scores that grow by more than any slack
    k[0, 0] = math.inf
    q = torch.zeros(n, 1, D)
    q[:, :, 0], q[:, :, 1] = -1, 8       # (the others' score of the first key is -inf)
    q[0, :, 0], q[0, :, 1] = 1, 0
    kb, vb, table = make_cache(gen(29), [kv], 1, D, 16, dtype)
    for j in range(kv):
        kb[int(table[0, j // 16]), 0, j % 16] = k[j].to(dtype)
    out, lse = fs.fs_paged_attention(step_of([n], [kv]), on_gpu(kb, vb, table), q.to(dtype).cuda(), scale,
                                     window, want_lse=True, sinks=sinks)
    assert float(lse[0, 0]) == math.inf and not bool(torch.isfinite(out[0]).any())
    assert bool(torch.isfinite(out[1:]).all())
    for t in range(1, n):
        pos = kv - n + t
        seen = [j for j in range(1, pos + 1) if window == 0 or j > pos - window or j < sinks]
        want = float(torch.logsumexp(k[seen, 1].double() * 8 * scale, 0))
        # scores are exact; a sum of at most 400 terms is off by 400 * 2^-24 < 3e-5, its
        # exponents (up to 145 = 100 / ln 2) by 145 * 2^-23 < 2e-5, and lse <= 106 itself by
        # 106 * 2^-23 < 2e-5
        assert abs(float(lse[t, 0]) - want) < 1e-4, (t, float(lse[t, 0]), want)


def test_sinks_in_a_graph_with_lengths_that_grow():
    g = gen(23)
    k, v, table = make_cache(g, [1300, 200], 2, 128, 16, BF)
    cache = on_gpu(k, v, table)
    q = normal(g, 2, 8, 128).cuda()
    kv_len = torch.tensor([3, 100], dtype=torch.int32).cuda()
    step, err = fs.Step([0, 1, 2], kv_len=kv_len, max_kv=1300), fs.cleared_err_word()
    need = fs._lib().fs_attention_sinks_workspace(step.ref, cache.ref, 8, 900, 4)
    ws, out = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda"), torch.empty_like(q)

    def call(out, ws):
        fs.fs_paged_attention(step, cache, q, 0.09, 900, out=out, ws=ws, err=err, check=False, sinks=4)

    call(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws)
    for n in (4, 890, 905, 1300):
        kv_len.copy_(torch.tensor([n, min(n, 199)], dtype=torch.int32))
        q.normal_()
        graph.replay()
        torch.cuda.synchronize()
        again = torch.empty_like(out)
        call(again, torch.empty_like(ws))
        assert torch.equal(again, out)
        want, tol, _, _ = cref.attention(q.cpu(), k, v, table, [0, 1, 2], [n, min(n, 199)], 0.09, 900, 4)
        within(out, want, tol, "out")
    assert int(err) == 0
