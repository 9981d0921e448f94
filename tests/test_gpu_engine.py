"""The engine step's operators against the 64-bit oracle in engine_ref.py: types, head
layouts, lengths from one token on, odd and ragged sizes, strides, masks that leave a row
empty, garbage in unused slots, page sizes, offsets beyond 32 bits, streams, graphs."""
import math

import numpy as np
import pytest
import torch

import engine_ref as ref
import paper_2411_15997_amd as fs
from gpu_common import say

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator("cpu").manual_seed(seed)


def normal(g, *shape, dtype=BF, std=1.0):
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def offsets(lens):
    return [0] + list(np.cumsum(lens))


def within(got, want, bound, what):
    got = got.double().cpu()
    want, bound = torch.as_tensor(want), torch.as_tensor(bound)
    bad = ~((got - want).abs() <= bound)
    assert not bool(bad.any()), (
        f"{what}: {int(bad.sum())} of {bad.numel()} outside, first at "
        f"{bad.nonzero()[0].tolist()}: {got[bad][0].item()} for {want[bad][0].item()} "
        f"(bound {bound[bad][0].item():.3g})")


# ----------------------------------------------------------------- adapters

LINEAR = [
    # rows of the requests, K, N, adapters, max rank
    ([1], 64, 64, 1, 8),
    ([1, 1, 1, 1], 520, 136, 3, 16),
    ([3, 0, 1, 17, 5], 1000, 72, 2, 24),
    ([1] * 64, 256, 520, 8, 16),
    ([33, 130, 1, 64, 29], 136, 264, 5, 32),
    ([200, 57], 512, 768, 2, 64),
    ([16, 40], 72, 8, 2, 128),
    ([300], 2056, 384, 1, 8),
    ([1, 2, 255, 130, 0, 127, 1], 320, 1032, 4, 40),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,K,N,n,R", LINEAR)
def test_linear(lens, K, N, n, R, dtype):
    say("linear", lens[:8], K, N, n, R, dtype)
    g = gen(K + N)
    q_off = offsets(lens)
    T = q_off[-1]
    wide = normal(g, T, K + 24, dtype=dtype)              # rows with a stride of their own
    x = wide[:, 8:8 + K]
    w = normal(g, N, K, dtype=dtype, std=K ** -0.5)
    a = normal(g, n, R, K, dtype=dtype, std=K ** -0.5)
    b = normal(g, n, N, R, dtype=dtype)
    rank = torch.randint(0, R + 1, (n,), generator=g, dtype=torch.int32)
    rank[0] = R
    for i in range(n):                                     # what lies beyond a rank is not used
        a[i, int(rank[i]):] = math.nan
        b[i, :, int(rank[i]):] = math.inf
    scale = torch.rand(n, generator=g) * 3 - 1
    adapter = torch.randint(-1, n, (len(lens),), generator=g, dtype=torch.int32)
    adapter[0] = 0
    want, bound = ref.linear(x, w, a, b, q_off, adapter, rank, scale)
    dev = [t.cuda() for t in (a, b, adapter, rank, scale)]
    out = torch.full((T, N + 16), 7.0, dtype=dtype, device="cuda")
    xd, wd = wide.cuda()[:, 8:8 + K], w.cuda()
    y = fs.fs_adapter_linear(fs.Step(q_off), fs.Adapters(*dev), xd, wd, y=out[:, 8:8 + N])
    within(y, want, bound, "y")
    assert bool((out[:, :8] == 7).all()) and bool((out[:, 8 + N:] == 7).all())
    again = fs.fs_adapter_linear(fs.Step(q_off), fs.Adapters(*dev), xd, wd)
    assert torch.equal(again, y)


@pytest.mark.parametrize("rows", [20, 50])
@pytest.mark.parametrize("N", [8200, 12304, 24600])
def test_linear_few_rows_many_columns(rows, N):
    g = gen(rows + N)
    K, lens = 136, [1] * (rows - 7) + [7]
    q_off = offsets(lens)
    x, w = normal(g, rows, K), normal(g, N, K, std=K ** -0.5)
    a, b = normal(g, 3, 16, K, std=K ** -0.5), normal(g, 3, N, 16)
    adapter = torch.randint(-1, 3, (len(lens),), generator=g, dtype=torch.int32)
    want, bound = ref.linear(x, w, a, b, q_off, adapter)
    ad = fs.Adapters(a.cuda(), b.cuda(), adapter.cuda())
    within(fs.fs_adapter_linear(fs.Step(q_off), ad, x.cuda(), w.cuda()), want, bound, "y")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,N", [(1, 64), (20, 136), (50, 9000), (130, 520), (1200, 2056), (5000, 4000)])
def test_linear_of_a_broken_adapter_is_its_own(rows, N, dtype):
    """Infinities and NaN in one adapter reach the rows of its requests alone."""
    g = gen(rows + N)
    K, R = 72, 24
    lens = [1] * min(rows, 40) + ([rows - 40] if rows > 40 else [])
    q_off = offsets(lens)
    x, w = normal(g, rows, K, dtype=dtype), normal(g, N, K, dtype=dtype, std=K ** -0.5)
    a, b = normal(g, 5, R, K, dtype=dtype, std=K ** -0.5), normal(g, 5, N, R, dtype=dtype)
    adapter = torch.randint(-1, 5, (len(lens),), generator=g, dtype=torch.int32)
    whole = fs.fs_adapter_linear(fs.Step(q_off), fs.Adapters(a.cuda(), b.cuda(), adapter.cuda()),
                                 x.cuda(), w.cuda())
    assert bool(torch.isfinite(whole).all())
    bad_a, bad_b = a.clone(), b.clone()
    bad_a[0, 3], bad_b[1], bad_b[2, :, 5] = math.inf, math.nan, -math.inf
    bad = fs.Adapters(bad_a.cuda(), bad_b.cuda(), adapter.cuda())
    y = fs.fs_adapter_linear(fs.Step(q_off), bad, x.cuda(), w.cuda())
    for s in range(len(lens)):
        rows_s = slice(q_off[s], q_off[s + 1])
        if int(adapter[s]) in (0, 1, 2):
            assert not bool(torch.isfinite(y[rows_s]).any()), s
        else:
            assert torch.equal(y[rows_s], whole[rows_s]), s


@pytest.mark.parametrize("size", [3e-5, 1e-2, 3e3])
@pytest.mark.parametrize("rows", [3, 200])
def test_linear_half_precision_beyond_its_range(rows, size):
    """x a^T from far below half precision's smallest numbers to far above its largest."""
    g = gen(rows)
    K, N, R = 512, 136, 16
    q_off = [0, 1, rows]
    x = normal(g, rows, K, dtype=HF, std=size)
    a = (normal(g, 2, R, K).abs() + 1).to(HF) * min(size, 10)
    b = normal(g, 2, N, R, dtype=HF, std=1e-4 if size > 1 else 1.0)
    w = torch.zeros(N, K, dtype=HF)
    x[:, :300] = x[:, :300].abs()
    adapter = torch.tensor([1, 0], dtype=torch.int32)
    want, bound = ref.linear(x, w, a, b, q_off, adapter)
    y = fs.fs_adapter_linear(fs.Step(q_off), fs.Adapters(a.cuda(), b.cuda(), adapter.cuda()),
                             x.cuda(), w.cuda())
    within(y, want, bound, "y")


@pytest.mark.parametrize("lens,N", [([700, 1, 1297], 2568), ([1400, 150], 4096), ([2000, 501], 4104)])
def test_linear_tiles_of_the_middle(lens, N):
    """Row and column counts whose tiles are 128 rows by 96 or 128 columns."""
    g = gen(N)
    K, q_off, T = 200, offsets(lens), sum(lens)
    x, w = normal(g, T, K, dtype=HF), normal(g, N, K, dtype=HF, std=K ** -0.5)
    a, b = normal(g, 2, 8, K, dtype=HF, std=K ** -0.5), normal(g, 2, N, 8, dtype=HF)
    adapter = torch.tensor([1, -1, 0][:len(lens)], dtype=torch.int32)
    want, bound = ref.linear(x, w, a, b, q_off, adapter)
    ad = fs.Adapters(a.cuda(), b.cuda(), adapter.cuda())
    within(fs.fs_adapter_linear(fs.Step(q_off), ad, x.cuda(), w.cuda()), want, bound, "y")


def test_linear_without_adapters_and_defaults():
    g = gen(5)
    lens, K, N = [5, 1, 70], 128, 200
    q_off = offsets(lens)
    x, w = normal(g, q_off[-1], K), normal(g, N, K)
    none = torch.full((3,), -1, dtype=torch.int32)
    a, b = normal(g, 2, 16, K), normal(g, 2, N, 16)
    want, bound = ref.linear(x, w, a, b, q_off, none)
    ad = fs.Adapters(a.cuda(), b.cuda(), none.cuda())
    within(fs.fs_adapter_linear(fs.Step(q_off), ad, x.cuda(), w.cuda()), want, bound, "no adapter")
    empty = fs.Adapters(a[:0].cuda(), b[:0].cuda(), none.cuda())
    within(fs.fs_adapter_linear(fs.Step(q_off), empty, x.cuda(), w.cuda()), want, bound, "none at all")
    one = torch.tensor([1, -1, 0], dtype=torch.int32)
    want, bound = ref.linear(x, w, a, b, q_off, one)
    ad = fs.Adapters(a.cuda(), b.cuda(), one.cuda())       # rank and scale by default
    within(fs.fs_adapter_linear(fs.Step(q_off), ad, x.cuda(), w.cuda()), want, bound, "defaults")


def test_linear_bad_adapter_is_an_error_not_an_address():
    g = gen(6)
    x, w = normal(g, 4, 64).cuda(), normal(g, 64, 64).cuda()
    a, b = normal(g, 2, 8, 64).cuda(), normal(g, 2, 64, 8).cuda()
    for bad, rank in (([0, 2], None), ([-2, 0], None), ([0, 1], [8, 9]), ([0, 1], [-1, 8])):
        ad = fs.Adapters(a, b, torch.tensor(bad, dtype=torch.int32).cuda(),
                         None if rank is None else torch.tensor(rank, dtype=torch.int32).cuda())
        with pytest.raises(fs.FairServeError) as e:
            fs.fs_adapter_linear(fs.Step([0, 2, 4]), ad, x, w)
        assert e.value.code == fs.FS_E_RANGE


# ----------------------------------------------------------------- the paged cache

def make_cache(g, kv_len, HK, D, page, dtype, garbage=math.nan, extra=3, token_major=False):
    """A cache whose pages lie in random order; unused slots and pages hold `garbage`."""
    need = [-(-n // page) for n in kv_len]
    width = max(max(need), 1)
    total = sum(need) + extra
    perm = torch.randperm(total, generator=g).to(torch.int32)
    table = torch.full((len(kv_len), width), -1, dtype=torch.int32)
    shape = (total, page, HK, D) if token_major else (total, HK, page, D)
    k, v = (torch.full(shape, garbage, dtype=dtype) for _ in range(2))
    kk, vv = (t.permute(0, 2, 1, 3) if token_major else t for t in (k, v))
    at = 0
    for s, n in enumerate(kv_len):
        ids = perm[at:at + need[s]]
        at += need[s]
        table[s, :need[s]] = ids
        j = torch.arange(n)
        kk[ids[j // page].long(), :, j % page] = normal(g, n, HK, D, dtype=dtype)
        vv[ids[j // page].long(), :, j % page] = normal(g, n, HK, D, dtype=dtype)
    return kk, vv, table


def on_gpu(k, v, table, token_major=False):
    kd, vd = k.cuda(), v.cuda()        # permuted views keep their strides
    return fs.KVCache(kd, vd, table.cuda())


def step_of(lens, kv_len):
    return fs.Step(offsets(lens), kv_len=torch.tensor(kv_len, dtype=torch.int32).cuda(),
                   max_kv=max(max(kv_len), 0))


# ----------------------------------------------------------------- rotary append

ROPE = [
    # rows, cached lengths, heads, kv heads, dim, page, rotary, interleaved
    ([1], [1], 8, 2, 64, 16, 64, False),
    ([1, 1, 1], [5, 17, 4000], 4, 4, 128, 16, 128, True),
    ([7, 0, 1, 30], [7, 3, 1, 61], 12, 3, 80, 8, 40, False),       # pairs across chunks
    ([5, 9], [3, 9], 6, 2, 64, 4, 24, False),                      # padding rows, scalar pairs
    ([5, 9], [3, 9], 6, 2, 64, 4, 24, True),
    ([33, 2], [100000, 70001], 2, 1, 256, 64, 128, True),
    ([13], [200], 1, 1, 8, 1, 2, False),
    ([6], [6], 3, 3, 96, 32, 0, False),                            # nothing turns
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,H,HK,D,page,rot,inter", ROPE)
def test_rope_append(lens, kv, H, HK, D, page, rot, inter, dtype):
    say("rope", lens, kv, H, HK, D, page, rot, inter, dtype)
    g = gen(D + rot)
    q_off = offsets(lens)
    T = q_off[-1]
    k, v, table = make_cache(g, kv, HK, D, page, dtype, garbage=5.0, token_major=inter)
    qkv = normal(g, T, H + 2 * HK, D, dtype=dtype)
    f, factor = fs.fs_rope_frequencies(rot, 10000.0, fs.FS_ROPE_PARTS, 4.0, 2048)
    inv = torch.from_numpy(f)
    cache = on_gpu(k, v, table)
    d = qkv.cuda()
    q = fs.fs_rope_append(step_of(lens, kv), cache, fs.Rope(inv.cuda(), inter, factor), d[:, :H],
                          d[:, H:H + HK], d[:, H + HK:])
    kw, kb = k.double().clone(), torch.zeros(k.shape, dtype=torch.float64)
    vw = v.clone()
    for s, pos in enumerate(ref.positions(q_off, kv)):
        rows = slice(q_off[s], q_off[s + 1])
        seen = [max(0, p) for p in pos]
        y, b = ref.rope_rows(qkv[rows, :H + HK], seen, inv, rot, inter, factor)
        within(q[rows], y[:, :H], b[:, :H], f"q of request {s}")
        for i, p in enumerate(pos):
            if p >= 0:
                at = int(table[s, p // page])
                kw[at, :, p % page] = torch.from_numpy(y[i, H:])
                kb[at, :, p % page] = torch.from_numpy(b[i, H:])
                vw[at, :, p % page] = qkv[q_off[s] + i, H + HK:]
    within(cache.k, kw, kb, "key cache")             # bound 0 where nothing is appended
    assert torch.equal(cache.v.cpu(), vw)
    # in place, with positions of its own
    pos = torch.randint(0, 1 << 20, (T,), generator=g, dtype=torch.int32)
    q2 = d[:, :H]
    fs.fs_rope_append(step_of(lens, kv), cache, fs.Rope(inv.cuda(), inter, factor, pos.cuda()), q2,
                      d[:, H:H + HK].clone(), d[:, H + HK:].clone(), q_out=q2)
    y, b = ref.rope_rows(qkv[:, :H], pos.numpy(), inv, rot, inter, factor)
    within(q2, y, b, "q in place")


def test_rope_append_without_queries_and_bad_pages():
    g = gen(3)
    k, v, table = make_cache(g, [4, 9], 2, 64, 8, BF, garbage=1.0)
    kv = normal(g, 3, 4, 64)
    rope = fs.Rope(torch.ones(32).cuda())
    cache = on_gpu(k, v, table)
    d = kv.cuda()
    assert fs.fs_rope_append(step_of([1, 2], [4, 9]), cache, rope, None, d[:, :2], d[:, 2:]) is None
    table2 = table.clone()
    table2[1, 1] = k.shape[0]
    bad = fs.KVCache(cache.k, cache.v, table2.cuda())
    before = cache.k.clone()
    with pytest.raises(fs.FairServeError) as e:
        fs.fs_rope_append(step_of([0, 1], [4, 9]), bad, rope, None, d[:1, :2], d[:1, 2:])
    assert e.value.code == fs.FS_E_RANGE and torch.equal(before, cache.k)
    over = fs.Step([0, 1], kv_len=torch.tensor([10], dtype=torch.int32).cuda(), max_kv=9)
    with pytest.raises(fs.FairServeError) as e:
        fs.fs_rope_append(over, cache, rope, None, d[:1, :2], d[:1, 2:])
    assert e.value.code == fs.FS_E_RANGE


# ----------------------------------------------------------------- attention

ATTENTION = [
    # rows, cached lengths, heads, kv heads, dim, page, window
    ([1], [1], 1, 1, 64, 16, 0),
    ([1, 1, 1], [5, 16, 333], 8, 2, 128, 16, 0),
    ([1] * 5, [0, 1, 64, 65, 1000], 32, 8, 128, 16, 0),
    ([1, 1], [5000, 70], 7, 1, 128, 32, 0),
    ([1, 1, 1], [700, 3, 129], 16, 16, 64, 8, 100),
    ([1], [40001], 8, 1, 64, 64, 0),                      # split over a long context
    ([1, 1], [9000, 20], 64, 1, 128, 16, 4097),
    ([3, 0, 1, 20], [3, 9, 50, 33], 6, 2, 64, 16, 0),
    ([40, 130], [40, 400], 8, 2, 128, 16, 0),
    ([65, 2, 1], [1000, 2, 600], 3, 3, 128, 4, 7),
    ([200], [200], 8, 8, 64, 16, 0),
    ([70, 5, 9], [64, 2, 9], 4, 1, 128, 1, 0),            # padding rows ahead
    ([17, 33], [517, 33], 14, 2, 64, 128, 50),
    ([5, 1, 2], [3000, 3000, 2500], 12, 4, 128, 16, 0),   # few rows, long contexts
    ([4], [300], 64, 1, 64, 16, 0),
    ([257], [771], 5, 1, 128, 16, 0),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,H,HK,D,page,window", ATTENTION)
def test_attention(lens, kv, H, HK, D, page, window, dtype):
    say("attention", lens[:6], kv[:6], H, HK, D, page, window, dtype)
    g = gen(H * 1000 + D + len(lens))
    q_off = offsets(lens)
    T = q_off[-1]
    token_major = page == 16
    k, v, table = make_cache(g, kv, HK, D, page, dtype, token_major=token_major)
    wide = normal(g, T, H + 2, D, dtype=dtype, std=2.0)
    q = wide[:, 1:1 + H]
    scale = 1.3 * D ** -0.5
    want, tol, lse, ltol = ref.attention(q, k, v, table, q_off, kv, scale, window)
    out = torch.full((T, H + 1, D), 9.0, dtype=dtype, device="cuda")
    step, cache, qd = step_of(lens, kv), on_gpu(k, v, table), wide.cuda()[:, 1:1 + H]
    o, l = fs.fs_paged_attention(step, cache, qd, scale, window, out=out[:, :H], want_lse=True)
    within(o, want, tol, "out")
    empty = torch.isinf(lse)
    assert bool((l.cpu()[empty] == -math.inf).all())
    within(l.cpu()[~empty], lse[~empty], ltol[~empty], "lse")
    assert bool((out[:, H:] == 9).all())
    again = fs.fs_paged_attention(step, cache, qd, scale, window)
    assert torch.equal(again, o)


@pytest.mark.parametrize("lens,kv", [([1, 1], [3000, 50]), ([60], [90])])
def test_attention_large_scores_and_a_loose_bound(lens, kv):
    """Scores in the thousands (no overflow), and a host bound far above the lengths."""
    g = gen(11)
    k, v, table = make_cache(g, kv, 2, 128, 16, BF)
    k = k * 20
    q_off = offsets(lens)
    q = normal(g, q_off[-1], 8, 128, std=20.0)
    want, tol, lse, ltol = ref.attention(q, k, v, table, q_off, kv, 0.5, 0)
    wide = torch.full((len(kv), 4000), -1, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    step = fs.Step(q_off, kv_len=torch.tensor(kv, dtype=torch.int32).cuda(), max_kv=60000)
    o, l = fs.fs_paged_attention(step, on_gpu(k, v, wide), q.cuda(), 0.5, want_lse=True)
    within(o, want, tol, "out")
    within(l, lse, ltol, "lse")


@pytest.mark.parametrize("lens,kv", [([1, 1], [300, 0]), ([90, 70, 3], [200, 40, 3])])
def test_attention_window_beyond_every_length(lens, kv):
    """The largest window there is, with padding rows: as without a window."""
    g = gen(17)
    k, v, table = make_cache(g, kv, 2, 64, 16, HF)
    q = normal(g, sum(lens), 6, 64, dtype=HF).cuda()
    step, cache = step_of(lens, kv), on_gpu(k, v, table)
    plain = fs.fs_paged_attention(step, cache, q, 0.2)
    for window in (2 ** 31 - 1, 300, 1 << 30):
        assert torch.equal(fs.fs_paged_attention(step, cache, q, 0.2, window=window), plain)


@pytest.mark.parametrize("lens", [[1] * 70, [80] * 3 + [1] * 67])
def test_attention_of_many_requests(lens):
    g = gen(18)
    kv = [n + int(x) for n, x in zip(lens, torch.randint(0, 150, (len(lens),), generator=g))]
    k, v, table = make_cache(g, kv, 1, 128, 16, BF)
    q_off = offsets(lens)
    q = normal(g, q_off[-1], 3, 128)
    want, tol, _, _ = ref.attention(q, k, v, table, q_off, kv, 0.1, 0)
    within(fs.fs_paged_attention(step_of(lens, kv), on_gpu(k, v, table), q.cuda(), 0.1), want, tol, "out")


@pytest.mark.parametrize("most", [1023, 1024, 1025, 2047, 2048, 2049])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_around_the_longest_whole_request(D, most):
    """Lengths and bounds at which single tokens go from one work-group a head to splits."""
    g = gen(most + D)
    lens, kv = [1, 1, 2, 1], [most, 1, most - 200, 257]
    k, v, table = make_cache(g, kv, 2, D, 16, BF)
    q_off = offsets(lens)
    q = normal(g, q_off[-1], 8, D)
    want, tol, lse, ltol = ref.attention(q, k, v, table, q_off, kv, 0.1, 0)
    got, l = fs.fs_paged_attention(step_of(lens, kv), on_gpu(k, v, table), q.cuda(), 0.1, want_lse=True)
    within(got, want, tol, "out")
    within(l, lse, ltol, "lse")


@pytest.mark.parametrize("window", [0, 150])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_attention_of_many_rows_without_small_requests(dtype, window):
    """Chunks alone, and so many heads that 256 rows share a tile of keys."""
    g = gen(19 + window)
    lens, kv = [261, 0, 77], [500, 9, 333]
    k, v, table = make_cache(g, kv, 16, 128, 16, dtype)
    q = normal(g, sum(lens), 256, 128, dtype=dtype)
    q_off = offsets(lens)
    want, tol, _, _ = ref.attention(q, k, v, table, q_off, kv, 0.09, window)
    got = fs.fs_paged_attention(step_of(lens, kv), on_gpu(k, v, table), q.cuda(), 0.09, window=window)
    within(got, want, tol, "out")


@pytest.mark.parametrize("lens", [[1, 1, 1], [50, 1, 20]])
def test_attention_offsets_beyond_32_bits_and_shared_pages(lens):
    g = gen(12)
    D, HK, page, stride = 64, 1, 16, 1_200_000_000           # elements between pages
    kv = [60, 50, 49]
    big = [torch.empty(3 * stride + 4096, dtype=BF, device="cuda") for _ in range(2)]
    view = [t.as_strided((4, HK, page, D), (stride, page * D, D, 1)) for t in big]
    k, v = (normal(g, 4, HK, page, D) for _ in range(2))
    for a, b in zip(view, (k, v)):
        a.copy_(b)
    table = torch.tensor([[3, 1, 0, 2], [3, 1, 2, 0], [3, 3, 3, 3]], dtype=torch.int32)
    q_off = offsets(lens)
    q = normal(g, q_off[-1], 4, D)
    want, tol, _, _ = ref.attention(q, k, v, table, q_off, kv, 0.125, 0)
    cache = fs.KVCache(view[0], view[1], table.cuda())
    step = step_of(lens, kv)
    within(fs.fs_paged_attention(step, cache, q.cuda(), 0.125), want, tol, "out")
    rope = fs.Rope(torch.ones(16).cuda())
    kvn = normal(g, q_off[-1], 2, D).cuda()
    fs.fs_rope_append(fs.Step([0, 1], kv_len=torch.tensor([17], dtype=torch.int32).cuda(), max_kv=17),
                      fs.KVCache(view[0], view[1], table.cuda()), rope, None, kvn[:1, :1], kvn[:1, 1:])
    assert torch.equal(view[1][1, 0, 0], kvn[0, 1])


def test_attention_bad_lengths_and_pages_are_errors():
    g = gen(13)
    for lens in ([1, 1], [40, 1]):
        k, v, table = make_cache(g, [90, 70], 2, 64, 16, BF)
        q = normal(g, offsets(lens)[-1], 4, 64).cuda()
        for where, value in (((0, 1), -1), ((1, 0), 1 << 30)):
            t2 = table.clone()
            t2[where] = value
            with pytest.raises(fs.FairServeError) as e:
                fs.fs_paged_attention(step_of(lens, [90, 70]), on_gpu(k, v, t2), q, 0.1)
            assert e.value.code == fs.FS_E_RANGE
        for n in (-1, 91):
            step = fs.Step(offsets(lens), kv_len=torch.tensor([n, 70], dtype=torch.int32).cuda(),
                           max_kv=90)
            with pytest.raises(fs.FairServeError) as e:
                fs.fs_paged_attention(step, on_gpu(k, v, torch.zeros_like(table)), q, 0.1)
            assert e.value.code == fs.FS_E_RANGE


# ----------------------------------------------------------------- sampling

def check_sample(x, u, t=None, k=None, p=None, m=None):
    dev = lambda v, d: None if v is None else torch.tensor(v, dtype=d).cuda()   # noqa: E731
    n = x.shape[0]
    xd = x.cuda() if x.is_contiguous() else x
    tok, lp, kept = fs.fs_sample(xd, dev(u, F32), fs.Sampling(dev(t, F32), dev(k, torch.int32),
                                                              dev(p, F32), dev(m, F32)))
    xs = x.float().cpu().numpy()
    for i in range(n):
        want = ref.sample_row(xs[i], u[i], 1.0 if t is None else t[i], 0 if k is None else k[i],
                              1.0 if p is None else p[i], 0.0 if m is None else m[i])
        got = (int(tok[i]), float(lp[i]), int(kept[i]))
        assert got[0] == want[0] and got[2] == want[2], (i, got, want)
        assert got[1] == want[1] or abs(got[1] - want[1]) <= 4 * ref.E32 * max(1.0, abs(want[1])), \
            (i, got, want)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("vocab", [1, 2, 63, 1000, 4099, 32000, 70001])
def test_sample_settings(vocab, dtype):
    say("sample", vocab, dtype)
    g = gen(vocab)
    n = 12
    x = normal(g, n, vocab, dtype=dtype, std=3.0)
    u = torch.rand(n, generator=g).tolist()
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -24
    rng = np.random.default_rng(vocab)
    t = rng.uniform(0.2, 2.0, n).astype(np.float32).tolist()
    t[2] = 0.0
    k = rng.integers(-1, 60, n).tolist()
    k[3], k[4] = 1, vocab + 5
    p = rng.uniform(0.05, 1.0, n).astype(np.float32).tolist()
    p[5], p[6] = 0.0, 1.0
    m = rng.uniform(0.0, 0.3, n).astype(np.float32).tolist()
    m[7], m[8] = 1.0, 0.0
    check_sample(x, u)
    check_sample(x, u, t=t)
    check_sample(x, u, t=t, k=k)
    check_sample(x, u, t=t, p=p)
    check_sample(x, u, m=m)
    check_sample(x, u, t, k, p, m)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_sample_ties_infinities_and_masks(dtype):
    g = gen(77)
    V = 5000
    rows = []
    rows.append(torch.zeros(V))                                       # all equal
    rows.append(torch.randint(0, 4, (V,), generator=g).float())       # many ties
    r = torch.randn(V, generator=g)
    r[torch.rand(V, generator=g) < 0.999] = -math.inf                 # a mask
    rows.append(r)
    rows.append(torch.full((V,), -math.inf))                          # nothing left
    r = torch.randn(V, generator=g)
    r[7] = r[4000] = math.inf
    rows.append(r)
    r = torch.randn(V, generator=g)
    r[::3] = math.nan
    rows.append(r)
    rows.append(torch.full((V,), torch.finfo(dtype).min))             # the type's lowest value
    r = torch.full((V,), torch.finfo(dtype).min)
    r[123] = 0.0
    r[124] = -0.0
    rows.append(r)
    r = torch.full((V,), -math.inf)
    r[V - 1] = -3.0
    rows.append(r)
    r = torch.full((V,), math.nan)
    rows.append(r)
    x = torch.stack(rows).to(dtype)
    n = x.shape[0]
    for u in (0.0, 0.31, 0.77, 1 - 2.0 ** -24):
        check_sample(x, [u] * n)
        check_sample(x, [u] * n, k=[37] * n)
        check_sample(x, [u] * n, p=[0.4] * n)
        check_sample(x, [u] * n, t=[0.5] * n, k=[2500] * n, p=[0.999] * n, m=[0.01] * n)
        check_sample(x, [u] * n, t=[0.0] * n)
        check_sample(x, [u] * n, t=[1e-30] * n, p=[0.9] * n)
        check_sample(x, [u] * n, t=[1e30] * n, p=[0.5] * n)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,vocab", [(1, 131072), (3, 262147), (40, 20011), (300, 1500)])
def test_sample_shapes_and_strides(rows, vocab, dtype):
    say("sample shapes", rows, vocab, dtype)
    g = gen(rows)
    wide = torch.randn(rows, vocab + 37, generator=g, dtype=F32).mul_(2.5).to(dtype).cuda()
    x = wide[:, 5:5 + vocab]                                          # odd alignment
    u = torch.rand(rows, generator=g).tolist()
    few = 8
    sel = list(range(min(few, rows))) + ([rows - 1] if rows > few else [])
    k = [50] * rows
    p = [0.9] * rows
    tok, lp, kept = fs.fs_sample(x, torch.tensor(u).cuda(),
                                 fs.Sampling(top_k=torch.tensor(k, dtype=torch.int32).cuda(),
                                             top_p=torch.tensor(p).cuda()))
    tok2, _, kept2 = fs.fs_sample(x, torch.tensor(u).cuda(), fs.Sampling(top_p=torch.tensor(p).cuda()))
    tok3, _, kept3 = fs.fs_sample(x, torch.tensor(u).cuda(), fs.Sampling())
    xs = x.float().cpu().numpy()
    for i in sel:
        a = ref.sample_row(xs[i], u[i], 1.0, 50, 0.9, 0.0)
        b = ref.sample_row(xs[i], u[i], 1.0, 0, 0.9, 0.0)
        c = ref.sample_row(xs[i], u[i], 1.0, 0, 1.0, 0.0)
        assert (int(tok[i]), int(kept[i])) == (a[0], a[2]), i
        assert (int(tok2[i]), int(kept2[i])) == (b[0], b[2]), i
        assert (int(tok3[i]), int(kept3[i])) == (c[0], c[2]), i


@pytest.mark.parametrize("dtype", [BF, F32])
def test_sample_large_k(dtype):
    """k beyond the work-group's threads, and beyond what is sorted in LDS."""
    g = gen(91)
    x = normal(g, 4, 60000, dtype=dtype, std=2.0)
    u = torch.rand(4, generator=g).tolist()
    check_sample(x, u, k=[513, 1500, 3900, 20000])
    check_sample(x, u, t=[0.3, 2.0, 1.0, 0.7], k=[1025, 4096, 59999, 5000], p=[0.9, 0.999, 0.5, 1.0])


def test_sample_bad_settings():
    x = torch.zeros(2, 100, device="cuda")
    ok = dict(t=[1.0, 1.0], p=[0.9, 0.9], m=[0.1, 0.1], u=[0.5, 0.5])
    for name, bad in (("t", -1.0), ("t", math.nan), ("t", math.inf), ("p", 1.5), ("p", -0.1),
                      ("p", math.nan), ("m", 2.0), ("m", math.nan), ("u", 1.0), ("u", -0.5),
                      ("u", math.nan)):
        a = {key: list(v) for key, v in ok.items()}
        a[name][1] = bad
        c = {key: torch.tensor(v).cuda() for key, v in a.items()}
        err = fs.cleared_err_word()
        tok, _, _ = fs.fs_sample(x, c["u"], fs.Sampling(c["t"], None, c["p"], c["m"]), err=err,
                                 check=False)
        assert fs.fs_sync_status(err) == fs.FS_E_RANGE, (name, bad)
        assert int(tok[1]) == -1 and int(tok[0]) >= 0
        fs.fs_clear_status(err)
        assert fs.fs_sync_status(err) == fs.FS_OK


# ----------------------------------------------------------------- a step together

def test_step_on_a_side_stream_and_in_a_graph():
    """The four calls of a decode step, captured once; the lengths, the tokens and the
    adapters then change between replays and every replay matches the eager calls."""
    g = gen(21)
    n, H, HK, D, K, V, page, cap = 5, 8, 2, 64, 256, 1000, 16, 900
    lens = [1] * n
    kv = [3, 40, 500, 1, 77]
    k, v, table = make_cache(g, [cap] * n, HK, D, page, BF)
    w = normal(g, (H + 2 * HK) * D, K, std=K ** -0.5).cuda()
    head = normal(g, V, H * D, std=0.2).cuda()
    a, b = normal(g, 3, 16, K, std=K ** -0.5).cuda(), normal(g, 3, (H + 2 * HK) * D, 16).cuda()
    ad = torch.tensor([0, 1, -1, 2, 0], dtype=torch.int32).cuda()
    kv_len = torch.tensor(kv, dtype=torch.int32).cuda()
    step = fs.Step(offsets(lens), kv_len=kv_len, max_kv=cap)
    none = fs.Adapters(torch.zeros(0, 8, H * D, dtype=BF).cuda(), torch.zeros(0, V, 8, dtype=BF).cuda(), ad)
    adapters = fs.Adapters(a, b, ad)
    rope = fs.Rope(torch.from_numpy(fs.fs_rope_frequencies(D)[0]).cuda())
    x = normal(g, n, K).cuda()
    u = torch.rand(n, generator=g).cuda()
    top_p = torch.full((n,), 0.9).cuda()

    def run(cache, err):
        qkv = fs.fs_adapter_linear(step, adapters, x, w, err=err, check=False).view(n, H + 2 * HK, D)
        q = fs.fs_rope_append(step, cache, rope, qkv[:, :H], qkv[:, H:H + HK], qkv[:, H + HK:],
                              err=err, check=False)
        o = fs.fs_paged_attention(step, cache, q, D ** -0.5, err=err, check=False)
        logits = fs.fs_adapter_linear(step, none, o.view(n, H * D), head, err=err, check=False)
        return o, logits, fs.fs_sample(logits, u, fs.Sampling(top_p=top_p), err=err, check=False)

    err = fs.cleared_err_word()
    eager_cache, graph_cache = on_gpu(k, v, table), on_gpu(k, v, table)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(graph_cache, err)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = run(graph_cache, err)
    torch.cuda.synchronize()
    for i in range(4):
        if i:
            kv_len += 1 + 60 * i
            x.copy_(normal(g, n, K))
            ad.copy_(torch.tensor([(j + i) % 4 - 1 for j in range(n)], dtype=torch.int32))
            u.copy_(torch.rand(n, generator=g))
            torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = run(eager_cache, err)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), i
        assert torch.equal(got[2][0], want[2][0]) and torch.equal(got[2][2], want[2][2]), i
    assert fs.fs_sync_status(err) == fs.FS_OK
