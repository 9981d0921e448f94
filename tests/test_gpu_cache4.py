"""The cache held in 4 bits against the oracle in cache_ref.py: the format, the append, the
rows read back, and attention over it (types, head layouts, lengths from one token on, odd
and ragged sizes, strides, masks, garbage in unused slots, NaN, offsets beyond 32 bits,
graphs)."""
import math

import numpy as np
import pytest
import torch

import cache_ref as cref
import engine_ref as ref
import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_engine import BF, HF, gen, normal, offsets, step_of, within

pytestmark = pytest.mark.gpu


def make_cache4(g, kv_len, HK, D, page, dtype, extra=3, token_major=False, spread=3):
    """(k, v, k_scale, v_scale, table): random codes and scales around 1, pages in random order;
    unused slots and pages hold scales that count as NaN."""
    need = [-(-n // page) for n in kv_len]
    total, width = sum(need) + extra, max(max(need), 1)
    perm = torch.randperm(total, generator=g).to(torch.int32)
    table = torch.full((len(kv_len), width), -1, dtype=torch.int32)
    shape = (total, page, HK) if token_major else (total, HK, page)
    out = []
    for per in (D // 2, D // 2, D // 32, D // 32):
        x = torch.randint(0, 256, (*shape, per), generator=g, dtype=torch.uint8)
        if per == D // 32:
            x.fill_(255)
        out.append(x.permute(0, 2, 1, 3) if token_major else x)
    at = 0
    for s, n in enumerate(kv_len):
        ids = perm[at:at + need[s]]
        at += need[s]
        table[s, :need[s]] = ids
        j = torch.arange(n)
        for x in out[2:]:
            x[ids[j // page].long(), :, j % page] = torch.randint(
                127 - spread, 127, (n, HK, D // 32), generator=g, dtype=torch.uint8)
    return (*out, table)


def on_gpu4(k, v, ks, vs, table):
    return fs.KVCache4(*(t.cuda() for t in (k, v, ks, vs, table)))


def both_values(c, dtype):
    """float64 keys and values of a cache on the host."""
    k, v, ks, vs, _ = c
    return cref.values(k, ks, cref.TOP[dtype]), cref.values(v, vs, cref.TOP[dtype])


# ----------------------------------------------------------------- the format

@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 256])
def test_every_code_and_scale_reads_as_its_value(D, dtype):
    top = cref.TOP[dtype]
    n = 256                                    # a token for every scale byte
    codes = (torch.arange(n * 2 * D // 2).view(n, 2, D // 2) * 37 % 256).to(torch.uint8)
    scales = torch.arange(n, dtype=torch.uint8)[:, None, None].expand(n, 2, D // 32).contiguous()
    k = codes.view(n // 16, 16, 2, D // 2).permute(0, 2, 1, 3)
    ks = scales.view(n // 16, 16, 2, D // 32).permute(0, 2, 1, 3)
    table = torch.arange(n // 16, dtype=torch.int32)[None]
    cache = on_gpu4(k, k.flip(0), ks, ks.flip(0), table)
    kk, vv = fs.fs_cache4_rows(step_of([n], [n]), cache, dtype)
    for got, x, b in ((kk, k, ks), (vv, k.flip(0), ks.flip(0))):
        want = cref.values(x, b, top).permute(0, 2, 1, 3).reshape(n, 2, D)
        nan = want.isnan()
        assert torch.equal(got.cpu().isnan(), nan)
        # rounded once to the type (exact but for half precision's smallest numbers)
        want = torch.where(nan, torch.zeros_like(want), want).to(dtype)
        assert torch.equal(torch.where(nan, torch.zeros_like(want), got.cpu()), want)


def test_rows_read_back_leave_the_rest_and_pad_with_zeros():
    g = gen(4)
    lens, kv = [3, 0, 5], [2, 7, 40]
    c = make_cache4(g, kv, 2, 64, 8, BF)
    out = torch.full((8, 3, 64), 5.0, dtype=BF, device="cuda")
    k, v = fs.fs_cache4_rows(step_of(lens, kv), on_gpu4(*c), k=out[:, :2])
    K, V = both_values(c, BF)
    tab, q_off = c[4].numpy(), offsets(lens)
    for s, pos in enumerate(ref.positions(q_off, kv)):
        for i, p in enumerate(pos):
            for got, of in ((k, K), (v, V)):
                want = of[tab[s][p // 8], :, p % 8] if p >= 0 else torch.zeros(2, 64)
                assert torch.equal(got[q_off[s] + i].double().cpu(), want.double())
    assert bool((out[:, 2] == 5).all())


# ----------------------------------------------------------------- append

APPEND = [
    # rows, cached lengths, heads, kv heads, dim, page, rotary, interleaved
    ([1], [1], 8, 2, 64, 16, 64, False),
    ([1, 1, 1], [5, 17, 4000], 4, 4, 128, 16, 128, True),
    ([7, 0, 1, 30], [7, 3, 1, 61], 11, 3, 96, 8, 48, False),       # groups of four lanes, odd heads
    ([5, 9], [3, 9], 6, 2, 64, 4, 24, False),                      # padding rows, scalar pairs
    ([5, 9], [3, 9], 7, 2, 64, 4, 26, True),
    ([33, 2], [100000, 70001], 2, 1, 256, 64, 128, True),
    ([13], [200], 1, 1, 32, 1, 2, False),
    ([6], [6], 3, 3, 96, 32, 0, False),                            # nothing turns
    ([40, 3], [1 << 20, 900], 2, 2, 128, 4096, 128, False),
    # four tokens a work-group, the last one's not all there; sides of 4, of 1, chunks turned in part
    ([1021, 5], [1021, 300], 3, 1, 64, 16, 24, False),
    ([5, 1021], [3, 2000], 2, 2, 96, 16, 22, False),
    ([1027], [1500], 1, 1, 32, 64, 20, False),
    ([1, 1026], [9, 1026], 3, 1, 64, 16, 20, True),
    ([1030], [1030], 2, 1, 128, 8, 128, False),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,H,HK,D,page,rot,inter", APPEND)
def test_rope_append4(lens, kv, H, HK, D, page, rot, inter, dtype):
    say("append4", lens, kv, H, HK, D, page, rot, inter, dtype)
    g = gen(D + rot)
    q_off, top = offsets(lens), cref.TOP[dtype]
    T = q_off[-1]
    c = make_cache4(g, kv, HK, D, page, dtype, token_major=inter)
    cache = on_gpu4(*c)
    qkv = normal(g, T, H + 2 * HK, D, dtype=dtype) * torch.exp(normal(g, 1, 1, D)).to(dtype)
    f, factor = fs.fs_rope_frequencies(rot, 10000.0, fs.FS_ROPE_PARTS, 4.0, 2048)
    inv, d = torch.from_numpy(f), qkv.cuda()
    q = fs.fs_rope_append4(step_of(lens, kv), cache, fs.Rope(inv.cuda(), inter, factor), d[:, :H],
                           d[:, H:H + HK], d[:, H + HK:])
    want = [x.clone() for x in c[:4]]
    factor = float(np.float32(factor))
    for s, pos in enumerate(ref.positions(q_off, kv)):
        rows = slice(q_off[s], q_off[s + 1])
        y, b = ref.rope_rows(qkv[rows, :H + HK], [max(0, p) for p in pos], inv, rot, inter, factor)
        within(q[rows], y[:, :H], b[:, :H], f"q of request {s}")
        live = [i for i, p in enumerate(pos) if p >= 0]
        if not live:
            continue
        # keys are turned in fp64 and rounded to fp32: their codes and scales are the oracle's
        kc, kb = cref.quantise(y[live, H:].astype(np.float32), top)
        vc, vb = cref.quantise(qkv[rows, H + HK:][live].float().numpy(), top)
        for i, at in enumerate(live):
            p = pos[at]
            where = (int(c[4][s, p // page]), slice(None), p % page)
            want[0][where], want[1][where] = cref.pack(kc[i]), cref.pack(vc[i])
            want[2][where], want[3][where] = torch.from_numpy(kb[i]), torch.from_numpy(vb[i])
    for got, x, name in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), want,
                            ("k", "v", "k_scale", "v_scale")):
        assert torch.equal(got.cpu(), x), name
    # in place, with positions of its own
    pos = torch.randint(0, 1 << 20, (T,), generator=g, dtype=torch.int32)
    q2 = d[:, :H]
    fs.fs_rope_append4(step_of(lens, kv), cache, fs.Rope(inv.cuda(), inter, factor, pos.cuda()), q2,
                       d[:, H:H + HK].clone(), d[:, H + HK:].clone(), q_out=q2)
    y, b = ref.rope_rows(qkv[:, :H], pos.numpy(), inv, rot, inter, factor)
    within(q2, y, b, "q in place")


@pytest.mark.parametrize("dtype", [BF, HF])
def test_append4_of_borders_extremes_and_broken_groups(dtype):
    """Values halfway between two codes, next to them, zeros, the type's largest and smallest
    numbers, infinities and NaN: codes and scales are the oracle's."""
    top, big = cref.TOP[dtype], float(torch.finfo(dtype).max)
    eps, tiny = float(torch.finfo(dtype).eps), float(torch.finfo(dtype).smallest_normal)
    mid = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    near = [m * (1 + s * eps) for m in mid for s in (-1, 0, 1)] + [6.0, 7.0, 6.5]
    rows = []
    for unit in (1.0, 2.0 ** -9, 2.0 ** 7):
        for most in (4.0, 6.0, 7.0 * (1 - eps), 7.0, 7.0 * (1 + eps), 7.5):
            rows.append([most * unit] + [x * unit * (-1) ** i for i, x in enumerate(near)] + [0.0] * 7)
    rows += [[0.0] * 32, [-0.0] * 32, [big] + [1.0] * 31, [-big, big / 2, big / 8] + [big / 32] * 29,
             [tiny] * 32, [tiny / 4, tiny / 2] + [0.0] * 30, [2 * tiny, tiny / 64] + [tiny] * 30,
             [math.inf] + [1.0] * 31, [1.0] * 31 + [-math.inf], [1.0] * 16 + [math.nan] + [2.0] * 15]
    x = torch.tensor(rows, dtype=torch.float64).to(dtype)
    n = x.shape[0]
    c = make_cache4(gen(1), [n], 1, 32, 16, dtype)
    cache = on_gpu4(*c)
    xd = x.cuda()[:, None]
    none = fs.Rope(torch.zeros(0, device="cuda"))
    fs.fs_rope_append4(step_of([n], [n]), cache, none, None, xd, xd.flip(0))
    code, byte = cref.quantise(x.float().numpy(), top)
    at, slot = c[4][0][torch.arange(n) // 16].long(), torch.arange(n) % 16
    bad = byte[:, 0] == 255
    for codes, scales, flip in ((cache.k, cache.k_scale, False), (cache.v, cache.v_scale, True)):
        got, gb = codes.cpu()[at, 0, slot].numpy(), scales.cpu()[at, 0, slot].numpy()
        got, gb = (got[::-1], gb[::-1]) if flip else (got, gb)
        assert np.array_equal(gb, byte)
        assert np.array_equal(got[~bad], cref.pack(code).numpy()[~bad])
    k, _ = fs.fs_cache4_rows(step_of([n], [n]), cache, dtype)
    assert bool(k[torch.from_numpy(bad).cuda()].isnan().all())
    assert bool(torch.isfinite(k[torch.from_numpy(~bad).cuda()]).all())


def test_append4_leaves_alone_what_is_not_its_own():
    """Bad pages and lengths raise the status word and nothing is written through them."""
    c = make_cache4(gen(3), [4, 9], 2, 64, 8, BF)
    kv = normal(gen(4), 3, 4, 64).cuda()
    rope = fs.Rope(torch.ones(32).cuda())
    cache = on_gpu4(*c)
    before = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    table = c[4].clone()
    table[1, 1] = c[0].shape[0]
    bad = fs.KVCache4(cache.k, cache.v, cache.k_scale, cache.v_scale, table.cuda())
    over = fs.Step([0, 1], kv_len=torch.tensor([10], dtype=torch.int32).cuda(), max_kv=9)
    for step, to in ((step_of([0, 1], [4, 9]), bad), (over, cache)):
        with pytest.raises(fs.FairServeError) as e:
            fs.fs_rope_append4(step, to, rope, None, kv[:1, :2], kv[:1, 2:])
        assert e.value.code == fs.FS_E_RANGE
        for a, b in zip(before, (cache.k, cache.v, cache.k_scale, cache.v_scale)):
            assert torch.equal(a, b)
        with pytest.raises(fs.FairServeError) as e:
            fs.fs_cache4_rows(step, to)
        assert e.value.code == fs.FS_E_RANGE


# ----------------------------------------------------------------- attention

ATTENTION = [
    # rows, cached lengths, heads, kv heads, dim, page, window, sinks
    ([1], [1], 1, 1, 64, 16, 0, 0),
    ([1, 1, 1], [5, 16, 333], 8, 2, 128, 16, 0, 0),
    ([1] * 5, [0, 1, 64, 65, 1000], 32, 8, 128, 16, 0, 3),
    ([1, 1], [5000, 70], 7, 1, 128, 32, 0, 0),
    ([1, 1, 1], [700, 3, 129], 16, 16, 64, 8, 100, 0),
    ([1], [40001], 8, 1, 64, 64, 0, 0),                   # split over a long context
    ([1, 1], [9000, 20], 64, 1, 128, 16, 4097, 5),
    ([3, 0, 1, 20], [3, 9, 50, 33], 6, 2, 64, 16, 0, 0),
    ([40, 130], [40, 400], 8, 2, 128, 16, 0, 0),
    ([65, 2, 1], [1000, 2, 600], 3, 3, 128, 4, 7, 2),
    ([200], [200], 8, 8, 64, 16, 0, 0),
    ([70, 5, 9], [64, 2, 9], 4, 1, 128, 1, 0, 0),         # padding rows ahead
    ([17, 33], [517, 33], 14, 2, 64, 128, 50, 16),
    ([5, 1, 2], [3000, 3000, 2500], 12, 4, 128, 16, 0, 0),
    ([4], [300], 64, 1, 64, 16, 0, 0),
    ([257], [771], 5, 1, 128, 16, 0, 0),
    ([300, 1, 3], [900, 2000, 700], 4, 2, 64, 16, 64, 40),
    ([261, 0, 77], [500, 9, 333], 64, 16, 128, 16, 150, 9),
    ([100], [4000], 4, 1, 128, 16, 0, 0),                 # chunks over split keys
    ([90, 80, 1], [2600, 700, 1500], 3, 3, 64, 32, 0, 0),
    ([65] * 67 + [1] * 3, [66 + 9 * i for i in range(66)] + [2500, 3, 0, 1400], 1, 1, 64, 16, 0, 0),  # > 64 requests
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,H,HK,D,page,window,sinks", ATTENTION)
def test_attention4(lens, kv, H, HK, D, page, window, sinks, dtype):
    say("attention4", lens[:6], kv[:6], H, HK, D, page, window, sinks, dtype)
    g = gen(H * 1000 + D + len(lens))
    q_off = offsets(lens)
    T = q_off[-1]
    c = make_cache4(g, kv, HK, D, page, dtype, token_major=page == 16)
    wide = normal(g, T, H + 2, D, dtype=dtype, std=2.0)
    q, scale = wide[:, 1:1 + H], 0.7 * D ** -0.5
    k, v = both_values(c, dtype)
    want, tol, lse, ltol = cref.attention(q, k, v, c[4], q_off, kv, scale, window, sinks)
    out = torch.full((T, H + 1, D), 9.0, dtype=dtype, device="cuda")
    step, cache, qd = step_of(lens, kv), on_gpu4(*c), wide.cuda()[:, 1:1 + H]
    o, l = fs.fs_paged_attention4(step, cache, qd, scale, window, sinks, out=out[:, :H], want_lse=True)
    within(o, want, tol, "out")
    empty = torch.isinf(lse)
    assert bool((l.cpu()[empty] == -math.inf).all())
    within(l.cpu()[~empty], lse[~empty], ltol[~empty], "lse")
    assert bool((out[:, H:] == 9).all())
    assert torch.equal(fs.fs_paged_attention4(step, cache, qd, scale, window, sinks), o)
    # a scale of the other sign
    want, tol, _, _ = cref.attention(q, k, v, c[4], q_off, kv, -scale, window, sinks)
    within(fs.fs_paged_attention4(step, cache, qd, -scale, window, sinks), want, tol, "out, flipped")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv", [([1, 2], [700, 30]), ([70, 1], [900, 40])])
def test_attention4_with_a_scale_of_zero(lens, kv, dtype):
    """Every visible token counts alike."""
    g = gen(41)
    c = make_cache4(g, kv, 1, 128, 16, dtype)
    k, v = both_values(c, dtype)
    q = normal(g, sum(lens), 2, 128, dtype=dtype)
    for scale in (0.0, -0.0):
        want, tol, lse, ltol = cref.attention(q, k, v, c[4], offsets(lens), kv, scale, 0, 0)
        o, l = fs.fs_paged_attention4(step_of(lens, kv), on_gpu4(*c), q.cuda(), scale, want_lse=True)
        within(o, want, tol, "out")
        within(l, lse, ltol, "lse")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,H,HK,D", [([1, 1], 4, 1, 128), ([1, 3], 16, 2, 64), ([4, 2], 8, 1, 128)])
def test_few_rows_keep_their_probabilities_to_two_parts(lens, H, HK, D, dtype):
    g = gen(D + H)
    kv = [40, 33]
    c = make_cache4(g, kv, HK, D, 16, dtype)
    k, v = both_values(c, dtype)
    q, q_off = normal(g, sum(lens), H, D, dtype=dtype), offsets(lens)
    want, tol, _, _ = cref.attention(q, k, v, c[4], q_off, kv, D ** -0.5, 0, 0)
    mag, _, _, _ = cref.attention(q, k, v.abs(), c[4], q_off, kv, D ** -0.5, 0, 0)
    u = ref.U16[dtype]
    # the bound has u |out| + (u + rel) (prob |V|): u^2 in the place of the second u
    bound = tol - (u - u * u) * mag
    assert bool((bound > 0).all())
    got = fs.fs_paged_attention4(step_of(lens, kv), on_gpu4(*c), q.cuda(), D ** -0.5)
    within(got, want, bound, "out")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,HK,D", [([1], [70001], 1, 64), ([2, 1], [66000, 130], 1, 128),
                                          ([1, 3], [140000, 90000], 1, 128)])
def test_attention4_of_very_many_splits(lens, kv, HK, D, dtype):
    g = gen(D + kv[0])
    c = make_cache4(g, kv, HK, D, 64, dtype)
    k, v = both_values(c, dtype)
    q, q_off = normal(g, sum(lens), 4, D, dtype=dtype), offsets(lens)
    want, tol, lse, ltol = cref.attention(q, k, v, c[4], q_off, kv, D ** -0.5, 0, 0)
    o, l = fs.fs_paged_attention4(step_of(lens, kv), on_gpu4(*c), q.cuda(), D ** -0.5, want_lse=True)
    within(o, want, tol, "out")
    within(l, lse, ltol, "lse")


@pytest.mark.parametrize("lens,kv", [([1, 1], [3000, 50]), ([60], [90])])
def test_attention4_with_a_loose_bound(lens, kv):
    """A host bound far above the lengths, and scores in the thousands."""
    g = gen(31)
    c = make_cache4(g, kv, 2, 128, 16, BF, spread=1)
    k, v = both_values(c, BF)
    q, q_off = normal(g, sum(lens), 8, 128, std=60.0), offsets(lens)
    want, tol, lse, ltol = cref.attention(q, k, v, c[4], q_off, kv, 0.5, 0, 0)
    wide = torch.full((len(kv), 4000), -1, dtype=torch.int32)
    wide[:, :c[4].shape[1]] = c[4]
    step = fs.Step(q_off, kv_len=torch.tensor(kv, dtype=torch.int32).cuda(), max_kv=60000)
    o, l = fs.fs_paged_attention4(step, on_gpu4(*c[:4], wide), q.cuda(), 0.5, want_lse=True)
    # Values are whole codes: where the largest score's one is 0, what is left is the others', whose
    # weights may lie beyond fp32.  An exponential is held in units of 2^-18 (and of up to 2^8
    # of the row's largest), so one below 2^-126 * 2^18 * 2^8 = 2^-100 of the largest may become
    # 0: each key loses less than 2^-100 of its value, at most 6 here (the scale bytes are at
    # most 2^-1), and the weights sum to one at least.
    tol = tol + max(kv) * 2.0 ** -100 * 6
    within(o, want, tol, "out")
    within(l, lse, ltol, "lse")


@pytest.mark.parametrize("lens,kv", [([1, 1, 1], [300, 90, 5000]), ([90, 80, 1], [150, 400, 40])])
def test_queries_that_are_not_finite_stay_in_their_rows(lens, kv):
    g = gen(32)
    c = make_cache4(g, kv, 2, 64, 16, HF)
    q = normal(g, sum(lens), 4, 64, dtype=HF)
    step, cache = step_of(lens, kv), on_gpu4(*c)
    want, wl = fs.fs_paged_attention4(step, cache, q.cuda(), 0.1, want_lse=True)
    q[0, 1, 3], q[sum(lens) - 1, 0, 60] = math.nan, math.inf
    out, lse = fs.fs_paged_attention4(step, cache, q.cuda(), 0.1, want_lse=True)
    touched = torch.zeros(sum(lens), 4, dtype=torch.bool)
    touched[0, 1] = touched[-1, 0] = True
    assert bool(out.cpu()[0, 1].isnan().all()) and bool(lse[0, 1].isnan())
    assert not bool(torch.isfinite(out.cpu()[-1, 0]).any())
    assert torch.equal(out.cpu()[~touched], want.cpu()[~touched])
    assert torch.equal(lse.cpu()[~touched], wl.cpu()[~touched])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("large", [1.0, 256.0, 2.0 ** 100])
def test_queries_of_chunks_keep_what_lies_far_below_their_largest_value(D, large):
    """The largest value of each group meets keys of 0, so the scores are the others'."""
    g, lens, kv = gen(D), [80], [150]
    c = make_cache4(g, kv, 1, D, 16, BF)
    c[0][..., ::16] &= 0xf0             # value 0 of each group of 32 is a zero
    q = normal(g, 80, 1, D, dtype=BF) * torch.exp2(-(torch.arange(D) % 23).float()).to(BF)
    q[..., ::32] = large
    k, v = both_values(c, BF)
    want, _, lse, ltol = cref.attention(q, k, v, c[4], [0, 80], kv, 1.0, 0, 0)
    _, l = fs.fs_paged_attention4(step_of(lens, kv), on_gpu4(*c), q.cuda(), 1.0, want_lse=True)
    within(l, lse, ltol, "lse")


@pytest.mark.parametrize("lens,kv", [([70, 1], [200, 40]), ([90], [3000]), ([70, 3], [64, 2])])
@pytest.mark.parametrize("D", [64, 128])
def test_a_nan_query_of_a_chunk_gives_nan_to_its_row(lens, kv, D):
    """A row that sees no token is 0 all the same."""
    g = gen(D + kv[0])
    c = make_cache4(g, kv, 1, D, 16, BF)
    q = normal(g, sum(lens), 1, D, dtype=BF)
    step, cache = step_of(lens, kv), on_gpu4(*c)
    want, wl = fs.fs_paged_attention4(step, cache, q.cuda(), 0.1, want_lse=True)
    rows = [0, 33, lens[0] - 1]
    for t, d in zip(rows, (0, D // 2 + 5, D - 1)):
        q[t, 0, d] = math.nan
    out, lse = fs.fs_paged_attention4(step, cache, q.cuda(), 0.1, want_lse=True)
    for t in range(sum(lens)):
        if t in rows and t + kv[0] - lens[0] >= 0:
            assert bool(out[t].isnan().all()) and bool(lse[t].isnan().all()), t
        else:
            assert torch.equal(out[t], want[t]) and torch.equal(lse[t], wl[t]), t
    if kv[0] < lens[0]:
        assert bool((out[0] == 0).all()) and float(lse[0, 0]) == -math.inf


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("byte", [1, 0, 30, 200, 252])
def test_attention4_of_far_scales(D, byte):
    """Keys of 0 weigh all values alike, however large or small these are (bfloat16's range)."""
    g = gen(D)
    lens, kv = [1, 70], [90, 200]
    k, v, ks, vs, table = make_cache4(g, kv, 1, D, 16, BF)
    k.zero_()
    vs[vs < 255] = byte
    c = (k, v, ks, vs, table)
    kk, vv = both_values(c, BF)
    q, q_off = normal(g, sum(lens), 2, D), offsets(lens)
    want, tol, _, _ = cref.attention(q, kk, vv, table, q_off, kv, 0.1, 0, 0)
    got = fs.fs_paged_attention4(step_of(lens, kv), on_gpu4(*c), q.cuda(), 0.1)
    if byte < 2:                               # (the type's smallest numbers may be lost)
        tol = tol + 6 * 2.0 ** -126
    within(got, want, tol, "out")


FORMS = [
    # rows, cached lengths, heads, kv heads, dim: whole and split, few rows and many, both at once
    ([1, 1, 1], [300, 90, 301], 8, 2, 128),
    ([1, 2, 1], [5000, 90, 2500], 4, 4, 64),
    ([40, 30], [200, 333], 6, 2, 128),
    ([90, 80], [1500, 4000], 3, 1, 64),
    ([90, 1, 2], [1500, 3000, 90], 6, 2, 64),
    ([300, 280], [400, 500], 32, 16, 128),
]


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,H,HK,D", FORMS)
def test_a_broken_group_stays_with_the_rows_that_see_it(lens, kv, H, HK, D, dtype, window, sinks):
    """A key's group that counts as NaN makes its rows NaN, a value's group the group's columns;
    rows (and heads) that do not see it are as without it."""
    say("broken", lens, kv, H, HK, D, dtype, window, sinks)
    g = gen(D + H)
    q_off, grp, page = offsets(lens), H // HK, 16
    c = list(make_cache4(g, kv, HK, D, page, dtype))
    q = normal(g, q_off[-1], H, D, dtype=dtype)
    step, scale = step_of(lens, kv), D ** -0.5
    plain, lplain = fs.fs_paged_attention4(step, on_gpu4(*c), q.cuda(), scale, window, sinks, want_lse=True)
    assert bool(torch.isfinite(plain).all())
    bad_v = [(0, kv[0] - 1, 0, D // 32 - 1), (1, max(0, kv[1] - 25), HK - 1, 0)]
    bad_k = [(len(lens) - 1, kv[-1] - 1, HK - 1, 1), (len(lens) - 1, 1, 0, 0)]
    c[2], c[3] = c[2].clone(), c[3].clone()
    for (s, j, m, grpno), x in [(b, c[3]) for b in bad_v] + [(b, c[2]) for b in bad_k]:
        x[int(c[4][s, j // page]), m, j % page, grpno] = cref.TOP[dtype] + 1
    out, lse = fs.fs_paged_attention4(step, on_gpu4(*c), q.cuda(), scale, window, sinks, want_lse=True)
    out, lse, plain, lplain = out.cpu(), lse.cpu(), plain.cpu(), lplain.cpu()
    for s, pos in enumerate(ref.positions(q_off, kv)):
        for i, p in enumerate(pos):
            at = set(cref.seen(p, kv[s], window, sinks))
            for h in range(H):
                t = q_off[s] + i
                if any(b[0] == s and b[1] in at and b[2] == h // grp for b in bad_k):
                    assert bool(out[t, h].isnan().all()) and bool(lse[t, h].isnan()), (t, h)
                    continue
                nan = torch.zeros(D, dtype=torch.bool)
                for b in bad_v:
                    if b[0] == s and b[1] in at and b[2] == h // grp:
                        nan[32 * b[3]:32 * b[3] + 32] = True
                assert torch.equal(out[t, h].isnan(), nan), (t, h)
                assert torch.equal(out[t, h][~nan], plain[t, h][~nan]) and lse[t, h] == lplain[t, h], (t, h)


def test_attention4_refuses_bad_pages_and_lengths():
    g = gen(14)
    for lens in ([1, 1], [70, 60]):
        kv = [90, 80]
        c = make_cache4(g, kv, 2, 64, 16, BF)
        q = normal(g, sum(lens), 4, 64).cuda()
        cache = on_gpu4(*c)
        for wrong in (c[0].shape[0], -1, 1 << 30):
            table = c[4].clone()
            table[1, 2] = wrong
            bad = fs.KVCache4(cache.k, cache.v, cache.k_scale, cache.v_scale, table.cuda())
            with pytest.raises(fs.FairServeError) as e:
                fs.fs_paged_attention4(step_of(lens, kv), bad, q, 0.1)
            assert e.value.code == fs.FS_E_RANGE
        for n in (-1, 91):
            step = fs.Step(offsets(lens), kv_len=torch.tensor([90, n], dtype=torch.int32).cuda(), max_kv=90)
            with pytest.raises(fs.FairServeError) as e:
                fs.fs_paged_attention4(step, cache, q, 0.1)
            assert e.value.code == fs.FS_E_RANGE


@pytest.mark.parametrize("lens", [[1, 1, 1], [50, 1, 20]])
def test_attention4_offsets_beyond_32_bits_and_shared_pages(lens):
    g = gen(12)
    D, HK, page, stride = 64, 1, 16, 1_700_000_000           # bytes between pages
    kv = [60, 50, 49]
    c = make_cache4(g, [160], HK, D, page, BF, extra=0)
    big = [torch.empty(3 * stride + 4096, dtype=torch.uint8, device="cuda") for _ in range(4)]
    ids = [0, 1, 2, 3]
    views = []
    for t, x, per in zip(big, c[:4], (D // 2, D // 2, D // 32, D // 32)):
        w = t.as_strided((4, HK, page, per), (stride, page * per, per, 1))
        w.copy_(x[ids].cuda())
        views.append(w)
    for x in views[2:]:
        x.clamp_(max=126)
    table = torch.tensor([[3, 0, 2, 1], [3, 0, 1, 2], [3, 2, 1, 0]], dtype=torch.int32)
    cache = fs.KVCache4(*views, table.cuda())
    host = [x.cpu() for x in views]
    k, v = cref.values(host[0], host[2], 252), cref.values(host[1], host[3], 252)
    q_off = offsets(lens)
    q = normal(g, q_off[-1], 4, D)
    want, tol, _, _ = cref.attention(q, k, v, table, q_off, kv, 0.1, 0, 0)
    within(fs.fs_paged_attention4(step_of(lens, kv), cache, q.cuda(), 0.1), want, tol, "out")
    kv_new = normal(g, q_off[-1], 2, D).cuda()
    table2 = torch.tensor([[0, 1, 2, 3]] * 3, dtype=torch.int32).cuda()
    one = fs.KVCache4(*views, table2)
    fs.fs_rope_append4(fs.Step([0, 2], kv_len=torch.tensor([64], dtype=torch.int32).cuda(), max_kv=64),
                       one, fs.Rope(torch.zeros(0, device="cuda")), None, kv_new[:2, :1], kv_new[:2, 1:])
    code, byte = cref.quantise(kv_new[:2, :1].float().cpu().numpy(), 252)
    assert torch.equal(views[0][3, :, 14:].cpu(), cref.pack(code).permute(1, 0, 2))
    assert torch.equal(views[2][3, :, 14:].cpu(), torch.from_numpy(byte).permute(1, 0, 2))


@pytest.mark.parametrize("lens,kv", [([1, 1], [3000, 50]), ([60, 100], [90, 1500])])
def test_attention4_in_a_graph_with_lengths_that_grow(lens, kv):
    """Replays with other lengths, pages and queries, eager work between them: each is the eager
    result."""
    g = gen(21)
    H, HK, D, page = 8, 2, 128, 16
    c = make_cache4(g, [n + 64 for n in kv], HK, D, page, BF)
    cache = on_gpu4(*c)
    q_off, T = offsets(lens), sum(lens)
    q = normal(g, T, H, D).cuda()
    kv_len = torch.tensor(kv, dtype=torch.int32).cuda()
    step = fs.Step(q_off, kv_len=kv_len, max_kv=max(kv) + 64)
    err, new = fs.cleared_err_word(), normal(g, T, 2 * HK, D).cuda()
    rope = fs.Rope(torch.rand(D // 2).cuda())
    need = fs._lib().fs_attention4_workspace(step.ref, cache.ref, H, 700, 4)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(T, H, device="cuda")

    def call(out, lse, ws):
        t = fs.fs_rope_append4(step, cache, rope, q, new[:, :HK], new[:, HK:], err=err, check=False)
        fs.fs_paged_attention4(step, cache, t, 0.09, 700, 4, out=out, lse=lse, ws=ws, err=err, check=False)

    call(out, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, lse, ws)
    for i in range(4):
        kv_len += 7
        q.normal_()
        new.normal_()
        graph.replay()
        torch.cuda.synchronize()
        o2, l2 = torch.empty_like(out), torch.empty_like(lse)
        call(o2, l2, torch.empty_like(ws))
        torch.cuda.synchronize()
        assert torch.equal(o2, out) and torch.equal(l2, lse), i
    assert int(err) == 0


def test_attention4_on_another_stream():
    g = gen(22)
    c = make_cache4(g, [500, 20], 2, 64, 16, HF)
    cache, q = on_gpu4(*c), normal(g, 2, 4, 64, dtype=HF).cuda()
    want = fs.fs_paged_attention4(step_of([1, 1], [500, 20]), cache, q, 0.1)
    s = torch.cuda.Stream()
    step = step_of([1, 1], [500, 20])
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        got = fs.fs_paged_attention4(step, cache, q, 0.1)
    assert torch.equal(got, want)
