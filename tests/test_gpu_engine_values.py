"""Attention of values that are not finite, or far apart: NaN and infinities in queries and
keys, in every form of the call (single tokens and chunks, whole and split over keys)."""
import math

import pytest
import torch

import engine_ref as ref
import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_engine import BF, HF, gen, make_cache, normal, offsets, on_gpu, step_of, within

pytestmark = pytest.mark.gpu

FORMS = [
    # rows, cached lengths, heads, kv heads, dim: whole and split, few rows and many, both at once
    ([1, 1, 1], [300, 90, 301], 8, 2, 128),
    ([1, 2, 1], [5000, 90, 2500], 4, 4, 64),
    ([40, 30], [200, 333], 6, 2, 128),
    ([90, 80], [1500, 4000], 3, 1, 64),
    ([90, 1, 2], [1500, 3000, 90], 6, 2, 64),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,H,HK,D", FORMS)
def test_rows_with_scores_that_are_not_finite(lens, kv, H, HK, D, dtype):
    """A NaN score makes out and lse NaN; one of +inf makes out NaN (inf / inf) and lse +inf;
    scores of -inf weigh nothing.  Other heads and rows are as they were."""
    say("not finite", lens, kv, H, HK, D, dtype)
    g = gen(D + H)
    q_off, grp = offsets(lens), H // HK
    T = q_off[-1]
    k, v, table = make_cache(g, kv, HK, D, 16, dtype)
    q = normal(g, T, H, D, dtype=dtype)
    # element 0 of the queries is 1, and -1 in one row: a key's element 0 of inf then makes its
    # scores inf, and -inf in that row
    q[:, :, 0] = 1.0
    q[0, 0, 0] = -1.0
    nan_row = T - 1
    q[nan_row, H - 1, 3] = math.nan
    bad = min(kv[0] - lens[0], 7)                   # a key that every row of request 0 sees
    page = int(table[0, bad // 16])
    k[page, 0, bad % 16, 0] = math.inf
    if HK > 1:
        k[page, 1, bad % 16, 5] = math.nan
    scale = D ** -0.5
    out, lse = fs.fs_paged_attention(step_of(lens, kv), on_gpu(k, v, table), q.cuda(), scale,
                                     want_lse=True)
    out, lse = out.double().cpu(), lse.double().cpu()
    # what must not have changed: the oracle on finite inputs, the key of -inf scores left out
    kf, qf = k.clone(), q.clone()
    kf[page, 0, bad % 16, 0] = 0.0
    if HK > 1:
        kf[page, 1, bad % 16, 5] = 0.0
    qf[nan_row, H - 1, 3] = 0.0
    want, tol, wl, ltol = ref.attention(qf, kf, v, table, q_off, kv, scale, 0)
    for t in range(T):
        for h in range(H):
            first = t < lens[0]
            if (t, h) == (nan_row, H - 1) or (first and HK > 1 and h // grp == 1):
                assert bool(out[t, h].isnan().all()) and bool(lse[t, h].isnan()), (t, h, lse[t, h])
            elif first and h // grp == 0 and (t, h) != (0, 0):
                assert bool(out[t, h].isnan().all()) and lse[t, h] == math.inf, (t, h, lse[t, h])
            elif (t, h) != (0, 0):
                within(out[t, h], want[t, h], tol[t, h], f"out {t} {h}")
                within(lse[t, h], wl[t, h], ltol[t, h], f"lse {t} {h}")
    # row 0, head 0: without the key whose score is -inf
    p = kv[0] - lens[0]
    K = ref.kv_rows(kf, table[0], p + 1, 16, 0)
    sc = scale * K @ q[0, 0].double()
    sc[bad] = -math.inf
    V = ref.kv_rows(v, table[0], p + 1, 16, 0)
    prob = torch.softmax(sc, 0)
    u = ref.U16[dtype]
    rel = u + 2 * (D + 4) * ref.E32 * scale * float((K.abs() @ q[0, 0].double().abs()).max()) + \
        (p + 9) * ref.E32 + 2.0 ** -20
    bound = u * (prob @ V).abs() + rel * (prob @ V.abs()) + ref.TINY[dtype]
    if p > 0:
        within(out[0, 0], prob @ V, bound, "out without a key")
        within(lse[0, 0], torch.logsumexp(sc, 0), rel + 2 * ref.E32 * float(lse[0, 0].abs()), "lse")
    else:
        assert lse[0, 0] == -math.inf


def test_rows_without_a_key_are_empty_and_nothing_else():
    """-inf is the log-sum-exp of rows that see nothing, and of rows whose scores are all -inf."""
    g = gen(5)
    k, v, table = make_cache(g, [3, 40], 1, 64, 16, BF)
    k[int(table[1, 0]), 0, 0:16, 0] = -math.inf
    k[int(table[1, 1]), 0, 0:16, 0] = -math.inf
    k[int(table[1, 2]), 0, 0:8, 0] = -math.inf
    q = normal(g, 6, 2, 64)
    q[:, :, 0] = 1.0
    out, lse = fs.fs_paged_attention(step_of([5, 1], [3, 40]), on_gpu(k, v, table), q.cuda(), 0.1,
                                     want_lse=True)
    assert bool((lse[:2] == -math.inf).all()) and bool((out[:2] == 0).all())
    assert bool(torch.isfinite(lse[2:5]).all())
    assert bool((lse[5] == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,H,HK,D", [([1, 1], 4, 1, 128), ([1, 3], 16, 2, 64), ([4, 2], 8, 1, 128)])
def test_few_rows_keep_their_probabilities_to_two_parts(lens, H, HK, D, dtype):
    """Up to 32 rows: no rounding of a probability to 16 bits shows, only one of what a first
    rounding left (u^2) and the result's own."""
    g = gen(D + H)
    kv = [40, 33]
    k, v, table = make_cache(g, kv, HK, D, 16, dtype)
    q = normal(g, sum(lens), H, D, dtype=dtype)
    q_off = offsets(lens)
    want, tol, _, _ = ref.attention(q, k, v, table, q_off, kv, D ** -0.5, 0)
    u = ref.U16[dtype]
    mag, _, _, _ = ref.attention(q, k, v.abs(), table, q_off, kv, D ** -0.5, 0)
    # ref's bound has u |out| + (u + rel) (prob |V|): u^2 in the place of the second u
    bound = tol - (u - u * u) * mag
    assert bool((bound > 0).all())
    got = fs.fs_paged_attention(step_of(lens, kv), on_gpu(k, v, table), q.cuda(), D ** -0.5)
    within(got, want, bound, "out")


@pytest.mark.parametrize("lens", [[1, 1], [90, 1]])
def test_a_window_beyond_32_bits_is_none(lens):
    g = gen(6)
    k, v, table = make_cache(g, [200, 33], 2, 64, 16, BF)
    q = normal(g, sum(lens), 4, 64).cuda()
    step, cache = step_of(lens, [200, 33]), on_gpu(k, v, table)
    plain = fs.fs_paged_attention(step, cache, q, 0.2)
    for window in ((1 << 31), (1 << 32) + 3, 1 << 40):
        assert torch.equal(fs.fs_paged_attention(step, cache, q, 0.2, window=window), plain)
    for window in (-1, -(1 << 32) + 3):
        with pytest.raises(fs.FairServeError) as e:
            fs.fs_paged_attention(step, cache, q, 0.2, window=window)
        assert e.value.code == fs.FS_E_ARG


def test_calls_go_to_their_tensors_gpu(monkeypatch):
    """With another GPU current, each call makes its tensors' own one current: the handle of a
    default stream names no GPU.  (One GPU is enough to see that the call asks for it.)"""
    g = gen(7)
    k, v, table = make_cache(g, [30, 9], 2, 64, 16, BF)
    step, cache = step_of([1, 2], [30, 9]), on_gpu(k, v, table)
    qkv = normal(g, 3, 8, 64).cuda()
    q, kn, vn = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    x, w = normal(g, 3, 64).cuda(), normal(g, 72, 64).cuda()
    ad = fs.Adapters(normal(g, 1, 8, 64).cuda(), normal(g, 1, 72, 8).cuda(),
                     torch.tensor([0, -1], dtype=torch.int32).cuda())
    rope = fs.Rope(torch.ones(32).cuda())
    err = fs.cleared_err_word()
    calls = (lambda: fs.fs_adapter_linear(step, ad, x, w, err=err, check=False),
             lambda: fs.fs_rope_append(step, cache, rope, q, kn, vn, err=err, check=False),
             lambda: fs.fs_paged_attention(step, cache, q, 0.1, err=err, check=False),
             lambda: fs.fs_sample(x, torch.rand(3).cuda() * 0, fs.Sampling(), err=err, check=False)[0],
             lambda: fs.fs_clear_status(err))
    want = [c() for c in calls]
    entered, current, device = [], [0], torch.cuda.device

    class Spy(device):
        def __enter__(self):
            entered.append(self.idx)
            current[0] = self.idx
            return super().__enter__()

        def __exit__(self, *a):
            current[0] = 1
            return super().__exit__(*a)

    monkeypatch.setattr(fs.engine, "_current_gpu", lambda: current[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", Spy)
    for i, c in enumerate(calls):
        current[0], entered[:] = 1, []
        got = c()
        assert entered == [0], (i, entered)
        assert got is None or torch.equal(got, want[i]), i


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,D", [(1, 128), (1, 64), (70, 128), (70, 64)])
def test_many_small_probabilities_are_not_lost(rows, D, dtype):
    """One key of weight 1 and value 0, and 1,000 of weight 2^-26 and value 64: all of the result
    is theirs.  The bound: a probability of half precision counts in units of 2^-31, and is
    rounded to half of that; a result to its own unit; sums of fp32; 2^-20 for exponentials."""
    n, small = 1000, 2.0 ** -26
    kv = [n + 1 + rows - 1]
    k, v, table = make_cache(gen(9), kv, 1, D, 16, dtype)
    for j in range(kv[0]):
        at = (int(table[0, j // 16]), 0, j % 16)
        k[at], v[at] = 0.0, 64.0
        k[at][0] = -13.0
        if j == 0:
            k[at][0], v[at] = 13.0, 0.0
    q = torch.zeros(rows, 1, D, dtype=dtype)
    q[:, 0, 0] = 1.0
    out, lse = fs.fs_paged_attention(step_of([rows], kv), on_gpu(k, v, table), q.cuda(), math.log(2.0),
                                     want_lse=True)
    count = torch.arange(n, n + rows, dtype=torch.float64)[:, None, None]
    want = (64 * small * count / (1 + small * count)).expand(rows, 1, D)
    u = ref.U16[dtype]
    off = 2.0 ** -32 if dtype == HF else u * small
    rel = u + 2 * 30 * ref.E32 + (n + rows) * ref.E32 + 2.0 ** -20
    within(out, want, want * rel + 64 * count * off + ref.TINY[dtype], "out")
    within(lse[:, 0], 13 * math.log(2.0) + torch.log1p(small * count[:, 0, 0]),
           torch.full((rows,), 2 * 30 * ref.E32 + (n + rows) * ref.E32 + 2.0 ** -20), "lse")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,kv,H,HK,D,window", [
    ([3, 1], [40, 9], 8, 2, 128, 0),
    ([5, 7], [3, 60], 4, 4, 64, 0),                     # padding rows
    ([8, 20], [5000, 900], 8, 4, 64, 0),                # few rows, split
    ([30, 9], [2500, 70], 4, 2, 128, 1100),             # the same with a window
    ([16, 2], [100, 300], 16, 4, 128, 0),               # 64 rows
    ([90, 70], [90, 400], 6, 3, 128, 0),
    ([150, 2, 1], [3000, 30, 3], 3, 1, 64, 0),          # chunks, split, beside few rows
    ([150, 2], [3100, 1300], 4, 1, 128, 1050),
    ([300], [300], 2, 1, 64, 40),
    ([130, 300], [130, 700], 64, 32, 128, 0),           # 256 rows a work-group
])
def test_values_that_are_not_finite_stay_with_the_rows_that_see_them(lens, kv, H, HK, D, window, dtype):
    """V of NaN or infinities at places that some rows see and others do not."""
    say("values not finite", lens, kv, H, HK, D, window, dtype)
    g = gen(D + H + len(lens))
    k, v, table = make_cache(g, kv, HK, D, 16, dtype)
    q_off = offsets(lens)
    q = normal(g, q_off[-1], H, D, dtype=dtype)
    for s, (n, c) in enumerate(zip(lens, kv)):
        def put(j, head, cols, value):
            if 0 <= j < c:
                v[int(table[s, j // 16]), head, j % 16, cols] = value
        put(c - 1, 0, slice(3, 4), math.nan)                       # the newest token
        put(c - 1 - n // 2, HK - 1, slice(0, D), math.inf)         # one of the middle
        put(c - n // 3, HK - 1, slice(9, 11), -math.inf)
        if window:
            put(c - n - window + 2, 0, slice(20, 30), math.nan)    # in the first rows' windows alone
    want, tol, lse, ltol = ref.attention(q, k, v, table, q_off, kv, D ** -0.5, window)
    out = torch.full((q_off[-1], H, D), 99.0, dtype=dtype, device="cuda")
    out, got = fs.fs_paged_attention(step_of(lens, kv), on_gpu(k, v, table), q.cuda(), D ** -0.5, window,
                                     out=out, want_lse=True)
    out = out.double().cpu()
    fine = torch.isfinite(want)
    assert bool(fine.any()) and not bool(fine.all())
    assert not bool(torch.isfinite(out[~fine]).any())
    within(out[fine], want[fine], tol[fine], "out")
    some = torch.isfinite(lse)
    within(got.cpu()[some], lse[some], ltol[some], "lse")
    again = fs.fs_paged_attention(step_of(lens, kv), on_gpu(k, v, table), q.cuda(), D ** -0.5, window)
    assert torch.equal(again.double().cpu()[fine], out[fine])
