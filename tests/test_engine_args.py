"""The engine step's operators: what is refused on the host (nothing is enqueued, no GPU
needed), the rotary frequencies, and the oracle of the GPU tests against plain cases."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import engine_ref as ref
import paper_2411_15997_amd as fs
from paper_2411_15997_amd import engine as E

A = fs.FS_E_ARG


def step(q_off=(0, 1, 3), max_kv=100, q_dev=256, kv=256):
    q = np.array(q_off, np.int32)
    s = E.fs_step(len(q_off) - 1, q.ctypes.data, q_dev, kv, max_kv)
    s.keep = q
    return s


def cache(**kw):
    v = dict(dtype=0, n_kv_heads=2, head_dim=64, page_size=16, n_pages=50, k=256, v=256,
             page_stride=2048, head_stride=1024, token_stride=64, table=256, table_stride=7)
    v.update(kw)
    return E.fs_kv_cache(**v)


def test_step_and_cache_arguments():
    lib = fs._lib()

    def attn(s=None, c=None, heads=4, scale=0.1, window=0, q=256, qs=256, out=256, os_=256,
             ws=256, wsb=1 << 30, err=16):
        s, c = s or step(), c or cache()
        return lib.fs_paged_attention(C.byref(s), C.byref(c), heads, scale, window, q, qs, out, os_,
                                      None, ws, wsb, err, None)

    for s in (step((1, 2)), step((0, 2, 1)), step(max_kv=-1), step(q_dev=None), step(kv=None),
              step((0, 1 << 30), max_kv=16), step((0, (1 << 24) + 1)),
              step([0] * 65537 + [1])):
        assert attn(s=s) == A
    for kw in (dict(dtype=2), dict(dtype=-1), dict(n_kv_heads=0), dict(head_dim=96),
               dict(head_dim=60), dict(head_dim=256), dict(page_size=0), dict(page_size=24),
               dict(page_size=8192), dict(n_pages=0), dict(page_stride=-8), dict(token_stride=68),
               dict(head_stride=1 << 31), dict(k=264), dict(v=None), dict(table=None),
               dict(table_stride=6)):
        assert attn(c=cache(**kw)) == A, kw
    for kw in (dict(heads=0), dict(heads=3), dict(heads=130), dict(scale=math.inf),
               dict(scale=math.nan), dict(window=-1), dict(q=None), dict(q=258), dict(qs=248),
               dict(qs=260), dict(out=None), dict(os_=255), dict(err=None)):
        assert attn(**kw) == A, kw
    assert lib.fs_paged_attention(None, None, 4, 0.1, 0, 256, 256, 256, 256, None, None, 0, 16,
                                  None) == A
    # a step without rows does nothing
    assert attn(s=step((0, 0, 0))) == fs.FS_OK and attn(s=step((0,))) == fs.FS_OK
    # few rows over a long context need a workspace
    long = step((0, 1), max_kv=200000)
    big = cache(n_pages=20000, table_stride=12500)
    need = lib.fs_attention_workspace(C.byref(long), C.byref(big), 4, 0)
    if need:
        assert attn(s=long, c=big, ws=None, wsb=0) == fs.FS_E_WORKSPACE
        assert attn(s=long, c=big, wsb=need - 1) == fs.FS_E_WORKSPACE
        assert attn(s=long, c=big, ws=128) == fs.FS_E_WORKSPACE


def test_rope_arguments():
    lib = fs._lib()

    def rope(rot=64, inter=0, f=256, heads=4, q=256, qs=256, k=256, ks=128, v=256, vs=128, out=256,
             os_=256, err=16, c=None, s=None):
        r = E.fs_rope(rot, inter, f, 1.0, None)
        s, c = s or step(), c or cache()
        return lib.fs_rope_append(C.byref(s), C.byref(c), C.byref(r), heads, q, qs, k, ks, v, vs,
                                  out, os_, err, None)

    for kw in (dict(rot=66), dict(rot=3), dict(rot=-2), dict(inter=2), dict(f=None), dict(heads=-1),
               dict(q=None), dict(qs=248), dict(qs=257), dict(k=None), dict(k=260), dict(ks=120),
               dict(v=None), dict(vs=132), dict(out=None), dict(os_=0), dict(err=None),
               dict(c=cache(head_dim=264)), dict(c=cache(dtype=2))):
        assert rope(**kw) == A, kw
    assert rope(s=step((0, 0))) == fs.FS_OK


def test_linear_arguments():
    lib = fs._lib()

    def lin(K=64, N=128, n=2, R=16, dtype=0, a=256, b=256, ad=256, x=256, xs=64, w=256, y=256,
            ys=128, ws=256, wsb=1 << 30, err=16):
        g = E.fs_adapters(dtype, K, N, n, R, a, b, None, None, ad)
        s = step()
        return lib.fs_adapter_linear(C.byref(s), C.byref(g), x, xs, w, y, ys, ws, wsb, err, None)

    for kw in (dict(K=60), dict(K=0), dict(N=4), dict(n=-1), dict(R=12), dict(R=136), dict(R=0),
               dict(dtype=2), dict(a=None), dict(b=264), dict(ad=None), dict(x=None), dict(x=248),
               dict(xs=56), dict(xs=68), dict(w=None), dict(y=None), dict(ys=120), dict(err=None)):
        assert lin(**kw) == A, kw
    assert lin(wsb=0) == fs.FS_E_WORKSPACE and lin(ws=None) == fs.FS_E_WORKSPACE


def test_sample_arguments():
    lib = fs._lib()
    p = E.fs_sampling(None, None, None, None)

    def sample(dtype=2, rows=2, vocab=100, x=256, stride=100, u=16, token=16, err=16, par=p,
               ws=256, wsb=1 << 30):
        return lib.fs_sample(dtype, rows, vocab, x, stride, None if par is None else C.byref(par), u,
                             token, None, None, ws, wsb, err, None)

    for kw in (dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(vocab=0), dict(vocab=(1 << 20) + 1),
               dict(x=None), dict(x=258), dict(stride=99), dict(u=None), dict(token=None),
               dict(err=None), dict(par=None)):
        assert sample(**kw) == A, kw
    assert sample(rows=0) == fs.FS_OK
    assert lib.fs_clear_status(None, None) == A


def test_binding_wants_one_device():
    m = torch.device("meta")
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    t = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        fs.KVCache(k, k, t.to(m))
    with pytest.raises(ValueError):
        fs.Sampling(torch.zeros(4), None, torch.zeros(4, device=m))
    step = fs.Step([0, 1], kv_len=t[0, :1].clone(), max_kv=5, device="cpu")
    with pytest.raises(ValueError):
        fs.fs_paged_attention(step, fs.KVCache(k, k, t), torch.zeros(1, 2, 64, dtype=k.dtype, device=m),
                              1.0)
    q = torch.zeros(1, 2, 64, dtype=k.dtype)
    rope = fs.Rope(torch.ones(32))
    for call in (lambda: fs.fs_paged_attention(step, fs.KVCache(k, k, t), q, 1.0),
                 lambda: fs.fs_rope_append(step, fs.KVCache(k, k, t), rope, q, q, q),
                 lambda: fs.fs_sample(q[0].float(), torch.zeros(2), fs.Sampling())):
        with pytest.raises(ValueError):                    # nothing of it is on a GPU
            call()


def test_binding_refuses_what_it_would_misread():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    t = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        fs.KVCache(k, k.transpose(1, 2), t)
    with pytest.raises(ValueError):
        fs.KVCache(k, k, t.long())
    with pytest.raises(ValueError):
        fs.KVCache(k, k, t.t())
    with pytest.raises(TypeError):
        fs.KVCache(k.double(), k.double(), t)
    a, b = torch.zeros(2, 8, 64), torch.zeros(2, 32, 16)
    with pytest.raises(ValueError):
        fs.Adapters(a, b, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        fs.Sampling(temperature=torch.zeros(4, dtype=torch.float64))


def test_rope_frequencies():
    f, m = fs.fs_rope_frequencies(64, 10000.0)
    want = 10000.0 ** (-np.arange(32) / 32.0)
    np.testing.assert_allclose(f, want, rtol=2.0 ** -23)
    assert m == 1.0
    f, m = fs.fs_rope_frequencies(64, 10000.0, fs.FS_ROPE_LINEAR, 4.0)
    np.testing.assert_allclose(f, want / 4, rtol=2.0 ** -23)
    f, m = fs.fs_rope_frequencies(64, 10000.0, fs.FS_ROPE_BASE, 4.0)
    assert f[0] == 1.0 and m == 1.0
    np.testing.assert_allclose(f[-1], want[-1] / 4, rtol=2.0 ** -22)
    f, m = fs.fs_rope_frequencies(64, 10000.0, fs.FS_ROPE_PARTS, 8.0, 4096, 32.0, 1.0)
    turns = 4096 * want / (2 * math.pi)
    np.testing.assert_allclose(f[turns >= 32], want[turns >= 32], rtol=2.0 ** -23)
    np.testing.assert_allclose(f[turns <= 1], want[turns <= 1] / 8, rtol=2.0 ** -23)
    assert (f <= want * (1 + 2.0 ** -23)).all() and (f >= want / 8 * (1 - 2.0 ** -23)).all()
    assert m == pytest.approx(0.1 * math.log(8.0) + 1, rel=2.0 ** -23)
    assert fs.fs_rope_frequencies(0)[0].shape == (0,)
    for bad in ((63,), (-2,), (64, 0.0), (64, math.nan), (64, 1e4, 4), (64, 1e4, 1, 0.5),
                (2, 1e4, 2, 2.0), (64, 1e4, 3, 2.0, 0), (64, 1e4, 3, 2.0, 10, 1.0, 1.0)):
        with pytest.raises(fs.FairServeError) as e:
            fs.fs_rope_frequencies(*bad)
        assert e.value.code == A


def test_oracle_on_cases_worked_by_hand():
    # two equal keys: the mean of the values; a window of one: the newest value
    q = torch.ones(1, 1, 64, dtype=torch.bfloat16)
    k = torch.ones(1, 1, 4, 64, dtype=torch.bfloat16)
    v = torch.arange(4.0)[None, None, :, None].expand(1, 1, 4, 64).to(torch.bfloat16)
    t = torch.zeros(1, 1, dtype=torch.int32)
    o, _, lse, _ = ref.attention(q, k, v, t, [0, 1], [2], 1.0, 0)
    assert o[0, 0, 0] == 0.5 and lse[0, 0] == pytest.approx(64 + math.log(2))
    o, _, _, _ = ref.attention(q, k, v, t, [0, 1], [4], 1.0, 1)
    assert o[0, 0, 0] == 3.0
    # weights 1, 1/2, 1/4 (logits ln 2 apart): W = 7/4
    x = np.array([0.0, math.log(2), -math.log(2)], np.float64)
    assert ref.sample_row(x, 0.0, 1.0, 0, 1.0, 0.0)[0] == 0
    assert ref.sample_row(x, 0.5, 1.0, 0, 1.0, 0.0)[0] == 1
    assert ref.sample_row(x, 0.9, 1.0, 0, 1.0, 0.0)[0] == 2
    assert ref.sample_row(x, 0.9, 1.0, 2, 1.0, 0.0)[::2] == (1, 2)
    assert ref.sample_row(x, 0.0, 1.0, 0, 0.5, 0.0)[::2] == (1, 1)
    assert ref.sample_row(x, 0.0, 1.0, 0, 0.6, 0.0)[::2] == (0, 2)
    assert ref.sample_row(x, 0.0, 1.0, 0, 1.0, 0.4)[::2] == (0, 2)
    # a quarter turn
    y, _ = ref.rope_rows(torch.tensor([[[1.0, 0.0]]], dtype=torch.bfloat16), [1],
                         torch.tensor([math.pi / 2]), 2, False, 1.0)
    np.testing.assert_allclose(y[0, 0], [0.0, 1.0], atol=1e-7)
