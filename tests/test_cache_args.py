"""The cache's operators: what is refused on the host (nothing is enqueued, no GPU needed), by
the library and by the binding, and the oracle of the GPU tests against plain cases."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import cache_ref as cref
import paper_2411_15997_amd as fs
from paper_2411_15997_amd import cache as CA
from paper_2411_15997_amd import engine as E
from test_engine_args import cache, step

A = fs.FS_E_ARG


def cache4(**kw):
    v = dict(n_kv_heads=2, head_dim=64, page_size=16, n_pages=50, k=256, v=256, page_stride=1024,
             head_stride=512, token_stride=32, k_scale=3, v_scale=5, scale_page_stride=64,
             scale_head_stride=32, scale_token_stride=2, table=256, table_stride=7)
    v.update(kw)
    return CA.fs_kv_cache4(**v)


BAD_CACHE4 = [dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=48), dict(head_dim=0),
              dict(head_dim=288), dict(page_size=0), dict(page_size=24), dict(page_size=8192),
              dict(n_pages=0), dict(page_stride=-16), dict(token_stride=40), dict(head_stride=8),
              dict(page_stride=1 << 31), dict(token_stride=1 << 27), dict(scale_page_stride=-1),
              dict(scale_head_stride=1 << 31), dict(scale_token_stride=1 << 27), dict(k=264),
              dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(table=None),
              dict(table_stride=6), dict(table_stride=-1)]


def test_attention4_arguments():
    lib = fs._lib()

    def attn(s=None, c=None, dtype=0, heads=4, scale=0.1, window=0, sinks=0, q=256, qs=256, out=256,
             os_=256, ws=256, wsb=1 << 30, err=16):
        s, c = s or step(), c or cache4()
        return lib.fs_paged_attention4(C.byref(s), C.byref(c), dtype, heads, scale, window, sinks, q,
                                       qs, out, os_, None, ws, wsb, err, None)

    for s in (step((1, 2)), step((0, 2, 1)), step(max_kv=-1), step(q_dev=None), step(kv=None)):
        assert attn(s=s) == A
    for kw in BAD_CACHE4 + [dict(head_dim=96, token_stride=48)]:
        assert attn(c=cache4(**kw)) == A, kw
    for kw in (dict(dtype=2), dict(dtype=-1), dict(heads=0), dict(heads=3), dict(heads=130),
               dict(scale=math.inf), dict(scale=math.nan), dict(window=-1), dict(sinks=-1),
               dict(q=None), dict(q=258), dict(qs=248), dict(qs=260), dict(out=None), dict(os_=255),
               dict(err=None)):
        assert attn(**kw) == A, kw
    assert lib.fs_paged_attention4(None, None, 0, 4, 0.1, 0, 0, 256, 256, 256, 256, None, None, 0, 16,
                                   None) == A
    assert attn(s=step((0, 0, 0))) == fs.FS_OK and attn(s=step((0,))) == fs.FS_OK
    long, big = step((0, 1), max_kv=200000), cache4(n_pages=20000, table_stride=12500)
    need = lib.fs_attention4_workspace(C.byref(long), C.byref(big), 4, 0, 0)
    assert need > 0
    assert attn(s=long, c=big, ws=None, wsb=0) == fs.FS_E_WORKSPACE
    assert attn(s=long, c=big, wsb=need - 1) == fs.FS_E_WORKSPACE
    assert attn(s=long, c=big, ws=128) == fs.FS_E_WORKSPACE
    assert lib.fs_attention4_workspace(C.byref(long), C.byref(big), 3, 0, 0) == 0


def test_append4_and_rows_arguments():
    lib = fs._lib()

    def rope(rot=64, inter=0, f=256, dtype=0, heads=4, q=256, qs=256, k=256, ks=128, v=256, vs=128,
             out=256, os_=256, err=16, c=None, s=None):
        r = E.fs_rope(rot, inter, f, 1.0, None)
        s, c = s or step(), c or cache4()
        return lib.fs_rope_append4(C.byref(s), C.byref(c), C.byref(r), dtype, heads, q, qs, k, ks, v,
                                   vs, out, os_, err, None)

    def rows(dtype=0, k=256, ks=128, v=256, vs=128, err=16, c=None, s=None):
        s, c = s or step(), c or cache4()
        return lib.fs_cache4_rows(C.byref(s), C.byref(c), dtype, k, ks, v, vs, err, None)

    for kw in (dict(rot=66), dict(rot=3), dict(rot=-2), dict(inter=2), dict(f=None), dict(dtype=2),
               dict(heads=-1), dict(q=None), dict(qs=248), dict(qs=257), dict(k=None), dict(k=260),
               dict(ks=120), dict(v=None), dict(vs=132), dict(out=None), dict(os_=0), dict(err=None)):
        assert rope(**kw) == A, kw
    for kw in (dict(dtype=2), dict(k=264), dict(ks=120), dict(v=8), dict(vs=129), dict(err=None)):
        assert rows(**kw) == A, kw
    for kw in BAD_CACHE4:
        assert rope(c=cache4(**kw)) == A and rows(c=cache4(**kw)) == A, kw
    assert rope(s=step((0, 0, 0))) == fs.FS_OK and rows(s=step((0, 0, 0))) == fs.FS_OK
    assert rows(k=None, v=None) == fs.FS_OK


def test_sinks_arguments():
    lib = fs._lib()

    def attn(s=None, c=None, heads=4, scale=0.1, window=5, sinks=2, q=256, qs=256, out=256, os_=256,
             ws=256, wsb=1 << 30, err=16):
        s, c = s or step(), c or cache()
        return lib.fs_paged_attention_sinks(C.byref(s), C.byref(c), heads, scale, window, sinks, q, qs,
                                            out, os_, None, ws, wsb, err, None)

    for kw in (dict(heads=0), dict(heads=3), dict(scale=math.nan), dict(window=-1), dict(sinks=-1),
               dict(q=None), dict(qs=248), dict(out=None), dict(os_=255), dict(err=None),
               dict(c=cache(dtype=2)), dict(s=step((0, 2, 1)))):
        assert attn(**kw) == A, kw
    assert attn(s=step((0, 0, 0))) == fs.FS_OK
    long, big = step((0, 1), max_kv=200000), cache(n_pages=20000, table_stride=12500)
    need = lib.fs_attention_sinks_workspace(C.byref(long), C.byref(big), 4, 150000, 8)
    assert need > 0 and attn(s=long, c=big, window=150000, wsb=need - 1) == fs.FS_E_WORKSPACE


def pool(**kw):
    v = dict(n_pages=50, page_size=16, n_rows=4, width=7, refs=256, table=256, held=256, table_stride=7)
    v.update(kw)
    return CA.fs_pages(**v)


def test_pages_arguments():
    lib = fs._lib()
    ok = 1 << 20

    def free(p=None, n=2, rows=256, err=16):
        return lib.fs_pages_free(C.byref(p or pool()), n, rows, err, None)

    def fork(p=None, n=2, parent=256, child=256, shared=256, room=256, src=256, dst=256, ws=256,
             wsb=ok, err=16):
        return lib.fs_pages_fork(C.byref(p or pool()), n, parent, child, shared, room, src, dst, ws,
                                 wsb, err, None)

    def compact(p=None, refs=256, table=512, stride=7, src=256, dst=256, count=256, ws=256, wsb=ok,
                err=16):
        return lib.fs_pages_compact(C.byref(p or pool()), refs, table, stride, src, dst, count, ws, wsb,
                                    err, None)

    for kw in (dict(n_pages=0), dict(n_pages=(1 << 24) + 1), dict(page_size=0), dict(page_size=12),
               dict(page_size=8192), dict(n_rows=-1), dict(n_rows=65536), dict(width=-1),
               dict(width=(1 << 30) + 1), dict(refs=None), dict(table=None), dict(held=None),
               dict(table_stride=6)):
        assert free(p=pool(**kw)) == fork(p=pool(**kw)) == compact(p=pool(**kw)) == A, kw
        assert lib.fs_pages_workspace(C.byref(pool(**kw)), 2) == 0
    for kw in (dict(n=-1), dict(rows=None), dict(err=None)):
        assert free(**kw) == A, kw
    for kw in (dict(n=-1), dict(n=65536), dict(parent=None), dict(child=None), dict(shared=None),
               dict(room=None), dict(src=None), dict(dst=None), dict(err=None)):
        assert fork(**kw) == A, kw
    for kw in (dict(refs=None), dict(table=None), dict(stride=6), dict(src=None), dict(dst=None),
               dict(count=None), dict(err=None), dict(table=256, stride=8)):
        assert compact(**kw) == A, kw
    need = lib.fs_pages_workspace(C.byref(pool()), 2)
    for call in (fork, compact):
        assert call(ws=None) == call(ws=100) == fs.FS_E_WORKSPACE
    assert fork(wsb=need - 1) == fs.FS_E_WORKSPACE
    assert free(n=0) == fork(n=0) == fs.FS_OK


def test_copy_arguments():
    lib = fs._lib()
    for fn, make, bad in ((lib.fs_pages_copy, cache, dict(dtype=1)),
                          (lib.fs_pages_copy4, cache4, dict(scale_head_stride=64))):
        def copy(*caches, layers=None, n=2, src=256, dst=256, err=16):
            arr = (type(make()) * max(1, len(caches)))(*caches)
            return fn(C.byref(arr), len(caches) if layers is None else layers, n, src, dst, None, err,
                      None)
        assert copy(make(), layers=-1) == copy(make(), layers=65537) == A
        assert copy(make(), n=-1) == copy(make(), n=(1 << 24) + 1) == copy(make(), src=None) == A
        assert copy(make(), dst=None) == copy(make(), err=None) == A
        assert copy(make(), n=0) == copy(layers=0) == fs.FS_OK
        for kw in (bad, dict(n_kv_heads=1), dict(page_size=8), dict(n_pages=49), dict(page_stride=4096),
                   dict(k=None), dict(v=264), dict(head_dim=512)):
            assert copy(make(), make(**kw)) == A, kw
        assert fn(None, 1, 2, 256, 256, None, 16, None) == A


# ----------------------------------------------------------------- the binding

U8, I32 = torch.uint8, torch.int32


def tensors4(D=64, table=None):
    k = torch.zeros(4, 2, 16, D // 2, dtype=U8)
    s = torch.zeros(4, 2, 16, D // 32, dtype=U8)
    return k, k.clone(), s, s.clone(), torch.zeros(2, 4, dtype=I32) if table is None else table


def test_cache4_takes_what_the_library_cannot_check():
    good = tensors4()
    fs.KVCache4(*good)
    wide = torch.zeros(4, 2, 16, 4, dtype=U8)
    for i, t in ((0, good[0].to(torch.int8)), (1, good[1][:, :1]), (1, good[1].transpose(0, 0)[:, :, :, ::2]),
                 (2, wide), (2, wide[..., ::2]), (3, good[3].float()), (0, torch.zeros(4, 2, 16, 24, dtype=U8)),
                 (4, good[4].long()), (4, good[4][0]), (4, torch.zeros(2, 8, dtype=I32)[:, ::2]),
                 (4, torch.zeros(1, 4, dtype=I32).expand(2, 4))):
        t5 = list(good)
        t5[i] = t
        with pytest.raises(ValueError):
            fs.KVCache4(*t5)


def a_step(max_kv, rows=2):
    return fs.Step(list(range(rows + 1)), kv_len=torch.ones(rows, dtype=I32), max_kv=max_kv, device="cpu")


def test_calls_over_cache4_keep_to_the_table_and_to_types():
    c = fs.KVCache4(*tensors4(table=torch.zeros(2, 9, dtype=I32)[:, :4]))
    q, kv = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    rope = fs.Rope(torch.ones(32))
    calls = (lambda s, c: fs.fs_paged_attention4(s, c, q, 1.0),
             lambda s, c: fs.fs_rope_append4(s, c, rope, q, kv, kv),
             lambda s, c: fs.fs_cache4_rows(s, c))
    for call in calls:
        with pytest.raises(fs.FairServeError) as e:
            call(a_step(65), c)
        assert e.value.code == A
        with pytest.raises(ValueError, match="on one GPU"):
            call(a_step(64), c)
        with pytest.raises(ValueError, match="a row for every request"):
            call(a_step(4, rows=3), c)
    with pytest.raises(TypeError):
        fs.fs_paged_attention4(a_step(4), c, q.float(), 1.0)
    with pytest.raises(TypeError):
        fs.fs_rope_append4(a_step(4), c, rope, None, kv.float(), kv.float())
    with pytest.raises(ValueError):
        fs.fs_rope_append4(a_step(4), c, rope, None, kv, kv.half())
    with pytest.raises(TypeError):
        fs.fs_cache4_rows(a_step(4), c, torch.float32)
    with pytest.raises(ValueError):
        fs.fs_paged_attention4(a_step(4), c, torch.zeros(2, 4, 128, dtype=torch.float16), 1.0)


def test_pools_and_layers_of_the_binding():
    refs, table, held = torch.zeros(9, dtype=I32), torch.zeros(2, 4, dtype=I32), torch.zeros(2, dtype=I32)
    p = fs.PagePool(refs, table, held, 16)
    for bad in ((refs.long(), table, held), (refs, table.long(), held), (refs, table, held[:1]),
                (refs, table, held.float()), (refs, table[0], held), (refs[::2], table, held),
                (refs, torch.zeros(2, 8, dtype=I32)[:, ::2], held)):
        with pytest.raises(ValueError):
            fs.PagePool(*bad, 16)
    ids = torch.zeros(2, dtype=I32)
    for call in (lambda: fs.fs_pages_free(p, ids), lambda: fs.fs_pages_fork(p, ids, ids, ids, ids),
                 lambda: fs.fs_pages_compact(p)):
        with pytest.raises(ValueError, match="on one GPU"):
            call()
    c4, c16 = fs.KVCache4(*tensors4()), fs.KVCache(*[torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)] * 2, table)
    fs.CacheLayers([c4, c4])
    for bad in ([], [c4, c16], [table]):
        with pytest.raises(ValueError):
            fs.CacheLayers(bad)
    with pytest.raises(ValueError, match="on one GPU"):
        fs.fs_pages_copy(c16, ids, ids)


# ----------------------------------------------------------------- the oracle

def test_oracle_of_the_format():
    x = np.zeros((1, 32), np.float32)
    x[0, :9] = [7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.01]
    code, byte = cref.quantise(x, 252)
    assert byte[0, 0] == 127 and code[0, :9].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 15]
    x[0, 0] = np.nextafter(np.float32(7), np.float32(8))
    assert cref.quantise(x, 252)[1][0, 0] == 128
    x[0, 0] = np.inf
    assert cref.quantise(x, 252)[1][0, 0] == 255
    assert cref.quantise(np.zeros((1, 32), np.float32), 252)[1][0, 0] == 1
    rng = np.random.default_rng(1)
    for scale in (1e-4, 1.0, 300.0):
        x = (rng.standard_normal((50, 64)) * scale).astype(np.float32)
        code, byte = cref.quantise(x, 252)
        y = cref.values(cref.pack(code), torch.from_numpy(byte), 252).numpy()
        unit = np.repeat(2.0 ** (byte.astype(float) - 127), 32, 1)
        assert (np.abs(y - x) <= unit).all()
        small = np.abs(x) <= 2 * unit              # steps of a half there
        assert (np.abs(y - x)[small] <= unit[small] / 4).all()


def test_oracle_of_what_a_row_sees():
    assert cref.seen(9, 10, 3, 2) == [0, 1, 7, 8, 9]
    assert cref.seen(3, 10, 3, 2) == [0, 1, 2, 3]
    assert cref.seen(4, 10, 3, 8) == [0, 1, 2, 3, 4]
    assert cref.seen(4, 10, 0, 8) == [0, 1, 2, 3, 4]


def test_oracle_of_the_pool():
    p = cref.Pool(10, 4, 3, 5)
    assert p.fork([-1], [0], [0], [10]) == ([-1], [-1])
    assert p.fork([0, 0], [1, 2], [6, 8], [8, 9]) == ([1, -1], [3, -1])
    assert p.table[1][:2] == [0, 3] and p.table[2][:3] == [0, 1, 4] and p.refs[:5] == [3, 2, 1, 1, 1]
    p.free([0])
    assert p.refs[:5] == [2, 1, 0, 1, 1]
    assert p.compact() == ([4], [2]) and p.table[2][:3] == [0, 1, 2]
