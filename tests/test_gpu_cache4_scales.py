"""Attention over the 4-bit cache in half precision at the ends of that type's range: groups whose
values are subnormal halves, and the largest scales that count."""
import pytest
import torch

import cache_ref as cref
import paper_2411_15997_amd as fs
from gpu_common import say
from test_gpu_cache4 import both_values, make_cache4, on_gpu4
from test_gpu_engine import HF, gen, normal, offsets, step_of, within

pytestmark = pytest.mark.gpu

# few rows, 33 to 64 of them, chunks; single and several splits
LENS = [([1, 2], [90, 40]), ([1], [5000]), ([20], [300]), ([70], [200]), ([100], [1500])]


@pytest.mark.parametrize("lens,kv", LENS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("byte", [104, 108, 113, 140])
def test_values_of_far_scales_in_half_precision(lens, kv, D, byte):
    """Positive values that are all of one far scale (2^-23 to 2^13): exact in the type, so weighed
    as any others."""
    say("far values", lens, kv, D, byte)
    g = gen(D + byte)
    k, v, ks, vs, table = make_cache4(g, kv, 1, D, 16, HF)
    v &= 0x77
    vs[vs < 255] = byte
    kk, vv = both_values((k, v, ks, vs, table), HF)
    q, q_off = normal(g, sum(lens), 2, D, dtype=HF), offsets(lens)
    want, tol, lse, ltol = cref.attention(q, kk, vv, table, q_off, kv, 0.1, 0, 0)
    assert byte == 104 or bool((want.abs() > 4 * tol).all())
    o, l = fs.fs_paged_attention4(step_of(lens, kv), on_gpu4(k, v, ks, vs, table), q.cuda(), 0.1, want_lse=True)
    within(o, want, tol, "out")
    within(l, lse, ltol, "lse")


@pytest.mark.parametrize("lens,kv", LENS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("byte,size", [(104, 2.0 ** 12), (108, 2.0 ** 10), (113, 2.0 ** 8), (140, 2.0 ** -14)])
def test_keys_of_far_scales_in_half_precision(lens, kv, D, byte, size):
    """Keys of one far scale and queries that bring their scores to the size of others."""
    say("far keys", lens, kv, D, byte)
    g = gen(D + byte)
    k, v, ks, vs, table = make_cache4(g, kv, 1, D, 16, HF)
    ks[ks < 255] = byte
    kk, vv = both_values((k, v, ks, vs, table), HF)
    q, q_off = normal(g, sum(lens), 2, D, dtype=HF, std=size), offsets(lens)
    scale = 0.1 / (size * 2.0 ** (byte - 127))
    want, tol, lse, ltol = cref.attention(q, kk, vv, table, q_off, kv, scale, 0, 0)
    o, l = fs.fs_paged_attention4(step_of(lens, kv), on_gpu4(k, v, ks, vs, table), q.cuda(), scale, want_lse=True)
    within(o, want, tol, "out")
    within(l, lse, ltol, "lse")
