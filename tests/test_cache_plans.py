"""The workspace that attention over the caches asks for, on the host alone (no GPU needed): the
split of a call's work is a function of the step, the heads, the window and the sinks that count."""
import ctypes as C

import pytest

import paper_2411_15997_amd as fs
from test_engine_args import cache, step


@pytest.mark.parametrize("n,max_kv", [(64, 1000), (64, 513), (40, 1024), (3, 5000), (300, 2000), (1, 1)])
def test_sinks_that_do_not_count_leave_the_split_as_it_is(n, max_kv):
    """No window, or one that no length can fill: fs_paged_attention's own workspace, whatever
    the sinks (more than 256 requests times key/value heads among the cases)."""
    lib = fs._lib()
    s = step(tuple(range(n + 1)), max_kv=max_kv)
    c = cache(n_kv_heads=8, head_dim=128, page_stride=1 << 14, head_stride=2048, token_stride=128,
              n_pages=1 << 20, table_stride=-(-max_kv // 16))
    plain = lib.fs_attention_workspace(C.byref(s), C.byref(c), 32, 0)
    assert plain > 0 or max_kv <= 512 or n * 8 <= 256
    for window in (0, max_kv, max_kv + 1, 2 ** 31 - 1):
        for sinks in (0, 1, 4, max_kv, 2 ** 31 - 1):
            assert lib.fs_attention_sinks_workspace(C.byref(s), C.byref(c), 32, window, sinks) == plain, \
                (window, sinks)
