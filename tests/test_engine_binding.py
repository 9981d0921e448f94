"""The binding of the engine step's operators: what it refuses before anything is enqueued,
because the library could not see it (no GPU needed)."""
import numpy as np
import pytest
import torch

import paper_2411_15997_amd as fs

BF = torch.bfloat16


def cache(width, page=16, rows=2, of=None, at=0):
    """A cache whose page table is `width` columns of a table of `of` columns."""
    k = torch.zeros(4, 2, page, 64, dtype=BF)
    table = torch.zeros(rows, of or width, dtype=torch.int32)[:, at:at + width]
    return fs.KVCache(k, k.clone(), table)


def step(max_kv, rows=2):
    return fs.Step(list(range(rows + 1)), kv_len=torch.ones(rows, dtype=torch.int32), max_kv=max_kv,
                   device="cpu")


@pytest.mark.parametrize("width,of,at", [(4, 9, 0), (4, 9, 5), (4, 4, 0), (0, 3, 1)])
def test_lengths_keep_to_the_page_tables_width(width, of, at):
    """Columns of a wider table: its rows' distance is no width."""
    q, kv = torch.zeros(2, 4, 64, dtype=BF), torch.zeros(2, 2, 64, dtype=BF)
    rope = fs.Rope(torch.ones(32))
    calls = (lambda s, c: fs.fs_paged_attention(s, c, q, 1.0),
             lambda s, c: fs.fs_rope_append(s, c, rope, q, kv, kv))
    for call in calls:
        with pytest.raises(fs.FairServeError) as e:
            call(step(width * 16 + 1), cache(width, of=of, at=at))
        assert e.value.code == fs.FS_E_ARG
        with pytest.raises(ValueError, match="on one GPU"):           # up to the width: goes on
            call(step(width * 16), cache(width, of=of, at=at))


def test_a_steps_offsets_are_its_own():
    """A serving loop fills one array of offsets again for each step."""
    off = np.array([0, 1, 3], np.int32)
    s = fs.Step(off, kv_len=torch.ones(2, dtype=torch.int32), max_kv=4, device="cpu")
    off[:] = [0, 500, 1000]
    assert s.q_off_h.tolist() == [0, 1, 3] and s.rows == 3
    assert s.s.q_off_h == s.q_off_h.ctypes.data


BIG = 1 << 32


@pytest.mark.parametrize("make", [
    lambda: fs.Step([0, BIG + 1], kv_len=torch.ones(1, dtype=torch.int32), max_kv=4, device="cpu"),
    lambda: fs.Step(np.array([0, 1, BIG + 2]), max_kv=4, device="cpu"),
    lambda: fs.Step([0, 1], kv_len=torch.ones(1, dtype=torch.int32), max_kv=BIG + 16, device="cpu"),
    lambda: fs.KVCache(*[torch.empty(1, BIG + 1, 1, 8, dtype=BF, device="meta")] * 2,
                       torch.empty(1, 1, dtype=torch.int32, device="meta")),
    lambda: fs.Adapters(torch.empty(1, 8, BIG + 8, dtype=BF, device="meta"),
                        torch.empty(1, 64, 8, dtype=BF, device="meta"),
                        torch.empty(1, dtype=torch.int32, device="meta")),
    lambda: fs.Rope(torch.empty(BIG // 2 + 32, device="meta")),
    lambda: fs.fs_sample(torch.empty(BIG + 3, 1, dtype=BF, device="meta"),
                         torch.empty(BIG + 3, device="meta"), fs.Sampling()),
    lambda: fs.fs_sample(torch.empty(1, BIG + 3, dtype=BF, device="meta"),
                         torch.empty(1, device="meta"), fs.Sampling()),
])
def test_sizes_beyond_32_bits_are_refused(make):
    with pytest.raises(ValueError, match="beyond 32 bits"):
        make()


def test_a_workspace_is_as_large_as_it_says():
    """A view that repeats one byte has many values and little memory."""
    like = torch.zeros(1)
    _, _, n = fs.engine._workspace(torch.zeros(1000, dtype=torch.uint8), 500, like)
    assert n == 1000
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1000), torch.zeros(2000, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="ws: packed"):
            fs.engine._workspace(ws, 500, like)
