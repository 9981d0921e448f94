"""Several calls of the cache's operators beside each other: captured graphs that share a workspace,
and two streams at once."""
import pytest
import torch

import paper_2411_15997_amd as fs
from test_gpu_cache4 import make_cache4, on_gpu4
from test_gpu_engine import BF, HF, gen, make_cache, normal, on_gpu, step_of
from test_gpu_pages import i32

pytestmark = pytest.mark.gpu


def calls(dtype):
    """(name, its workspace's bytes, call(q, out, lse, ws), q) of attention that is split: few rows,
    chunks and both, over 4 bits and over 16 with sinks."""
    out = []
    for lens, kv in (([1, 2], [5000, 700]), ([100, 90], [2600, 1800]), ([90, 1, 3], [2600, 4000, 9])):
        g = gen(len(lens) + kv[0])
        q, step, err = normal(g, sum(lens), 8, 128, dtype=dtype).cuda(), step_of(lens, kv), fs.cleared_err_word()
        c4 = on_gpu4(*make_cache4(g, kv, 2, 128, 16, dtype))
        c16 = on_gpu(*make_cache(g, kv, 2, 128, 16, dtype))
        lib = fs._lib()

        def four(q, o, l, ws, step=step, c=c4, err=err):
            fs.fs_paged_attention4(step, c, q, 0.09, out=o, lse=l, ws=ws, err=err, check=False)

        def sinks(q, o, l, ws, step=step, c=c16, err=err):
            fs.fs_paged_attention(step, c, q, 0.09, 2400, out=o, lse=l, ws=ws, err=err, check=False, sinks=5)
        out.append((f"4 bits {lens}", lib.fs_attention4_workspace(step.ref, c4.ref, 8, 0, 0), four, q))
        out.append((f"sinks {lens}", lib.fs_attention_sinks_workspace(step.ref, c16.ref, 8, 2400, 5), sinks, q))
    assert all(n > 0 for _, n, _, _ in out)
    return out


@pytest.mark.parametrize("dtype", [BF, HF])
def test_graphs_that_share_a_workspace(dtype):
    """Replayed in turn, with eager calls between that use it too: each as with a workspace alone."""
    all_calls = calls(dtype)
    ws = torch.empty(max(n for _, n, _, _ in all_calls), dtype=torch.uint8, device="cuda")
    graphs = []
    for name, n, call, q in all_calls:
        o, l = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        call(q, o, l, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(q, o, l, ws)
        graphs.append((graph, o, l))
    for turn in range(3):
        for _, _, _, q in all_calls[::2]:
            q.normal_()
        for i in range(len(graphs)):
            graphs[(i * 5 + turn) % len(graphs)][0].replay()
            if i == turn:
                ws.fill_(255)
        torch.cuda.synchronize()
        for (name, n, call, q), (_, o, l) in zip(all_calls, graphs):
            o2, l2 = torch.empty_like(o), torch.empty_like(l)
            call(q, o2, l2, torch.full((n,), 255, dtype=torch.uint8, device="cuda"))
            assert torch.equal(o2, o) and torch.equal(l2, l), (name, turn)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_two_streams_at_once(dtype):
    """Calls over the same caches on two streams, a workspace for each."""
    all_calls = calls(dtype)
    want = []
    for name, n, call, q in all_calls:
        o, l = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        call(q, o, l, torch.empty(n, dtype=torch.uint8, device="cuda"))
        want.append((o, l))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    spaces = [torch.empty(max(n for _, n, _, _ in all_calls), dtype=torch.uint8, device="cuda") for _ in streams]
    outs = [[(torch.empty_like(o), torch.empty_like(l)) for o, l in want] for _ in range(6)]
    torch.cuda.synchronize()
    for turn, mine in enumerate(outs):
        for i, ((name, n, call, q), (o, l)) in enumerate(zip(all_calls, mine)):
            s = (i + turn) % 2
            with torch.cuda.stream(streams[s]):
                call(q, o, l, spaces[s])
    torch.cuda.synchronize()
    for mine in outs:
        for (name, *_), (o, l), (a, b) in zip(all_calls, mine, want):
            assert torch.equal(o, a) and torch.equal(l, b), name


def test_pools_on_two_streams_with_a_workspace_each():
    """Forks and compactions of two pools at once: as one after the other."""
    def pool():
        refs, table = [0] * 3000, torch.zeros(600, 8, dtype=torch.int32)
        table[0, :4] = torch.tensor([2990, 7, 2000, 13])
        for p in table[0, :4].tolist():
            refs[p] = 1
        return fs.PagePool(i32(refs), table.cuda(), i32([4] + [0] * 599), 16)

    def steps(p, ws, err):
        n = 300
        fs.fs_pages_fork(p, i32([0] * n), i32(list(range(1, n + 1))), i32([50] * n), i32([90] * n), ws=ws,
                         err=err, check=False)
        fs.fs_pages_free(p, i32(list(range(1, n + 1, 2))), err=err, check=False)
        fs.fs_pages_compact(p, ws=ws, err=err, check=False)

    pools, spaces = [pool() for _ in range(3)], [torch.empty(1 << 16, dtype=torch.uint8, device="cuda") for _ in range(3)]
    err = [fs.cleared_err_word() for _ in range(3)]
    steps(pools[0], spaces[0], err[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s, p, ws, e in zip(streams, pools[1:], spaces[1:], err[1:]):
        with torch.cuda.stream(s):
            steps(p, ws, e)
    torch.cuda.synchronize()
    assert [int(e) for e in err] == [0, 0, 0]
    for p in pools[1:]:
        for a, b in ((p.refs, pools[0].refs), (p.table, pools[0].table), (p.held, pools[0].held)):
            assert torch.equal(a, b)
    live = int((pools[0].refs > 0).sum())
    # row 0's four pages, three of them shared, and of 150 forks three pages of their own each
    assert live == 4 + 150 * 3 and int(pools[0].held.sum()) == 4 + 150 * 6
