"""The oracle of calls with many heads against the row-by-row one (no GPU needed)."""
import pytest
import torch

import cache_ref as cref
import cache_wide_ref as wide


@pytest.mark.parametrize("window,sinks", [(0, 0), (7, 0), (7, 3), (20, 40), (1, 1)])
@pytest.mark.parametrize("lens,kv", [([1, 3, 0, 5], [9, 30, 4, 5]), ([6, 1], [4, 0]), ([17], [33])])
def test_both_oracles_agree(lens, kv, window, sinks):
    g = torch.Generator().manual_seed(len(lens) + window)
    q_off = [sum(lens[:i]) for i in range(len(lens) + 1)]
    page, HK, H, D = 4, 2, 6, 32
    table = torch.randperm(40, generator=g)[:len(lens) * 9].view(len(lens), 9).int()
    k, v = (torch.randn(40, HK, page, D, generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(q_off[-1], H, D, generator=g).to(torch.bfloat16)
    a = cref.attention(q, k, v, table, q_off, kv, 0.3, window, sinks)
    b = wide.attention(q, k, v, table, q_off, kv, 0.3, window, sinks)
    for x, y in zip(a, b):
        assert torch.equal(torch.isinf(x), torch.isinf(y))
        fine = torch.isfinite(x)
        assert bool(((x[fine] - y[fine]).abs() <= 1e-12 * (1 + x[fine].abs())).all())
