"""The example that plays the literal engine's schedule with the engine-step operators:
every admitted call gets its output tokens within the engine's KV capacity, and decoding
token by token gives what prefilling the same tokens at once gives."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2411_15997_amd as fs
from gpu_common import say

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("engine_steps",
                                                  os.path.join(ROOT, "examples", "engine_steps.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.gpu
def test_schedule_is_played_out():
    ex = example()
    model, tr, done, s = ex.play(requests=40, layers=1)
    say("engine steps", s)
    assert len(done) == s["admitted"] > 0
    for g, r in done.items():
        assert len(r["out"]) == max(int(tr.len_out[g]), 1)
        assert all(0 <= t < model.vocab for t in r["out"])
    # the engine's admissions keep to its capacity (one larger call may run alone)
    assert s["most_tokens"] <= max(s["cap"], s["largest"])


@pytest.mark.gpu
def test_decoding_matches_prefilling():
    """Two layers round to bfloat16 (unit roundoff 2^-8) at some sixteen places a token; the
    two orders of work differ by those roundings at most: 2^-5 of the logits' norm."""
    ex = example()
    pages = 200
    rng = np.random.default_rng(4)
    model = ex.Decoder(3, pages, layers=2, seed=9)
    lens, more = [37, 5, 130], 12
    ids = [rng.integers(0, model.vocab, n + more).tolist() for n in lens]
    tables = rng.permutation(pages)[:2 * 3 * 10].reshape(2, 3, 10).astype(np.int32)
    app = [0, 2, 1]
    err = fs.cleared_err_word()
    u = torch.zeros(3, device="cuda")
    greedy = fs.Sampling(temperature=torch.zeros(3, device="cuda"))

    def run(new, kv, table):
        q_off = [0] + list(np.cumsum([len(x) for x in new]))
        return model.step([t for x in new for t in x], q_off, kv, table, app, u, greedy, err)

    _, whole = run(ids, [n + more for n in lens], tables[0])
    run([x[:n] for x, n in zip(ids, lens)], lens, tables[1])
    for i in range(more):
        token, one = run([[x[n + i]] for x, n in zip(ids, lens)], [n + i + 1 for n in lens], tables[1])
    assert fs.fs_sync_status(err) == fs.FS_OK
    a, b = whole.double(), one.double()
    off = ((a - b).norm(dim=1) / a.norm(dim=1)).max().item()
    say("decode against prefill", off)
    assert off <= 2.0 ** -5
    assert (token.cpu() == one.float().cpu().argmax(1)).all()
