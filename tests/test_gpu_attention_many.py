"""is_attention on batches of more than a wave of sequences with row tiles among them, and on chunks whose keys are cut into more than a
wave of pieces."""
import numpy as np
import pytest
import torch

import paper_2405_14597_amd as P
from test_gpu_attention import DEV, check, make, oracle, run

pytestmark = pytest.mark.gpu


def lengths(n, seed):
    """Rows of n sequences: many of one or none, every ninth a prompt of 20 to 150, the last among them."""
    g = np.random.default_rng(seed)
    rows = g.integers(0, 3, n)
    rows[8::9] = g.integers(20, 150, len(rows[8::9]))
    rows[-1] = 141
    return rows.tolist()


@pytest.mark.parametrize("hq,hk,d", [(4, 2, 64), (8, 1, 128), (3, 3, 64)])
@pytest.mark.parametrize("n", [65, 100, 193])
def test_row_tiles_of_many_sequences(n, hq, hk, d):
    rows = lengths(n, n + d)
    g = np.random.default_rng(n)
    # with pasts, some without keys or with fewer than rows
    seqs = [(r, int(k)) for r, k in zip(rows, np.array(rows) + g.integers(-5, 120, n).clip(min=-np.array(rows)))]
    c = make(seqs, hq, hk, d, n, gap=1, tail=3)
    for causal in (True, False):
        print("many", n, hq, hk, d, causal, flush=True)
        check(run(c, causal), oracle(c, causal), ("cached", causal))
    # straight from the projection: every sequence on row tiles
    c = make([(r, r) for r in rows], hq, hk, d, n + 1)
    order = [i for s, r in zip(c["starts"], rows) for i in range(s, s + r)]
    c["k"], c["v"], c["starts"] = c["k"][order], c["v"][order], c["off"][:-1]
    for causal in (True, False):
        check(run(c, causal, kv_starts=None, kv_lens=None), oracle(c, causal), ("packed", causal))


@pytest.mark.parametrize("seqs,hq,hk", [([(20, 33000)], 32, 8), ([(100, 50000)], 1, 1), ([(3, 10), (70, 40000), (1, 30000)], 4, 1)])
def test_a_chunk_over_more_than_a_wave_of_pieces(seqs, hq, hk):
    c = make(seqs, hq, hk, 64, 97, tail=1)
    c["q"] = c["q"] * 2
    rows = np.unique(np.concatenate([np.arange(o, o + n)[[0, n // 2, n - 1]] for o, (n, _) in zip(c["off"], seqs)])).tolist()
    got = run(c, True)
    # the oracle on some rows: each as a sequence of its own over the keys that it sees
    one = {**c, "q": c["q"][rows], "off": list(range(len(rows) + 1)), "starts": [], "lens": []}
    for r in rows:
        s = next(i for i in range(len(seqs)) if r < c["off"][i + 1])
        one["starts"].append(c["starts"][s])
        one["lens"].append(r - c["off"][s] + seqs[s][1] - seqs[s][0] + 1)
    check(got[rows], oracle(one, True), "some rows")
    assert (got[-1] == 7).all() and torch.isfinite(got).all()


def test_pieces_of_a_chunk_among_many_sequences():
    seqs = [(0, 5), (1, 40)] * 40 + [(30, 21000)] + [(1, 300)] * 20
    c = make(seqs, 8, 1, 64, 101)
    check(run(c, True), oracle(c, True), "many")


@pytest.mark.parametrize("some", [{0: (1, 900), 70000: (1, 5000), 70001: (1, 3), 149999: (1, 2500)}, {3: (1, 40), 70000: (100, 700), 149999: (90, 90)},
                                  {149999: (30, 21000)}], ids=["singles", "prompts", "chunk"])
def test_a_hundred_thousand_sequences_without_rows(some):
    # between the few that have some: a look at all of them in every workgroup, or one after the other, would take seconds
    n = 150000
    c = make([some[i] for i in sorted(some)], 4, 2, 64, 103, gap=2, tail=1)
    for x, rest in (("off", None), ("starts", 7), ("lens", 11)):
        v = torch.full((n,), 0 if rest is None else rest)
        for i, s in enumerate(sorted(some)):
            v[s] = some[s][0] if rest is None else c[x][i]
        big = torch.cat([torch.zeros(1, dtype=v.dtype), v.cumsum(0)]) if rest is None else v
        c["big_" + x] = big.to(DEV, torch.int64 if x == "starts" else torch.int32)
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    got = run(c, True, q_offsets=c["big_off"], kv_starts=c["big_starts"], kv_lens=c["big_lens"])
    e1.record()
    check(got, oracle(c, True), "some")
    print("many sequences: %.2f ms" % e0.elapsed_time(e1), flush=True)
