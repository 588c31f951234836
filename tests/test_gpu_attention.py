"""is_attention against the 64-bit oracle: lengths, heads, chunks of prompts, caches, what is masked, the split of the keys."""
import numpy as np
import pytest
import torch

import paper_2405_14597_amd as P
from oracle import block as B

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def make(seqs, hq, hk, d, seed, gap=0, tail=0):
    """Sequences [(rows of q, keys)] with their keys in a cache in reverse order, `gap` unused rows behind each, and `tail` rows of q
    behind the last sequence."""
    g = torch.Generator().manual_seed(seed)
    M = sum(n for n, _ in seqs) + tail
    starts, rows = [0] * len(seqs), 0
    for i in reversed(range(len(seqs))):
        starts[i] = rows
        rows += seqs[i][1] + gap
    c = {"q": (torch.randn((M, hq * d), generator=g) * 1.5).half(), "k": torch.randn((rows, hk * d), generator=g).half(),
         "v": torch.randn((rows, hk * d), generator=g).half(), "off": np.cumsum([0] + [n for n, _ in seqs]).tolist(), "starts": starts,
         "lens": [m for _, m in seqs], "d": d, "mq": max([n for n, _ in seqs], default=0), "mkv": max([m for _, m in seqs], default=0)}
    return c


def oracle(c, causal, scale=None, untouched=7.0):
    return B.attention(c["q"].numpy(), c["k"].numpy(), c["v"].numpy(), c["off"], c["starts"], c["lens"], c["d"],
                       float(np.float32(c["d"] ** -0.5 if scale is None else scale)), causal, np.full(tuple(c["q"].shape), untouched))


def run(c, causal, scale=None, workspace=None, **kw):
    whole = lambda v, t: torch.tensor(v, dtype=t, device=DEV)  # noqa: E731
    a = dict(q=c["q"].to(DEV), k=c["k"].to(DEV), v=c["v"].to(DEV), q_offsets=whole(c["off"], torch.int32), head_dim=c["d"], max_q_len=c["mq"],
             max_kv_len=c["mkv"], scale=scale, causal=causal, kv_starts=whole(c["starts"], torch.int64), kv_lens=whole(c["lens"], torch.int32),
             out=torch.full(tuple(c["q"].shape), 7.0, dtype=torch.float16, device=DEV))
    a.update(kw)
    return P.is_attention(**a)


def check(got, ref, what):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    worst = (np.abs(got - ref[0]) / np.maximum(ref[1], 1e-30)).max(initial=0.0)
    assert worst <= 1.0, (what, worst)


HEADS = [(4, 4, 128), (8, 2, 128), (8, 1, 64), (6, 2, 64), (3, 3, 64), (33, 1, 128)]


@pytest.mark.parametrize("hq,hk,d", HEADS)
@pytest.mark.parametrize("seqs", [
    [(1, 1)], [(1, 63), (1, 64), (1, 65), (1, 128), (1, 1000)], [(1, 5000)], [(2, 2), (3, 70), (5, 5)], [(0, 5), (3, 0), (4, 2), (0, 0), (1, 9)],
    [(65, 65), (33, 97), (1, 300), (130, 130)], [(31, 700), (1, 1500)]],
    ids=["one", "singles", "long_single", "small", "empty", "mixed", "chunk"])
def test_against_oracle(seqs, hq, hk, d):
    c = make(seqs, hq, hk, d, len(seqs) * 100 + d + hq, gap=3, tail=2)
    for causal in (True, False):
        print("attention", seqs, hq, hk, d, causal, flush=True)
        check(run(c, causal), oracle(c, causal), causal)


@pytest.mark.parametrize("causal", [True, False])
def test_longer_prompts_from_one_buffer(causal):
    # q, k, v columns of one projection's output, keys where the queries are; out wider than its rows
    hq, hk, d, lens = 4, 2, 128, [513, 1, 300, 64]
    g = torch.Generator().manual_seed(3)
    M = sum(lens)
    qkv = torch.randn((M, (hq + 2 * hk) * d), generator=g).half()
    off = np.cumsum([0] + lens).tolist()
    c = {"q": qkv[:, : hq * d], "k": qkv[:, hq * d : (hq + hk) * d], "v": qkv[:, (hq + hk) * d :], "off": off, "starts": off[:-1], "lens": lens, "d": d}
    x = qkv.to(DEV)
    wide = torch.full((M, hq * d + 40), 7.0, dtype=torch.float16, device=DEV)
    P.is_attention(x[:, : hq * d], x[:, hq * d : (hq + hk) * d], x[:, (hq + hk) * d :], torch.tensor(off, dtype=torch.int32, device=DEV), d, 513, 513,
                   causal=causal, out=wide[:, : hq * d])
    check(wide[:, : hq * d], oracle(c, causal), causal)
    assert (wide[:, hq * d :] == 7).all()


def test_many_sequences():
    # more than a wave of them, every third without rows of q, some without keys
    seqs = [((i * 7) % 3 * (1 + i % 5), (i * 37) % 150 if i % 11 else 0) for i in range(150)]
    c = make(seqs, 4, 2, 64, 17, gap=1, tail=5)
    for causal in (True, False):
        check(run(c, causal), oracle(c, causal), causal)


@pytest.mark.parametrize("hq,hk,d", [(64, 1, 128), (65, 1, 64), (16, 1, 128), (4, 4, 128)])
def test_groups_at_the_kernels_limits(hq, hk, d):
    # packed rows of a token at and past what the kernel for few rows takes; drafts of a few tokens; loose maxima
    for seqs in ([(1, 900), (1, 33)], [(2, 700), (4, 64), (1, 1)]):
        c = make(seqs, hq, hk, d, hq + d, gap=2)
        ref = oracle(c, True)
        check(run(c, True), ref, seqs)
        check(run(c, True, max_q_len=4096, max_kv_len=100000), ref, "loose")


def test_ragged_decode_batch_over_many_workgroups():
    # more than a wave of sequences whose keys are dealt out over workgroups that begin and end inside them
    g = np.random.default_rng(5)
    seqs = [(1, int(n)) for n in np.exp(g.uniform(0, np.log(4000), 90))]
    seqs[40], seqs[41], seqs[42] = (0, 3000), (1, 0), (1, 9000)
    c = make(seqs, 2, 1, 128, 61, gap=5)
    check(run(c, True), oracle(c, True), "90 sequences")
    c = make(seqs[:64], 2, 1, 64, 62)
    check(run(c, False), oracle(c, False), "64 sequences")
    # beside prompts
    c = make(seqs[:20] + [(70, 300), (150, 150)] + seqs[50:60], 4, 2, 128, 63, gap=1)
    check(run(c, True), oracle(c, True), "beside prompts")


def test_two_calls_at_once():
    # on two streams, each with its own workspace
    c, d = make([(1, 5000), (1, 77)], 8, 2, 128, 68), make([(60, 1000), (1, 2000)], 8, 2, 128, 69)
    want = [run(x, True) for x in (c, d)]
    whole = lambda v, t: torch.tensor(v, dtype=t, device=DEV)  # noqa: E731
    streams, args = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for x in (c, d):
        args.append((x["q"].to(DEV), x["k"].to(DEV), x["v"].to(DEV), whole(x["off"], torch.int32), 128, x["mq"], x["mkv"], whole(x["starts"], torch.int64),
                     whole(x["lens"], torch.int32), torch.zeros(tuple(x["q"].shape), dtype=torch.float16, device=DEV)))
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (q, k, v, off, hd, mq, mkv, starts, lens, out) in zip(streams, args):
            with torch.cuda.stream(s):
                P.is_attention(q, k, v, off, hd, mq, mkv, kv_starts=starts, kv_lens=lens, out=out)
    torch.cuda.synchronize()
    assert torch.equal(args[0][-1], want[0]) and torch.equal(args[1][-1], want[1])


def test_scale_and_large_scores():
    # scores of some hundreds: one key takes nearly all, the maximum moves far and often
    c = make([(40, 300), (1, 900)], 4, 2, 128, 23)
    c["q"] *= 8
    for scale in (0.7, 1e-4):
        check(run(c, True, scale=scale), oracle(c, True, scale=scale), scale)
    # scores that rise from key to key: every tile raises the maximum
    c["k"] = (c["k"].float() * 0.01 + torch.arange(len(c["k"]))[:, None] * 2e-3).half()
    c["q"] = c["q"].abs().clamp_(max=4.0)
    check(run(c, True, scale=0.5), oracle(c, True, scale=0.5), "rising")


@pytest.mark.parametrize("seqs", [[(100, 100), (70, 200)], [(1, 130), (1, 64), (1, 3)], [(9, 2500)]], ids=["prompts", "singles", "chunk"])
@pytest.mark.parametrize("hq,hk,d", [(4, 2, 128), (4, 4, 64)])
def test_what_a_row_does_not_see_does_not_reach_it(seqs, hq, hk, d):
    # NaN and infinities behind the sequences' ends and among the keys that only later rows see
    c = make(seqs, hq, hk, d, 31, gap=70)
    ref = oracle(c, True)
    rows = torch.ones(len(c["k"]), dtype=torch.bool)
    clean = np.ones(len(c["q"]), dtype=bool)
    for (n, m), start, q0 in zip(seqs, c["starts"], c["off"]):
        rows[start : start + m] = False
        if n > 5:  # the last keys are for the last rows alone
            for j, bad in ((m - 1, float("nan")), (m - 3, float("inf")), (m - 5, float("-inf"))):
                c["k"][start + j], c["v"][start + j] = (0.0 if bad != bad else 1.0), bad
            clean[q0 + n - 5 : q0 + n] = False
    c["k"][rows], c["v"][rows] = float("nan"), float("inf")
    got = run(c, True)
    check(got[torch.from_numpy(clean).to(DEV)], (ref[0][clean], ref[1][clean]), "rows that see sound keys")
    if not clean.all():  # what a row does see reaches it
        assert not torch.isfinite(got[torch.from_numpy(~clean).to(DEV)]).any()
        late = [q0 + n - 1 for (n, _), q0 in zip(seqs, c["off"]) if n > 5]
        assert torch.isnan(got[late]).all()
        first = [q0 + n - 5 for (n, _), q0 in zip(seqs, c["off"]) if n > 5]
        assert (got[first] == float("-inf")).all()


def test_lowest_keys_and_not_a_number():
    # keys of the type's lowest and largest values: finite scores of great size; a NaN in a query stays in its row
    c = make([(4, 90)], 4, 2, 64, 37)
    c["k"][10], c["k"][20] = -65504.0, 65504.0
    c["q"] = c["q"] * 0.01
    check(run(c, True, scale=1e-3), oracle(c, True, scale=1e-3), "extremes")
    c["q"][2, 64:128] = float("nan")
    got = run(c, True, scale=1e-3)
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[2, 64:128] = True
    assert torch.isnan(got[bad]).all() and torch.isfinite(got[~bad]).all()


def test_scores_of_minus_infinity_are_the_formulas_nan():
    c = make([(3, 70)], 2, 2, 64, 41)
    c["q"] = c["q"].abs() + 0.1
    c["k"][:, 0] = float("-inf")
    got = run(c, False)
    assert torch.isnan(got[:, :64]).all() and torch.isfinite(got[:, 64:]).all()


def test_lengths_and_places_outside_are_bounded():
    c = make([(3, 50), (2, 40), (4, 60), (1, 30)], 4, 2, 64, 43)
    rows = len(c["k"])
    c["starts"][1] = -5          # before the cache: no keys
    c["starts"][2] = rows - 20   # runs over its end: the 20 keys there
    ref = oracle({**c, "lens": [50, 0, 20, 0], "starts": [c["starts"][0], 0, rows - 20, 0]}, True)
    c["starts"][3] = rows + 1
    check(run(c, True), ref, "bounded")
    c["lens"][0] = -4            # no keys either
    ref2 = oracle({**c, "lens": [0, 0, 20, 0], "starts": [0, 0, rows - 20, 0]}, True)
    check(run(c, True), ref2, "negative")
    # offsets past the rows of q end there; keys past max_kv_len are left out
    c = make([(3, 50), (5, 40)], 4, 2, 64, 44)
    whole = lambda v, t: torch.tensor(v, dtype=t, device=DEV)  # noqa: E731
    got = run(c, False, q_offsets=whole([0, 3, 9000], torch.int32), max_kv_len=45)
    check(got, oracle({**c, "lens": [45, 40]}, False), "past the end")


def test_offsets_past_32_bits():
    # rows 16 KB apart, a sequence whose keys begin past 4 GB
    hq, hk, d, n = 8, 2, 128, 310000
    g = torch.Generator().manual_seed(47)
    lens = [700, 130]
    starts = [n - 700, 270001]
    c = {"q": torch.randn((3, hq * d), generator=g).half(), "off": [0, 1, 3], "starts": starts, "lens": lens, "d": d, "mq": 2, "mkv": 700}
    small = {x: torch.randn((830, hk * d), generator=g).half() for x in "kv"}
    ref = oracle({**c, "k": small["k"], "v": small["v"], "starts": [0, 700]}, True)
    big = {}
    for x in "kv":
        buf = torch.empty((n, 8192), dtype=torch.float16, device=DEV)
        big[x] = buf[:, 512 : 512 + hk * d]
        big[x][starts[0] :], big[x][starts[1] : starts[1] + 130] = small[x][:700].to(DEV), small[x][700:].to(DEV)
    assert starts[1] * 8192 * 2 > 2 ** 32
    check(run({**c, "k": big["k"], "v": big["v"]}, True), ref, "far rows")


def test_shared_rows_and_the_order_of_sequences():
    # two sequences over the same prefix; the batch in another order; the same call gives the same bits
    c = make([(1, 600), (1, 550), (20, 400)], 8, 2, 128, 53)
    c["starts"][1] = c["starts"][0]
    a, ref = run(c, True), oracle(c, True)
    check(a, ref, "shared")
    assert torch.equal(a, run(c, True))
    perm = [2, 0, 1]
    rows = [list(range(c["off"][s], c["off"][s + 1])) for s in perm]
    b = run({**c, "q": c["q"][sum(rows, [])], "off": np.cumsum([0] + [len(r) for r in rows]).tolist(), "starts": [c["starts"][s] for s in perm],
             "lens": [c["lens"][s] for s in perm]}, True)
    check(b, (ref[0][sum(rows, [])], ref[1][sum(rows, [])]), "another order")


def test_captured_calls_replay():
    # a decode step's call captured once and replayed on other lengths and values, eager work between the replays
    c = make([(1, 900), (1, 70), (1, 2000)], 8, 2, 128, 59, gap=64)
    d = {x: c[x].to(DEV) for x in "qkv"}
    off = torch.tensor(c["off"], dtype=torch.int32, device=DEV)
    starts = torch.tensor(c["starts"], dtype=torch.int64, device=DEV)
    lens = torch.tensor(c["lens"], dtype=torch.int32, device=DEV)
    ws = torch.empty((P.is_attention_workspace_bytes(3, 3, 1, 2064, 8, 2, 128),), dtype=torch.uint8, device=DEV)
    out = torch.zeros_like(d["q"])
    step = lambda o, w: P.is_attention(d["q"], d["k"], d["v"], off, 128, 1, 2064, kv_starts=starts, kv_lens=lens, out=o, workspace=w)  # noqa: E731
    step(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, ws)
    for i in range(4):
        lens.copy_(torch.tensor([900 + i, 70 - i, 2000 + 9 * i], dtype=torch.int32))
        d["q"].mul_(1.0 + 0.1 * i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step(torch.zeros_like(out), None))
        torch.cuda.synchronize()


def test_another_stream():
    c = make([(50, 80), (1, 3000)], 4, 2, 128, 61)
    want = run(c, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = run(c, True)
    torch.cuda.synchronize()
    q = c["q"].to(DEV)
    torch.cuda.synchronize()
    b = run(c, True, q=q, stream=side)
    side.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)


def test_nothing_to_do_and_refusals():
    c = make([(4, 9)], 4, 2, 64, 67)
    assert run({**c, "q": c["q"][:0], "off": [0]}, True, kv_starts=None, kv_lens=None).shape == (0, 256)
    assert (run({**c, "k": c["k"][:0], "v": c["v"][:0], "starts": [0]}, True) == 0).all()
    for kw in (dict(q=c["q"].to(DEV).float()), dict(k=c["k"].to(DEV)[:5]), dict(head_dim=48), dict(kv_lens=torch.zeros(1, dtype=torch.int64, device=DEV)),
               dict(q_offsets=torch.zeros(2, dtype=torch.int64, device=DEV)), dict(out=torch.zeros((4, 128), dtype=torch.float16, device=DEV)),
               dict(kv_starts=torch.zeros(2, dtype=torch.int64, device=DEV)), dict(q=c["q"])):
        with pytest.raises(ValueError):
            run(c, True, **kw)
    with pytest.raises(P.IntScaleError):
        run(c, True, head_dim=32)
    with pytest.raises(P.IntScaleError):
        run(c, True, scale=-1.0)
