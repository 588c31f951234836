"""is_attention where values are not ordinary: scores of great size, long tails beside a dominant key, infinities among the values."""
import numpy as np
import pytest
import torch

import paper_2405_14597_amd as P
from oracle import block as B
from test_gpu_attention import DEV, check, make, run

pytestmark = pytest.mark.gpu
SEQS = pytest.mark.parametrize("seqs", [[(1, 700), (1, 40)], [(100, 100), (70, 200)], [(70, 6000)], [(3, 20000)]],
                               ids=["singles", "prompts", "chunk", "far"])
HEADS = pytest.mark.parametrize("hq,hk,d", [(4, 2, 128), (8, 2, 64), (20, 1, 64)])
H = 2.0 ** -11


def oracle(c, causal, scale=None, **kw):
    return B.attention(c["q"].numpy(), c["k"].numpy(), c["v"].numpy(), c["off"], c["starts"], c["lens"], c["d"],
                       float(np.float32(c["d"] ** -0.5 if scale is None else scale)), causal, np.full(tuple(c["q"].shape), 7.0), **kw)


@SEQS
@HEADS
def test_finite_scores_of_any_size(seqs, hq, hk, d):
    # products of powers of two, exact in single precision: one key (or two alike) takes all
    c = make(seqs, hq, hk, d, 71)
    c["q"][:], c["k"][:] = 0.0, 0.0
    c["q"][:, ::d] = 2.0 ** 15
    for sign in (1.0, -1.0):
        place = torch.arange(len(c["k"]))
        c["k"][:, ::d] = (sign * 2.0 ** 10 * (1 + (place * 37 % 1021)[:, None] / 1024.0)).half()
        for scale in (2.0 ** -20, 2.0 ** -8, 0.125, 1.0, 2.0 ** 20):
            # (neighbouring keys are 2^15 * scale apart: at 2^-20 all count, from 2^-8 on one alone)
            got = run(c, True, scale=scale)
            if scale < 2.0 ** -10:
                check(got, oracle(c, True, scale=scale), (sign, scale))
                continue
            got = got.double().cpu().numpy()
            for (n, m), start, q0 in zip(seqs, c["starts"], c["off"]):
                for i in range(0, n, 7):
                    seen = i + m - n + 1
                    z = c["k"][start : start + seen, 0].double().numpy()
                    v = c["v"][start : start + seen].double().numpy()[z == z.max()]
                    want, size = (np.repeat(x.mean(0).reshape(hk, 1, d), hq // hk, 1).reshape(-1) for x in (v, np.abs(v)))
                    # (half a step of fp16 in the probabilities, which the sum below the line does not have, and half a step of the output)
                    assert (np.abs(got[q0 + i] - want) <= 1.01 * H * (np.abs(want) + size) + 2.0 ** -24).all(), (sign, scale, i)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mass", [0.98, 0.92, 0.5])
@pytest.mark.parametrize("form", ["row_tiles", "few_rows"])
def test_a_long_tail_beside_a_dominant_key(form, mass, d):
    # the first key takes most of the weight and has next to no value: what comes out is the tail's, all alike and 2^-20 or less of it
    # each.  Enough rows that a workgroup walks all keys; every sequence over the same ones, and a few rows compared.
    heads, keys, seqs = 8, 131072, 32
    rows = 6400 // seqs if form == "row_tiles" else 1
    g = torch.Generator(device=DEV).manual_seed(73)
    normal = lambda n: torch.randn((n, heads * d), generator=g, device=DEV)  # noqa: E731
    q, k, v = torch.zeros_like(normal(seqs * rows)).half(), normal(keys).half(), (normal(keys) * 0.3 + 1.0).half()
    scale = d ** -0.5
    q[:, ::d], k[:, ::d] = 4.0, 0.0
    k[0, ::d], v[0] = float(np.log(mass / (1.0 - mass) * keys)) / (4.0 * scale), 0.01
    whole = lambda x, t: torch.tensor(x, dtype=t, device=DEV)  # noqa: E731
    got = P.is_attention(q, k, v, whole([i * rows for i in range(seqs + 1)], torch.int32), d, rows, keys, causal=False,
                         kv_starts=whole([0] * seqs, torch.int64), kv_lens=whole([keys] * seqs, torch.int32))
    at = [0, seqs * rows // 2, seqs * rows - 1]
    head = slice(3 * d, 4 * d)   # (one head of the eight)
    ref = B.attention(q[at, head].cpu().numpy(), k[:, head].cpu().numpy(), v[:, head].cpu().numpy(), [0, 3], [0], [keys], d,
                      float(np.float32(scale)), False, np.zeros((3, d)))
    check(got[at, head], ref, "tail")


@pytest.mark.parametrize("seqs", [[(1, 700), (1, 40), (1, 1)], [(100, 100), (70, 200)], [(70, 6000)], [(3, 20000)], [(40, 9000), (1, 3000)]],
                         ids=["singles", "prompts", "chunk", "far", "beside"])
@pytest.mark.parametrize("causal", [True, False])
@HEADS
def test_infinities_among_the_values_a_row_sees(seqs, causal, hq, hk, d):
    # however small the key's probability, wherever it lies: its column is infinite (NaN for two of unlike sign and for a NaN), the other
    # columns are as ever.  Scores of some hundreds, so that most probabilities vanish.
    c = make(seqs, hq, hk, d, 79, gap=5)
    c["q"] = c["q"] * 8
    g = torch.Generator().manual_seed(83)
    ref = oracle(c, causal, scale=0.7)
    odd = torch.zeros_like(c["v"])
    for (n, m), start in zip(seqs, c["starts"]):
        place = torch.randint(0, m, (6,), generator=g)
        for j, x in zip(place.tolist(), (float("inf"), float("-inf"), float("inf"), float("nan"), float("-inf"), float("inf"))):
            odd[start + j, torch.randint(0, hk * d, (9,), generator=g)] = x
    late = [start + m - 1 for (_, m), start in zip(seqs, c["starts"])]
    odd[late, 5] = float("inf")
    c["v"] = torch.where(odd != 0, odd, c["v"])
    got = run(c, causal, scale=0.7).cpu().double().numpy()
    odd = odd.numpy().astype(np.float64)
    want, bound = ref[0].copy(), ref[1].copy()
    for (n, m), start, q0 in zip(seqs, c["starts"], c["off"]):
        for i in range(n):
            seen = i + m - n + 1 if causal else m
            with np.errstate(invalid="ignore"):
                w = np.repeat(odd[start : start + seen].sum(0).reshape(hk, 1, d), hq // hk, 1).reshape(-1)
            hit = w != 0
            # (two of unlike sign: NaN + anything, as it should)
            assert np.array_equal(got[q0 + i][hit], w[hit], equal_nan=True), (n, m, i)
            assert (np.abs(got[q0 + i][~hit] - want[q0 + i][~hit]) <= bound[q0 + i][~hit]).all(), (n, m, i)


@SEQS
@HEADS
def test_an_infinity_behind_a_score_of_minus_infinity(seqs, hq, hk, d):
    # the formula's 0 * infinity in its column; a finite value there does not count
    c = make(seqs, hq, hk, d, 89)
    c["q"][:, ::d] = c["q"][:, ::d].abs() + 0.1
    ref = oracle(c, False)
    gone = [start + m // 2 for (_, m), start in zip(seqs, c["starts"])]
    for j in gone:
        c["k"][j, ::d] = float("-inf")
    base = {**c, "k": c["k"].clone()}
    base["k"][gone] = 0.0
    c["v"][gone, 3] = float("inf")
    c["v"][gone, 4] = 60000.0
    keep = torch.ones(len(c["k"]), dtype=torch.bool)
    keep[gone] = False
    # the oracle without those keys
    at = np.cumsum(keep.numpy()) - 1
    less = {**c, "k": c["k"][keep], "v": c["v"][keep], "starts": [int(at[s]) for s in c["starts"]], "lens": [m - 1 for m in c["lens"]]}
    ref = oracle(less, False)
    got = run(c, False)
    cols = torch.ones(hq * d, dtype=torch.bool)
    for h in range(hq // hk):
        cols[h * d + 3] = False
    assert torch.isnan(got[:, (~cols).to(DEV)]).all()
    check(got[:, cols.to(DEV)], (ref[0][:, cols.numpy()], ref[1][:, cols.numpy()]), "the other columns")
