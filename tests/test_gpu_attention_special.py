"""is_attention where values are not ordinary: scores of great size, long tails beside a dominant key, infinities among the values."""
import numpy as np
import pytest
import torch

from test_gpu_attention import DEV, check, make, oracle, run

pytestmark = pytest.mark.gpu
SEQS = pytest.mark.parametrize("seqs", [[(1, 700), (1, 40)], [(100, 100), (70, 200)], [(70, 6000)], [(3, 20000)]],
                               ids=["singles", "prompts", "chunk", "far"])
HEADS = pytest.mark.parametrize("hq,hk,d", [(4, 2, 128), (8, 2, 64), (20, 1, 64)])
H = 2.0 ** -11


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
