"""is_lora_add where values are not ordinary: in the form by rows and in that by tiles (narrow and wide stores), which have to agree with
the formula alike."""
import numpy as np
import pytest
import torch

import paper_2405_14597_amd as P
from oracle import block as B
from test_gpu_lora import DEV, FORMS, check, make, on, want

pytestmark = pytest.mark.gpu


def add(c):
    d = on(c)
    return P.is_lora_add(d["x"], d["a"], d["b"], d["e"], d["base"], scales=d["scales"], ranks=d["ranks"])


@FORMS
def test_an_infinity_in_x_and_what_lies_past_the_rank(M, N, R):
    # adapters of rank 0, 1, 5 and all of R; what a row of A past the rank makes of an infinity does not count
    c = make(M, N, 72, R, 4, 17, "rows")
    c["ranks"] = torch.tensor([0, 1, 5, R], dtype=torch.int32)
    c["e"] = (torch.arange(M) % 5 - 1).int()
    odd = torch.arange(M) % 3 == 1
    c["a"][:, :, 7] = c["a"][:, :, 7].abs() + 0.1
    c["b"] = c["b"].abs() + 0.01
    ref = want(c)
    c["x"][odd, 7] = float("inf")
    got = add(c)
    fine = (~odd | (c["e"] < 1)).numpy()      # (no adapter or one of rank 0: the base, whatever x is)
    assert odd[torch.from_numpy(fine)].any()
    check(got[torch.from_numpy(fine).to(DEV)], (ref[0][fine], ref[1][fine]), "rows that no infinity reaches")
    nothing = (c["e"] < 1).to(DEV)
    assert torch.equal(got[nothing], c["base"].to(DEV)[nothing])
    assert (got[torch.from_numpy(~fine).to(DEV)] == float("inf")).all()


@FORMS
def test_inner_products_of_very_different_size(M, N, R):
    # from r to r the inner products fall by 2^24 in all and B's columns grow by as much: every r counts alike
    K = 4 * R
    c = make(M, N, K, R, 3, 19, "rows")
    c["ranks"][:] = torch.tensor([R, R - 3, R])
    fall = torch.exp2(-12.0 * torch.arange(R) / (R - 1))
    own = (torch.arange(K) // 4 == torch.arange(R)[:, None])
    g = torch.Generator().manual_seed(21)
    c["x"] = ((torch.rand((M, K), generator=g) + 0.5) * 64 * fall.repeat_interleave(4)).half()
    c["a"] = ((torch.rand((3, R, K), generator=g) + 0.5) * own * fall[:, None]).half()
    c["b"] = (torch.randn((3, N, R), generator=g) * 2.0 ** -12 / fall ** 2).half()
    c["base"] *= 0.01
    ref = want(c)
    part = lambda e, lo, hi: c["b"][e, :, lo:hi].double() @ (c["a"][e, lo:hi].double() @ c["x"][0].double())  # noqa: E731
    assert part(0, 0, 2).abs().mean() < 4 * part(0, R - 2, R).abs().mean() and part(0, R - 2, R).abs().mean() < 4 * part(0, 0, 2).abs().mean()
    check(add(c), ref, "spread")


@FORMS
def test_infinities_of_the_rows_own_adapter(M, N, R):
    # in B: their columns are infinite with the product's sign, or NaN where two of unlike sign meet, and no other column is touched; a row
    # whose inner products are infinite and large: infinite as well
    c = make(M, N, 72, R, 3, 23, "rows")
    c["ranks"][:] = torch.tensor([R, R - 3, R])
    g = torch.Generator().manual_seed(25)
    odd = torch.rand((3, N, R), generator=g) < 0.1 / R
    ref = want(c)
    c["b"][odd] = float("inf")
    c["b"][odd & (torch.rand((3, N, R), generator=g) < 0.3)] = float("-inf")
    # inner products far below their row's largest among them, which both terms of it round to little or nothing
    c["a"][1, 2] *= 2.0 ** -13
    got = add(c).cpu().numpy()
    rows = [(m, e) for m, e in enumerate(c["e"].tolist()) if e >= 0]
    seen = 0
    for m, e in rows[:: max(1, len(rows) // 60)]:
        r = int(c["ranks"][e])
        t = c["a"][e, :r].double() @ c["x"][m].double()
        with np.errstate(invalid="ignore"):
            y = (np.where(odd[e, :, :r], c["b"][e, :, :r], 0.0).astype(np.float64) * t.numpy()).sum(-1) * float(c["scales"][e])
        hit = odd[e, :, :r].any(-1).numpy()
        seen += int(hit.sum())
        assert np.array_equal(got[m][hit].astype(np.float64), y[hit], equal_nan=True), (m, e)
        if e != 1:
            assert (np.abs(got[m][~hit] - ref[0][m][~hit]) <= ref[1][m][~hit]).all(), (m, e)
        assert np.isfinite(got[m][~hit]).all()
    assert seen > 20
    # an infinite inner product beside large finite ones of the other sign
    c = make(M, N, 72, R, 3, 27, "rows")
    c["ranks"][:] = R
    c["a"][:, 1:] = -(c["a"][:, 1:].abs() + 0.1) * 3000
    c["a"][:, 0, 5] = float("inf")
    c["x"] = c["x"].abs() + 60
    c["b"] = c["b"].abs() + 0.01
    assert ((c["x"].double() @ c["a"][0, 1].double()) < -1e6).all()
    mine = (c["e"] >= 0).to(DEV)
    assert (add(c)[mine] == float("inf")).all()


@FORMS
def test_the_largest_scales(M, N, R):
    # a scale that overflows with the row's power of two: columns whose product is zero stay the base, the others are infinite
    c = make(M, N, 72, R, 3, 29, "rows")
    c["ranks"][:] = R
    c["x"] = c["x"].abs() + 50
    c["a"] = c["a"].abs() + 0.1
    c["b"] = c["b"].abs() + 0.01
    c["b"][:, 3::7] = 0.0
    c["scales"][:] = 3e38
    got = add(c)
    mine = c["e"] >= 0
    zero = torch.zeros(N, dtype=torch.bool)
    zero[3::7] = True
    assert torch.equal(got[:, zero.to(DEV)], c["base"][:, zero].to(DEV)) and torch.equal(got[(~mine).to(DEV)], c["base"][~mine].to(DEV))
    assert (got[mine.to(DEV)][:, (~zero).to(DEV)] == float("inf")).all()
