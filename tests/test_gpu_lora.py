"""is_lora_add against the 64-bit oracle: row and adapter mixes, odd widths, ranks, strides, in place, foreign adapters' infinities."""
import numpy as np
import pytest
import torch

import paper_2405_14597_amd as P
from oracle import block as B

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def make(M, N, K, R, E, seed, mix):
    g = torch.Generator().manual_seed(seed)
    c = {"x": torch.randn((M, K), generator=g), "a": (torch.randn((E, R, K), generator=g) * K ** -0.5).half(),
         "b": (torch.randn((E, N, R), generator=g) * 0.3).half(), "base": torch.randn((M, N), generator=g).half(),
         "scales": torch.rand((E,), generator=g) + 0.5, "ranks": torch.randint(0, R + 1, (E,), generator=g, dtype=torch.int32)}
    c["x"][:, : max(1, K // 100)] *= 20
    c["x"] = c["x"].half()
    if mix == "rows":       # every row its own request
        c["e"] = torch.randint(-1, E, (M,), generator=g, dtype=torch.int32)
    elif mix == "runs":
        c["e"] = (torch.arange(M) * E // M - (torch.arange(M) % 64 == 63).int() * (E + 1)).clamp_(min=-3).int()
    else:
        c["e"] = torch.full((M,), mix, dtype=torch.int32)
    c["ranks"][0] = R
    return c


def want(c, base=True, ranks=True, scales=True):
    E, R = c["a"].shape[:2]
    return B.lora_add(c["x"].numpy(), c["a"].numpy(), c["b"].numpy(), c["e"].tolist(), c["base"].numpy() if base else np.zeros(c["base"].shape),
                      c["scales"].tolist() if scales else [1.0] * E, c["ranks"].tolist() if ranks else [R] * E)


def on(c):
    return {k: v.to(DEV) for k, v in c.items()}


def check(got, ref, what):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    worst = (np.abs(got - ref[0]) / np.maximum(ref[1], 1e-30)).max(initial=0.0)
    assert worst <= 1.0, (what, worst)


@pytest.mark.parametrize("M,N,K,R,E,mix", [
    (1, 1024, 4096, 8, 4, 2), (1, 1, 8, 8, 1, 0), (16, 64, 136, 16, 3, "rows"), (17, 100, 4096, 16, 20, "rows"), (64, 4096, 4096, 16, 32, "rows"),
    (5, 5003, 256, 64, 2, "rows"), (100, 257, 1000, 24, 5, "runs"), (300, 384, 520, 128, 7, "runs"), (33, 72, 40, 40, 6, "rows"),
    (1000, 136, 264, 32, 3, "runs"), (40, 48, 64, 8, 2, -1), (40, 48, 64, 8, 2, 2), (2000, 96, 128, 96, 1, 0),
    # from 2^26 products of the wider side on: by tiles
    (1101, 1003, 72, 64, 5, "runs"), (530, 256, 2056, 64, 3, "rows"), (4207, 1000, 40, 16, 9, "runs"), (1050, 520, 1000, 128, 2, "runs"),
    (2100, 2008, 8, 24, 1, -1), (1800, 1168, 96, 40, 40, "rows"), (4097, 2049, 64, 8, 2, 1)])
def test_against_oracle(M, N, K, R, E, mix):
    print("lora", M, N, K, R, E, mix, flush=True)
    c = make(M, N, K, R, E, M + N + K, mix)
    d = on(c)
    check(P.is_lora_add(d["x"], d["a"], d["b"], d["e"], d["base"], scales=d["scales"], ranks=d["ranks"]), want(c), "all arguments")
    check(P.is_lora_add(d["x"], d["a"], d["b"], d["e"], None), want(c, False, False, False), "none of the optional ones")
    y = d["base"].clone()
    assert P.is_lora_add(d["x"], d["a"], d["b"], d["e"], y, scales=d["scales"], ranks=d["ranks"], out=y) is y
    check(y, want(c), "in place")
    # the same bits whatever the rows around: a row's result does not depend on its tile
    if M > 1:
        keep = torch.arange(M - 1, -1, -2)
        part = P.is_lora_add(d["x"][keep.to(DEV)], d["a"], d["b"], d["e"][keep.to(DEV)].contiguous(), d["base"][keep.to(DEV)],
                             scales=d["scales"], ranks=d["ranks"])
        ref = want(c)
        check(part, (ref[0][keep.numpy()], ref[1][keep.numpy()]), "every second row")


FORMS = pytest.mark.parametrize("M,N,R", [(50, 90, 16), (2100, 1002, 32), (2100, 1000, 32)], ids=["rows", "tiles", "tiles_wide"])


@FORMS
def test_strides_and_what_lies_between(M, N, R):
    c = make(M, N, 64, R, 3, 9, "rows")
    d = on(c)
    x = torch.full((M, 96), float("nan"), dtype=torch.float16, device=DEV)
    x[:, 16:80] = d["x"]
    wide = torch.full((M, N + (41 if M == 50 else 40)), 7.0, dtype=torch.float16, device=DEV)
    wide[:, :N] = d["base"]
    y = wide[:, :N]
    P.is_lora_add(x[:, 16:80], d["a"], d["b"], d["e"], y, scales=d["scales"], ranks=d["ranks"], out=y)
    check(y, want(c), "strided")
    assert (wide[:, N:] == 7).all()


@FORMS
def test_nothing_of_another_adapter_reaches_a_row(M, N, R):
    # NaN and infinities in adapters, ranks' rests and rows of other requests
    c = make(M, N, 72, R, 4, 11, "rows")
    c["ranks"] = torch.tensor([R, 5, R, 9], dtype=torch.int32)
    c["e"] = torch.randint(0, 4, (M,), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    ref = want(c)
    c["a"][2], c["b"][2] = float("inf"), float("nan")
    for e in (1, 3):
        r = int(c["ranks"][e])
        c["a"][e, r:], c["b"][e, :, r:] = float("nan"), float("inf")
    odd = c["e"] == 2
    c["x"][5], c["e"][5], odd[5] = float("nan"), 0, True
    d = on(c)
    got = P.is_lora_add(d["x"], d["a"], d["b"], d["e"], d["base"], scales=d["scales"], ranks=d["ranks"])
    fine = ~odd.numpy()
    check(got[torch.from_numpy(fine).to(DEV)], (ref[0][fine], ref[1][fine]), "rows of sound adapters")
    assert torch.isnan(got[5]).all() and not torch.isfinite(got[odd.to(DEV)]).any()


@FORMS
def test_large_inner_products(M, N, R):
    # x a^T far past fp16's largest number, b small: the output is ordinary
    c = make(M, N, 512, R, 2, 13, "rows")
    c["x"], c["a"], c["b"] = c["x"] * 400, (c["a"].float() * 400).half(), (c["b"].float() * 2e-6).half()
    d = on(c)
    assert (c["x"].float() @ c["a"][0].float().t()).abs().max() > 1e6
    check(P.is_lora_add(d["x"], d["a"], d["b"], d["e"], d["base"], scales=d["scales"], ranks=d["ranks"]), want(c), "large t")


def test_no_rows_and_refusals():
    d = on(make(4, 48, 64, 8, 2, 1, "rows"))
    z = lambda t: t[:0]  # noqa: E731
    assert P.is_lora_add(z(d["x"]), d["a"], d["b"], z(d["e"]), z(d["base"])).shape == (0, 48)
    ok = lambda **kw: P.is_lora_add(**{**dict(x=d["x"], a=d["a"], b=d["b"], row_adapter=d["e"], base=d["base"]), **kw})  # noqa: E731
    ok()
    for kw in (dict(x=d["x"].float()), dict(a=d["a"][:, :, :32]), dict(b=d["b"][:1]), dict(row_adapter=d["e"].long()), dict(row_adapter=d["e"][:3]),
               dict(base=d["base"][:, :40]), dict(scales=d["scales"].half()), dict(ranks=d["ranks"][:1]), dict(out=d["base"].t())):
        with pytest.raises(ValueError):
            ok(**kw)
    with pytest.raises(P.IntScaleError):
        ok(workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
