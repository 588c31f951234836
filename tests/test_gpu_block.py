"""The attention half of a block as a serving program runs it: RMSNorm folded into the quantiser, qkv GEMM, adapters of the
requests, per-head norm and rotation into the cache, attention, output projection.  Prompts of three requests, then decode steps
(captured and replayed); every operator's output against the 64-bit oracle on the inputs it had, and the decode steps against the
same tokens as part of a longer prompt."""
import numpy as np
import pytest
import torch

import paper_2405_14597_amd as P
from oracle import block as B

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
HIDDEN, HEADS, KV, D, G, ALPHA, EPS, R, E = 512, 4, 2, 128, 128, 10, 1e-5, 16, 2
WIDE = (HEADS + 2 * KV) * D
ROOM = 96                     # rows of the cache a request has


def projection(gen, n, k):
    q = P.is_quantize_weights_int4_group((torch.randn((n, k), generator=gen) * 0.04).half().to(DEV), G, ALPHA, P.IS_SCALE_NORM)
    return P.is_prepack_w4(q.qweight, q.scale_i32, G), q.chan_scale


class Block:
    def __init__(self):
        g = torch.Generator().manual_seed(71)
        self.gamma, self.gq, self.gk = ((torch.rand(n, generator=g) + 0.5).half().to(DEV) for n in (HIDDEN, D, D))
        self.qkv, self.o = projection(g, WIDE, HIDDEN), projection(g, HIDDEN, HEADS * D)
        self.a = (torch.randn((E, R, HIDDEN), generator=g) * HIDDEN ** -0.5).half().to(DEV)
        self.b = (torch.randn((E, WIDE, R), generator=g) * 0.3).half().to(DEV)
        self.scales = torch.tensor([1.5, 0.5], device=DEV)
        self.freq = (1.0 / 10000.0 ** (torch.arange(0, D, 2, dtype=torch.float64) / D)).float().to(DEV)
        self.kc, self.vc = (torch.zeros((3 * ROOM, KV * D), dtype=torch.float16, device=DEV) for _ in "kv")
        self.starts = torch.tensor([0, ROOM, 2 * ROOM], dtype=torch.int64, device=DEV)

    def step(self, x, adapter, positions, places, offsets, lens, longest):
        xq, sa = P.is_rmsnorm_quantize_act_int8_token(x, self.gamma, EPS)
        qkv, _ = P.is_gemm_w4a8_intscale_prepacked(xq, sa, self.qkv[0], self.qkv[1], ALPHA)
        full = P.is_lora_add((x.float() * 0.1).half(), self.a, self.b, adapter, qkv, scales=self.scales)
        h = HEADS * D
        q, _, _ = P.is_qk_norm_rope(full[:, :h], full[:, h : h + KV * D], positions, self.freq, D, gamma_q=self.gq, gamma_k=self.gk, eps=EPS,
                                    v=full[:, h + KV * D :], kv_rows=places, k_out=self.kc, v_out=self.vc)
        out = P.is_attention(q, self.kc, self.vc, offsets, D, longest, ROOM, kv_starts=self.starts, kv_lens=lens)
        y, _ = P.is_linear_w4a8_intscale_prepacked(out, self.o[0], self.o[1], ALPHA)
        return {"x": x, "qkv": qkv, "full": full, "q": q, "out": out, "y": y}


def tokens(lens, past):
    pos = np.concatenate([np.arange(p, p + n) for n, p in zip(lens, past)])
    place = np.concatenate([i * ROOM + np.arange(p, p + n) for i, (n, p) in enumerate(zip(lens, past))])
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    adapter = np.concatenate([np.full(n, e) for n, e in zip(lens, (0, -1, 1))])
    return (i32(adapter), i32(pos), torch.tensor(place, dtype=torch.int64, device=DEV), i32(np.cumsum([0] + list(lens))),
            i32([p + n for n, p in zip(lens, past)])), max(lens)


def check(got, want, bound, what):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    worst = (np.abs(got - want) / np.maximum(bound, 1e-30)).max(initial=0.0)
    assert worst <= 1.0, (what, worst)


def check_step(blk, r, args):
    adapter, pos, place, off, lens = (t.cpu().numpy() for t in args)
    n = lambda t: t.cpu().numpy()  # noqa: E731
    want, bound = B.lora_add(n((r["x"].float() * 0.1).half()), n(blk.a), n(blk.b), adapter.tolist(), n(r["qkv"]), blk.scales.tolist(), [R] * E)
    check(r["full"], want, bound, "adapters")
    h, f = HEADS * D, n(r["full"])
    want, bound = B.qk_norm_rope(f[:, :h], n(blk.gq), EPS, n(blk.freq), pos, D, False)
    check(r["q"], want, bound, "queries")
    want, bound = B.qk_norm_rope(f[:, h : h + KV * D], n(blk.gk), EPS, n(blk.freq), pos, D, False)
    check(blk.kc[args[2]], want, bound, "keys")
    assert np.array_equal(n(blk.vc[args[2]]), f[:, h + KV * D :])
    want, bound = B.attention(n(r["q"]), n(blk.kc), n(blk.vc), off.tolist(), blk.starts.tolist(), lens.tolist(), D, float(np.float32(D ** -0.5)), True,
                              np.zeros(tuple(r["q"].shape)))
    check(r["out"], want, bound, "attention")


def test_prompts_then_decode_steps():
    g = torch.Generator().manual_seed(73)
    lens = (40, 7, 65)
    x = [torch.randn((n + 3, HIDDEN), generator=g).half().to(DEV) for n in lens]
    blk = Block()
    args, longest = tokens(lens, (0, 0, 0))
    r = blk.step(torch.cat([t[:n] for t, n in zip(x, lens)]), *args, longest)
    check_step(blk, r, args)
    # three decode steps: the first as it is, then captured and replayed with new inputs in the same places
    args, longest = tokens((1, 1, 1), lens)
    xin = torch.stack([t[n] for t, n in zip(x, lens)])
    first = blk.step(xin, *args, longest)
    check_step(blk, first, args)
    steps = [first["out"].clone()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = blk.step(xin, *args, longest)
    for s in (1, 2):
        new, _ = tokens((1, 1, 1), [n + s for n in lens])
        for a, b in zip(args, new):
            a.copy_(b)
        xin.copy_(torch.stack([t[n + s] for t, n in zip(x, lens)]))
        graph.replay()
        torch.cuda.synchronize()
        check_step(blk, r, args)
        again = blk.step(xin, *args, longest)           # (writes the same rows of the cache)
        assert torch.equal(again["out"], r["out"]) and torch.equal(again["y"], r["y"])
        steps.append(r["out"].clone())
    # the same tokens in one longer prompt, over the keys that the steps wrote
    args, longest = tokens([n + 3 for n in lens], (0, 0, 0))
    whole = Block()
    r = whole.step(torch.cat(x), *args, longest)
    check_step(whole, r, args)
    at = np.cumsum([n + 3 for n in lens]) - 3
    for s in range(3):
        rows = r["out"][torch.tensor(at + s, device=DEV)]
        # (the GEMM of many rows and that of few agree to the bit, so the queries, keys and values do; attention sums in another order)
        _, bound = B.attention(r["q"].cpu().numpy(), whole.kc.cpu().numpy(), whole.vc.cpu().numpy(), args[3].tolist(), whole.starts.tolist(),
                               args[4].tolist(), D, float(np.float32(D ** -0.5)), True, np.zeros(tuple(r["q"].shape)))
        check(steps[s], rows.double().cpu().numpy(), 2 * bound[at + s], f"step {s}")
    assert torch.equal(whole.kc, blk.kc) and torch.equal(whole.vc, blk.vc)
