"""The attention half of a block with adapters on its projections, on the route that has their inputs in fp16: the normed rows go to the
linear call and to the adapters alike, and attention's rows to the output projection and its adapters.  Prompts of three requests, every
operator against the 64-bit oracle on the inputs it had, and the same tokens one at a time."""
import numpy as np
import pytest
import torch

import paper_2405_14597_amd as P
from oracle import block as B
from test_gpu_block import ALPHA, D, DEV, E, EPS, HEADS, HIDDEN, KV, R, WIDE, check, projection

pytestmark = pytest.mark.gpu
ROOM, LENS, ADAPTERS = 96, (40, 7, 65), (1, -1, 0)


class Block:
    def __init__(self):
        g = torch.Generator().manual_seed(107)
        self.gamma, self.gq, self.gk = ((torch.rand(n, generator=g) + 0.5).half().to(DEV) for n in (HIDDEN, D, D))
        self.qkv, self.o = projection(g, WIDE, HIDDEN), projection(g, HIDDEN, HEADS * D)
        self.lora = [[(torch.randn(s, generator=g) * f).half().to(DEV) for s, f in (((E, R, k), k ** -0.5), ((E, n, R), 0.3))]
                     for n, k in ((WIDE, HIDDEN), (HIDDEN, HEADS * D))]
        self.scales, self.ranks = torch.tensor([1.5, 0.5], device=DEV), torch.tensor([R, 5], dtype=torch.int32, device=DEV)
        self.freq = (1.0 / 10000.0 ** (torch.arange(0, D, 2, dtype=torch.float64) / D)).float().to(DEV)
        self.kc, self.vc = (torch.zeros((3 * ROOM, KV * D), dtype=torch.float16, device=DEV) for _ in "kv")
        self.starts = torch.tensor([0, ROOM, 2 * ROOM], dtype=torch.int64, device=DEV)

    def norm(self, x):
        x = x.float()
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * self.gamma.float()).half()

    def step(self, x, past, new):
        """`new` rows of each request behind `past` of its own."""
        whole = lambda v, t=torch.int32: torch.tensor(np.asarray(v), dtype=t, device=DEV)  # noqa: E731
        pos = np.concatenate([np.arange(p, p + n) for p, n in zip(past, new)])
        place = whole(np.concatenate([i * ROOM + np.arange(p, p + n) for i, (p, n) in enumerate(zip(past, new))]), torch.int64)
        e = whole(np.repeat(ADAPTERS, new))
        off, lens = whole(np.cumsum([0] + list(new))), whole(np.add(past, new))
        n = lambda t: t.cpu().numpy()  # noqa: E731
        add = lambda which, rows, base: P.is_lora_add(rows, *self.lora[which], e, base, scales=self.scales, ranks=self.ranks)  # noqa: E731

        def check_add(which, rows, base, got, what):
            want, bound = B.lora_add(n(rows), n(self.lora[which][0]), n(self.lora[which][1]), e.tolist(), n(base), self.scales.tolist(),
                                     self.ranks.tolist())
            check(got, want, bound, what)

        h = self.norm(x)
        base, _ = P.is_linear_w4a8_intscale_prepacked(h, *self.qkv, ALPHA)
        qkv = add(0, h, base)
        check_add(0, h, base, qkv, "qkv and its adapters")
        w = HEADS * D
        q, _, _ = P.is_qk_norm_rope(qkv[:, :w], qkv[:, w : w + KV * D], whole(pos), self.freq, D, gamma_q=self.gq, gamma_k=self.gk, eps=EPS,
                                    v=qkv[:, w + KV * D :], kv_rows=place, k_out=self.kc, v_out=self.vc)
        want, bound = B.qk_norm_rope(n(qkv)[:, :w], n(self.gq), EPS, n(self.freq), pos, D, False)
        check(q, want, bound, "queries")
        out = P.is_attention(q, self.kc, self.vc, off, D, max(new), ROOM, kv_starts=self.starts, kv_lens=lens)
        want, bound = B.attention(n(q), n(self.kc), n(self.vc), off.tolist(), self.starts.tolist(), lens.tolist(), D, float(np.float32(D ** -0.5)),
                                  True, np.zeros(tuple(q.shape)))
        check(out, want, bound, "attention")
        base, _ = P.is_linear_w4a8_intscale_prepacked(out, *self.o, ALPHA)
        y = P.is_lora_add(out, *self.lora[1], e, base, scales=self.scales, ranks=self.ranks, out=base.clone())
        check_add(1, out, base, y, "output projection and its adapters")
        return {"qkv": qkv, "q": q, "bound": bound, "out": out, "y": y}


def test_prompts_and_single_tokens():
    g = torch.Generator().manual_seed(109)
    x = [torch.randn((n + 2, HIDDEN), generator=g).half().to(DEV) for n in LENS]
    blk, whole = Block(), Block()
    blk.step(torch.cat([t[:n] for t, n in zip(x, LENS)]), (0, 0, 0), LENS)
    one = [blk.step(torch.stack([t[n + s] for t, n in zip(x, LENS)]), [n + s for n in LENS], (1, 1, 1)) for s in range(2)]
    r = whole.step(torch.cat(x), (0, 0, 0), [n + 2 for n in LENS])
    at = np.cumsum([n + 2 for n in LENS]) - 2
    for s in range(2):
        # the linear call and the adapters' form by rows agree to the bit whatever the number of rows; attention sums in another order
        assert torch.equal(one[s]["qkv"], r["qkv"][at + s]) and torch.equal(one[s]["q"], r["q"][at + s])
        check(one[s]["out"], r["out"][at + s].double().cpu().numpy(), 2 * r["bound"][at + s], f"step {s}")
    assert torch.equal(blk.kc, whole.kc) and torch.equal(blk.vc, whole.vc)
