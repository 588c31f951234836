"""The operators between a decoder block's qkv projection and its output projection, and the low-rank adapters beside any
projection, as cases that can be timed: in their plain form (elementary torch operations in 32 bits, rounded once) and by
the framework's own kernels (`own`).

Kinds of case
  attention  softmax(q k^T scale) v over sequences of different lengths packed behind each other, grouped heads.  A
             "prompt" brings several new tokens over a past of earlier ones, a "single" is one new token over its past.
             "cached": keys and values lie in a cache in which every sequence has a run of rows of its own; otherwise q, k
             and v are the columns of one qkv projection's output.
  rope       per-head RMSNorm of q and k and the rotation by position, from the columns of a qkv projection's output; the
             new keys and values go to their rows of the cache.
  lora       base + scale * (x A^T) B^T with the adapter of each row: rows of one request share an adapter, about one
             request in eight has none, some adapters have half the stacked rank.

Head counts and widths are those of the LLaMA and Mixtral blocks that the benchmark's linears belong to (32 heads of 128
with 32 or 8 key heads, 64 with 8), hidden sizes 4096 and 8192; rope bases 10^4 and 5 * 10^5.
"""
import math
import random

import torch

own = False

EPS = 1e-5


def listed():
    def attention(name, heads, kv_heads, dim=128, prompts=0, new=(0, 0), past=(0, 0), singles=0, context=(0, 0), cached=True,
                  causal=True, lens=1):
        return {"name": name, "kind": "attention", "heads": heads, "kv_heads": kv_heads, "dim": dim, "prompts": prompts,
                "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1], "singles": singles,
                "context_lo": context[0], "context_hi": context[1], "cached": cached, "causal": causal, "lens": lens}

    def rope(name, tokens, heads, kv_heads, dim=128, rot=128, interleaved=False, norm=True, cached=True, base=500000.0, far=8192):
        return {"name": name, "kind": "rope", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rot,
                "interleaved": interleaved, "norm": norm, "cached": cached, "base": base, "far": far}

    def lora(name, rows, requests, adapters, rank, k, n, lens=1):
        return {"name": name, "kind": "lora", "rows": rows, "requests": requests, "adapters": adapters, "rank": rank, "k": k,
                "n": n, "lens": lens}

    return [
        # one user's next token early in an answer: latency alone
        attention("attention_one_token", 32, 8, singles=1, context=(333, 333)),
        # a decode step of 64 requests, contexts of a few hundred to eight thousand tokens
        attention("attention_decode_b64", 32, 8, singles=64, context=(200, 8000)),
        # a decode step over long contexts at 64 heads: a gigabyte of keys and values
        attention("attention_decode_long", 64, 8, singles=8, context=(20000, 36000)),
        # what a scheduler with chunked prompts sends: a chunk over its past beside the other requests' next tokens
        attention("attention_chunk_mixed", 32, 8, prompts=1, new=(300, 300), past=(4000, 4000), singles=24, context=(100, 6000)),
        # a batch of prompts of ragged lengths, straight from the qkv projection
        attention("attention_prompts", 32, 8, prompts=12, new=(17, 2048), cached=False),
        # a whole prompt at 64 heads
        attention("attention_prompt_8192", 64, 8, prompts=1, new=(8192, 8192), cached=False),
        # heads of 64, keys of both directions (an encoder's batch), as many key heads as query heads
        attention("attention_both_ways", 32, 32, dim=64, prompts=5, new=(301, 1777), cached=False, causal=False),
        # a decode step's queries and keys
        rope("rope_decode_16", 16, 32, 8),
        # a long prompt's, at 64 heads
        rope("rope_prompt_8192", 8192, 64, 8, far=131072),
        # a decode step of 64 requests that use 32 adapters
        lora("lora_decode_64", 64, 64, 32, 16, 4096, 4096),
        # one request's next token, a narrow key projection
        lora("lora_one_token", 1, 1, 4, 8, 4096, 1024, lens=3),
        # prompts of nine requests on the qkv projection
        lora("lora_prompts", 4096, 9, 6, 64, 4096, 6144),
    ]


def draw(rng):
    """One more case of the same ranges."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choices(("attention", "rope", "lora"), (0.56, 0.18, 0.26))[0]
    heads, kv_heads = rng.choice(((32, 32), (32, 8), (64, 8), (16, 4), (24, 8), (8, 1)))
    if kind == "rope":
        dim = rng.choice((64, 128, 128, 96))
        return {"kind": kind, "tokens": log_int(1, 8192), "heads": heads, "kv_heads": kv_heads, "dim": dim,
                "rot": rng.choice((dim, dim, dim // 2)), "interleaved": rng.random() < 0.3, "norm": rng.random() < 0.7,
                "cached": rng.random() < 0.7, "base": rng.choice((10000.0, 500000.0)), "far": log_int(8192, 131072)}
    if kind == "lora":
        rows = log_int(1, 4096)
        requests = rows if rows <= 64 and rng.random() < 0.7 else min(rows, log_int(1, 16))
        return {"kind": kind, "rows": rows, "requests": requests, "adapters": log_int(1, 32), "rank": rng.choice((8, 16, 16, 32, 64)),
                "k": 128 * log_int(8, 64), "n": log_int(500, 6144), "lens": rng.randrange(1 << 30)}
    c = {"kind": kind, "heads": heads, "kv_heads": kv_heads, "dim": rng.choice((64, 128, 128, 128)), "prompts": 0, "new_lo": 0,
         "new_hi": 0, "past_lo": 0, "past_hi": 0, "singles": 0, "context_lo": 0, "context_hi": 0, "cached": True, "causal": True,
         "lens": rng.randrange(1 << 30)}
    form = rng.choice(("decode", "decode", "mixed", "prompts", "prompts"))
    if form == "decode":
        c["singles"] = log_int(1, 64)
        c["context_hi"] = log_int(64, 32768 if c["singles"] <= 8 else 8192)
        c["context_lo"] = max(1, c["context_hi"] // rng.choice((1, 2, 10)))
    elif form == "mixed":
        c["prompts"], c["singles"] = rng.randint(1, 3), rng.randint(1, 24)
        c["new_hi"], c["past_hi"], c["context_hi"] = log_int(2, 512), log_int(1, 6000), log_int(50, 6000)
        c["new_lo"], c["past_lo"], c["context_lo"] = max(1, c["new_hi"] // 2), c["past_hi"] // 4, max(1, c["context_hi"] // 10)
    else:
        c["prompts"], c["new_hi"], c["cached"], c["causal"] = log_int(1, 16), log_int(64, 4096), rng.random() < 0.3, rng.random() < 0.8
        c["new_lo"] = max(1, c["new_hi"] // rng.choice((1, 2, 30)))
    # no more than the largest listed case takes, in pairs of a padded batch too
    while heads * (c["prompts"] + c["singles"]) * max(1, c["new_hi"]) * (max(c["new_hi"] + c["past_hi"], c["context_hi"])) > 64 * 8192 * 8192:
        if c["prompts"] + c["singles"] > 2:
            c["prompts"], c["singles"] = -(-c["prompts"] // 2), c["singles"] // 2
        else:
            c["new_hi"] = -(-c["new_hi"] // 2)
            c["new_lo"] = min(c["new_lo"], c["new_hi"])
    return c


# ---- lengths: a case's own, whatever the seed of its values
def _sequences(c):
    """[(new tokens, keys)] of an attention case, in the order of the batch."""
    r = random.Random(c["lens"])
    got = []
    for _ in range(c["prompts"]):
        n = r.randint(c["new_lo"], c["new_hi"])
        got.append((n, n + r.randint(c["past_lo"], c["past_hi"])))
    got += [(1, r.randint(c["context_lo"], c["context_hi"])) for _ in range(c["singles"])]
    return got


def _row_adapters(c):
    """The adapter of every row of a lora case, -1 where there is none."""
    r = random.Random(c["lens"])
    cuts = sorted(r.sample(range(1, c["rows"]), c["requests"] - 1)) if c["requests"] > 1 else []
    rows = []
    for a, b in zip([0] + cuts, cuts + [c["rows"]]):
        rows += [-1 if c["requests"] > 1 and r.random() < 0.125 else r.randrange(c["adapters"])] * (b - a)
    return rows


def _ranks(c):
    r = random.Random(c["lens"] + 1)
    return [c["rank"] // 2 if r.random() < 0.25 else c["rank"] for _ in range(c["adapters"])]


def work(c):
    if c["kind"] == "attention":
        seqs, h, hk, d = _sequences(c), c["heads"], c["kv_heads"], c["dim"]
        pairs = sum(q * kv - (q * (q - 1) // 2 if c["causal"] else 0) for q, kv in seqs)
        return {"bytes": 2.0 * d * (2 * h * sum(q for q, _ in seqs) + 2 * hk * sum(kv for _, kv in seqs)), "flops": 4.0 * d * h * pairs}
    if c["kind"] == "rope":
        rows = c["heads"] + c["kv_heads"] * (2 if c["cached"] else 1)
        return {"bytes": 4.0 * c["tokens"] * rows * c["dim"], "flops": 8.0 * c["tokens"] * (c["heads"] + c["kv_heads"]) * c["dim"]}
    rows, ranks = _row_adapters(c), _ranks(c)
    used = sum(ranks[a] for a in set(rows) if a >= 0)
    inner = sum(ranks[a] for a in rows if a >= 0)
    with_one = sum(a >= 0 for a in rows)
    return {"bytes": 2.0 * (with_one * c["k"] + 2 * c["rows"] * c["n"] + used * (c["k"] + c["n"])), "flops": 2.0 * inner * (c["k"] + c["n"])}


# ---- inputs and what a program keeps
def prepare(c, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float16)

    def whole(values, dtype):
        return torch.tensor(values, dtype=dtype, device=dev)

    if c["kind"] == "attention":
        seqs, h, hk, d = _sequences(c), c["heads"], c["kv_heads"], c["dim"]
        m = sum(q for q, _ in seqs)
        s = {"kind": "attention", "heads": h, "kv_heads": hk, "dim": d, "causal": c["causal"], "scale": d ** -0.5, "m": m,
             "max_q": max(q for q, _ in seqs), "max_kv": max(kv for _, kv in seqs)}
        offsets = [0]
        for q, _ in seqs:
            offsets.append(offsets[-1] + q)
        s["q_offsets"] = whole(offsets, torch.int32)
        if c["cached"]:
            # every sequence has a run of rows in the cache, longer than what it has used, in no order
            order, starts, rows = list(range(len(seqs))), [0] * len(seqs), 0
            random.Random(c["lens"] + 2).shuffle(order)
            for i in order:
                starts[i] = rows
                rows += seqs[i][1] + 37
            s["q"] = normal(m, h * d).mul_(1.5)
            s["k"], s["v"] = normal(rows, hk * d), normal(rows, hk * d)
            s["kv_starts"], s["kv_lens"] = whole(starts, torch.int64), whole([kv for _, kv in seqs], torch.int32)
        else:
            qkv = normal(m, (h + 2 * hk) * d)
            s["q"], s["k"], s["v"] = qkv[:, : h * d], qkv[:, h * d : (h + hk) * d], qkv[:, (h + hk) * d :]
            s["q"].mul_(1.5)
            s["kv_starts"] = s["kv_lens"] = None
        s["out"] = torch.zeros((m, h * d), dtype=torch.float16, device=dev)
        return s
    if c["kind"] == "rope":
        t, h, hk, d = c["tokens"], c["heads"], c["kv_heads"], c["dim"]
        qkv = normal(t, (h + 2 * hk) * d).mul_(0.7)
        s = {"kind": "rope", "dim": d, "interleaved": c["interleaved"], "q": qkv[:, : h * d], "k": qkv[:, h * d : (h + hk) * d],
             "v": qkv[:, (h + hk) * d :] if c["cached"] else None, "gamma_q": None, "gamma_k": None, "kv_rows": None}
        s["inv_freq"] = (1.0 / c["base"] ** (torch.arange(0, c["rot"], 2, dtype=torch.float64, device=dev) / c["rot"])).float()
        if c["norm"]:
            s["gamma_q"], s["gamma_k"] = (torch.rand((2, d), generator=gen, device=dev).add_(0.5)).half()
        rows = t
        if t > 64:  # a prompt's positions run on from its past
            start = c["far"] - t if c["far"] > t else 0
            s["positions"] = torch.arange(start, start + t, dtype=torch.int32, device=dev)
        else:       # every row is another request's
            s["positions"] = torch.randint(0, c["far"], (t,), generator=gen, device=dev, dtype=torch.int32)
        if c["cached"]:
            rows = t + 64
            s["kv_rows"] = torch.randperm(rows, generator=gen, device=dev)[:t] if t <= 64 else torch.arange(31, 31 + t, device=dev)
        s["q_out"] = torch.zeros((t, h * d), dtype=torch.float16, device=dev)
        s["k_out"] = torch.zeros((rows, hk * d), dtype=torch.float16, device=dev)
        s["v_out"] = torch.zeros((rows, hk * d), dtype=torch.float16, device=dev) if c["cached"] else None
        return s
    m, n, k, e, r = c["rows"], c["n"], c["k"], c["adapters"], c["rank"]
    x = torch.randn((m, k), generator=gen, device=dev)
    x[:, torch.randperm(k, generator=gen, device=dev)[: k // 100]] *= 20.0
    return {"kind": "lora", "x": x.half(), "base": normal(m, n), "a": normal(e, r, k).mul_(k ** -0.5), "b": normal(e, n, r).mul_(0.1),
            "scales": torch.rand((e,), generator=gen, device=dev).add_(0.5), "ranks": whole(_ranks(c), torch.int32),
            "row_adapter": whole(_row_adapters(c), torch.int32), "out": torch.zeros((m, n), dtype=torch.float16, device=dev)}


# ---- one pass
def run(s):
    if s["kind"] == "attention":
        return _attention_own(s) if own else _attention(s)
    if s["kind"] == "rope":
        return _rope_own(s) if own else _rope(s)
    return _lora_own(s) if own else _lora(s)


def _attention_own(s):
    import paper_2405_14597_amd as P
    if "ws" not in s:  # kept by the program from its first call on
        nbytes = P.is_attention_workspace_bytes(s["m"], s["q_offsets"].numel() - 1, s["max_q"], s["max_kv"], s["heads"], s["kv_heads"], s["dim"])
        s["ws"] = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=s["q"].device)
    return P.is_attention(s["q"], s["k"], s["v"], s["q_offsets"], s["dim"], s["max_q"], s["max_kv"], scale=s["scale"], causal=s["causal"],
                          kv_starts=s["kv_starts"], kv_lens=s["kv_lens"], out=s["out"], workspace=s["ws"])


def _rope_own(s):
    import paper_2405_14597_amd as P
    return P.is_qk_norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], s["dim"], gamma_q=s["gamma_q"], gamma_k=s["gamma_k"], eps=EPS,
                             interleaved=s["interleaved"], v=s["v"], kv_rows=s["kv_rows"], q_out=s["q_out"], k_out=s["k_out"], v_out=s["v_out"])


def _lora_own(s):
    import paper_2405_14597_amd as P
    if "ws" not in s:
        m, k = s["x"].shape
        nbytes = P.is_lora_workspace_bytes(m, s["b"].shape[1], k, s["a"].shape[1], s["a"].shape[0])
        s["ws"] = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=s["x"].device)
    return P.is_lora_add(s["x"], s["a"], s["b"], s["row_adapter"], s["base"], scales=s["scales"], ranks=s["ranks"], out=s["out"], workspace=s["ws"])


def _attention(s):
    """As a padded batch: [sequence, key head, query head of its group and row, key]."""
    h, hk, d, offsets = s["heads"], s["kv_heads"], s["dim"], s["q_offsets"].long()
    dev, n, lq, lk = s["q"].device, offsets.numel() - 1, s["max_q"], s["max_kv"]
    q_len = offsets[1:] - offsets[:-1]
    kv_len = q_len if s["kv_lens"] is None else s["kv_lens"].long()
    kv_start = offsets[:-1] if s["kv_starts"] is None else s["kv_starts"]
    i, j = torch.arange(lq, device=dev), torch.arange(lk, device=dev)
    q_in, k_in = i < q_len[:, None], j < kv_len[:, None]                                     # [n, lq], [n, lk]
    q_at = torch.where(q_in, offsets[:-1, None] + i, 0)
    k_at = torch.where(k_in, kv_start[:, None] + j, 0)
    q = s["q"][q_at].float().view(n, lq, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(n, hk, h // hk * lq, d)
    k = s["k"][k_at].float().view(n, lk, hk, d).permute(0, 2, 3, 1).contiguous()
    v = s["v"][k_at].float().view(n, lk, hk, d).permute(0, 2, 1, 3).contiguous()
    seen = k_in[:, None, :].expand(n, lq, lk)
    if s["causal"]:
        seen = seen & (j <= i[:, None] + (kv_len - q_len)[:, None, None])
    p = torch.matmul(q.mul_(s["scale"]), k).view(n, hk, h // hk, lq, lk)
    p.masked_fill_(~seen[:, None, None], float("-inf"))
    top = p.amax(-1, keepdim=True)
    p.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, hk, h // hk * lq, lk), v).view(n, hk, h // hk, lq, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(n, lq, h * d).half()
    s["out"][q_at[q_in]] = o[q_in]
    return s["out"]


def _rope(s):
    d, rot = s["dim"], 2 * s["inv_freq"].numel()
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(x, gamma):
        x = x.float().unflatten(-1, (-1, d))
        if gamma is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gamma.float()
        x1, x2 = (x[..., 0:rot:2], x[..., 1:rot:2]) if s["interleaved"] else (x[..., : rot // 2], x[..., rot // 2 : rot])
        y = torch.stack((x1 * cos - x2 * sin, x2 * cos + x1 * sin), -1 if s["interleaved"] else -2).flatten(-2)
        return torch.cat((y, x[..., rot:]), -1).flatten(-2).half()

    s["q_out"].copy_(turned(s["q"], s["gamma_q"]))
    k = turned(s["k"], s["gamma_k"])
    if s["kv_rows"] is None:
        s["k_out"].copy_(k)
        return s["q_out"], s["k_out"]
    s["k_out"][s["kv_rows"]] = k
    s["v_out"][s["kv_rows"]] = s["v"]
    return s["q_out"], s["k_out"], s["v_out"]


def _lora(s):
    """All adapters side by side, the products of another adapter than the row's masked out."""
    e, r, k = s["a"].shape
    n = s["b"].shape[1]
    mine = s["row_adapter"][:, None] == torch.arange(e, device=s["x"].device)                # [m, e]
    factor = (mine * s["scales"])[:, :, None] * (torch.arange(r, device=s["x"].device) < s["ranks"][:, None])
    t = (s["x"].float() @ s["a"].float().view(e * r, k).t()).view(-1, e, r) * factor
    delta = t.view(-1, e * r) @ s["b"].float().permute(0, 2, 1).reshape(e * r, n)
    s["out"].copy_(s["base"].float() + delta)
    return s["out"]


# ---- the definitions in 64 bits, one sequence, head or adapter at a time
def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "attention":
        h, hk, d = c["heads"], c["kv_heads"], c["dim"]
        out, at, dev = torch.zeros((s["m"], h, d), dtype=torch.float64, device=s["q"].device), 0, s["q"].device
        for i, (nq, nk) in enumerate(_sequences(c)):
            first = at if s["kv_starts"] is None else int(s["kv_starts"][i])
            for g in range(hk):
                keys = s["k"][first : first + nk, g * d : (g + 1) * d].double()
                values = s["v"][first : first + nk, g * d : (g + 1) * d].double()
                for head in range(g * (h // hk), (g + 1) * (h // hk)):
                    z = s["q"][at : at + nq, head * d : (head + 1) * d].double() @ keys.t() * s["scale"]
                    if c["causal"]:
                        z = z + torch.full((nq, nk), float("-inf"), dtype=torch.float64, device=dev).triu(nk - nq + 1)
                    out[at : at + nq, head] = torch.softmax(z, -1) @ values
            at += nq
        return out.flatten(1)
    if c["kind"] == "rope":
        d, half = c["dim"], c["rot"] // 2
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=s["q"].device), s["positions"].double()[:, None] * s["inv_freq"].double())
        first = torch.arange(half, device=s["q"].device) * (2 if c["interleaved"] else 1)
        second = first + (1 if c["interleaved"] else half)
        got = []
        for x, gamma in ((s["q"], s["gamma_q"]), (s["k"], s["gamma_k"])):
            y = x.double().reshape(c["tokens"], -1, d).clone()
            if gamma is not None:
                y = y / (y.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * gamma.double()
            z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
            y[..., first], y[..., second] = z.real, z.imag
            got.append(y.reshape(c["tokens"], -1))
        if not c["cached"]:
            return tuple(got)
        keys, values = s["k_out"].double(), s["v_out"].double()
        keys[s["kv_rows"]], values[s["kv_rows"]] = got[1], s["v"].double()
        return got[0], keys, values
    out, rows, ranks = s["base"].double(), _row_adapters(c), _ranks(c)
    for e in sorted(set(rows) - {-1}):
        at = torch.tensor([i for i, a in enumerate(rows) if a == e], device=out.device)
        inner = s["x"][at].double() @ s["a"][e, : ranks[e]].double().t()
        out[at] += s["scales"][e].double() * (inner @ s["b"][e, :, : ranks[e]].double().t())
    return out
