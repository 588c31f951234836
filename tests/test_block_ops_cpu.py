"""Per-head norm with rotation, attention and low-rank adapters: what needs no GPU.  The 64-bit oracle against independent forms,
and the refusals of the C ABI and of the binding (before any HIP call)."""
import numpy as np
import pytest
import torch

import paper_2405_14597_amd as P
from oracle import block as B

A = 0x10000  # a fake, 16-byte aligned "device pointer": validation must fail before it is ever dereferenced
BAD, UNSUP = P.IS_ERR_INVALID_ARG, P.IS_ERR_UNSUPPORTED


# ---- the oracle
def test_attention_oracle_against_torch():
    g = np.random.default_rng(1)
    q, k, v = g.standard_normal((7, 4 * 8)), g.standard_normal((9, 2 * 8)), g.standard_normal((9, 2 * 8))
    for causal in (True, False):
        out, bound = B.attention(q, k, v, [0, 7], [0], [9], 8, 0.3, causal, np.zeros_like(q))
        t = lambda x, h: torch.from_numpy(x).view(len(x), h, 8).transpose(0, 1)  # noqa: E731
        mask = torch.ones(7, 9, dtype=torch.bool).tril(2) if causal else None
        want = torch.nn.functional.scaled_dot_product_attention(t(q, 4), t(k, 2).repeat_interleave(2, 0), t(v, 2).repeat_interleave(2, 0),
                                                                attn_mask=mask, scale=0.3)
        assert np.allclose(out, want.transpose(0, 1).reshape(7, 32).numpy(), atol=1e-12)
        assert (bound > 0).all() and (bound < 0.01).all()


def test_attention_oracle_empty_rows_and_rows_of_no_sequence():
    g = np.random.default_rng(2)
    q, k, v = g.standard_normal((6, 8)), g.standard_normal((2, 8)), g.standard_normal((2, 8))
    out, _ = B.attention(q, k, v, [0, 4], [0], [2], 8, 1.0, True, np.full((6, 8), 7.0))
    assert (out[:2] == 0).all() and np.allclose(out[2], v[0]) and (out[4:] == 7).all()
    out, _ = B.attention(q, k, v, [0, 4], [0], [0], 8, 1.0, False, np.full((6, 8), 7.0))
    assert (out[:4] == 0).all()


def test_rope_oracle_is_a_rotation():
    g = np.random.default_rng(3)
    x = g.standard_normal((5, 3 * 16))
    f = (1.0 / 100.0 ** (np.arange(6) / 6)).astype(np.float32)
    pos = [0, 1, 9, 1000, 131071]
    for inter in (False, True):
        y, _ = B.qk_norm_rope(x, None, 0.0, f, pos, 16, inter)
        assert np.allclose(y[0], x[0])
        z, w = x.reshape(5, 3, 16), y.reshape(5, 3, 16)
        assert np.allclose(z[..., 12:], w[..., 12:]) and np.allclose((z * z).sum(-1), (w * w).sum(-1))
        a, b = (slice(0, 12, 2), slice(1, 12, 2)) if inter else (slice(0, 6), slice(6, 12))
        turn = np.exp(1j * np.array(pos)[:, None] * f.astype(np.float64))[:, None]
        assert np.allclose((z[..., a] + 1j * z[..., b]) * turn, w[..., a] + 1j * w[..., b])
    y, _ = B.qk_norm_rope(x, np.ones(16), 1e-30, f, [0] * 5, 16, False)
    assert np.allclose((y.reshape(5, 3, 16) ** 2).mean(-1), 1.0)


def test_lora_oracle_is_a_matrix_product():
    g = np.random.default_rng(4)
    x, a, b, base = g.standard_normal((4, 8)), g.standard_normal((2, 3, 8)), g.standard_normal((2, 5, 3)), g.standard_normal((4, 5))
    out, _ = B.lora_add(x, a, b, [0, -1, 1, 2], base, [2.0, 0.5], [3, 2])
    assert np.allclose(out[0], base[0] + 2 * (b[0] @ a[0]) @ x[0])
    assert np.allclose(out[2], base[2] + 0.5 * (b[1][:, :2] @ a[1][:2]) @ x[2])
    assert (out[1] == base[1]).all() and (out[3] == base[3]).all()


# ---- refusals of the C ABI
def rope(**kw):
    a = dict(q=A, ldq=256, k=A * 2, ldk=128, v=None, ldv=0, gq=None, gk=None, eps=1e-5, f=A, rot=64, inter=0, pos=A, rows=None, M=4,
             hq=4, hk=2, d=64, cache=4, qo=A * 3, ldqo=256, ko=A * 4, ldko=128, vo=None, ldvo=0)
    assert set(kw) <= set(a)
    a.update(kw)
    return P.load_library().is_qk_norm_rope(*a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(M=-1), dict(hq=-1), dict(hk=-1), dict(hq=0, hk=0), dict(d=0), dict(d=60, rot=8), dict(rot=-8), dict(rot=12), dict(rot=72),
    dict(inter=2), dict(ldq=248), dict(ldq=260), dict(ldqo=128), dict(ldk=64), dict(ldko=132), dict(q=A + 8), dict(k=None), dict(qo=None),
    dict(ko=A + 2), dict(f=None), dict(f=A + 2), dict(pos=None), dict(pos=A + 2), dict(rows=A + 4), dict(gq=A + 8), dict(gk=A, eps=0.0),
    dict(gq=A, eps=float("nan")), dict(gq=A, eps=float("inf")), dict(v=A), dict(vo=A), dict(v=A, vo=A * 5, ldv=64, ldvo=128), dict(cache=-1),
    dict(cache=3), dict(rows=A, ko=A * 2), dict(qo=A, ldqo=512), dict(rows=A, v=A * 5, vo=A * 5, ldv=128, ldvo=128)])
def test_rope_refusals(kw):
    assert rope(**kw) == BAD


def test_rope_unsupported_and_empty():
    assert rope(d=264, rot=8, ldq=2048, ldqo=2048, ldk=1024, ldko=1024) == UNSUP
    assert rope(M=(1 << 20) + 1, cache=1 << 21) == UNSUP
    assert rope(M=0, q=None, k=None, qo=None, ko=None, pos=None, f=None, cache=0) == P.IS_OK


def attention(**kw):
    a = dict(q=A, ldq=512, k=A * 2, ldk=256, v=A * 3, ldv=256, off=A, starts=None, lens=None, M=4, rows=4, seqs=1, mq=4, mkv=4, hq=4, hkv=2,
             d=128, scale=0.1, causal=1, out=A * 4, ldo=512, ws=None, wsb=0)
    assert set(kw) <= set(a)
    a.update(kw)
    return P.load_library().is_attention(*a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(M=-1), dict(seqs=-1), dict(mq=-1), dict(mkv=-1), dict(hq=0), dict(hkv=0), dict(hkv=3), dict(d=0), dict(rows=-1), dict(scale=0.0),
    dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(causal=2), dict(ldq=504), dict(ldq=516), dict(ldk=128),
    dict(ldv=260), dict(ldo=256), dict(q=None), dict(k=None), dict(v=A + 8), dict(out=None), dict(off=None), dict(off=A + 2),
    dict(starts=A + 4), dict(lens=A + 2), dict(ws=A + 8)])
def test_attention_refusals(kw):
    assert attention(**kw) == BAD


def test_attention_unsupported_empty_and_workspace():
    assert attention(d=96, ldq=384, ldk=192, ldv=192, ldo=384) == UNSUP
    assert attention(M=(1 << 20) + 1) == UNSUP
    assert attention(ldk=(1 << 23) + 8) == UNSUP
    assert attention(seqs=1 << 22, hq=8, ldq=1024, ldo=1024) == UNSUP
    assert attention(mkv=(1 << 30) + 1) == UNSUP
    assert attention(M=0, q=None, out=None, off=None) == P.IS_OK
    assert attention(seqs=0, off=None) == P.IS_OK
    need = P.is_attention_workspace_bytes(4, 1, 4, 100000, 4, 2, 128)
    assert need > 0
    assert attention(mkv=100000, rows=100000) == P.IS_ERR_WORKSPACE
    assert attention(mkv=100000, rows=100000, ws=A, wsb=need - 1) == P.IS_ERR_WORKSPACE
    assert P.is_attention_workspace_bytes(4, 1, 4, 64, 4, 2, 128) == 0
    assert P.is_attention_workspace_bytes(4, 1, 4, 100000, 4, 2, 96) == 0
    assert P.is_attention_workspace_bytes(0, 0, 4, 100000, 4, 2, 128) == 0 and P.is_attention_workspace_bytes(4, 0, 4, 100000, 4, 2, 128) == 0


def lora(**kw):
    a = dict(x=A, ldx=64, a=A * 2, b=A * 3, rows=A, scales=None, ranks=None, M=4, N=33, K=64, R=16, E=2, base=A * 4, ldb=33, out=A * 5, ldo=33,
             ws=A * 6, wsb=1 << 30)
    assert set(kw) <= set(a)
    a.update(kw)
    return P.load_library().is_lora_add(*a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(M=-1), dict(N=0), dict(K=0), dict(K=60, ldx=64), dict(R=0), dict(R=12), dict(E=-1), dict(ldx=56), dict(ldx=68), dict(ldo=32),
    dict(ldb=32), dict(base=A * 5, ldb=40, ldo=48), dict(x=None), dict(x=A + 8), dict(a=None), dict(b=A + 4), dict(base=A + 2), dict(out=None),
    dict(rows=None), dict(rows=A + 2), dict(scales=A + 2), dict(ranks=A + 2), dict(ws=A + 8)])
def test_lora_refusals(kw):
    assert lora(**kw) == BAD


def test_lora_unsupported_empty_and_workspace():
    assert lora(R=136) == UNSUP
    assert lora(M=(1 << 20) + 1) == UNSUP
    assert lora(M=0, x=None, out=None, rows=None, ws=None, wsb=0) == P.IS_OK
    need = P.is_lora_workspace_bytes(4, 33, 64, 16, 2)
    assert need > 0 and lora(ws=None, wsb=0) == P.IS_ERR_WORKSPACE and lora(wsb=need - 1) == P.IS_ERR_WORKSPACE
    assert P.is_lora_workspace_bytes(0, 33, 64, 16, 2) == 0 and P.is_lora_workspace_bytes(4, 33, 60, 16, 2) == 0


# ---- refusals of the binding
def test_binding_refuses_host_tensors():
    half = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    whole = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="current cuda device"):
        P.is_qk_norm_rope(half(4, 64), half(4, 64), whole, torch.zeros(32), 64)
    with pytest.raises(ValueError, match="current cuda device"):
        P.is_attention(half(4, 64), half(4, 64), half(4, 64), whole[:2], 64, 4, 4)
    with pytest.raises(ValueError, match="current cuda device"):
        P.is_lora_add(half(4, 64), half(2, 8, 64), half(2, 5, 8), whole, half(4, 5))
