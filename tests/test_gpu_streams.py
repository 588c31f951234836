"""Calls on a stream of their own while the current stream has work queued: what a call allocates and fills is its stream's."""
import pytest
import torch

import paper_2405_14597_amd as P

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def busy():
    """Some tens of milliseconds of work on the current stream."""
    a = torch.zeros((8192, 8192), dtype=torch.float16, device=DEV)
    for _ in range(40):
        a = a @ a
    return a


def test_attention_with_an_output_of_its_own():
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn((n, 256), generator=g).half().to(DEV) for n in (70, 300, 300))
    off, starts, lens = (torch.tensor(x, dtype=t, device=DEV) for x, t in (([0, 66, 68], torch.int32), ([0, 100], torch.int64), ([300, 200], torch.int32)))
    call = lambda **kw: P.is_attention(q, k, v, off, 64, 66, 300, kv_starts=starts, kv_lens=lens, **kw)  # noqa: E731
    want = call()
    assert (want[68:] == 0).all() and (want[:68] != 0).any()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    keep = busy()
    got = call(stream=side)
    side.synchronize()
    now = got.clone()            # (behind the current stream's work)
    torch.cuda.synchronize()
    assert torch.equal(now, want) and torch.equal(got, want)
    del keep


def test_prepacked_gemm_with_a_workspace_of_its_own():
    # K cut over workgroups, which meet by arrival counters in the workspace
    M, N, K, G = 4, 64, 65536, 128
    g = torch.Generator().manual_seed(5)
    q = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, generator=g).to(DEV)
    si = torch.randint(1, 1025, (N, K // G), dtype=torch.int32, generator=g).to(DEV)
    xq = torch.randint(-127, 128, (M, K), dtype=torch.int8, generator=g).to(DEV)
    sa, chan = (torch.rand(n, generator=g).to(DEV) * 1e-3 for n in (M, N))
    packed = P.is_prepack_w4(q, si, G)
    assert P.is_gemm_prepacked_workspace_bytes(M, N, K, G) > 0 and P.is_describe_prepacked(M, N, K, G)[0].startswith("gemm_decode_pk_kernel<")
    want = P.is_gemm_w4a8_intscale_prepacked(xq, sa, packed, chan, 10, want_acc=True)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    keep = busy()
    got = P.is_gemm_w4a8_intscale_prepacked(xq, sa, packed, chan, 10, want_acc=True, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    del keep


def test_new_outputs_leave_alone_what_the_current_stream_still_reads():
    # a tensor given up on the current stream whose last reader is still queued there: the call's new output must not lie in it
    g = torch.Generator().manual_seed(7)
    q = torch.randn((2048, 4096), generator=g).half().to(DEV)
    pos, freq = torch.arange(2048, dtype=torch.int32, device=DEV), torch.ones(64, device=DEV)
    k = torch.empty((2048, 0), dtype=torch.float16, device=DEV)
    want, _ = P.is_qk_norm_rope(q, k, pos, freq, 128)
    side = torch.cuda.Stream()
    last = torch.full((2048, 4096), 3.0, dtype=torch.float16, device=DEV)
    read = torch.zeros_like(last)
    torch.cuda.synchronize()
    keep = busy()
    read.copy_(last)
    del last
    got, _ = P.is_qk_norm_rope(q, k, pos, freq, 128, stream=side)
    torch.cuda.synchronize()
    assert (read == 3).all() and torch.equal(got, want)
    del keep


def test_no_rows_on_another_stream():
    side = torch.cuda.Stream()
    half = lambda *s: torch.zeros(s, dtype=torch.float16, device=DEV)  # noqa: E731
    whole = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
    assert P.is_lora_add(half(0, 64), half(2, 8, 64), half(2, 40, 8), whole(0), half(0, 40), stream=side).shape == (0, 40)
    assert P.is_attention(half(0, 128), half(0, 64), half(0, 64), whole(1), 64, 0, 0, stream=side).shape == (0, 128)
    assert P.is_qk_norm_rope(half(0, 128), half(0, 64), whole(0), torch.zeros(32, device=DEV), 64, stream=side)[0].shape == (0, 128)
    torch.cuda.synchronize()
