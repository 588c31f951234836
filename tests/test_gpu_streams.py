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
