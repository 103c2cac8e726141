"""Calls on a stream that is not torch's current one: tensors that a call makes itself belong to the stream that it works on.

The current stream is kept busy for some 100 ms, so that whatever a call put there by mistake comes after its kernels."""
import numpy as np
import pytest
import torch

from paper_2407_15891_b200 import binding as rz

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _randn(*shape, dtype=torch.bfloat16):
    return torch.randn(*shape, device=DEV).to(dtype)


def _beside_a_busy_stream(call, sizes):
    """call(stream) on a stream of its own, while the current one has a wait, then fills of freed blocks of these sizes, to do."""
    side = torch.cuda.Stream()
    call(None)                                             # (memory that torch has to ask the device for, and kernels that are
    call(side.cuda_stream)                                 # loaded, make both streams wait: all there from here on)
    blocks = [torch.zeros(n, dtype=torch.uint8, device=DEV) for n in sizes]
    torch.cuda._sleep(1000)
    for x in blocks:
        x.fill_(1)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    for x in blocks:
        x.fill_(0xff)
    del blocks, x                                          # freed, with the fill still to come
    done = torch.cuda.Event()
    done.record()
    got = call(side.cuda_stream)
    side.synchronize()
    assert not done.query()                                # the current stream has been busy all the while
    torch.cuda.synchronize()
    return got


@pytest.mark.parametrize("T,N", [(1, 5000), (40, 40), (700, 900)])
def test_window_attention(T, N):
    q, K, V = _randn(2, T, 8, 128), _randn(2, 2, N, 128), _randn(2, 2, N, 128)
    want = rz.razor_window_attention(q, K, V, 4)
    need = rz.razor_window_attention_workspace_bytes(2, 8, 2, 128, T)
    got = _beside_a_busy_stream(lambda s: rz.razor_window_attention(q, K, V, 4, stream=s), [q.numel() * 2, need])
    assert torch.equal(got, want)
    # rows that the call does not write are zeros
    new = torch.tensor([0, T // 2], dtype=torch.int32, device=DEV)
    got = _beside_a_busy_stream(lambda s: rz.razor_window_attention(q, K, V, 4, q_len=new, stream=s), [q.numel() * 2, need])
    assert not got[0].any() and not got[1, T // 2:].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rope(dtype):
    q, k = _randn(2, 300, 8, 128, dtype=dtype), _randn(2, 300, 2, 128, dtype=dtype)
    w, _ = rz.razor_rope_frequencies(128)
    want = rz.razor_rope(q, k, w)
    got = _beside_a_busy_stream(lambda s: rz.razor_rope(q, k, w, stream=s), [x.numel() * x.element_size() for x in (q, k)])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_verify_tree_and_head_scores():
    B, T, V = 4, 7, 1000
    target = torch.softmax(_randn(B, T + 1, V, dtype=torch.float32), -1)
    draft = torch.softmax(_randn(B, T + 1, V, dtype=torch.float32), -1)
    tokens = torch.randint(V, (B, T), dtype=torch.int32, device=DEV)
    parent = torch.arange(-1, T - 1, dtype=torch.int32, device=DEV).repeat(B, 1)
    ua, us = torch.rand(B, T, device=DEV), torch.rand(B, device=DEV)
    call = lambda s: rz.razor_verify_tree(target, draft, tokens, parent, ua, us, stream=s)  # noqa: E731
    want, got = call(None), _beside_a_busy_stream(call, [B * (T + 2) * 4])
    for x in want:
        assert torch.equal(got[x], want[x])
    Q, K = _randn(4, 512, 128), _randn(4, 512, 128)
    want = rz.razor_head_scores(Q, K, 128)
    got = _beside_a_busy_stream(lambda s: rz.razor_head_scores(Q, K, 128, stream=s), [1 << 12, 1 << 16, 1 << 20, 1 << 22])
    assert np.array_equal(got[0].cpu(), want[0].cpu()) and np.array_equal(got[1].cpu(), want[1].cpu())
