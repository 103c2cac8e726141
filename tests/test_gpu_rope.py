"""Rotary positions on the GPU against the oracle in 64 bits.

Tolerance: an angle reaches the sine as half turns in fp32 (off by pi 2^-25), the sine is good to 2 units of 2^-24, gain and
the two products round once each: under 4e-7 (|x_a| + |x_b|) |gain| in all; a bf16 result is off by half a step more."""
import numpy as np
import pytest
import torch

from oracle import razor_oracle as orc
from paper_2407_15891_b200 import binding as rz

from _harness import to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _check(x, got, positions, w, interleaved, inverse, gain):
    X = to_f64(x)
    pos = np.broadcast_to(np.asarray(positions)[:, :, None], X.shape[:3])
    want = orc.rope(X, pos, w, interleaved, inverse, gain)
    size = orc.rope(np.abs(X), np.zeros_like(pos), w, interleaved)
    R = 2 * w.size
    pair = np.zeros_like(size)
    if interleaved:
        pair[..., 0:R:2] = pair[..., 1:R:2] = size[..., 0:R:2] + size[..., 1:R:2]
    else:
        pair[..., :R // 2] = pair[..., R // 2:R] = size[..., :R // 2] + size[..., R // 2:R]
    tol = 4e-7 * pair * abs(gain)
    if x.dtype is torch.bfloat16:
        tol = tol + (np.abs(want) + tol) * 2.0 ** -8 * (np.arange(X.shape[-1]) < R)
    err = np.abs(to_f64(got) - want)
    assert (err <= tol).all(), (err - tol).max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,T,Hq,Hk,D,R", [(1, 1, 1, 0, 128, 128), (3, 1, 32, 8, 128, 128), (2, 37, 5, 1, 64, 64),
                                           (2, 3, 4, 4, 128, 32), (1, 5, 3, 2, 128, 38), (4, 2, 8, 2, 256, 240),
                                           (1, 129, 2, 2, 8, 2), (1, 700, 40, 40, 128, 96)])
def test_rope_matches_the_oracle(dtype, interleaved, B, T, Hq, Hk, D, R):
    g = torch.Generator().manual_seed(B * 1000 + T + R)
    x = torch.randn(B, T, Hq + 2 * Hk + 1, D, generator=g).to(dtype).to(DEV)     # a fused projection, a column range unused
    q, k = x[:, :, :Hq], x[:, :, Hq:Hq + Hk] if Hk else None
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (B, T), generator=g).to(torch.int32)
    w, gain = rz.razor_rope_frequencies(R, 10000.0, "yarn", 4.0, 8192)
    for inverse in (False, True):
        qo, ko = rz.razor_rope(q, k, w, pos.to(DEV), interleaved, inverse, gain)
        for a, b in ((q, qo), (k, ko)):
            if a is not None:
                _check(a, b, pos.numpy(), w, interleaved, inverse, gain)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R", [128, 64, 6])
def test_in_place_other_layouts_and_default_positions(dtype, R):
    B, T, H, D = 2, 9, 4, 128
    x = torch.randn(B, T, 3 * H, D, device=DEV).to(dtype)
    w, _ = rz.razor_rope_frequencies(R)
    before = x.clone()
    pos = np.tile(np.arange(T), (B, 1))
    dense = torch.full((B, H, T + 5, D), 7.0, device=DEV).to(dtype)              # keys as the prompt's dense buffer has them
    rz.razor_rope(x[:, :, :H], x[:, :, H:2 * H], w, q_out=x[:, :, :H], k_out=dense[:, :, 2:2 + T].transpose(1, 2))
    _check(before[:, :, :H], x[:, :, :H], pos, w, False, False, 1.0)
    _check(before[:, :, H:2 * H], dense[:, :, 2:2 + T].transpose(1, 2), pos, w, False, False, 1.0)
    assert torch.equal(x[:, :, H:], before[:, :, H:])                            # nothing else is touched
    assert (dense[:, :, :2] == 7).all() and (dense[:, :, 2 + T:] == 7).all()


def test_values_that_are_not_finite_stay_in_their_pair():
    x = torch.randn(1, 2, 3, 64, device=DEV)
    x[0, 0, 1, 5] = float("inf")
    x[0, 1, 2, 40] = float("nan")
    w, _ = rz.razor_rope_frequencies(64)
    y, _ = rz.razor_rope(x, None, w)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[0, 0, 1, [5, 37]] = True
    bad[0, 1, 2, [8, 40]] = True
    assert torch.equal(~torch.isfinite(y), bad)


def test_captured_on_another_stream_and_empty():
    x = torch.randn(2, 5, 4, 128, device=DEV).to(torch.bfloat16)
    pos = torch.arange(10, dtype=torch.int32, device=DEV).view(2, 5)
    w, _ = rz.razor_rope_frequencies(128)
    out = torch.zeros_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        rz.razor_rope(x, None, w, pos, q_out=out)
    x.copy_(torch.randn_like(x))
    pos += 1000                                                                 # a replay reads what is there then
    graph.replay()
    torch.cuda.synchronize()
    _check(x, out, pos.cpu().numpy(), w, False, False, 1.0)
    q, k = rz.razor_rope(x[:, :0], x[:, :0], w)
    assert q.shape == (2, 0, 4, 128) and k.shape == q.shape
