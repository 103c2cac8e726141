"""Small rotary angles keep their relative precision: slow pairs at near positions.

Off by: the frequency as a 64-bit fraction of a turn 2^-65 turns a position (under 1e-9 of the angle at 1e-9 radians a
position), the angle's rounding to fp32 2^-24, the sine 2^-23, gain and product 2^-24 each: under 6 2^-24 of sin(p w), which
changes by no larger a share than the angle does.  (Angles below 0.1, x_a = 0 and x_b = 1: y_a is -sin alone.)"""
import numpy as np
import pytest
import torch

from paper_2407_15891_b200 import binding as rz

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("R,interleaved", [(128, False), (128, True), (6, False), (6, True)])
@pytest.mark.parametrize("inverse", [False, True])
def test_sines_of_small_angles(R, interleaved, inverse):
    T, D = 1000, 128
    w = np.geomspace(1e-9, 1e-4, R // 2)
    a, b = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    x = torch.zeros(1, T, 1, D, device=DEV)
    x[..., b] = 1
    for sign in (1, -1):
        pos = sign * torch.arange(T, dtype=torch.int32, device=DEV)[None]
        y, _ = rz.razor_rope(x, None, w, pos, interleaved, inverse)
        angle = pos.cpu().numpy()[0][:, None].astype(np.float64) * w
        want = np.sin(angle) * (1 if inverse else -1)
        got = y[0, :, 0, a].double().cpu().numpy()
        assert (np.abs(got - want) <= 6 * 2.0 ** -24 * np.abs(want)).all()
        assert (np.abs(y[0, :, 0, b].double().cpu().numpy() - np.cos(angle)) <= 6 * 2.0 ** -24).all()
