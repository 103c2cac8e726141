"""Calls of the prompt attention that its documentation allows: strides of dimensions of one, a buffer for every call, scores of
-infinity."""
import numpy as np
import pytest
import torch

from paper_2407_15891_b200 import binding as rz

from test_gpu_window import _check, _dev, _inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("B,Hk,N", [(1, 1, 200), (1, 2, 200), (2, 1, 200), (2, 2, 1)])
def test_strides_of_dimensions_of_one_do_not_matter(B, Hk, N):
    q, K, V = _inputs(B, min(N, 5), N, 2 * Hk, Hk, 64, seed=B)
    want = rz.razor_window_attention(q, K, V, 4)
    K2, V2 = (x.as_strided(x.shape, [odd if n == 1 else s for n, s in zip(x.shape, x.stride())]) for x, odd in ((K, 24), (V, 7)))
    assert K2.stride() != V2.stride()
    assert torch.equal(rz.razor_window_attention(q, K2, V2, 4), want)
