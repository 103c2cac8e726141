"""Calls of the prompt attention that its documentation allows: strides of dimensions of one, a buffer for every call, scores of
-infinity."""
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


@pytest.mark.parametrize("T,N", [(300, 300), (1, 9000), (64, 5000)])
def test_a_score_of_minus_infinity_hides_its_key(T, N):
    """Keys with an infinity against queries that are negative there: the oracle's weights of such keys are zero as well."""
    q, K, V = _inputs(1, T, N, 4, 2, 128, seed=8)
    q[..., 17] = -q[..., 17].abs() - 0.25
    for n in sorted({0, 3, 40, N // 2, N - 60, N - 1}):
        K[:, :, n, 17] = float("inf")
    window = [[90, -1]]
    out = rz.razor_window_attention(q, K, V, 3, _dev(window))
    assert torch.isfinite(out).all()
    _check(q, K, V, out, 3, window)


def test_a_row_whose_keys_are_all_hidden_is_zeros():
    q, K, V = _inputs(2, 4, 4, 2, 1, 64, seed=2)
    q[..., 5], K[..., 5] = -1, float("inf")
    assert not rz.razor_window_attention(q, K, V, 4).any()
    q[..., 5] = 1
    assert rz.razor_window_attention(q, K, V, 4).isnan().all()


@pytest.mark.parametrize("D,size", [(64, 21635328), (128, 42607872)])
def test_one_buffer_serves_calls_of_all_sizes(D, size):
    ws = torch.full((size,), 0x7f, dtype=torch.uint8, device=DEV)
    calls = []
    for B, T, N, Hq, Hk in ((1, 600, 600, 32, 8), (1, 1, 5000, 8, 2), (70, 1, 100, 16, 16), (4, 1, 3000, 32, 8), (1, 257, 900, 2, 1)):
        q, K, V = _inputs(B, T, N, Hq, Hk, D, seed=T)
        calls.append((q, K, V, rz.razor_window_attention(q, K, V, 4)))
    for _ in range(2):
        for q, K, V, want in calls:
            assert torch.equal(rz.razor_window_attention(q, K, V, 4, workspace=ws), want)
