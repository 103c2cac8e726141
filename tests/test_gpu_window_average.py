"""A row of the prompt attention is an average of the values it sees: its weights, in whatever bits, add up to one.

Where every value of a dimension is the same bf16 number c, numerator and denominator hold the same rounded weights: c times a
sum over up to 2000 of them in fp32, off by less than 2000 2^-23 of it however the additions round or cut off, and the quotient
is nearer to c than half the smallest step of bf16 below it (2^-10 c): the result is c itself."""
import pytest
import torch

from paper_2407_15891_b200 import binding as rz

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,N,Hk,G,window", [(300, 2000, 2, 1, None), (1, 1999, 2, 4, None), (256, 256, 2, 2, [[-1, 60]]),
                                             (40, 1500, 1, 8, [[700]])])
def test_equal_values_come_out_as_they_are(D, T, N, Hk, G, window):
    g = torch.Generator(DEV).manual_seed(T + N + D)
    q, K = (torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16) for s in ((1, T, Hk * G, D), (1, Hk, N, D)))
    K *= torch.linspace(0.1, 3, N, device=DEV)[None, None, :, None].to(torch.bfloat16)   # late keys weigh most: the reference lags
    c = (torch.randn(D, generator=g, device=DEV) * 10).to(torch.bfloat16)
    V = c.expand(1, Hk, N, D).contiguous()
    w = None if window is None else torch.tensor(window, dtype=torch.int32, device=DEV)
    out = rz.razor_window_attention(q, K, V, 4, w)
    assert torch.equal(out, c.expand_as(out))
