"""What the prompt attention leaves when a wait runs out: rows that are NaN, rows as they were, and right ones, never rows folded
from records that nobody wrote.  One thread block gives up its waits at once; the launch itself runs to its end."""
import pytest
import torch

from paper_2407_15891_b200 import binding as rz

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _inputs(B, T, N, Hq, Hk, D, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    return [torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16) for s in ((B, T, Hq, D), (B, Hk, N, D), (B, Hk, N, D))]


# (cut: every unit is cut up, so that no row of it can have been left as it was)
@pytest.mark.parametrize("B,T,N,Hq,Hk,D,cut", [(1, 1, 40000, 8, 2, 128, True), (2, 130, 20000, 2, 1, 64, True), (2, 64, 3000, 8, 2, 128, False),
                                               (1, 2000, 2000, 4, 4, 64, False), (65, 1, 300, 16, 16, 64, False)])
def test_a_block_that_gives_up_leaves_no_made_up_rows(B, T, N, Hq, Hk, D, cut):
    q, K, V = _inputs(B, T, N, Hq, Hk, D, T)
    ws = torch.zeros(rz.razor_window_attention_workspace_bytes(B, Hq, Hk, D, T), dtype=torch.uint8, device=DEV)
    good = rz.razor_window_attention(q, K, V, 4, workspace=ws)
    other = _inputs(B, T, N, Hq, Hk, D, 1000)
    for cta in (0, 1, 17, 100, 147):
        rz.razor_window_attention(*other, 4, workspace=ws)             # records of another call lie there
        out = torch.full_like(good, 7.0)
        rz.razor_window_attention_wait_selftest(q, K, V, 4, cta, out=out, workspace=ws)
        nan, kept = out.isnan().all(-1), (out == 7.0).all(-1)
        right = (out == good).all(-1)
        assert (nan | kept | right).all(), cta
        if cut:
            assert nan.any() and not (kept & ~right).any(), cta
        # nothing of it stays behind
        assert torch.equal(rz.razor_window_attention(q, K, V, 4, workspace=ws), good)
    beyond = rz.razor_window_attention_wait_selftest(q, K, V, 4, 100000, workspace=ws)
    assert torch.equal(beyond, good)


def test_refused():
    q, K, V = _inputs(1, 4, 16, 2, 2, 64, 0)
    with pytest.raises(rz.RazorError) as e:
        rz.razor_window_attention_wait_selftest(q, K, V, 4, -1)
    assert e.value.status == -1
