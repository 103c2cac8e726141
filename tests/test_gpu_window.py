"""Attention of prompt tokens with windows and sinks on the GPU against the oracle in 64 bits.

Tolerance: a weight is rounded to bf16 for the product with V (half a step, 2^-8 of it), the result to bf16 once more: 2^-8 of
sum p |v| / sum p and 2^-8 of |out|; scores, exponentials and sums in fp32 add a few 2^-20, taken as 1e-4 of the former."""
import math

import numpy as np
import pytest
import torch

from oracle import razor_oracle as orc
from paper_2407_15891_b200 import binding as rz

from _harness import to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _want(q, K, V, ctx, window, n_sink, scale):
    """[T, D], vectorised form of the oracle's window attention, and the same of |V|."""
    T, pos = q.shape[0], ctx - q.shape[0] + np.arange(q.shape[0])[:, None]
    n = np.arange(K.shape[0])[None]
    see = (n <= pos) & ((n < n_sink) | (window < 0) | (pos - n < window))
    s = np.where(see, q @ K.T * scale, -np.inf)
    top = s.max(1, keepdims=True, initial=-np.inf)
    w = np.where(see, np.exp(s - np.where(np.isfinite(top), top, 0)), 0)
    den = np.maximum(w.sum(1, keepdims=True), 1e-300)
    return (w @ V) / den, (w @ np.abs(V)) / den


def _check(q, K, V, out, n_sink, window=None, q_len=None, ctx_len=None, scale=0.0, rows=None):
    B, T, Hq, D = q.shape
    Hk, N = K.shape[1], K.shape[2]
    G = Hq // Hk
    scale = scale or 1 / math.sqrt(D)
    for b in range(B):
        t_n = T if q_len is None else min(max(q_len[b], 0), T)
        ctx = N if ctx_len is None else min(max(ctx_len[b], 0), N)
        for g in range(Hk):
            Kh, Vh = to_f64(K[b, g, :ctx]), to_f64(V[b, g, :ctx])
            w = -1 if window is None else window[b][g]
            for h in range(g * G, (g + 1) * G):
                qh, got = to_f64(q[b, :t_n, h]), to_f64(out[b, :t_n, h])
                if rows is not None:      # a few rows of a long prompt, each as the last query of what came before it
                    for t in [r for r in rows if r < t_n]:
                        want, size = _want(qh[t:t + 1], Kh, Vh, ctx - t_n + t + 1, w, n_sink, scale)
                        assert (np.abs(got[t] - want[0]) <= 2.0 ** -8 * (size[0] + np.abs(want[0])) + 1e-4 * size[0]).all(), (b, h, t)
                    continue
                want, size = _want(qh, Kh, Vh, ctx, w, n_sink, scale)
                err = np.abs(got - want) - (2.0 ** -8 * (size + np.abs(want)) + 1e-4 * size)
                assert (err <= 0).all(), (b, h, np.argwhere(err > 0)[:3], err.max())


def _inputs(B, T, N, Hq, Hk, D, seed=0):
    g = torch.Generator(DEV).manual_seed(seed)
    q, K, V = (torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16) for s in ((B, T, Hq, D), (B, Hk, N, D), (B, Hk, N, D)))
    K[:, :, :4] *= 4
    return q, K, V


def _dev(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (4, 4), (8, 2), (16, 2)])
@pytest.mark.parametrize("T,N", [(1, 1), (1, 700), (5, 5), (127, 127), (128, 128), (129, 129), (257, 300), (300, 1000)])
def test_everything_in_sight(D, Hq, Hk, T, N):
    q, K, V = _inputs(2, T, N, Hq, Hk, D)
    _check(q, K, V, rz.razor_window_attention(q, K, V, 4), 4)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_sink", [0, 1, 4, 130, 300])
@pytest.mark.parametrize("T,N,W", [(1, 900, 100), (300, 300, 1), (300, 300, 128), (400, 900, 129), (513, 513, 57), (200, 777, 5000),
                                   (260, 640, 0)])
def test_windows_and_sinks(D, n_sink, T, N, W):
    q, K, V = _inputs(1, T, N, 8, 4, D, seed=W)
    window = [[W, -1, max(0, W - 40), W + 1]]
    _check(q, K, V, rz.razor_window_attention(q, K, V, n_sink, _dev(window)), n_sink, window)


@pytest.mark.parametrize("G", [1, 2, 3, 5, 7, 8, 12, 71, 128])
def test_groups(G):
    q, K, V = _inputs(2, 150, 333, 2 * G, 2, 64, seed=G)
    window = [[100, -1], [-1, 31]]
    _check(q, K, V, rz.razor_window_attention(q, K, V, 3, _dev(window)), 3, window)


@pytest.mark.parametrize("seed", range(40))
def test_ragged_batches(seed):
    rng = np.random.default_rng(seed)
    B, Hk, G, D = int(rng.integers(1, 6)), int(rng.choice([1, 2, 3])), int(rng.choice([1, 2, 4, 8])), int(rng.choice([64, 128]))
    N = int(rng.integers(1, 1500))
    T = int(rng.choice([1, 3, 64, 200, 600]))
    ctx = rng.integers(-1, N + 3, B).tolist()
    new = rng.integers(-1, T + 3, B).tolist()
    window = rng.integers(-1, 700, (B, Hk)).tolist()
    n_sink = int(rng.choice([0, 2, 50, 200]))
    q, K, V = _inputs(B, T, N, Hk * G, Hk, D, seed)
    for b in range(B):                               # what no query sees may hold anything
        K[b, :, max(ctx[b], 0):] = float("nan")
        V[b, :, max(ctx[b], 0):] = float("inf")
        q[b, max(new[b], 0):] = float("nan")
    out = torch.full_like(q, 7.0)
    rz.razor_window_attention(q, K, V, n_sink, _dev(window), _dev(new), _dev(ctx), out=out)
    _check(q, K, V, out, n_sink, window, new, ctx)
    for b in range(B):
        assert (out[b, min(max(new[b], 0), T):] == 7.0).all()


def test_strides_scale_and_a_fused_projection():
    B, T, Hq, Hk, D, N = 2, 200, 4, 2, 128, 260
    fused = torch.randn(B, T, Hq + 2 * Hk, D, device=DEV).to(torch.bfloat16)
    big = torch.randn(B, N + 6, Hk, 2 * D, device=DEV).to(torch.bfloat16)         # K and V side by side, tokens outermost
    K, V = big[:, 3:3 + N, :, :D].transpose(1, 2), big[:, 3:3 + N, :, D:].transpose(1, 2)
    q = fused[:, :, :Hq]
    _check(q, K, V, rz.razor_window_attention(q, K, V, 4, sm_scale=0.31), 4, scale=0.31)
    # batch and heads of one: their strides do not matter
    one = rz.razor_window_attention(q[:1, :, :2], K[:1, :1], V[:1, :1], 4)
    _check(q[:1, :, :2], K[:1, :1], V[:1, :1], one, 4)


def test_a_large_batch_of_single_tokens_captured():
    """More units than the spans are made for, lengths that change between replays."""
    q, K, V = _inputs(65, 1, 300, 32, 16, 64, seed=3)
    rng = np.random.default_rng(1)
    window = rng.integers(-1, 200, (65, 16)).tolist()
    out, ctx = torch.zeros_like(q), _dev([300] * 65)
    w = _dev(window)
    ws = torch.empty(rz.razor_window_attention_workspace_bytes(65, 32, 16, 64, 1), dtype=torch.uint8, device=DEV)
    rz.razor_window_attention(q, K, V, 4, w, None, ctx, out=out, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        rz.razor_window_attention(q, K, V, 4, w, None, ctx, out=out, workspace=ws)
    for _ in range(2):
        lens = rng.integers(0, 301, 65).tolist()
        ctx.copy_(_dev(lens))
        graph.replay()
        torch.cuda.synchronize()
        _check(q, K, V, out, 4, window, None, lens)


@pytest.mark.parametrize("T,N", [(200, 260), (1, 9000)])
def test_out_at_a_16_byte_boundary(T, N):
    q, K, V = _inputs(1, T, N, 4, 2, 128, seed=9)
    buffer = torch.zeros(q.numel() + 16, dtype=torch.bfloat16, device=DEV)
    out = buffer[8:8 + q.numel()].view(q.shape)
    assert out.data_ptr() % 32 == 16
    rz.razor_window_attention(q, K, V, 4, out=out)
    assert torch.equal(out, rz.razor_window_attention(q, K, V, 4)) and not buffer[:8].any() and not buffer[-8:].any()


@pytest.mark.parametrize("T,N,Hq,Hk,D,ctx", [(1, 40000, 8, 2, 128, [40000, 33]), (2, 20011, 2, 2, 64, [20011, 20000]),
                                             (130, 9000, 4, 1, 128, [9000, 8000])])
def test_few_queries_over_a_long_context_are_cut_into_spans(T, N, Hq, Hk, D, ctx):
    q, K, V = _inputs(2, T, N, Hq, Hk, D)
    window = [[-1, 3000], [2000, -1]]
    window = [w[:Hk] for w in window]
    _check(q, K, V, rz.razor_window_attention(q, K, V, 4, _dev(window), None, _dev(ctx)), 4, window, None, ctx)


def test_many_units_come_from_the_queue():
    q, K, V = _inputs(9, 700, 700, 64, 64, 64)       # 3 pairs of tiles x 9 x 64 units
    window = np.random.default_rng(0).integers(-1, 400, (9, 64)).tolist()
    out = rz.razor_window_attention(q, K, V, 4, _dev(window))
    _check(q, K, V, out, 4, window, rows=[0, 1, 127, 128, 255, 256, 400, 699])
    assert torch.equal(out, rz.razor_window_attention(q, K, V, 4, _dev(window)))


@pytest.mark.parametrize("G", [1, 4])
def test_a_long_prompt_at_chosen_rows(G):
    q, K, V = _inputs(1, 8192, 8192, 2 * G, 2, 128)
    window = [[1000, -1]]
    out = rz.razor_window_attention(q, K, V, 4, _dev(window))
    _check(q, K, V, out, 4, window, rows=[0, 3, 4, 127, 128, 999, 1000, 1003, 1004, 5000, 8191])


def test_rows_with_far_apart_scores():
    """Maxima that grow along the context (the accumulator is rescaled again and again), and scores beyond e^80 of each other."""
    q, K, V = _inputs(1, 300, 1500, 2, 2, 128)
    K *= torch.linspace(0.1, 6, 1500, device=DEV)[None, None, :, None].to(torch.bfloat16)
    window = [[-1, 400]]
    _check(q, K, V, rz.razor_window_attention(q, K, V, 4, _dev(window)), 4, window)


@pytest.mark.parametrize("T,N", [(300, 300), (1, 9000), (64, 5000)])
@pytest.mark.parametrize("what", ["k_nan", "k_inf", "v_nan", "v_inf", "v_both", "q_nan"])
def test_what_is_not_finite_shows_where_it_is_seen(T, N, what):
    """Poison at tokens inside and outside of windows, in the future and behind the end: the rows that see it get it, the others
    are what they are without it."""
    q, K, V = _inputs(1, T, N, 4, 2, 128, seed=5)
    window, n_sink, ctx = [[90, -1]], 3, [N - 7 if N > 299 and T < N else N]
    clean = rz.razor_window_attention(q, K, V, n_sink, _dev(window), None, _dev(ctx))
    tokens = sorted({1, 40, N // 2, N - 60, N - 30, N - 9, N - 1})
    value = {"k_nan": float("nan"), "k_inf": float("inf"), "v_nan": float("nan"), "v_inf": float("-inf"), "v_both": float("inf"),
             "q_nan": float("nan")}[what]
    bad = torch.zeros(T, 4, 128, dtype=torch.bool, device=DEV)
    signs = torch.zeros(T, 4, 128, device=DEV)
    pos = ctx[0] - T + torch.arange(T, device=DEV)
    for i, n in enumerate(tokens):
        for g in range(2):
            w = window[0][g]
            see = (n <= pos) & ((n < n_sink) | (w < 0) | (pos - n < (w if w >= 0 else 0)))
            heads = slice(2 * g, 2 * g + 2)
            if what == "q_nan":
                t = (n * 7) % T
                q[0, t, 2 * g] = value
                bad[t, 2 * g] = True
            elif what[0] == "k":
                K[0, g, n, 17] = value
                bad[:, heads] |= see[:, None, None]
            else:
                d = (i * 3) % 128 if what != "v_both" else 5
                x = value if what != "v_both" or i % 2 else -value
                V[0, g, n, d] = x
                bad[:, heads, d] |= see[:, None]
                signs[:, heads, d] = torch.where(see[:, None], signs[:, heads, d] + x, signs[:, heads, d])
    out = rz.razor_window_attention(q, K, V, n_sink, _dev(window), None, _dev(ctx))
    got = out[0]
    if what == "k_inf":   # a score of -infinity hides the key, one of +infinity makes the row NaN: sign of q decides
        up = (q[0, :, :, 17].float() > 0)
        for t in range(T):
            for h in range(4):
                if bad[t, h].any() and up[t, h]:
                    assert got[t, h].isnan().all()
                elif not bad[t, h].any():
                    assert torch.equal(got[t, h], clean[0, t, h])
        return
    assert torch.equal(~torch.isfinite(got), bad)
    if what[0] == "v":
        assert torch.equal(got.float()[bad].nan_to_num(123.0, 9e9, -9e9), signs[bad].nan_to_num(123.0, 9e9, -9e9))
    # one rounding step of another sum's order at most: the paths differ only in what was taken out and put back
    assert torch.equal(got[~bad], clean[0][~bad])


def test_captured_lengths_are_read_at_replay_and_streams():
    q, K, V = _inputs(2, 64, 3000, 8, 2, 128)
    window, ctx, new = _dev([[500, -1], [-1, 100]]), _dev([2000, 3000]), _dev([64, 10])
    out = torch.zeros_like(q)
    ws = torch.empty(rz.razor_window_attention_workspace_bytes(2, 8, 2, 128, 64), dtype=torch.uint8, device=DEV)
    rz.razor_window_attention(q, K, V, 4, window, new, ctx, out=out, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        rz.razor_window_attention(q, K, V, 4, window, new, ctx, out=out, workspace=ws)
    for c, n, w in (([3000, 40], [1, 64], [[7, 7], [-1, 64]]), ([64, 1500], [64, 64], [[-1, -1], [1, 2000]])):
        ctx.copy_(_dev(c)); new.copy_(_dev(n)); window.copy_(_dev(w))
        out.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        _check(q, K, V, out, 4, w, n, c)
    # two calls at once, each with a workspace of its own
    other = torch.cuda.Stream()
    outs = [torch.zeros_like(q) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o in zip((side, other), outs):
            with torch.cuda.stream(s):
                rz.razor_window_attention(q, K, V, 4, window, new, ctx, out=o)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], out) and torch.equal(outs[1], out)


def test_refused_on_the_device_too():
    q, K, V = _inputs(1, 4, 16, 2, 2, 64)
    with pytest.raises(rz.RazorError) as e:
        rz.razor_window_attention(q, K, V, 4, workspace=torch.empty(0, dtype=torch.uint8, device=DEV))
    assert e.value.status in (-2, -4)
    with pytest.raises(rz.RazorError) as e:
        rz.razor_window_attention(q, K, V, -1)
    assert e.value.status == -1
    assert rz.razor_window_attention(q[:, :0], K, V, 4).shape == (1, 0, 2, 64)
