"""The cache of 8-bit rows on the GPU: codes and scales exactly the definition's, attention against the oracle in 64 bits over
the values held.

Tolerance of attention: products are exact, sums of them are fp32 (tensor cores: eight additions that may drop a 2^-23 each,
2^-20 of sum |q k|), exponentials good to 2^-21, weights to 2^-22 (an fp16 head and remainder), sums over tokens fp32: taken as
2^-19 (1 + the largest scale * sum |q_d k_d| of the row) of sum p |v| / sum p.  A weight p v_scale is given to fp16 as a
share of 2^14 / R, R < 2 max v_scale; below fp16's smallest step, 2^-24, nothing is left of it: at most half of that, with codes
up to 127 an error of 2^-25 2^-14 127 R < 2^-38 max |v| a token, against the largest weight.  The compensation token is a mean of n rows that
were added up in fp32, one by one: off by at most n 2^-24 of the mean of |rows| in every dimension, whatever cancels in the
mean itself.  In V that reaches the result with the token's share p_c / sum p; in K it moves the token's score by
n 2^-24 scale sum |q_d| mean |k_d|, and a result by at most twice that of sum p |v| / sum p."""
import math

import numpy as np
import pytest
import torch

from oracle import razor_oracle as orc
from paper_2407_15891_b200 import binding as rz

from _harness import to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Head:
    """One KV head: its rows as held, the sums of what it dropped (64 bits)."""

    def __init__(self, D, n_sink, window):
        self.n_sink, self.window, self.pos, self.K, self.V = n_sink, window, [], [], []
        self.n, self.n_drop, self.sums, self.size = 0, 0, np.zeros((2, D)), np.zeros((2, D))   # (size: sums of |rows|)

    def compress(self, K, V):
        n, W = len(K), self.window
        keep = list(range(n)) if W < 0 or n <= self.n_sink + W else [*range(self.n_sink), *range(n - W, n)]
        self.pos, self.n, self.n_drop = keep, n, n - len(keep)
        gone = sorted(set(range(n)) - set(keep))
        if gone:
            self.sums = np.stack([K[gone].sum(0), V[gone].sum(0)])
            self.size = np.stack([np.abs(K[gone]).sum(0), np.abs(V[gone]).sum(0)])
        self.K, self.V = (list(orc.quantise_rows(x[keep])[2]) for x in (K, V))

    def append(self, k, v):
        held = [orc.quantise_rows(x[None])[2][0] for x in (k, v)]
        if self.window >= 0 and len(self.pos) >= self.n_sink + self.window:
            self.n_drop += 1
            if self.window == 0:                             # dropped without having been held
                self.sums += np.stack([k, v])
                self.size += np.abs(np.stack([k, v]))
                self.n += 1
                return
            i = self.n_sink
            old = np.stack([self.K.pop(i), self.V.pop(i)]).astype(np.float64)
            self.sums += old
            self.size += np.abs(old)
            self.pos.pop(i)
        self.pos.append(self.n)
        self.K.append(held[0])
        self.V.append(held[1])
        self.n += 1

    def attend(self, q, scale, q_pos=None, slope=0.0, more=0.0):
        """q [D] -> (out, tolerance).  more: size of further terms of the scores."""
        D = len(q)
        K, V = (np.array(x, dtype=np.float64).reshape(-1, D) for x in (self.K, self.V))
        bias = np.zeros(len(K))
        if q_pos is not None:
            pos = np.array(self.pos)
            bias = np.where(pos <= q_pos, slope * (pos - q_pos) * 1.0, -np.inf)
        mean = bool(self.n_drop and self.window >= 0 and self.comp)
        if mean:
            m = self.sums / self.n_drop
            K, V, bias = np.vstack([K, m[:1]]), np.vstack([V, m[1:]]), np.append(bias, math.log(self.n_drop))
        if not len(K):
            return np.zeros(D), np.zeros(D)
        s = K @ q * scale + bias
        p = np.exp(s - s.max())
        p /= p.sum()
        size, smax = p @ np.abs(V), (np.abs(K) @ np.abs(q)).max() * scale
        tol = 2.0 ** -19 * (1 + smax + more) * size + len(V) * 2.0 ** -38 * np.abs(V).max() * p.max() + 1e-30
        if mean:
            off = self.size * 2.0 ** -24                     # n 2^-24 of the mean of |rows|
            tol = tol + p[-1] * off[1] + 2 * scale * (np.abs(q) @ off[0]) * size
        return p @ V, tol

    comp = True


class Case:
    def __init__(self, B=2, Hk=2, G=2, D=128, lens=(300, 77), window=40, n_sink=4, retr=(1, 0), max_new=64, shuffle=0, comp=1, seed=0,
                 scale=0.0, options=None):
        self.B, self.Hk, self.G, self.D, self.n_sink = B, Hk, G, D, n_sink
        self.gen = torch.Generator(DEV).manual_seed(seed)
        self.lens, self.retr, self.win = list(lens), np.array(retr, dtype=np.uint8), [window] * B
        N = max(max(lens), 1)
        self.K, self.V = self.randn(B, Hk, N, D), self.randn(B, Hk, N, D)
        self.K[..., 3] *= 8
        self.K[:, :, :4] *= 4
        self.scale = scale or 1 / math.sqrt(D)
        cfg = rz.make_config(B, 1, Hk * G, Hk, D, "i8", n_sink, N, max_new, comp, shuffle, scale)
        self.cache = rz.RazorCache(cfg, self.lens, self.win, self.retr, device=DEV)
        for o, v in (options or {}).items():
            self.cache.set_option(o, v)
        self.heads = [[Head(D, n_sink, -1 if retr[g] else window) for g in range(Hk)] for _ in range(B)]
        for row in self.heads:
            for h in row:
                h.comp = bool(comp)

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.gen, device=DEV).to(torch.bfloat16)

    def compress(self):
        self.cache.compress(0, self.K, self.V, self.lens, self.retr, self.win)
        for b in range(self.B):
            for g in range(self.Hk):
                n = self.lens[b]
                self.heads[b][g].compress(to_f64(self.K[b, g, :n]), to_f64(self.V[b, g, :n]))
        return self

    def append(self, T=None, how="append"):
        k, v = self.randn(self.B, T or 1, self.Hk, self.D), self.randn(self.B, T or 1, self.Hk, self.D)
        if T is None:
            self.cache.append(0, k[:, 0].contiguous(), v[:, 0].contiguous()) if how == "append" else None
        else:
            self.cache.append_many(0, k, v)
        for t in range(T or 1):
            for b in range(self.B):
                for g in range(self.Hk):
                    self.heads[b][g].append(to_f64(k[b, t, g]), to_f64(v[b, t, g]))
        return k[:, 0].contiguous(), v[:, 0].contiguous()

    def check_state(self):
        kept = 0
        for b in range(self.B):
            for g in range(self.Hk):
                h, ex = self.heads[b][g], self.cache.export(0, b, g)
                assert ex["kept_pos"].tolist() == h.pos and ex["n_drop"] == h.n_drop
                kept += len(h.pos)
                for x, y in ((ex["K"], h.K), (ex["V"], h.V)):
                    assert x.dtype is torch.float32
                    want = np.array(y, dtype=np.float32).reshape(-1, self.D)
                    assert np.array_equal(x.cpu().numpy(), want, equal_nan=True)
                for x, y, size in ((ex["sum_k"], h.sums[0], h.size[0]), (ex["sum_v"], h.sums[1], h.size[1])):
                    assert (np.abs(to_f64(x) - y) <= h.n_drop * 2.0 ** -24 * size).all()
        assert self.cache.stats(0)[0] == kept * 2 * (self.D + 4)

    def check_out(self, q, out, heads=None):
        q, out = to_f64(q), to_f64(out)
        for b in range(self.B):
            for h in range(self.Hk * self.G):
                want, tol = self.heads[b][h // self.G].attend(q[b, h], self.scale)
                assert (np.abs(out[b, h] - want) <= tol).all(), (b, h, (np.abs(out[b, h] - want) / tol).max())

    def check_decode(self):
        q = self.randn(self.B, self.Hk * self.G, self.D)
        self.check_out(q, self.cache.decode(0, q))
        assert self.cache.device_status() == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,window,n_sink", [((0, 1), 5, 2), ((16, 17), 8, 0), ((300, 77), 40, 4), ((1000, 5), 0, 3), ((999, 250), 100, 0),
                                                ((64, 31), 500, 4)])
def test_compressed_rows_are_the_definitions(D, lens, window, n_sink):
    c = Case(D=D, lens=lens, window=window, n_sink=n_sink, shuffle=lens[0] % 2).compress()
    c.check_state()
    c.check_decode()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_groups(D, G):
    c = Case(B=3, Hk=2, G=G, D=D, lens=(2000, 3, 513), window=300, seed=G).compress()
    c.check_decode()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [0, 1, 5, 40])
def test_appends_one_by_one_in_short_and_in_long_runs(D, window):
    c = Case(D=D, lens=(60, 3), window=window, max_new=300, seed=window).compress()
    for T in (None, None, 3, 7, None, 8, 45, None, 130, 2):
        c.append(T)
        c.check_decode()
    c.check_state()


def test_chunked_prefill_from_an_empty_layer():
    c = Case(lens=(0, 0), window=50, max_new=700)
    c.cache.start_empty(0, c.retr, c.win)
    for T in (100, 64, 200, 3, 300):
        c.append(T)
        c.check_state()
    c.check_decode()


@pytest.mark.parametrize("window", [0, 9, 64])
def test_decode_steps(window):
    c = Case(lens=(70, 20), window=window, max_new=40, seed=3).compress()
    for _ in range(30):
        k, v = c.append(how="mirror only")
        q = c.randn(c.B, c.Hk * c.G, c.D)
        c.check_out(q, c.cache.decode_step(0, k, v, q))
    c.check_state()


@pytest.mark.parametrize("G,T", [(1, 1), (1, 2), (1, 7), (2, 3), (2, 9), (4, 2), (4, 5), (8, 1), (8, 3)])
def test_rounds(G, T):
    c = Case(G=G, lens=(400, 90), window=60, max_new=40, seed=G + T).compress()
    c.append(T)
    q = c.randn(c.B, T, c.Hk * G, c.D)
    out = to_f64(c.cache.decode_multi(0, q))
    for b in range(c.B):
        for t in range(T):
            for h in range(c.Hk * G):
                head = c.heads[b][h // G]
                want, tol = head.attend(to_f64(q[b, t, h]), c.scale, head.n - T + t)
                assert (np.abs(out[b, t, h] - want) <= tol).all(), (b, t, h)


@pytest.mark.parametrize("n_sink", [0, 3])
def test_alibi(n_sink):
    c = Case(G=2, lens=(300, 40), window=50, n_sink=n_sink, comp=0, max_new=8).compress()
    slopes = np.array([0.5, 0.25, 0.03, 0.001], dtype=np.float32)
    rz.razor_cache_set_alibi(c.cache.handle, slopes)
    c.append()
    q = c.randn(c.B, 4, c.D)
    out = to_f64(c.cache.decode(0, q))
    for b in range(c.B):
        for h in range(4):
            head = c.heads[b][h // 2]
            # (the penalty, up to 0.5 * 300, is a term of the score as well)
            want, tol = head.attend(to_f64(q[b, h]), c.scale, head.n - 1, float(slopes[h]), more=150.0)
            assert (np.abs(out[b, h] - want) <= tol).all(), (b, h)


@pytest.mark.parametrize("options", [{}, {rz.OPT_DECODE_STATIC_PERCENT: 0, rz.OPT_DECODE_MIN_CHUNK_PAGES: 1}, {rz.OPT_DECODE_RING_KB: 40},
                                     {rz.OPT_DECODE_CONSUMER_WARPS: 12}])
def test_long_heads_in_many_parts(options):
    c = Case(B=1, Hk=2, G=4, lens=(30000,), window=4000, options=options).compress()
    c.check_decode()
    c.append(5)
    c.check_decode()


def test_rows_of_very_different_sizes():
    """Scales that span the range of bf16, tiny rows first and last, and zero rows."""
    c = Case(B=1, Hk=2, G=2, lens=(800,), window=300, seed=11)
    size = 10.0 ** torch.linspace(-12, 6, 800, device=DEV)
    c.V *= size[None, None, torch.randperm(800, generator=c.gen, device=DEV), None].to(torch.bfloat16)
    c.V[0, 0, 5] = 0
    c.K[0, 0, 700] = 0
    c.V[0, 1, 790:] *= 1e-25
    c.K[0, 1, 100] = 1e-33
    c.compress()
    c.check_state()
    c.check_decode()
    big = Case(B=1, Hk=1, G=4, lens=(50,), window=20, retr=(0,), seed=4)
    big.K *= 1e18
    big.compress()
    q = (big.randn(1, 4, 128).float() * 1e-18).to(torch.bfloat16)
    big.check_out(q, big.cache.decode(0, q))
    q0 = torch.zeros_like(q)
    big.check_out(q0, big.cache.decode(0, q0))


def test_what_is_not_finite():
    c = Case(B=1, Hk=2, G=2, lens=(200,), window=50, n_sink=0, comp=0, seed=2)
    c.V[0, 0, 120, 7] = float("inf")                 # in the retrieval head
    c.V[0, 1, 10, 7] = float("nan")                  # dropped by the other head (no compensation token)
    c.K[0, 1, 180, 1] = float("nan")                 # in its window
    c.compress()
    ex = c.cache.export(0, 0, 0)
    assert ex["V"][120].isnan().all() and torch.isfinite(ex["V"][119]).all() and torch.isfinite(ex["K"]).all()
    q = c.randn(1, 4, 128)
    out = c.cache.decode(0, q)
    assert out.isnan().all()                         # each head sees one
    clean = Case(B=1, Hk=2, G=2, lens=(200,), window=50, n_sink=0, comp=0, seed=2).compress()
    clean.cache.compress(0, torch.where(torch.isfinite(c.K), c.K, torch.zeros_like(c.K)),
                         torch.where(torch.isfinite(c.V), c.V, torch.zeros_like(c.V)), clean.lens, clean.retr, clean.win)
    assert torch.isfinite(clean.cache.decode(0, q)).all()
    # a later token of a round, unseen by the earlier ones
    r = Case(B=1, Hk=1, G=1, lens=(100,), window=50, retr=(1,), max_new=8, seed=6).compress()
    k, v = r.randn(1, 3, 1, 128), r.randn(1, 3, 1, 128)
    v[0, 2] = float("nan")
    k[0, 1] = float("inf")
    r.cache.append_many(0, k, v)
    out = r.cache.decode_multi(0, r.randn(1, 3, 1, 128))
    assert torch.isfinite(out[0, 0]).all() and out[0, 1].isnan().all() and out[0, 2].isnan().all()


def test_many_sequences_one_at_a_time_and_again():
    c = Case(B=5, Hk=3, G=1, D=64, lens=(10, 400, 33, 129, 0), window=30, retr=(0, 1, 0), shuffle=7)
    for b in (3, 0, 4, 2, 1):
        c.cache.compress_seq(0, b, c.K[b], c.V[b], c.lens[b], c.retr, c.win[b])
    c.compress()                                      # over it, in place
    c.check_state()
    c.check_decode()
    c.cache.close()


def test_the_whole_path_of_a_layer():
    """Projection -> rotary positions -> prompt attention with windows -> 8-bit cache -> decode steps, against the oracle."""
    B, T, Hk, G, D, W, n_sink = 2, 150, 2, 2, 128, 40, 4
    gen = torch.Generator(DEV).manual_seed(0)
    fused = torch.randn(B, T + 6, Hk * (G + 2), D, generator=gen, device=DEV).to(torch.bfloat16)
    w, gain = rz.razor_rope_frequencies(D, 10000.0, "yarn", 4.0, 100)
    q, k, v = fused[:, :, :Hk * G], fused[:, :, Hk * G:Hk * (G + 1)], fused[:, :, Hk * (G + 1):]
    kd = torch.zeros(B, Hk, T, D, dtype=torch.bfloat16, device=DEV)
    qr, _ = rz.razor_rope(q[:, :T], k[:, :T], w, gain=gain, k_out=kd.transpose(1, 2))
    vd = v[:, :T].transpose(1, 2).contiguous()
    lens = torch.tensor([T, 101], dtype=torch.int32, device=DEV)
    window = torch.tensor([[-1, W]] * B, dtype=torch.int32, device=DEV)
    out = rz.razor_window_attention(qr, kd, vd, n_sink, window, lens, lens)
    retr = np.array([1, 0], dtype=np.uint8)
    cfg = rz.make_config(B, 1, Hk * G, Hk, D, "i8", n_sink, T, 8)
    cache = rz.RazorCache(cfg, lens.tolist(), [W] * B, retr, device=DEV)
    cache.compress(0, kd, vd, lens.tolist(), retr, [W] * B)
    heads = [[Head(D, n_sink, -1 if retr[g] else W) for g in range(Hk)] for _ in range(B)]
    for b, n in enumerate(lens.tolist()):
        for g in range(Hk):
            K, V = to_f64(kd[b, g, :n]), to_f64(vd[b, g, :n])
            heads[b][g].compress(K, V)
            for h in range(g * G, (g + 1) * G):
                Q = to_f64(qr[b, :n, h])
                want = orc.window_attention(Q, K, V, n, -1 if retr[g] else W, n_sink, 1 / math.sqrt(D))
                size = orc.window_attention(Q, K, np.abs(V), n, -1 if retr[g] else W, n_sink, 1 / math.sqrt(D))
                assert (np.abs(to_f64(out[b, :n, h]) - want) <= 2.0 ** -8 * (size + np.abs(want)) + 1e-4 * size).all()
    for t in range(6):
        pos = (lens + t)[:, None].contiguous()
        q1, k1 = rz.razor_rope(q[:, T + t:T + t + 1], k[:, T + t:T + t + 1], w, pos, gain=gain)
        v1 = v[:, T + t].contiguous()
        got = to_f64(cache.decode_step(0, k1[:, 0].contiguous(), v1, q1[:, 0].contiguous()))
        for b in range(B):
            for g in range(Hk):
                heads[b][g].append(to_f64(k1[b, 0, g]), to_f64(v1[b, g]))
                for h in range(g * G, (g + 1) * G):
                    want, tol = heads[b][g].attend(to_f64(q1[b, 0, h]), 1 / math.sqrt(D))
                    assert (np.abs(got[b, h] - want) <= tol).all()


def test_tree_calls_are_refused():
    c = Case(max_new=8).compress()
    q, k = c.randn(2, 3, 4, 128), c.randn(2, 3, 2, 128)
    parent = torch.full((2, 3), -1, dtype=torch.int32, device=DEV)
    with pytest.raises(rz.RazorError) as e:
        c.cache.decode_tree(0, q, k, k, parent)
    assert e.value.status == -3
    with pytest.raises(rz.RazorError) as e:
        c.cache.append_tree(0, k, k, None, [1, 2])
    assert e.value.status == -3
