"""Tree attention where the other tests' bars would not notice a loss: spans of 150 steps, in which the matrix unit's additions
pile up, and ALiBi over fp32 caches."""
import math

import numpy as np
import pytest
import torch

from oracle import razor_oracle as orc
from paper_2407_15891_b200 import binding as rz
from paper_2407_15891_b200 import synth

from _harness import TOL_OUT, HeadRef, make_cache, to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("group,T,D,alibi", [(1, 4, 64, False), (1, 50, 64, False), (8, 128, 128, False), (8, 100, 64, True)])
def test_long_spans_keep_their_precision(group, T, D, alibi):
    """One head so long that every CTA has about 150 steps of 128 tokens (148 spans, or 148 / 8 under eight tiles of rows; seven
    of them here with 100 nodes).  Bar: 1e-5 of the result's norm, from the arithmetic.  A weight, a bf16 head plus a bf16
    remainder, is within 2^-18 = 3.8e-6; its logit adds 16 products at a time, eight truncated additions of 2^-23 on sums of about
    11 = sqrt(128), 1e-5 / sqrt(128) = 0.9e-6; the exponential 2^-22 = 0.2e-6; an output accumulator loses half a place of 2^-23
    in each of the 64 additions before it is taken out, on sums that grow like a root, 64 * 2^-24 * 2/3 = 2.5e-6; the sum of
    weights rounds 150 times to nearest, sqrt(150) * 2^-24 = 0.7e-6.  Together 8.1e-6.  (Errors of single weights, of either
    sign, weigh on the norm as the weights themselves do.)  1200 additions without taking out would lose 4.7e-5."""
    tiles = -(-group * T // 128) if group * T > 64 else 1
    n = (148 // tiles) * 150 * 128 + 77
    cfg = rz.make_config(1, 1, group, 1, D, "bf16", 4, n, 1, 0 if alibi else 1)
    cache = rz.RazorCache(cfg, [n], [64], [1])
    if alibi:
        slopes = (2.0 ** -(18.0 + np.arange(group))).astype(np.float32)      # a penalty of up to two over the whole context
        rz.razor_cache_set_alibi(cache.handle, slopes)
    gen = torch.Generator(DEV)
    gen.manual_seed(T)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=DEV, dtype=torch.bfloat16)  # noqa: E731
    K, V = normal(1, 1, n, D), normal(1, 1, n, D)
    q, k, v = normal(1, T, group, D), normal(1, T, 1, D), normal(1, T, 1, D)
    cache.compress(0, K, V, [n], [1], [64])
    got = cache.decode_tree(0, q, k, v, torch.full((1, T), -1, dtype=torch.int32, device=DEV))
    assert cache.device_status() == 0
    cache.close()
    want = torch.empty(T, group, D, dtype=torch.float64, device=DEV)
    Kd, Vd = K[0, 0].double(), V[0, 0].double()
    dist = torch.arange(n, 0, -1, device=DEV, dtype=torch.float64)
    for t in range(T):
        for j in range(group):
            x = q[0, t, j].double() / math.sqrt(D)
            s = Kd @ x - (float(slopes[j]) * dist if alibi else 0.0)
            own = k[0, t, 0].double() @ x
            top = torch.maximum(s.max(), own)
            w, w_own = (s - top).exp(), (own - top).exp()
            want[t, j] = (w @ Vd + w_own * v[0, t, 0].double()) / (w.sum() + w_own)
    err = (got[0].double() - want).norm() / want.norm()
    assert err <= 1e-5, float(err)


@pytest.mark.parametrize("group,D,n_sink,T", [(1, 128, 0, 9), (4, 64, 0, 30), (2, 128, 4, 40), (8, 128, 0, 64), (4, 128, 3, 5), (2, 64, 1, 1)])
def test_alibi_trees_over_fp32_caches(group, D, n_sink, T):
    """Eq. 1 in a tree over an fp32 cache: positions are the tokens seen plus the depth; rings that have wrapped, absent nodes.
    Bar: the framework's 1e-5.  A logit in powers of two is 17 at most where it counts (the sinks' keys are four times as long):
    three roundings of it 17 * 3 * 2^-24 * ln 2 = 2.1e-6, 32 additions of a lane's quarter of a dot product of up to 136,
    136 * 2^-24 * sqrt(32) / sqrt(128) = 4e-6, of a weight; an output between values a few apart moves by less than 1e-5."""
    Hkv, rounds, extra = 2, 50, 64
    w = synth.Workload("alibi_f32", 2, 1, Hkv * group, Hkv, D, "f32", [700, 90], [120, 40], n_sink, 1, extra, 61 + T)
    cache = make_cache(w, use_comp=0, max_new=extra)
    K, V = synth.make_dense_kv(w, 0, DEV)
    cache.compress(0, K, V, w.ctx_len, w.retrieval(0), w.window)
    slopes = (2.0 ** -(1.0 + np.arange(w.n_q_heads) * 8.0 / w.n_q_heads)).astype(np.float32)
    rz.razor_cache_set_alibi(cache.handle, slopes)
    normal = lambda tag, *shape, sub: synth.normal_bf16(w.seed, tag, shape, DEV, sub=sub).float()  # noqa: E731
    ka, va = (normal(tag, 2, rounds, Hkv, D, sub=6) for tag in (synth.TAG_KNEW, synth.TAG_VNEW))
    cache.append_many(0, ka, va)
    q = normal(synth.TAG_Q, 2, T, w.n_q_heads, D, sub=7)
    k, v = (normal(tag, 2, T, Hkv, D, sub=7) for tag in (synth.TAG_KNEW, synth.TAG_VNEW))
    rng = np.random.default_rng(T)
    parent = np.array([[rng.integers(-1, t) for t in range(T)] for _ in range(2)], dtype=np.int32)
    if T > 1:
        parent[1, T // 2] = -2
    mark = 12345.0
    out = torch.full(q.shape, mark, dtype=torch.float32, device=DEV)
    cache.decode_tree(0, q, k, v, torch.from_numpy(parent).to(DEV), out=out)
    assert cache.device_status() == 0
    out, qh, kh, vh, retr = to_f64(out), to_f64(q), to_f64(k), to_f64(v), w.retrieval(0)
    for b in range(2):
        for g in range(Hkv):
            ref = HeadRef(0, b, g, K[b, g], V[b, g], w.ctx_len[b], extra)
            for t in range(rounds):
                ref.append(ka[b, t, g].cpu(), va[b, t, g].cpu())
            hc = orc.compress_head(ref.K[:ref.n], ref.V[:ref.n], ref.n, n_sink, w.window[b], bool(retr[g]))
            for h in range(g * group, (g + 1) * group):
                want = orc.tree_attention(qh[b, :, h], hc, kh[b, :, g], vh[b, :, g], parent[b].tolist(), 1 / math.sqrt(D), False, float(slopes[h]))
                gone = np.isnan(want).all(1)
                assert (out[b, gone, h] == mark).all()
                assert np.abs(out[b, ~gone, h] - want[~gone]).max() <= TOL_OUT["f32"], (b, g, h)
    cache.close()
