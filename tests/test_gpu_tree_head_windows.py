"""The tree calls on a layer whose heads each have a window of their own (the vision scopes of ALiBi heads, Section 3.1), with and
without the ALiBi penalty: a path appended, then the attention of a tree over it, per head against the oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import razor_oracle as orc
from paper_2407_15891_b200 import binding as rz
from paper_2407_15891_b200 import synth

from _harness import TOL_OUT, HeadRef, check_head_state, make_cache, to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype,alibi,n_sink,T", [("bf16", True, 0, 20), ("bf16", False, 4, 20), ("f32", True, 2, 9), ("bf16", True, 4, 40)])
def test_a_window_to_each_head(dtype, alibi, n_sink, T):
    w = synth.Workload("scopes", 2, 1, 10, 5, 128, dtype, [400, 77], [300, 50], n_sink, 1, 128, 33 + T)
    cache = make_cache(w, max_new=128, use_comp=0 if alibi else 1)
    own = [500, 0, 7, 64, 129]
    rz.razor_cache_set_head_windows(cache.handle, 0, own)
    slopes = (2.0 ** -(1.0 + np.arange(10) * 8.0 / 10)).astype(np.float32) if alibi else np.zeros(10, np.float32)
    if alibi:
        rz.razor_cache_set_alibi(cache.handle, slopes)
    K, V = synth.make_dense_kv(w, 0, DEV)
    retr = w.retrieval(0)
    cache.compress(0, K, V, w.ctx_len, retr, w.window)
    refs = {(b, g): HeadRef(0, b, g, K[b, g], V[b, g], w.ctx_len[b], 128) for b in range(2) for g in range(5)}
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    normal = lambda tag, *shape, sub: synth.normal_bf16(w.seed, tag, shape, DEV, sub=sub).to(dt)  # noqa: E731
    rng = np.random.default_rng(T)
    for rnd in range(3):
        q = normal(synth.TAG_Q, 2, T, 10, 128, sub=rnd)
        k, v = (normal(tag, 2, T, 5, 128, sub=rnd) for tag in (synth.TAG_KNEW, synth.TAG_VNEW))
        parent = np.array([[rng.integers(-1, t) for t in range(T)] for _ in range(2)], dtype=np.int32)
        out = to_f64(cache.decode_tree(0, q, k, v, torch.from_numpy(parent).to(DEV)))
        qh, kh, vh = to_f64(q), to_f64(k), to_f64(v)
        counts = [int(rng.integers(1, T + 1)), int(rng.integers(0, T + 1))]
        path = np.full((2, T), -1, dtype=np.int32)
        for b in range(2):
            path[b, :counts[b]] = np.sort(rng.permutation(T)[:counts[b]])
        cache.append_tree(0, k, v, torch.from_numpy(path).to(DEV), counts)
        for (b, g), ref in refs.items():
            window = min(w.window[b], own[g])
            hc = orc.compress_head(ref.K[:ref.n], ref.V[:ref.n], ref.n, n_sink, window, bool(retr[g]))
            for h in (2 * g, 2 * g + 1):
                want = orc.tree_attention(qh[b, :, h], hc, kh[b, :, g], vh[b, :, g], parent[b].tolist(), 1 / math.sqrt(128), not alibi, float(slopes[h]))
                assert np.abs(out[b, :, h] - want).max() <= TOL_OUT[dtype], (rnd, b, h)
            for n in path[b, :counts[b]]:
                ref.append(k[b, n, g].cpu(), v[b, n, g].cpu())
            check_head_state(cache, ref, n_sink, window, bool(retr[g]))
    assert cache.device_status() == 0
    cache.close()
