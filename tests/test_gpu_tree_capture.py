"""Attention calls captured while appends are in flight or behind an empty start: a capture runs nothing, so what is launched next
has to behave as if it were not there.  (What the host decides is checked in test_host_tracking.py; here the results.)"""
import math

import numpy as np
import pytest
import torch

from oracle import razor_oracle as orc
from paper_2407_15891_b200 import synth

from _harness import TOL_OUT, HeadRef, check_head_state, make_cache, to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_appends_around_a_capture():
    """Single appends back to back with a tree call captured on another stream between them, nothing synchronised; then the
    state of some heads, and a replay against the eager call."""
    B, rounds, T = 16, 24, 5
    w = synth.Workload("around", B, 1, 16, 8, 128, "bf16", [100] * B, [20] * B, 4, 1, 2 * rounds, 47)
    cache = make_cache(w, max_new=2 * rounds)
    K, V = synth.make_dense_kv(w, 0, DEV)
    cache.compress(0, K, V, w.ctx_len, w.retrieval(0), w.window)
    heads = [(0, 0), (7, 3), (15, 7), (15, 0)]
    refs = {(b, g): HeadRef(0, b, g, K[b, g], V[b, g], 100, 2 * rounds) for b, g in heads}
    new = [[synth.normal_bf16(w.seed, tag, (B, 8, 128), DEV, sub=10 + i) for tag in (synth.TAG_KNEW, synth.TAG_VNEW)] for i in range(4)]
    q = synth.normal_bf16(w.seed, synth.TAG_Q, (B, T, 16, 128), DEV, sub=1)
    k, v = (synth.normal_bf16(w.seed, tag, (B, T, 8, 128), DEV, sub=1) for tag in (synth.TAG_KNEW, synth.TAG_VNEW))
    parent = torch.tensor([[-1, 0, 0, 1, -1]] * B, dtype=torch.int32, device=DEV)
    out = torch.zeros(B, T, 16, 128, device=DEV)
    side, graphs = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    for i in range(rounds):
        cache.append(0, *new[i % 4])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            graph.capture_begin(capture_error_mode="thread_local")
            cache.decode_tree(0, q, k, v, parent, out=out)
            graph.capture_end()
        graphs.append(graph)
        cache.append(0, *new[(i + 1) % 4])
    torch.cuda.synchronize()
    for (b, g), ref in refs.items():
        for i in range(rounds):
            for j in (i % 4, (i + 1) % 4):
                ref.append(new[j][0][b, g].cpu(), new[j][1][b, g].cpu())
        check_head_state(cache, ref, 4, 20, bool(w.retrieval(0)[g]))
    assert not out.any()
    graphs[0].replay()
    assert torch.equal(out, cache.decode_tree(0, q, k, v, parent))
    assert cache.device_status() == 0
    cache.close()


@pytest.mark.parametrize("shuffle,B,Hkv", [(0, 3, 4), (5, 40, 16)])
def test_a_first_decode_captured_behind_an_empty_start(shuffle, B, Hkv):
    """An empty layer, a few tokens appended, the first decode only captured: the eager decode behind it and the replay are right,
    and so they are after more appends and after the layer was started again."""
    w = synth.Workload("empty", B, 1, 2 * Hkv, Hkv, 128, "bf16", [0] * B, [20 + b for b in range(B)], 4, 1, 100, 57)
    cache = make_cache(w, max_new=100, shuffle=shuffle)
    k, v = (synth.normal_bf16(w.seed, tag, (B, 60, Hkv, 128), DEV, sub=1) for tag in (synth.TAG_KNEW, synth.TAG_VNEW))
    q = synth.normal_bf16(w.seed, synth.TAG_Q, (B, 2 * Hkv, 128), DEV, sub=1)
    out = torch.zeros(B, 2 * Hkv, 128, device=DEV)
    kh, vh, qh, retr = to_f64(k), to_f64(v), to_f64(q), w.retrieval(0)

    def check(got, n):
        got = to_f64(got)
        for b in {0, B // 2, B - 1}:
            for g in range(Hkv):
                hc = orc.compress_head(kh[b, :n, g], vh[b, :n, g], n, 4, w.window[b], bool(retr[g]))
                for h in (2 * g, 2 * g + 1):
                    assert np.abs(got[b, h] - orc.decode_head(qh[b, h], hc, 1 / math.sqrt(128))).max() <= TOL_OUT["bf16"]

    side = torch.cuda.Stream()
    for start in range(2):
        cache.start_empty(0, retr, w.window)
        cache.append_many(0, k[:, :5].contiguous(), v[:, :5].contiguous())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            graph.capture_begin(capture_error_mode="thread_local")
            cache.decode(0, q, out=out)
            graph.capture_end()
        out.zero_()
        check(cache.decode(0, q), 5)
        graph.replay()
        check(out, 5)
        cache.append_many(0, k[:, 5:].contiguous(), v[:, 5:].contiguous())
        check(cache.decode(0, q), 60)
        graph.replay()
        check(out, 60)
    assert cache.device_status() == 0
    cache.close()
