"""Tree attention captured while appends are in flight: the capture runs nothing, so what is launched next has to behave as if
it were not there.  (What the host decides is checked in test_host_tracking.py; here the results.)"""
import pytest
import torch

from paper_2407_15891_b200 import synth

from _harness import HeadRef, check_head_state, make_cache

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
