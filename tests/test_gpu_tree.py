"""GPU parity of the speculative-decoding operators (tree attention, verification, append of the accepted path) against
the fp64 oracle.

Bars.  Attention: the framework's own for bf16 (3e-3) and fp32 (1e-5) outputs, and for bf16 a tighter one where inputs
are standard normal, derived from the arithmetic: a weight enters the product as a bf16 head plus a bf16 remainder
(relative error at most 2^-17 = 7.6e-6, the remainder's rounding), an exponential of the hardware's adds 2^-22 and the
fp32 logit (128 products of about one) 128 * 2^-24 = 7.6e-6 of its size, a few units: an output, an average of values
below 6, stays within 6 * (7.6e-6 + 8 * 7.6e-6) < 5e-4.  Verification: whole numbers, equal.  Appends: layout bit for
bit, means 1e-3 (the framework's bar)."""
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
TIGHT = {"bf16": 5e-4, "f32": 1e-5}


def _random_parents(rng, batch, nodes, chain=False, holes=False):
    p = np.zeros((batch, nodes), dtype=np.int32)
    for b in range(batch):
        for t in range(nodes):
            p[b, t] = t - 1 if chain else rng.integers(-1, t)
        if holes and nodes > 1:
            p[b, rng.integers(0, nodes)] = rng.choice([-2, nodes, 1 << 30, -(1 << 31)])
    return p


def _drafts(w, T, sub, fused=False):
    """q [B, T, Hq, D], k, v [B, T, Hkv, D]; `fused`: column ranges of one projection's buffer."""
    dt = torch.bfloat16 if w.dtype == "bf16" else torch.float32
    H, Hq, D = w.n_kv_heads, w.n_q_heads, w.head_dim
    if fused:
        x = synth.normal_bf16(w.seed, synth.TAG_Q, (w.batch, T, (Hq + 2 * H) * D), DEV, sub=100 + sub).to(dt)
        return (x[:, :, :Hq * D].unflatten(2, (Hq, D)), x[:, :, Hq * D:(Hq + H) * D].unflatten(2, (H, D)),
                x[:, :, (Hq + H) * D:].unflatten(2, (H, D)))
    return (synth.normal_bf16(w.seed, synth.TAG_Q, (w.batch, T, Hq, D), DEV, sub=sub).to(dt),
            synth.normal_bf16(w.seed, synth.TAG_KNEW, (w.batch, T, H, D), DEV, sub=sub).to(dt),
            synth.normal_bf16(w.seed, synth.TAG_VNEW, (w.batch, T, H, D), DEV, sub=sub).to(dt))


def _compress(w, **kw):
    cache = make_cache(w, **kw)
    K, V = synth.make_dense_kv(w, 0, DEV)
    cache.compress(0, K, V, w.ctx_len, w.retrieval(0), w.window)
    return cache, K, V


def _check(w, cache, refs, q, k, v, parent, scale=None, use_comp=True, slopes=None, tol=None, heads=None):
    """The whole output against the oracle; absent rows must be as they were."""
    T, G = q.shape[1], w.n_q_heads // w.n_kv_heads
    mark = 12345.0
    out = torch.full((w.batch, T, w.n_q_heads, w.head_dim), mark, dtype=torch.float32, device=DEV)
    cache.decode_tree(0, q, k, v, torch.from_numpy(parent).to(DEV), out=out)
    assert cache.device_status() == 0
    out, qh, kh, vh = out.cpu().numpy().astype(np.float64), to_f64(q), to_f64(k), to_f64(v)
    scale = 1.0 / math.sqrt(w.head_dim) if scale is None else scale
    tol = TIGHT[w.dtype] if tol is None else tol
    retr = w.retrieval(0)
    for (b, g), ref in refs.items():
        if heads is not None and (b, g) not in heads:
            continue
        hc = orc.compress_head(ref.K[:ref.n], ref.V[:ref.n], ref.n, w.n_sink, w.window[b], bool(retr[g]))
        for j in range(G):
            h = g * G + j
            want = orc.tree_attention(qh[b, :, h], hc, kh[b, :, g], vh[b, :, g], parent[b].tolist(), scale, use_comp,
                                      0.0 if slopes is None else float(slopes[h]))
            gone = np.isnan(want).all(1)
            assert (out[b, gone, h] == mark).all()
            err = float(np.abs(out[b, ~gone, h] - want[~gone]).max()) if (~gone).any() else 0.0
            assert err <= tol, (err, b, g, j)
    return out


def _refs(w, K, V, extra=0):
    return {(b, g): HeadRef(0, b, g, K[b, g], V[b, g], w.ctx_len[b], extra)
            for b in range(w.batch) for g in range(w.n_kv_heads)}


# ----------------------------------------------------------------------------- attention
@pytest.mark.parametrize("group,T,D,dtype", [
    (1, 1, 128, "bf16"), (1, 5, 128, "bf16"), (1, 33, 64, "bf16"), (2, 16, 128, "bf16"), (4, 1, 64, "bf16"),
    (4, 8, 128, "bf16"), (4, 26, 128, "bf16"), (8, 17, 128, "bf16"), (8, 64, 64, "bf16"), (1, 64, 128, "bf16"),
    (1, 127, 128, "bf16"), (2, 128, 64, "bf16"), (8, 128, 128, "bf16"), (4, 128, 128, "bf16"),
    (1, 3, 64, "f32"), (4, 9, 128, "f32"), (8, 40, 64, "f32"), (2, 128, 128, "f32")])
def test_tree_attention_matches_the_oracle(group, T, D, dtype):
    """Ragged batch: a context that ends inside a page and a block, one shorter than its window, one of a single token, one
    that is empty; trees with absent nodes."""
    Hkv = 3
    w = synth.Workload("tree", 4, 1, Hkv * group, Hkv, D, dtype, [1003, 70, 1, 0], [200, 90, 40, 5], 4, 1, 0, 900 + T + group)
    cache, K, V = _compress(w, shuffle=3)
    rng = np.random.default_rng(T * 10 + group)
    q, k, v = _drafts(w, T, 1)
    refs = _refs(w, K, V)
    _check(w, cache, refs, q, k, v, _random_parents(rng, w.batch, T, holes=True))
    _check(w, cache, refs, q, k, v, _random_parents(rng, w.batch, T, chain=True))
    cache.close()


@pytest.mark.parametrize("n_ctx,window,n_sink", [(15, 4, 0), (16, 16, 0), (17, 0, 0), (17, 0, 1), (127, 40, 4), (128, 40, 4),
                                                 (129, 128, 1), (255, 3, 17), (256, 90, 4), (257, 200, 4), (640, 639, 1)])
def test_lengths_around_pages_and_blocks(n_ctx, window, n_sink):
    """Every length of a page's and a block's border, windows of zero (the whole context is the compensation token) and
    sinks that fill more than a page."""
    w = synth.Workload("edge", 2, 1, 8, 4, 128, "bf16", [n_ctx, max(0, n_ctx - 1)], [window, window], n_sink, 1, 0, n_ctx)
    cache, K, V = _compress(w)
    q, k, v = _drafts(w, 12, 2)
    _check(w, cache, _refs(w, K, V), q, k, v, _random_parents(np.random.default_rng(n_ctx), 2, 12))
    cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_drafts_out_of_one_fused_projection(dtype):
    """q, k, v as column ranges of one buffer: strided over sequences and nodes."""
    w = synth.Workload("fused", 3, 1, 8, 4, 128, dtype, [300, 77, 512], [100, 40, 60], 4, 1, 0, 31)
    cache, K, V = _compress(w)
    q, k, v = _drafts(w, 11, 3, fused=True)
    assert not q.is_contiguous() and not k.is_contiguous()
    _check(w, cache, _refs(w, K, V), q, k, v, _random_parents(np.random.default_rng(5), 3, 11))
    cache.close()


@pytest.mark.parametrize("sm_scale,use_comp", [(1.0, 1), (0.05, 1), (0.0, 0)])
def test_scale_and_truncation(sm_scale, use_comp):
    """sm_scale = 1 (the printed form of Eq. 5: logits of standard deviation 11, 45 at the sinks, so the running maximum
    climbs far) and the scheme without compensation.  With logits up to about 180 the 128 roundings of a logit's partial
    sums leave 180 * sqrt(128) * 2^-24 = 1.2e-4 in it, so in a weight; an output, an average of values below 6 over
    weights that are off so in numerator and denominator, 2 * 6 * 1.2e-4 = 1.5e-3: within the framework's 3e-3."""
    w = synth.Workload("scale", 2, 1, 4, 2, 128, "bf16", [900, 333], [150, 60], 4, 1, 0, 77)
    cache, K, V = _compress(w, sm_scale=sm_scale, use_comp=use_comp)
    q, k, v = _drafts(w, 20, 4)
    _check(w, cache, _refs(w, K, V), q, k, v, _random_parents(np.random.default_rng(6), 2, 20),
           scale=sm_scale or None, use_comp=bool(use_comp), tol=TOL_OUT["bf16"])
    cache.close()


@pytest.mark.parametrize("group,D,n_sink,T", [(1, 128, 0, 9), (4, 64, 0, 30), (2, 128, 4, 40), (8, 128, 0, 64), (4, 128, 3, 5)])
def test_alibi_trees(group, D, n_sink, T):
    """Eq. 1 in a tree: a node's position is the tokens seen plus its depth; with and without sink tokens, rings that have
    wrapped."""
    Hkv = 2
    w = synth.Workload("alibi_tree", 2, 1, Hkv * group, Hkv, D, "bf16", [700, 90], [120, 40], n_sink, 1, 64, 41 + T)
    cache, K, V = _compress(w, use_comp=0, max_new=64)
    slopes = (2.0 ** -(1.0 + np.arange(w.n_q_heads) * 8.0 / w.n_q_heads)).astype(np.float32)
    rz.razor_cache_set_alibi(cache.handle, slopes)
    refs = _refs(w, K, V, extra=64)
    _, ka, va = _drafts(w, 50, 6)
    cache.append_many(0, ka, va)       # the rings wrap
    for (b, g), ref in refs.items():
        for t in range(50):
            ref.append(ka[b, t, g].cpu(), va[b, t, g].cpu())
    q, k, v = _drafts(w, T, 7)
    _check(w, cache, refs, q, k, v, _random_parents(np.random.default_rng(T), 2, T, holes=True), use_comp=False, slopes=slopes)
    cache.close()


def test_a_late_maximum_far_above_the_first():
    """The running maximum has to follow: a needle in the last page whose logit is 200 (in powers of two: 288) above all
    before it, and drafts whose logits are higher still for some nodes only."""
    w = synth.Workload("needle", 1, 1, 2, 1, 128, "bf16", [2000], [300], 4, 1, 0, 5)
    cache = make_cache(w)
    K, V = synth.make_dense_kv(w, 0, DEV)
    q, k, v = _drafts(w, 6, 8)
    unit = q[0, 0, 0].float() / q[0, 0, 0].float().norm() ** 2
    K[0, 0, 1990] = (200.0 * math.sqrt(128) * unit).to(torch.bfloat16)
    k[0, 3, 0] = (400.0 * math.sqrt(128) * unit).to(torch.bfloat16)
    cache.compress(0, K, V, w.ctx_len, w.retrieval(0), w.window)
    parent = np.array([[-1, 0, 0, 1, 3, -1]], dtype=np.int32)
    # logits near 400 with fp32 partial sums: 400 * 2^-24 * 2 relative in the weights of the runner-ups, which are nothing
    _check(w, cache, _refs(w, K, V), q, k, v, parent, tol=TOL_OUT["bf16"])
    cache.close()


@pytest.mark.parametrize("dtype,group,D,more", [("bf16", 4, 128, 0), ("f32", 4, 128, 0), ("bf16", 1, 128, 0),
                                                  ("bf16", 8, 128, 0), ("bf16", 8, 64, 20), ("bf16", 1, 128, 119)])
def test_what_a_node_does_not_see_cannot_reach_it(dtype, group, D, more):
    """NaN and infinities in the K and V of nodes on other branches, in absent nodes and in the pool beyond a head's last
    token leave a node's output as it is, bit for bit; nodes that see them get what the arithmetic gives."""
    w = synth.Workload("poison", 2, 1, 2 * group, 2, D, dtype, [130, 37], [60, 30], 4, 1, 0, 15)
    cache = make_cache(w)
    cache.pool.fill_(0xFF)             # every 16- and 32-bit pattern of it is a NaN
    K, V = synth.make_dense_kv(w, 0, DEV)
    cache.compress(0, K, V, w.ctx_len, w.retrieval(0), w.window)
    q, k, v = _drafts(w, 9 + more, 9)
    # 2, 4: the clean line; 5, 6 absent; `more` nodes behind them that follow node 4
    parent = np.array([[-1, 0, 0, 1, 2, -2, 5, -1, 7] + [4] * more] * 2, dtype=np.int32)
    pd = torch.from_numpy(parent).to(DEV)
    clean = cache.decode_tree(0, q, k, v, pd).clone()
    assert torch.isfinite(clean).all()
    for bad in (float("nan"), float("inf"), -float("inf")):
        k2, v2 = k.clone(), v.clone()
        for n in (1, 5, 6, 7):
            v2[:, n, :, ::3] = bad
            k2[:, n, :, 5] = bad
        got = cache.decode_tree(0, q, k2, v2, pd)
        for t in (0, 2, 4, *range(9, 9 + more)):
            assert torch.equal(got[:, t], clean[:, t]), (bad, t)
        assert (got[:, 5:7] == 0).all()
        # V alone: the nodes that see it get non-finite values there and the clean ones elsewhere
        v3 = v.clone()
        v3[:, 1, :, 10] = bad
        got = cache.decode_tree(0, q, k, v3, pd)
        for t in (1, 3):
            assert not torch.isfinite(got[:, t, :, 10]).any()
            if not math.isnan(bad):
                assert (got[:, t, :, 10] == bad).all()
            keep = [d for d in range(D) if d != 10]
            assert torch.equal(got[:, t][..., keep], clean[:, t][..., keep])
        assert torch.equal(got[:, 0], clean[:, 0]) and torch.equal(got[:, 4], clean[:, 4])
    assert cache.device_status() == 0
    cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_long_context_in_many_parts_is_repeatable(dtype):
    """32K tokens of few heads: every head is cut into parts.  Against the oracle, and twice the same bits."""
    w = synth.Workload("long", 2, 1, 8, 2, 128, dtype, [32771, 20000], [5000, 3000], 4, 1, 0, 19)
    cache, K, V = _compress(w)
    q, k, v = _drafts(w, 24, 10)
    parent = _random_parents(np.random.default_rng(1), 2, 24)
    a = _check(w, cache, _refs(w, K, V), q, k, v, parent)
    b = _check(w, cache, {}, q, k, v, parent)
    assert np.array_equal(a, b)
    cache.close()


@pytest.mark.parametrize("nodes,group,D,dtype,n_ctx", [
    (1, 1, 128, "bf16", 40000), (20, 4, 128, "bf16", 40001), (7, 8, 64, "bf16", 40015), (33, 4, 64, "bf16", 12345),
    (128, 8, 128, "bf16", 9001), (3, 2, 128, "f32", 40000), (40, 1, 64, "f32", 20001), (2, 1, 128, "bf16", 1500)])
def test_a_single_head_cut_into_many_parts(nodes, group, D, dtype, n_ctx):
    """One KV head alone: as many parts as spans, or as the shorter contexts have steps for, folded by several warps to a row."""
    w = synth.Workload("single", 1, 1, group, 1, D, dtype, [n_ctx], [64], 4, 1, 0, nodes)
    cache, K, V = _compress(w)
    q, k, v = _drafts(w, nodes, 6)
    _check(w, cache, _refs(w, K, V), q, k, v, _random_parents(np.random.default_rng(nodes), 1, nodes, holes=True))
    cache.close()


def test_tree_attention_in_a_graph_follows_the_cache():
    """Captured on a stream of its own and replayed after appends have grown the cache: a replay attends to the cache as it
    then is, and another call's shape in between does not disturb it."""
    w = synth.Workload("graph", 2, 1, 8, 4, 128, "bf16", [900, 400], [200, 90], 4, 1, 64, 23)
    cache, K, V = _compress(w, max_new=64)
    refs = _refs(w, K, V, extra=64)
    q, k, v = _drafts(w, 10, 11)
    parent = _random_parents(np.random.default_rng(2), 2, 10)
    pd = torch.from_numpy(parent).to(DEV)
    out = torch.zeros(2, 10, 8, 128, dtype=torch.float32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.decode_tree(0, q, k, v, pd, out=out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.decode_tree(0, q, k, v, pd, out=out)
    for rnd in range(2):
        out.zero_()
        graph.replay()
        want = cache.decode_tree(0, q, k, v, pd)
        assert torch.equal(out, want)
        _check(w, cache, refs, q, k, v, parent)
        q2, k2, v2 = _drafts(w, 40, 12 + rnd)
        cache.decode_tree(0, q2, k2, v2, torch.from_numpy(_random_parents(np.random.default_rng(3), 2, 40)).to(DEV))
        _, ka, va = _drafts(w, 30, 20 + rnd)
        cache.append_many(0, ka, va)
        for (b, g), ref in refs.items():
            for t in range(30):
                ref.append(ka[b, t, g].cpu(), va[b, t, g].cpu())
    out.zero_()
    graph.replay()
    assert torch.equal(out, cache.decode_tree(0, q, k, v, pd))
    _check(w, cache, refs, q, k, v, parent)
    cache.close()


def test_refusals_leave_the_cache_usable():
    w = synth.Workload("refuse", 2, 1, 8, 4, 128, "bf16", [300, 77], [60, 30], 4, 1, 6, 3)
    fresh = make_cache(w, max_new=6)
    q, k, v = _drafts(w, 4, 1)
    parent = torch.zeros(2, 4, dtype=torch.int32, device=DEV) - 1
    with pytest.raises(rz.RazorError) as e:
        fresh.decode_tree(0, q, k, v, parent)
    assert e.value.status == -6
    with pytest.raises(rz.RazorError) as e:
        fresh.append_tree(0, k, v, None, [1, 1])
    assert e.value.status == -6
    fresh.close()
    cache, K, V = _compress(w, max_new=6)
    out = torch.zeros(2, 4, 8, 128, device=DEV)
    good = dict(q=q, qb=4096, qt=1024, k=k, v=v, kb=2048, kt=512, parent=parent, n=4, out=out)

    def call(layer=0, **kw):
        a = dict(good, **kw)
        rz.razor_decode_attention_tree(cache.handle, layer, a["q"], a["qb"], a["qt"], a["k"], a["v"], a["kb"], a["kt"],
                                       a["parent"], a["n"], a["out"])

    for kw, code in [(dict(layer=1), -1), (dict(layer=-1), -1), (dict(n=0), -1), (dict(n=129), -1), (dict(q=None), -2),
                     (dict(k=None), -2), (dict(v=None), -2), (dict(parent=None), -2), (dict(out=None), -2),
                     (dict(q=q.data_ptr() + 2), -8), (dict(out=out.data_ptr() + 4), -8), (dict(parent=parent.data_ptr() + 2), -8),
                     (dict(qt=1028), -8), (dict(kt=516), -8), (dict(qb=4100), -8), (dict(qt=1016), -1), (dict(kt=504), -1),
                     (dict(kb=504), -1), (dict(qb=-4096), -1), (dict(kt=1 << 37), -1)]:
        with pytest.raises(rz.RazorError) as e:
            call(**kw)
        assert e.value.status == code, kw

    def commit(n_accept, layer=0, **kw):
        a = dict(dict(k=k, v=v, kb=2048, kt=512, path=None, n=4), **kw)
        rz.razor_append_tree(cache.handle, layer, a["k"], a["v"], a["kb"], a["kt"], a["path"], a["n"], n_accept)

    for n_accept, kw, code in [([5, 0], {}, -1), ([-1, 0], {}, -1), ([1, 1], dict(layer=2), -1), ([1, 1], dict(k=None), -2),
                               ([1, 1], dict(n=0), -1), ([1, 1], dict(n=200), -1), ([1, 1], dict(kt=508), -8),
                               ([1, 1], dict(path=parent.data_ptr() + 1), -8), ([1, 1], dict(kb=8), -1)]:
        with pytest.raises(rz.RazorError) as e:
            commit(n_accept, **kw)
        assert e.value.status == code, (n_accept, kw)
    commit([4, 0])
    with pytest.raises(rz.RazorError) as e:
        commit([3, 1])                      # sequence 0 has room for two more
    assert e.value.status == -5
    with pytest.raises(rz.RazorError) as e:
        cache.append_many(0, *_drafts(w, 3, 2)[1:])
    assert e.value.status == -5
    commit([2, 3])
    with pytest.raises(rz.RazorError) as e:
        cache.append(0, k[:, 0].contiguous(), v[:, 0].contiguous())
    assert e.value.status == -5
    assert [cache.export(0, b, 0)["kept_pos"].numel() + cache.export(0, b, 0)["n_drop"] for b in (0, 1)] == [306, 80]
    call()
    assert cache.device_status() == 0
    for bad in (dict(q=q.float()), dict(k_draft=k[:, :3]), dict(parent=parent.long()), dict(q=q[:, :, :4]),
                dict(q=q.transpose(2, 3).contiguous().transpose(2, 3))):
        with pytest.raises(AssertionError):
            cache.decode_tree(0, **dict(dict(q=q, k_draft=k, v_draft=v, parent=parent), **bad))
    cache.close()


@pytest.mark.parametrize("seed", range(14))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_random_shapes(dtype, seed):
    """Groups, head sizes, lengths, windows, sinks and trees at random: heads that spans cut anywhere, several tiles of rows,
    more heads than SMs."""
    rng = np.random.default_rng(7000 + seed)
    group, D = int(rng.choice([1, 2, 4, 8])), int(rng.choice([64, 128]))
    B, Hkv = (int(rng.integers(1, 4)), int(rng.integers(1, 5))) if seed % 3 else (9, 40 // group)
    top = 40 if seed % 3 == 0 else int(rng.choice([30, 600, 5000]))
    lens = [int(x) for x in rng.integers(0, top + 1, B)]
    wins = [int(x) for x in rng.integers(0, max(1, top // 2) + 1, B)]
    T = int(rng.integers(1, rz.TREE_MAX_NODES + 1))
    w = synth.Workload("any", B, 1, Hkv * group, Hkv, D, dtype, lens, wins, int(rng.integers(0, 20)), min(1, Hkv - 1), 0, seed)
    use_comp = int(rng.integers(0, 4) > 0)
    cache, K, V = _compress(w, shuffle=int(rng.integers(0, 3)), use_comp=use_comp)
    q, k, v = _drafts(w, T, 3, fused=bool(rng.integers(0, 2)))
    heads = {(b, g) for b in range(B) for g in range(Hkv)} if seed % 3 else {(b, int(rng.integers(Hkv))) for b in range(B)}
    _check(w, cache, _refs(w, K, V), q, k, v, _random_parents(rng, B, T, chain=seed % 5 == 0, holes=True),
           use_comp=bool(use_comp), heads=heads)
    cache.close()


def test_tree_attention_on_another_stream():
    """Every call on a stream of its own, ordered by events: inputs written there just before, results read there."""
    w = synth.Workload("stream", 2, 1, 8, 2, 128, "bf16", [1500, 77], [300, 50], 4, 1, 16, 29)
    cache, K, V = _compress(w, max_new=16)
    q, k, v = _drafts(w, 30, 1)
    parent = torch.from_numpy(_random_parents(np.random.default_rng(1), 2, 30)).to(DEV)
    want = cache.decode_tree(0, q, k, v, parent).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        q2, k2, v2 = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        for _ in range(20):
            q2.zero_(), k2.zero_(), v2.zero_()
            q2.copy_(q), k2.copy_(k), v2.copy_(v)
            got = cache.decode_tree(0, q2, k2, v2, parent)
        q2.fill_(float("nan"))       # (behind the call: it has read its queries)
    side.synchronize()
    assert torch.equal(got, want)
    cache.close()


@pytest.mark.parametrize("B", [37, 38, 75, 149, 300, 700])
def test_verification_of_large_batches(B):
    """More sequences than CTAs fit at eight to a sequence, then at four, two and one."""
    assert _verify_check(*_verify_case(np.random.default_rng(B), B, 4, 700, True)) > 0


# ----------------------------------------------------------------------------- append of a path
@pytest.mark.parametrize("dtype,D,T,n_sink,windows", [
    ("bf16", 128, 6, 4, [60, 30, 3]), ("bf16", 64, 40, 4, [12, 100, 0]), ("f32", 128, 9, 0, [1, 2, 50]),
    ("f32", 64, 128, 17, [40, 7, 300]), ("bf16", 128, 128, 4, [5, 64, 129])])
def test_append_of_a_path_is_as_many_single_appends(dtype, D, T, n_sink, windows):
    """Every sequence its own count and path, several rounds: windows fill, evict, wrap, and are shorter than the run; one
    window of zero drops every token at once.  Layout bit for bit, means, and the attention over the result."""
    w = synth.Workload("path", 3, 1, 8, 4, D, dtype, [70, 9, 200], windows, n_sink, 1, 4 * T, 60 + T)
    cache, K, V = _compress(w, max_new=4 * T, shuffle=2)
    refs = _refs(w, K, V, extra=4 * T)
    rng = np.random.default_rng(T)
    retr = w.retrieval(0)
    for rnd in range(4):
        _, k, v = _drafts(w, T, 30 + rnd, fused=rnd % 2 == 1)
        counts = [int(rng.integers(0, T + 1)) for _ in range(3)] if rnd else [T, 0, 1]
        path = np.full((3, T), -1, dtype=np.int32)
        for b in range(3):
            path[b, :counts[b]] = np.sort(rng.permutation(T)[:counts[b]])
        cache.append_tree(0, k, v, None if rnd == 3 else torch.from_numpy(path).to(DEV), counts)
        kh, vh = k.cpu(), v.cpu()
        for (b, g), ref in refs.items():
            for i in range(counts[b]):
                n = i if rnd == 3 else path[b, i]
                ref.append(kh[b, n, g], vh[b, n, g])
            check_head_state(cache, ref, n_sink, windows[b], bool(retr[g]))
    q, k, v = _drafts(w, 5, 50)
    _check(w, cache, refs, q, k, v, _random_parents(rng, 3, 5))
    # and the older calls go on from there
    _, k1, v1 = _drafts(w, 1, 51)
    if max(int(x) for x in [refs[(b, 0)].n - w.ctx_len[b] for b in range(3)]) < 4 * T:
        cache.append(0, k1[:, 0].contiguous(), v1[:, 0].contiguous())
        for (b, g), ref in refs.items():
            ref.append(k1[b, 0, g].cpu(), v1[b, 0, g].cpu())
            check_head_state(cache, ref, n_sink, windows[b], bool(retr[g]))
    cache.close()


def test_layers_appended_to_in_turn_without_a_decode_between():
    """Paths and single tokens appended to two layers in turn, with nothing in between that waits: an append may start
    while the one before is in flight, and has to find what the last append of its own layer left."""
    w = synth.Workload("turn", 16, 2, 8, 8, 128, "bf16", [100] * 16, [20] * 16, 4, 1, 200, 41)
    cache = make_cache(w, max_new=200)
    heads = [(0, 0), (7, 3), (15, 7), (15, 0)]
    refs = []
    for layer in range(2):
        K, V = synth.make_dense_kv(w, layer, DEV)
        cache.compress(layer, K, V, w.ctx_len, w.retrieval(layer), w.window)
        refs.append({(b, g): HeadRef(layer, b, g, K[b, g], V[b, g], 100, 200) for b, g in heads})
    drafts = [_drafts(w, 12, 300 + i) for i in range(2)]
    ones = [[x[:, i].contiguous() for x in drafts[0][1:]] for i in range(3)]
    counts = [12, 5] * 8
    torch.cuda.synchronize()
    for _ in range(6):
        cache.append_tree(0, drafts[0][1], drafts[0][2], None, counts)
        for i in range(3):
            cache.append(1, *ones[i])
            cache.append(0, *ones[i])
        cache.append_tree(1, drafts[1][1], drafts[1][2], None, counts)
    for layer in range(2):
        kv = [x.cpu() for x in drafts[layer][1:]]
        for (b, g), ref in refs[layer].items():
            for _ in range(6):
                path = [(kv[0][b, i, g], kv[1][b, i, g]) for i in range(counts[b])]
                single = [(ones[i][0][b, g].cpu(), ones[i][1][b, g].cpu()) for i in range(3)]
                for k, v in (path + single if layer == 0 else single + path):
                    ref.append(k, v)
            check_head_state(cache, ref, 4, 20, bool(w.retrieval(layer)[g]))
    assert cache.device_status() == 0
    cache.close()


def test_path_entries_outside_the_tree_read_the_nearest_node():
    w = synth.Workload("clamp", 1, 1, 2, 2, 128, "bf16", [20], [50], 4, 1, 8, 4)
    cache, K, V = _compress(w, max_new=8)
    refs = _refs(w, K, V, extra=8)
    _, k, v = _drafts(w, 4, 1)
    cache.append_tree(0, k, v, torch.tensor([[-1, 2, 9, 1 << 30]], dtype=torch.int32, device=DEV), [4])
    for (b, g), ref in refs.items():
        for n in (0, 2, 3, 3):
            ref.append(k[b, n, g].cpu(), v[b, n, g].cpu())
        check_head_state(cache, ref, 4, 50, bool(w.retrieval(0)[g]))
    cache.close()


def test_append_of_a_path_is_refused_on_a_capturing_stream():
    """A replay would move the device's lengths and not the host's."""
    w = synth.Workload("capture", 1, 1, 2, 2, 128, "bf16", [20], [50], 4, 1, 8, 4)
    cache, K, V = _compress(w, max_new=8)
    _, k, v = _drafts(w, 4, 1)
    graph, x = torch.cuda.CUDAGraph(), torch.zeros(4, device=DEV)
    with torch.cuda.graph(graph):
        x.add_(1)
        with pytest.raises(rz.RazorError) as e:
            cache.append_tree(0, k, v, None, [2])
    assert e.value.status == -1
    graph.replay()
    assert cache.export(0, 0, 0)["kept_pos"].numel() == 20
    cache.append_tree(0, k, v, None, [2])
    assert cache.export(0, 0, 0)["kept_pos"].numel() == 22
    cache.close()


def test_a_large_batch_takes_several_launches_of_counts():
    """2100 sequences: the counts travel 1024 at a time."""
    B = 2100
    w = synth.Workload("wide", B, 1, 1, 1, 64, "bf16", [0] * B, [4] * B, 1, 0, 8, 9)
    cfg = rz.make_config(B, 1, 1, 1, 64, "bf16", 1, 0, 8)
    cache = rz.RazorCache(cfg, [0] * B, [4] * B, [0])
    cache.start_empty(0, [0], [4] * B)
    _, k, v = _drafts(w, 8, 1)
    counts = [(7 * b + 3) % 9 for b in range(B)]
    cache.append_tree(0, k, v, None, counts)
    for b in (0, 1, 1023, 1024, 1025, 2047, 2048, B - 1):
        ex = cache.export(0, b, 0)
        keep = orc.kept_positions(counts[b], 1, 4, False)
        assert ex["kept_pos"].cpu().numpy().tolist() == keep.tolist() and ex["n_drop"] == counts[b] - len(keep)
        assert torch.equal(ex["K"], k[b, keep.tolist(), 0])
    cache.close()


# ----------------------------------------------------------------------------- verification
def _verify_case(rng, B, T, V, sampled, chain=False, holes=False, sharp=1.0):
    parent = _random_parents(rng, B, T, chain=chain, holes=holes)
    logits = rng.standard_normal((B, T + 1, V)) * sharp
    p = np.exp(logits - logits.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    q = None
    tokens = np.zeros((B, T), dtype=np.int32)
    lq = logits + 0.7 * rng.standard_normal((B, T + 1, V))
    if sampled:
        q = np.exp(lq - lq.max(-1, keepdims=True))
        q /= q.sum(-1, keepdims=True)
    for b in range(B):
        used = {}
        for t in range(T):
            a = int(parent[b, t])
            row = a + 1 if -1 <= a < t else 0
            order = used.setdefault(row, list(np.argsort(-(lq[b, row] + rng.gumbel(size=V)))))
            tokens[b, t] = order.pop(0) if order else 0
    return parent, p, q, tokens, rng.random((B, T), dtype=np.float32), rng.random(B, dtype=np.float32)


def _verify_check(parent, p, q, tokens, u, r, dtype=torch.float32):
    dev = lambda x, dt: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(DEV).to(dt)  # noqa: E731
    P, Q = dev(p, dtype), dev(q, dtype)
    got = rz.razor_verify_tree(P, Q, dev(tokens, torch.int32), dev(parent, torch.int32), dev(u, torch.float32), dev(r, torch.float32))
    got = {k: x.cpu().numpy() for k, x in got.items()}
    P, Q = to_f64(P), None if Q is None else to_f64(Q)
    n_kept = 0
    for b in range(tokens.shape[0]):
        path, token = orc.verify_tree(P[b], None if Q is None else Q[b], tokens[b], parent[b], u[b], r[b])
        assert got["accepted"][b] == len(path), b
        assert got["path"][b].tolist() == path + [-1] * (tokens.shape[1] - len(path)), b
        assert got["token"][b] == token, b
        n_kept += len(path)
    return n_kept


@pytest.mark.parametrize("B,T,V,sampled,chain,dtype", [
    (64, 1, 2, True, True, torch.float32), (40, 7, 5, True, False, torch.float32), (30, 12, 255, False, False, torch.float32),
    (30, 12, 256, True, False, torch.bfloat16), (20, 5, 257, True, True, torch.float32), (9, 128, 1000, True, False, torch.float32),
    (9, 128, 1000, False, False, torch.bfloat16), (5, 127, 2049, True, True, torch.bfloat16), (4, 7, 32000, True, True, torch.float32),
    (3, 26, 50257, False, False, torch.float32), (2, 30, 128256, True, False, torch.float32), (3, 4, 1, True, False, torch.float32),
    (2, 9, 140001, True, False, torch.bfloat16), (40, 20, 2000, True, False, torch.bfloat16), (1, 2, 2200001, True, False, torch.float32)])
def test_verification_matches_the_oracle(B, T, V, sampled, chain, dtype):
    rng = np.random.default_rng(B * 1000 + T)
    kept = _verify_check(*_verify_case(rng, B, T, V, sampled, chain=chain, holes=not chain), dtype=dtype)
    # (drafts that were not drawn from a distribution near the target's are seldom kept: nothing to count there)
    assert kept > 0 or not sampled


def test_looked_up_drafts_that_are_often_right():
    """Peaked rows, so that drafts without probabilities are kept in long paths too."""
    kept = _verify_check(*_verify_case(np.random.default_rng(77), 40, 24, 300, False, sharp=6.0))
    assert kept >= 20


@pytest.mark.parametrize("copies", [1, 2])
def test_verification_on_the_borders(copies):
    """u and r of zero, r of the largest fp32 below one, rows with long runs of zeros, one-hot rows, rows without any
    weight, NaN and infinite entries, sibling tokens that repeat, tokens outside the vocabulary; rows kept in registers and,
    with more sequences, streamed."""
    rng = np.random.default_rng(4)
    B, T, V = 12, 6, 700
    parent, p, q, tokens, u, r = _verify_case(rng, B, T, V, True)
    p[0, :, 100:] = 0
    p[1, :, :650] = 0
    p[2] = 0
    p[2, :, 350] = 1
    p[3] = 0                                   # no weight anywhere
    p[4, :, 10] = np.nan
    p[5, :, 20] = np.inf
    p[6, :, 30] = -1
    q[7] = np.nan
    q[8, :, :] = 1.0 / V
    tokens[9] = tokens[9, 0]                   # siblings of one token
    tokens[10, ::2] = [-1, V, 1 << 30]
    parent[11] = [-1] * T
    parent, p, q, tokens = (np.concatenate([x] * copies) for x in (parent, p, q, tokens))
    B *= copies
    for rr in (0.0, 0.5, float(np.nextafter(np.float32(1), np.float32(0)))):
        for uu in (0.0, 0.3, float(np.nextafter(np.float32(1), np.float32(0)))):
            uv, rv = np.full((B, T), uu, np.float32), np.full(B, rr, np.float32)
            _verify_check(parent, p, q, tokens, uv, rv)
            _verify_check(parent, p, None, tokens, uv, rv)


def test_verification_in_a_graph():
    rng = np.random.default_rng(12)
    cases = [_verify_case(rng, 5, 9, 3001, True) for _ in range(2)]
    bufs = [torch.from_numpy(np.ascontiguousarray(x)).to(DEV) for x in cases[0]]
    bufs[1:3] = [x.float() for x in bufs[1:3]]
    call = lambda: rz.razor_verify_tree(bufs[1], bufs[2], bufs[3], bufs[0], bufs[4], bufs[5])  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for case in cases:
        for buf, x in zip(bufs, case):
            buf.copy_(torch.from_numpy(np.ascontiguousarray(x)))
        graph.replay()
        P, Q = to_f64(bufs[1]), to_f64(bufs[2])
        for b in range(5):
            path, token = orc.verify_tree(P[b], Q[b], case[3][b], case[0][b], case[4][b], case[5][b])
            assert got["accepted"][b].item() == len(path) and got["token"][b].item() == token
            assert got["path"][b].tolist() == path + [-1] * (9 - len(path))


def test_verification_of_strided_rows():
    """Rows of a padded vocabulary inside a larger buffer, at an odd offset, and a chain's draft rows without a last one."""
    rng = np.random.default_rng(8)
    parent, p, q, tokens, u, r = _verify_case(rng, 5, 6, 1003, True, chain=True)
    for dtype in (torch.float32, torch.bfloat16):
        big = torch.full((5, 9, 1101), 7.0, dtype=dtype, device=DEV)
        P = big[:, 1:8, 33:1036]
        P.copy_(torch.from_numpy(p))
        Q = torch.from_numpy(q[:, :6]).to(DEV).to(dtype)
        args = [torch.from_numpy(x).to(DEV) for x in (tokens, parent, u, r)]
        a = rz.razor_verify_tree(P, Q, *args)
        b = rz.razor_verify_tree(P.contiguous(), torch.from_numpy(q).to(DEV).to(dtype), *args)
        for key in a:
            assert torch.equal(a[key], b[key])


# ----------------------------------------------------------------------------- together
def test_rounds_of_speculative_decoding():
    """The three calls as a serving loop makes them: tree attention over two layers, verification, the counts read back
    once, the path appended in both layers; eight rounds, states and outputs against the oracle every round."""
    w = synth.Workload("spec", 3, 2, 8, 4, 128, "bf16", [90, 300, 17], [40, 64, 8], 4, 1, 80, 99)
    cache = make_cache(w, max_new=80)
    refs, V, T = [], 64, 10
    for layer in range(2):
        K, Vd = synth.make_dense_kv(w, layer, DEV)
        cache.compress(layer, K, Vd, w.ctx_len, w.retrieval(layer), w.window)
        refs.append({(b, g): HeadRef(layer, b, g, K[b, g], Vd[b, g], w.ctx_len[b], 80) for b in range(3) for g in range(4)})
    rng = np.random.default_rng(0)
    moved = 0
    for rnd in range(8):
        parent, p, q, tokens, u, r = _verify_case(rng, 3, T, V, rnd % 2 == 0, sharp=1.5)
        pd = torch.from_numpy(parent).to(DEV)
        drafts = [_drafts(w, T, 200 + 2 * rnd + layer, fused=layer == 1) for layer in range(2)]
        outs = [cache.decode_tree(layer, *drafts[layer], pd) for layer in range(2)]
        res = rz.razor_verify_tree(torch.from_numpy(p).float().to(DEV), None if q is None else torch.from_numpy(q).float().to(DEV),
                                   torch.from_numpy(tokens).to(DEV), pd, torch.from_numpy(u).to(DEV), torch.from_numpy(r).to(DEV))
        counts = res["accepted"].cpu().tolist()
        for layer in range(2):
            cache.append_tree(layer, drafts[layer][1], drafts[layer][2], res["path"], counts)
        for layer in range(2):
            qh, kh, vh = (to_f64(x) for x in drafts[layer])
            out, retr = to_f64(outs[layer]), w.retrieval(layer)
            kb, vb = drafts[layer][1].cpu(), drafts[layer][2].cpu()
            for (b, g), ref in refs[layer].items():
                hc = orc.compress_head(ref.K[:ref.n], ref.V[:ref.n], ref.n, 4, w.window[b], bool(retr[g]))
                for j in range(2):
                    want = orc.tree_attention(qh[b, :, 2 * g + j], hc, kh[b, :, g], vh[b, :, g], parent[b].tolist(), 1 / math.sqrt(128))
                    assert np.abs(out[b, :, 2 * g + j] - want).max() <= TIGHT["bf16"]
                for n in res["path"][b, :counts[b]].tolist():
                    ref.append(kb[b, n, g], vb[b, n, g])
                check_head_state(cache, ref, 4, w.window[b], bool(retr[g]))
        moved += sum(counts)
    assert moved > 8 and cache.device_status() == 0
    cache.close()


@pytest.mark.parametrize("seed", range(4))
def test_tree_calls_among_the_others(seed):
    """Random sessions that mix the tree calls with single steps, long appends, rounds and decodes on one layer: each of
    them goes on from the state the one before has left."""
    rng = np.random.default_rng(400 + seed)
    group, D, cap = int(rng.choice([1, 4])), int(rng.choice([64, 128])), 260
    w = synth.Workload("mixed", 2, 1, 2 * group, 2, D, "bf16", [int(rng.integers(0, 400)), 90], [int(rng.integers(8, 120)), 30], 4, 1, cap, 800 + seed)
    cache, K, V = _compress(w, max_new=cap, shuffle=seed)
    refs, retr, scale = _refs(w, K, V, extra=cap), w.retrieval(0), 1 / math.sqrt(D)
    used = [0, 0]

    def appended(k, v, rows):
        kb, vb = k.cpu(), v.cpu()
        for (b, g), ref in refs.items():
            for n in rows[b]:
                ref.append(kb[b, n, g], vb[b, n, g])
        for b in range(2):
            used[b] += len(rows[b])

    def expect(q, out):
        qh, out = to_f64(q), to_f64(out)
        for (b, g), ref in refs.items():
            for j in range(group):
                want = orc.multi_query_attention(qh[b, :, g * group + j], ref.K[:ref.n], ref.V[:ref.n], 4, w.window[b], bool(retr[g]), scale)
                assert np.abs(out[b, :, g * group + j] - want).max() <= TOL_OUT["bf16"]

    for step in range(24):
        kind = rng.choice(["tree", "path", "step", "append", "round", "decode"])
        T = int(rng.integers(1, 30))
        q, k, v = _drafts(w, T, 1000 * seed + step)
        if kind == "tree":
            _check(w, cache, refs, q, k, v, _random_parents(rng, 2, T, holes=True))
        elif kind == "path":
            counts = [int(min(rng.integers(0, T + 1), cap - u)) for u in used]
            path = np.full((2, T), -1, dtype=np.int32)
            for b in range(2):
                path[b, :counts[b]] = np.sort(rng.permutation(T)[:counts[b]])
            cache.append_tree(0, k, v, torch.from_numpy(path).to(DEV), counts)
            appended(k, v, [path[b, :counts[b]].tolist() for b in range(2)])
        elif max(used) + T > cap:
            continue
        elif kind == "step":
            out = cache.decode_step(0, k[:, 0].contiguous(), v[:, 0].contiguous(), q[:, 0].contiguous())
            appended(k, v, [[0], [0]])
            expect(q[:, :1], out[:, None])
        elif kind == "append":
            cache.append_many(0, k, v)
            appended(k, v, [list(range(T))] * 2)
        elif kind == "round":
            T = min(T, 8)                          # (no window is shorter)
            q, k, v = (x[:, :T].contiguous() for x in (q, k, v))
            cache.append_many(0, k, v)
            appended(k, v, [list(range(T))] * 2)
            expect(q, cache.decode_multi(0, q))
        elif min(ref.n for ref in refs.values()) > 0:
            expect(q[:, :1], cache.decode(0, q[:, 0].contiguous())[:, None])
        for (b, g), ref in refs.items():
            check_head_state(cache, ref, 4, w.window[b], bool(retr[g]))
    assert cache.device_status() == 0
    cache.close()
