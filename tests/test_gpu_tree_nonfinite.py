"""Tree attention with NaN and infinities that a node DOES see: its row shows them, whatever way the heads were cut between
CTAs, and no other row does.  `out` holds a mark before every call, so a row that is not written is noticed."""
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
MARK = 12345.0
LONG, SHORT = 6000, 100      # 53 units of 128 tokens and fixed cost: cut into eight spans; seven units: one span


def _setup(dtype, group, D, T, alibi, n_ctx, poison_cache=False):
    """One KV head, one sequence, T nodes: 0 <- 1 <- 3, 0 <- 2 <- 4, 5 absent with 6 under it, the others after node 4."""
    w = synth.Workload("nonfinite", 1, 1, group, 1, D, dtype, [n_ctx], [64], 4, 1, 0, 70 + T + D)
    cache = make_cache(w, use_comp=0 if alibi else 1)
    slopes = None
    if alibi:
        slopes = (2.0 ** -(1.0 + np.arange(group) * 8.0 / group)).astype(np.float32)
        rz.razor_cache_set_alibi(cache.handle, slopes)
    K, V = synth.make_dense_kv(w, 0, DEV)
    if poison_cache:
        K[0, 0, n_ctx - 1, 3] = float("nan")
    cache.compress(0, K, V, w.ctx_len, w.retrieval(0), w.window)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = synth.normal_bf16(w.seed, synth.TAG_Q, (1, T, group, D), DEV, sub=1).to(dt)
    k = synth.normal_bf16(w.seed, synth.TAG_KNEW, (1, T, 1, D), DEV, sub=1).to(dt)
    v = synth.normal_bf16(w.seed, synth.TAG_VNEW, (1, T, 1, D), DEV, sub=1).to(dt)
    parent = [-1, 0, 0, 1, 2, -2, 5] + [4] * (T - 7)
    return w, cache, K, V, q, k, v, parent, slopes


def _call(cache, q, k, v, parent):
    out = torch.full(q.shape, MARK, dtype=torch.float32, device=DEV)
    cache.decode_tree(0, q, k, v, torch.tensor([parent], dtype=torch.int32, device=DEV), out=out)
    assert cache.device_status() == 0
    return out[0]


KERNELS = [("bf16", 4, 128, 9, False),     # up to 64 rows of a KV head
           ("bf16", 1, 64, 64, False),
           ("bf16", 8, 128, 20, False),    # more: tiles of 128 rows
           ("bf16", 2, 64, 100, False),
           ("bf16", 2, 128, 9, True),      # ALiBi, 32 and 128 columns
           ("bf16", 8, 64, 20, True),
           ("f32", 2, 128, 9, False),
           ("f32", 4, 64, 12, True)]


@pytest.mark.parametrize("n_ctx", [LONG, SHORT])
@pytest.mark.parametrize("dtype,group,D,T,alibi", KERNELS)
def test_a_nan_reaches_every_row_that_sees_it(dtype, group, D, T, alibi, n_ctx):
    """A NaN in one query row (that row alone), in a draft's K (the node and its descendants) and in the last cached token's K
    (every row); the others keep every bit, absent nodes' rows the mark."""
    w, cache, K, V, q, k, v, parent, _ = _setup(dtype, group, D, T, alibi, n_ctx)
    lines = orc.tree_lines(parent)
    absent = [t for t in range(T) if lines[t] is None]
    clean = _call(cache, q, k, v, parent)
    assert (clean[absent] == MARK).all() and torch.isfinite(clean).all()

    def expect(out, poisoned):
        """poisoned: bool [T, group]."""
        for t in range(T):
            for j in range(group):
                if t in absent:
                    assert (out[t, j] == MARK).all(), (t, j)
                elif poisoned[t, j]:
                    assert torch.isnan(out[t, j]).all(), (t, j)
                else:
                    assert torch.equal(out[t, j], clean[t, j]), (t, j)

    for t, j in ((2, group - 1), (0, 0), (T - 1, 0)):
        q2 = q.clone()
        q2[0, t, j, 7] = float("nan")
        hit = np.zeros((T, group), dtype=bool)
        hit[t, j] = True
        expect(_call(cache, q2, k, v, parent), hit)
    q2 = q.clone()
    q2[0, absent] = float("nan")
    expect(_call(cache, q2, k, v, parent), np.zeros((T, group), dtype=bool))
    for node in (1, 4, T - 1):
        k2 = k.clone()
        k2[0, node, 0, 5] = float("nan")
        hit = np.zeros((T, group), dtype=bool)
        hit[[t for t in range(T) if lines[t] is not None and node in lines[t]]] = True
        expect(_call(cache, q, k2, v, parent), hit)
    cache.close()
    _, cache, *_ = _setup(dtype, group, D, T, alibi, n_ctx, poison_cache=True)
    expect(_call(cache, q, k, v, parent), np.ones((T, group), dtype=bool))
    cache.close()


@pytest.mark.parametrize("n_ctx", [LONG, SHORT])
@pytest.mark.parametrize("dtype,group,D,T,alibi", [KERNELS[0], KERNELS[2], KERNELS[4], KERNELS[7]])
def test_an_infinity_in_a_drafts_k(dtype, group, D, T, alibi, n_ctx):
    """A logit of plus infinity makes its row NaN (infinity over infinity), one of minus infinity is a weight of zero: which
    rows are which is the query's sign, and the finite ones are the oracle's.  Bar: the framework's own, 3e-3 and 1e-5."""
    w, cache, K, V, q, k, v, parent, slopes = _setup(dtype, group, D, T, alibi, n_ctx)
    k[0, 1, 0, 5] = float("inf")
    out = _call(cache, q, k, v, parent).double().cpu().numpy()
    ref = HeadRef(0, 0, 0, K[0, 0], V[0, 0], n_ctx, 0)
    hc = orc.compress_head(ref.K, ref.V, n_ctx, 4, 64, bool(w.retrieval(0)[0]))
    lines, seen = orc.tree_lines(parent), set()
    with np.errstate(invalid="ignore"):
        for j in range(group):
            want = orc.tree_attention(to_f64(q)[0, :, j], hc, to_f64(k)[0, :, 0], to_f64(v)[0, :, 0], parent, 1 / math.sqrt(D),
                                      not alibi, float(slopes[j]) if alibi else 0.0)
            for t in range(T):
                if lines[t] is None:
                    assert (out[t, j] == MARK).all()
                elif np.isnan(want[t]).any():
                    assert np.isnan(out[t, j]).all(), (t, j)
                    seen.add("nan")
                else:
                    assert np.abs(out[t, j] - want[t]).max() <= TOL_OUT[dtype], (t, j)
                    seen.add("below" if 1 in lines[t] else "away")
    assert seen == {"nan", "below", "away"}
    cache.close()


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("n_ctx", [LONG, SHORT])
@pytest.mark.parametrize("dtype,group,D,T,alibi", KERNELS)
def test_a_cached_v_that_is_not_finite(dtype, group, D, T, alibi, n_ctx, bad):
    """Dimension 10 of the last cached token's V: that dimension of every live row is not finite - the infinity itself from fp32
    caches, which weigh a row once, possibly a NaN from bf16 ones, whose weights come in two parts of either sign - and every
    other dimension keeps its bits.  (The last token: the weight that ALiBi's penalty leaves it is not zero.)"""
    w, cache, K, V, q, k, v, parent, _ = _setup(dtype, group, D, T, alibi, n_ctx)
    live = [t for t, line in enumerate(orc.tree_lines(parent)) if line is not None]
    clean = _call(cache, q, k, v, parent)
    V[0, 0, n_ctx - 1, 10] = bad
    cache.compress(0, K, V, w.ctx_len, w.retrieval(0), w.window)
    out = _call(cache, q, k, v, parent)
    assert not torch.isfinite(out[live][..., 10]).any()
    if dtype == "f32" and not math.isnan(bad):
        assert (out[live][..., 10] == bad).all()
    rest = [d for d in range(D) if d != 10]
    assert torch.equal(out[..., rest], clean[..., rest])
    absent = [t for t in range(T) if t not in live]
    assert (out[absent] == MARK).all()
    cache.close()
