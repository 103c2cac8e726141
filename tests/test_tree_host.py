"""CPU tests of the speculative-decoding operators: the oracle's tree attention and verification pinned by special cases,
closed forms and the distribution they promise, and the library's refusals that need no device."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import razor_oracle as orc
from paper_2407_15891_b200 import binding as rz
from paper_2407_15891_b200 import build as rz_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    rz_build.build()


def _head(rng, n, D=8, n_sink=2, window=5, retr=False):
    K, V = rng.standard_normal((n, D)), rng.standard_normal((n, D))
    return K, V, orc.compress_head(K, V, n, n_sink, window, retr)


# ----------------------------------------------------------------------------- oracle pins
def test_tree_lines():
    assert orc.tree_lines([-1, 0, 0, 1, -1, 4]) == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5]]
    assert orc.tree_lines([-2, 0, -1, 3, 7, 2]) == [None, None, [2], None, None, [2, 5]]


@pytest.mark.parametrize("retr", [True, False])
def test_a_chain_over_a_cache_that_dropped_nothing_is_causal_attention(retr):
    rng = np.random.default_rng(1)
    n, T, D = 6, 5, 8
    K, V = rng.standard_normal((n + T, D)), rng.standard_normal((n + T, D))
    q = rng.standard_normal((T, D))
    hc = orc.compress_head(K, V, n, 4, 100, retr)
    got = orc.tree_attention(q, hc, K[n:], V[n:], [-1, 0, 1, 2, 3], 0.4)
    want = orc.multi_query_attention(q, K, V, 4, 100, retr, 0.4)
    assert np.abs(got - want).max() < 1e-12


def test_every_line_of_a_tree_is_a_chain_of_its_own():
    rng = np.random.default_rng(2)
    K, V, hc = _head(rng, 30)
    parent = [-1, 0, 0, 2, -1, 4, 2]
    q, k, v = (rng.standard_normal((7, 8)) for _ in range(3))
    got = orc.tree_attention(q, hc, k, v, parent, 0.3)
    for t, line in enumerate(orc.tree_lines(parent)):
        alone = orc.tree_attention(q[line], hc, k[line], v[line], list(range(-1, len(line) - 1)), 0.3)
        assert np.abs(got[t] - alone[-1]).max() < 1e-12
    # and the compensation token counts as N_d copies of the mean
    K2 = np.concatenate([hc.K, np.repeat(hc.k_hat[None], hc.n_drop, 0), k[:1]])
    V2 = np.concatenate([hc.V, np.repeat(hc.v_hat[None], hc.n_drop, 0), v[:1]])
    assert np.abs(got[0] - orc.full_attention(q[0], K2, V2, 0.3)).max() < 1e-12


def test_an_empty_cache_and_absent_nodes():
    rng = np.random.default_rng(3)
    hc = orc.compress_head(np.zeros((0, 8)), np.zeros((0, 8)), 0, 2, 5, False)
    q, k, v = (rng.standard_normal((3, 8)) for _ in range(3))
    got = orc.tree_attention(q, hc, k, v, [-1, 5, 0], 0.3)
    assert np.abs(got[0] - v[0]).max() < 1e-15 and np.isnan(got[1]).all() and np.isfinite(got[2]).all()


def test_alibi_penalty_counts_depth_not_index():
    rng = np.random.default_rng(4)
    K, V = rng.standard_normal((9, 8)), rng.standard_normal((9, 8))
    hc = orc.compress_head(K, V, 9, 0, 4, False)
    q, k, v = (rng.standard_normal((3, 8)) for _ in range(3))
    got = orc.tree_attention(q, hc, k, v, [-1, -1, 1], 0.3, slope=0.25)
    want = orc.alibi_attention(q[2], np.concatenate([K[5:], k[1:]]), np.concatenate([V[5:], v[1:]]),
                               np.array([5, 6, 7, 8, 9, 10]), 10, 0.25, 0.3)
    assert np.abs(got[2] - want).max() < 1e-12


def _rows(rng, n, V):
    x = rng.random((n, V)) ** 2 + 1e-3
    return x / x.sum(1, keepdims=True)


def _draw_children(rng, q, count):
    """Distinct tokens drawn from q one after the other."""
    q, got = q.copy(), []
    for _ in range(count):
        x = int(rng.choice(len(q), p=q / q.sum()))
        got.append(x)
        q[x] = 0
    return got


@pytest.mark.parametrize("children,sampled", [(1, True), (3, True), (2, False), (5, False)])
def test_the_kept_tokens_are_distributed_as_the_target_says(children, sampled):
    """The promise of verification: the first token kept (an accepted child of the root, or the drawn one) follows the
    target's row.  20000 runs over six tokens: a frequency is off by more than 5 sigma = 5 sqrt(1/4 / 20000) = 0.018
    with probability below 1e-6."""
    rng = np.random.default_rng(children + 10 * sampled)
    V, N = 6, 20000
    p, q = _rows(rng, 1 + children, V), _rows(rng, 1 + children, V)
    count = np.zeros(V)
    fixed = list(np.argsort(-q[0])[:children])
    for _ in range(N):
        tokens = _draw_children(rng, q[0], children) if sampled else fixed
        path, nxt = orc.verify_tree(p, q if sampled else None, tokens, [-1] * children, rng.random(children), rng.random())
        count[tokens[path[0]] if path else nxt] += 1
    assert np.abs(count / N - p[0]).max() < 0.018


def test_verification_in_closed_form():
    p = np.array([[0.5, 0.3, 0.2], [0.1, 0.6, 0.3], [0.2, 0.2, 0.6]])
    q = np.array([[0.25, 0.5, 0.25], [0.3, 0.3, 0.4], [0, 0, 0]])
    # accepted where q <= p whatever u is; u q < p decides otherwise: 0.5 u < 0.3
    assert orc.verify_tree(p, q, [0], [-1], [0.999], 0.0)[0] == [0]
    assert orc.verify_tree(p, q, [1], [-1], [0.59], 0.0)[0] == [0]
    path, tok = orc.verify_tree(p, q, [1], [-1], [0.61], 0.99)
    assert (path, tok) == ([], 0)                     # what is left of p is (0.25, 0, 0): token 0 whatever r is
    # a chain kept whole: the token comes from the last node's row
    path, tok = orc.verify_tree(p, q, [0, 1], [-1, 0], [0.1, 0.1], 0.41)
    assert path == [0, 1] and tok == 2
    # identical rows: always kept
    assert orc.verify_tree(p, p, [2, 0], [-1, 0], [0.999999, 0.999999], 0.5)[0] == [0, 1]
    # without draft probabilities: kept with the target's own probability
    assert orc.verify_tree(p, None, [1], [-1], [0.29], 0.0)[0] == [0]
    assert orc.verify_tree(p, None, [1], [-1], [0.31], 0.0) == ([], 0)
    # the second of two: u times what is left (0.7) against 0.2
    assert orc.verify_tree(p, None, [1, 2], [-1, -1], [0.31, 0.28], 0.0)[0] == [1]
    assert orc.verify_tree(p, None, [1, 2], [-1, -1], [0.31, 0.29], 0.99) == ([], 0)


def test_verification_corners():
    p = np.array([[0.0, np.nan, -1.0, 0.0], [0.25] * 4, [0.25] * 4])
    assert orc.verify_tree(p, None, [0], [-1], [0.0], 0.5) == ([], -1)        # no weight at all
    p[0] = [0.0, 0.0, 1.0, np.inf]
    assert orc.verify_tree(p, None, [3], [-1], [0.0], 0.5) == ([], 2)
    assert orc.verify_tree(p, None, [9, 2], [-1, -1], [0.0, 0.5], 0.5)[0] == [1]   # a token outside the vocabulary
    assert orc.verify_tree(p, None, [2], [0], [0.0], 0.5)[0] == []                 # a node that is its own parent
    # p nowhere above the draft and the child rejected (rows that do not sum to one): the target's own row is used
    p, q = np.array([[0.1, 0.2]] * 2), np.array([[0.5, 0.5]] * 2)
    assert orc.verify_tree(p, q, [0], [-1], [0.9], 0.0) == ([], 0)


# ----------------------------------------------------------------------------- refusals without a device
def test_cache_calls_refuse_a_null_handle():
    lib = rz.load()
    assert lib.razor_decode_attention_tree(None, 0, 256, 0, 0, 256, 256, 0, 0, 256, 1, 256, None) == -2
    assert lib.razor_append_tree(None, 0, 256, 256, 0, 0, None, 1, 256, None) == -2


def test_verify_tree_refusals():
    """Every refusal comes before anything is launched; the addresses are never read."""
    good = dict(target=256, tsb=3000, tsr=1000, draft=256, dsb=3000, dsr=1000, dtype=0, tokens=256, parent=256, u=256,
                r=256, batch=2, n=2, vocab=1000, acc=256, path=256, tok=256)

    def call(**kw):
        a = dict(good, **kw)
        return rz.load().razor_verify_tree(a["target"], a["tsb"], a["tsr"], a["draft"], a["dsb"], a["dsr"], a["dtype"],
                                           a["tokens"], a["parent"], a["u"], a["r"], a["batch"], a["n"], a["vocab"],
                                           a["acc"], a["path"], a["tok"], None)

    for name in ("target", "tokens", "parent", "u", "r", "acc", "path", "tok"):
        assert call(**{name: None}) == -2, name
    for kw in (dict(batch=0), dict(batch=(1 << 20) + 1), dict(n=0), dict(n=rz.TREE_MAX_NODES + 1), dict(vocab=0),
               dict(vocab=1001), dict(tsr=999), dict(dsr=999), dict(tsb=-1), dict(dsb=-1), dict(vocab=-5)):
        assert call(**kw) == -1, kw
    for dtype in (-1, 2, 7):
        assert call(dtype=dtype) == -3
    for kw in (dict(target=258), dict(draft=257, dtype=1), dict(tokens=257), dict(parent=258), dict(u=254), dict(r=255),
               dict(acc=257), dict(path=258), dict(tok=254)):
        assert call(**kw) == -8, kw


def test_the_binding_checks_shapes_before_the_call():
    B, T, V = 2, 3, 11
    p = torch.zeros(B, T + 1, V)
    ok = dict(target=p, draft=None, tokens=torch.zeros(B, T, dtype=torch.int32), parent=torch.zeros(B, T, dtype=torch.int32),
              u_accept=torch.zeros(B, T), u_sample=torch.zeros(B))
    for kw in (dict(target=p[:, :T]), dict(target=p.transpose(1, 2).contiguous().transpose(1, 2)),
               dict(draft=p.to(torch.bfloat16)), dict(draft=p[:, :, :V - 1]), dict(tokens=ok["tokens"].long()),
               dict(parent=ok["parent"][:, :2]), dict(u_accept=ok["u_accept"].double()), dict(u_sample=torch.zeros(B, 1))):
        with pytest.raises(AssertionError):
            rz.razor_verify_tree(**dict(ok, **kw))
    with pytest.raises(KeyError):
        rz.razor_verify_tree(**dict(ok, target=p.to(torch.float16)))


def test_the_node_limit_is_the_headers():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "razor.h")).read()
    assert int(re.search(r"#define RAZOR_TREE_MAX_NODES (\d+)", text).group(1)) == rz.TREE_MAX_NODES
