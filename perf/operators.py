"""The speculative-decoding operators, measured: attention for a tree of drafted tokens over the compressed cache,
verification of the drafts against the target's probabilities, and the append of an accepted path.

`run` computes the plain form (elementary torch operations) while `own` is false and makes the framework's calls while
it is true; `exact` computes the same from the definitions in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
ABSENT = -2          # parent of an unused node


# ----------------------------------------------------------------------------- the cases
def listed():
    def tree(name, **kw):
        base = dict(name=name, kind="tree", batch=1, q_heads=32, kv_heads=32, head_dim=128, ctx=4096, ragged=False,
                    window=1024, sinks=4, retrieval=2, nodes=8, padded=False, chain=False)
        base.update(kw)
        return base

    return [
        # one user's short conversation, five drafted tokens: latency is all that counts
        tree("tree_5_short", kv_heads=8, ctx=509, window=128, nodes=5),
        # a decode step through the same entry point: one node a sequence, small batch
        tree("tree_1_gqa_4k", kv_heads=8, batch=8, nodes=1),
        # eight drafted tokens over the 32K multi-head shape
        tree("tree_8_mha_32k", batch=8, ctx=32768, window=6553, retrieval=5, nodes=8),
        # a full tree of 64 over the same cache
        tree("tree_64_mha_32k", batch=8, ctx=32768, window=6553, retrieval=5, nodes=64),
        # a ragged serving batch of a grouped-query model, trees of different sizes
        tree("tree_26_gqa_ragged", kv_heads=8, batch=16, ctx=32768, ragged=True, window=4000, nodes=26, padded=True),
        # the long grouped-query context with a wide tree: 256 query rows per KV head
        tree("tree_64_gqa_128k", kv_heads=8, batch=2, ctx=131072, window=16384, nodes=64),
        # small heads, two queries each, an odd chain
        tree("tree_33_d64", q_heads=16, kv_heads=8, head_dim=64, batch=4, ctx=10007, ragged=True, window=2000, nodes=33,
             chain=True),
        # drafts looked up in the prompt (no draft probabilities), one user
        dict(name="verify_fixed_4", kind="verify", batch=1, nodes=4, vocab=32000, dtype="f32", chain=True, sampled=False),
        # a serving batch verifying chains of seven
        dict(name="verify_chain_7", kind="verify", batch=64, nodes=7, vocab=128256, dtype="f32", chain=True, sampled=True),
        # wide trees, probabilities kept in 16 bits
        dict(name="verify_tree_63", kind="verify", batch=16, nodes=63, vocab=128256, dtype="bf16", chain=False, sampled=True),
        # the first round of a fresh layer: a few accepted tokens committed, then a tree over them
        dict(name="round_small", kind="round", batch=4, q_heads=32, kv_heads=8, head_dim=128, window=64, sinks=4,
             retrieval=2, first=7, nodes=8),
        # a large batch whose committed tokens outgrow the window (rows are evicted and folded into the mean)
        dict(name="round_large", kind="round", batch=64, q_heads=32, kv_heads=8, head_dim=128, window=40, sinks=4,
             retrieval=2, first=128, nodes=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "verify", "verify", "round"])
    if kind == "verify":
        nodes, vocab = _log_int(rng, 1, 100), _log_int(rng, 1000, 160000)
        batch = max(1, min(_log_int(rng, 1, 64), 130_000_000 // ((nodes + 1) * vocab)))
        return dict(kind=kind, batch=batch, nodes=nodes, vocab=vocab, dtype=rng.choice(["f32", "bf16"]),
                    chain=rng.random() < 0.4, sampled=rng.random() < 0.7)
    kv, group = rng.choice([2, 4, 8, 10, 32, 40]), rng.choice([1, 2, 4, 8])
    head_dim = rng.choice([64, 128, 128])
    sinks = rng.choice([0, 1, 4, 4, 17])
    if kind == "round":
        return dict(kind=kind, batch=_log_int(rng, 1, 64), q_heads=kv * group, kv_heads=kv, head_dim=head_dim,
                    window=_log_int(rng, 1, 300), sinks=sinks, retrieval=rng.randint(0, 2),
                    first=_log_int(rng, 1, 128), nodes=_log_int(rng, 1, 64))
    ctx, nodes, retrieval = _log_int(rng, 1, 131072), _log_int(rng, 1, 128), rng.randint(0, 2)
    window = max(1, int(ctx * rng.uniform(0.05, 0.5)))
    # no more kept tokens, and no more query rows times tokens, than the largest listed cases have
    kept = min(retrieval, kv) * ctx + max(0, kv - retrieval) * min(ctx, sinks + window)
    batch = max(1, min(_log_int(rng, 1, 64), 2_600_000 // kept, 8 * 32 * 32768 // (ctx * kv)))
    nodes = max(1, min(nodes, 180_000_000 // (batch * kept * group)))
    return dict(kind=kind, batch=batch, q_heads=kv * group, kv_heads=kv, head_dim=head_dim, ctx=ctx,
                ragged=rng.random() < 0.5, window=window, sinks=sinks, retrieval=retrieval, nodes=nodes,
                padded=rng.random() < 0.4, chain=rng.random() < 0.3)


# ----------------------------------------------------------------------------- inputs
def _parents(host, batch, nodes, chain, padded):
    """[batch][nodes]: the node each drafted token follows, -1 for the sequence itself; unused nodes at the end."""
    rows = []
    for _ in range(batch):
        row = [t - 1 if chain else int(host.random() ** 1.5 * t * 0.8) - 1 for t in range(nodes)]
        used = host.randint(1, nodes) if padded else nodes
        rows.append(row[:used] + [ABSENT] * (nodes - used))
    return rows


def _retrieval(case, host):
    flags = [0] * case["kv_heads"]
    for g in host.sample(range(case["kv_heads"]), min(case["retrieval"], case["kv_heads"])):
        flags[g] = 1
    return flags


def _lengths(case, host):
    n = case["ctx"]
    return [host.randint(max(1, n // 4), n) for _ in range(case["batch"])] if case["ragged"] else [n] * case["batch"]


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.bfloat16)


def _tree_inputs(case, seed):
    """What both sides and `exact` start from: the whole context's K and V and one round of drafts."""
    host, gen = random.Random(seed), torch.Generator(DEV)
    gen.manual_seed(seed)
    B, H, D, T = case["batch"], case["kv_heads"], case["head_dim"], case["nodes"]
    x = dict(lens=_lengths(case, host), flags=_retrieval(case, host),
             parent=_parents(host, B, T, case["chain"], case["padded"]))
    x["K"], x["V"] = _randn(gen, B, H, case["ctx"], D), _randn(gen, B, H, case["ctx"], D)
    x["K"][:, :, :4] *= 4     # the first tokens of a context draw a large share of the attention
    x["q"] = _randn(gen, B, T, case["q_heads"], D)
    x["k"], x["v"] = _randn(gen, B, T, H, D), _randn(gen, B, T, H, D)
    return x


def _round_inputs(case, seed):
    host, gen = random.Random(seed), torch.Generator(DEV)
    gen.manual_seed(seed)
    B, H, D, T, F = case["batch"], case["kv_heads"], case["head_dim"], case["nodes"], case["first"]
    x = dict(flags=_retrieval(case, host), parent=_parents(host, B, T, False, False),
             counts=[host.randint(0, F) for _ in range(B)])
    # the accepted path of a sequence: ascending draft indices, unused entries -1
    x["path"] = [sorted(host.sample(range(F), n)) + [-1] * (F - n) for n in x["counts"]]
    x["k0"], x["v0"] = _randn(gen, B, F, H, D), _randn(gen, B, F, H, D)
    x["q"] = _randn(gen, B, T, case["q_heads"], D)
    x["k"], x["v"] = _randn(gen, B, T, H, D), _randn(gen, B, T, H, D)
    return x


def _verify_inputs(case, seed):
    host, gen = random.Random(seed), torch.Generator(DEV)
    gen.manual_seed(seed)
    B, T, V = case["batch"], case["nodes"], case["vocab"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    parent = torch.tensor(_parents(host, B, T, case["chain"], not case["chain"]), dtype=torch.int32)
    rank = torch.zeros(B, T, dtype=torch.int64)          # place of a node among its siblings
    for b in range(B):
        seen = {}
        for t in range(T):
            a = int(parent[b, t])
            rank[b, t] = seen.get(a, 0)
            seen[a] = int(rank[b, t]) + 1
    x = dict(parent=parent.to(DEV), q=None)
    x["p"] = torch.empty(B, T + 1, V, dtype=dtype, device=DEV)
    if case["sampled"]:
        x["q"] = torch.empty(B, T + 1, V, dtype=dtype, device=DEV)
    x["tokens"] = torch.zeros(B, T, dtype=torch.int32, device=DEV)
    k = min(V, int(rank.max()) + 1)
    rank = rank.clamp(max=k - 1).to(DEV)
    for b in range(B):
        target = 2.5 * torch.randn(T + 1, V, generator=gen, device=DEV)
        draft = target + 0.7 * torch.randn(T + 1, V, generator=gen, device=DEV)
        x["p"][b] = torch.softmax(target, -1).to(dtype)
        if case["sampled"]:                              # children drawn from q without replacement
            x["q"][b] = torch.softmax(draft, -1).to(dtype)
            draft = draft - torch.log(-torch.log(torch.rand(T + 1, V, generator=gen, device=DEV).clamp(1e-20, 1 - 1e-7)))
        best = draft.topk(k, dim=-1).indices             # otherwise the draft's most likely ones
        row = (x["parent"][b].long() + 1).clamp(min=0)
        x["tokens"][b] = best[row, rank[b]].to(torch.int32)
    x["u"] = torch.rand(B, T, generator=gen, device=DEV)
    x["r"] = torch.rand(B, generator=gen, device=DEV)
    return x


# ----------------------------------------------------------------------------- prepare
def _visible(parent, device):
    """bool [B, T, T]: node n is node t or one of its ancestors; all false for an unused node."""
    see = torch.zeros(len(parent), len(parent[0]), len(parent[0]), dtype=torch.bool)
    for b, row in enumerate(parent):
        for t, a in enumerate(row):
            if -1 <= a < t and (a < 0 or see[b, a, a]):
                if a >= 0:
                    see[b, t] = see[b, a]
                see[b, t, t] = True
    return see.to(device)


def prepare(case, seed):
    if case["kind"] == "verify":
        s = dict(case=case, **_verify_inputs(case, seed))
        if own:
            from paper_2407_15891_b200 import binding
            s["rz"] = binding
        return s
    x = _tree_inputs(case, seed) if case["kind"] == "tree" else _round_inputs(case, seed)
    s = dict(case=case, q=x["q"], k=x["k"], v=x["v"], flags=x["flags"],
             parent=torch.tensor(x["parent"], dtype=torch.int32, device=DEV))
    B, T, D, n_sink, W = case["batch"], case["nodes"], case["head_dim"], case["sinks"], case["window"]
    s["out"] = torch.zeros(B, T, case["q_heads"], D, dtype=torch.float32, device=DEV)
    lens = x["lens"] if case["kind"] == "tree" else [0] * B
    if case["kind"] == "round":
        s.update(k0=x["k0"], v0=x["v0"], counts=x["counts"],
                 path=torch.tensor(x["path"], dtype=torch.int32, device=DEV))
    if own:
        from paper_2407_15891_b200 import binding as rz
        new = 0 if case["kind"] == "tree" else case["first"]
        cfg = rz.make_config(B, 1, case["q_heads"], case["kv_heads"], D, "bf16", n_sink, max(lens), new)
        s["window"] = [W] * B
        s["cache"] = rz.RazorCache(cfg, lens, s["window"], np.array(x["flags"], dtype=np.uint8))
        if case["kind"] == "tree":
            s["cache"].compress(0, x["K"], x["V"], lens, x["flags"], s["window"])
        return s
    s["see"] = _visible(x["parent"], DEV)
    if case["kind"] == "round":
        return s
    # the compressed cache in plain tensors, one group for the heads that keep everything, one for the others
    n = torch.tensor(lens, device=DEV)[:, None]
    s["groups"] = []
    for flag in (1, 0):
        heads = [g for g, f in enumerate(x["flags"]) if f == flag]
        if not heads:
            continue
        K, V = x["K"][:, heads], x["V"][:, heads]
        pos = torch.arange(case["ctx"], device=DEV)[None]
        keep = pos < n
        if not flag:
            kept = keep & ((pos < n_sink) | (pos >= n - W))
            gone = keep & ~kept
            cnt = gone.sum(1)
            # (a sequence at a time: the context in 32 bits need not fit beside its 16-bit form)
            mean = [torch.stack([(t[b].float() * gone[b][None, :, None]).sum(1, dtype=torch.float64)
                                 / cnt[b].clamp(min=1) for b in range(B)]).float() for t in (K, V)]
            order = torch.where(kept, pos, case["ctx"] + pos).argsort(1)[:, :min(case["ctx"], n_sink + W)]
            at = order[:, None, :, None].expand(-1, len(heads), -1, D)
            s["groups"].append((heads, K.gather(2, at), V.gather(2, at), kept.gather(1, order), mean, cnt))
        else:
            s["groups"].append((heads, K, V, keep, None, None))
    return s


# ----------------------------------------------------------------------------- run
def run(state):
    kind = state["case"]["kind"]
    if own:
        if kind == "verify":
            return state["rz"].razor_verify_tree(state["p"], state["q"], state["tokens"], state["parent"], state["u"],
                                                 state["r"])
        cache = state["cache"]
        if kind == "round":
            cache.start_empty(0, state["flags"], state["window"])
            cache.append_tree(0, state["k0"], state["v0"], state["path"], state["counts"])
        return cache.decode_tree(0, state["q"], state["k"], state["v"], state["parent"], out=state["out"])
    if kind == "verify":
        return _plain_verify(state)
    groups = state["groups"] if kind == "tree" else _plain_commit(state)
    for heads, K, V, keep, mean, cnt in groups:
        _plain_attention(state, heads, K, V, keep, mean, cnt)
    return state["out"]


def _plain_attention(state, heads, K, V, keep, mean, cnt):
    """Attention of the tree's nodes over kept tokens, compensation token and their own ancestors, for some KV heads."""
    case = state["case"]
    B, T, D, H = case["batch"], case["nodes"], case["head_dim"], case["kv_heads"]
    G, n = case["q_heads"] // H, K.shape[2]
    q = state["q"].float().view(B, T, H, G, D)[:, :, heads].permute(0, 2, 1, 3, 4).reshape(B, len(heads), T * G, D)
    k, v = (state[x].float()[:, :, heads].transpose(1, 2) for x in ("k", "v"))
    q = q / math.sqrt(D)
    old = (q @ K.float().transpose(2, 3)).masked_fill(~keep[:, None, None], -math.inf)
    see = state["see"].repeat_interleave(G, dim=1)                        # [B, T G, T]
    new = (q @ k.transpose(2, 3)).masked_fill(~see[:, None], -math.inf)
    top = new.amax(-1, keepdim=True)
    if n:
        top = torch.maximum(top, old.amax(-1, keepdim=True))
    if mean is not None:
        comp = (q @ mean[0][..., None]) + cnt.float().log()[:, None, None, None]
        top = torch.maximum(top, comp)
    top = top.clamp(min=-1e30)
    old, new = (old - top).exp(), (new - top).exp()
    num, den = old @ V.float() + new @ v, old.sum(-1, keepdim=True) + new.sum(-1, keepdim=True)
    if mean is not None:
        w = (comp - top).exp()
        num, den = num + w * mean[1][:, :, None], den + w
    out = (num / den).view(B, len(heads), T, G, D).permute(0, 2, 1, 3, 4)
    live = state["see"].any(-1)[:, :, None, None, None]
    at = state["out"].view(B, T, H, G, D)
    at[:, :, heads] = torch.where(live, out, at[:, :, heads])


def _plain_commit(state):
    """The cache that appending the accepted path to an empty layer leaves, in the form _plain_attention reads."""
    case = state["case"]
    B, F, D = case["batch"], case["first"], case["head_dim"]
    n = torch.tensor(state["counts"], device=DEV)[:, None]
    pos = torch.arange(F, device=DEV)[None]
    at = state["path"].long().clamp(min=0)[:, :, None, None].expand(-1, -1, case["kv_heads"], D)
    K, V = (state[x].gather(1, at).transpose(1, 2) for x in ("k0", "v0"))
    there = pos < n
    kept = there & ((pos < case["sinks"]) | (pos >= n - case["window"]))
    gone = there & ~kept
    cnt = gone.sum(1)
    groups = []
    for flag in (1, 0):
        heads = [g for g, f in enumerate(state["flags"]) if f == flag]
        if heads and flag:
            groups.append((heads, K[:, heads], V[:, heads], there, None, None))
        elif heads:
            mean = [(t[:, heads].float() * gone[:, None, :, None]).sum(2) / cnt.clamp(min=1)[:, None, None] for t in (K, V)]
            groups.append((heads, K[:, heads], V[:, heads], kept, mean, cnt))
    return groups


def _weight(x):
    """Probabilities in 64 bits; what is not a positive finite number counts as nothing."""
    x = x.double()
    return torch.where((x > 0) & (x < math.inf), x, 0.0)


def _plain_verify(state):
    """The walk down the tree for all sequences at once, one node at a time."""
    case, p, q, tokens, parent = (state[x] for x in ("case", "p", "q", "tokens", "parent"))
    B, T, V = case["batch"], case["nodes"], case["vocab"]
    every = torch.arange(B, device=p.device)
    cur = torch.full((B,), -1, device=p.device)
    taken, path = torch.zeros_like(cur), torch.full((B, T), -1, dtype=torch.int64, device=p.device)
    away = torch.zeros(B, V, dtype=torch.bool, device=p.device)           # rejected children of the current node
    one = torch.ones(B, dtype=torch.float64, device=p.device)
    minus, left, total = 0 * one, one, one                               # A, Z and S of the definition
    for t in range(T):
        x = tokens[:, t].long()
        here = (parent[:, t] == cur) & (x >= 0) & (x < V)
        x = x.clamp(0, V - 1)
        there = ~away[every, x]
        qx = _weight(q[every, cur + 1, x]) * there if q is not None else one
        w = (_weight(p[every, cur + 1, x]) - (minus * qx if q is not None else 0)).clamp(min=0) * there
        yes = here & (state["u"][:, t].double() * qx * total < w * left)
        no = here & ~yes
        away[every, x] |= no
        if q is not None:
            minus = torch.where(no, minus + torch.where(left > 0, total / left, 0.0), minus)
            left = torch.where(no, left - qx, left)
            rest = ((_weight(p[every, cur + 1]) - minus[:, None] * _weight(q[every, cur + 1])).clamp(min=0) * ~away).sum(1)
        else:
            rest = (total - w).clamp(min=0)
        total = torch.where(no, rest, total)
        cur = torch.where(yes, t, cur)
        path[every, taken.clamp(max=T - 1)] = torch.where(yes, t, path[every, taken.clamp(max=T - 1)])
        taken = taken + yes
        away &= ~yes[:, None]
        minus, left, total = (torch.where(yes, a, b) for a, b in ((0 * one, minus), (one, left), (one, total)))
    w = _weight(p[every, cur + 1])
    rest = (w - (minus[:, None] * _weight(q[every, cur + 1]) if q is not None else 0)).clamp(min=0) * ~away
    w = torch.where(rest.sum(1, keepdim=True) > 0, rest, w)
    upto = w.cumsum(1)
    over = (upto > state["r"].double()[:, None] * upto[:, -1:]) & (w > 0)
    last = V - 1 - (w > 0).flip(1).to(torch.uint8).argmax(1)
    token = torch.where(over.any(1), over.to(torch.uint8).argmax(1), last)
    token = torch.where((w > 0).any(1), token, -1)
    return dict(accepted=taken.to(torch.int32), path=path.to(torch.int32), token=token.to(torch.int32))


# ----------------------------------------------------------------------------- work
def work(case):
    if case["kind"] == "verify":
        esz = 2 if case["dtype"] == "bf16" else 4
        rows = 2 if case["sampled"] else 1               # the rows the last token is drawn from; the walk reads single values
        return dict(bytes=case["batch"] * (rows * case["vocab"] * esz + case["nodes"] * (12 + rows * esz)),
                    flops=4 * rows * case["batch"] * case["vocab"])
    B, H, D, T, G = case["batch"], case["kv_heads"], case["head_dim"], case["nodes"], case["q_heads"] // case["kv_heads"]
    draft = B * T * (2 * H * D * 2 + H * G * D * 6 + 4)  # K and V, queries in 16 bits, outputs in 32, parents
    whole = min(case["retrieval"], H)
    if case["kind"] == "tree":
        n = case["ctx"] * 0.625 if case["ragged"] else case["ctx"]      # ragged lengths: a quarter of it to all of it
        kept = whole * n + (H - whole) * min(n, case["sinks"] + case["window"])
        return dict(bytes=B * kept * 4 * D + draft, flops=B * T * G * (kept + H * T / 2) * 4 * D)
    n = case["first"] / 2
    kept = whole * n + (H - whole) * min(n, case["sinks"] + case["window"])
    return dict(bytes=B * (n * H + 2 * kept) * 4 * D + draft, flops=B * T * G * (kept + H * T / 2) * 4 * D)


# ----------------------------------------------------------------------------- exact
def exact(case, seed):
    return _exact_verify(case, seed) if case["kind"] == "verify" else _exact_attention(case, seed)


def _exact_attention(case, seed):
    B, H, T, D = case["batch"], case["kv_heads"], case["nodes"], case["head_dim"]
    G = case["q_heads"] // H
    x = _tree_inputs(case, seed) if case["kind"] == "tree" else _round_inputs(case, seed)
    out = torch.zeros(B, T, case["q_heads"], D, dtype=torch.float64, device=DEV)
    for b in range(B):
        lines = []                                       # every node with the nodes from the root down to it
        for t, a in enumerate(x["parent"][b]):
            lines.append(None if not -1 <= a < t or (a >= 0 and lines[a] is None) else (lines[a] if a >= 0 else []) + [t])
        hidden = torch.ones(T, T, dtype=torch.bool)
        for t, line in enumerate(lines):
            if line:
                hidden[t, line] = False
        alive = [t for t in range(T) if lines[t]]
        hidden = hidden[alive].to(DEV)
        if not alive:
            continue
        for g in range(H):
            if case["kind"] == "tree":
                K, V = (x[c][b, g, :x["lens"][b]].double() for c in ("K", "V"))
            else:
                K, V = (x[c][b, x["path"][b][:x["counts"][b]], g].double() for c in ("k0", "v0"))
            n = K.shape[0]
            lo, hi = (n, n) if x["flags"][g] else (case["sinks"], n - case["window"])
            extra = torch.zeros(0, dtype=torch.float64, device=DEV)
            if lo < hi:                                  # positions lo .. hi - 1 are dropped: one mean with their count
                extra = torch.full((1,), math.log(hi - lo), dtype=torch.float64, device=DEV)
                K, V = (torch.cat([c[:lo], c[hi:], c[lo:hi].mean(0, keepdim=True)]) for c in (K, V))
            bias = torch.zeros(K.shape[0], dtype=torch.float64, device=DEV)
            if len(extra):
                bias[-1] = extra[0]
            K, V = torch.cat([K, x["k"][b, :, g].double()]), torch.cat([V, x["v"][b, :, g].double()])
            for j in range(G):
                s = x["q"][b, alive, g * G + j].double() @ K.T / math.sqrt(D)
                s[:, :len(bias)] += bias
                s[:, len(bias):][hidden] = -math.inf
                out[b, alive, g * G + j] = torch.softmax(s, -1) @ V
    return out


def _exact_verify(case, seed):
    B, T, V = case["batch"], case["nodes"], case["vocab"]
    x = _verify_inputs(case, seed)
    parent, tokens, u, r = (x[c].cpu().numpy() for c in ("parent", "tokens", "u", "r"))
    accepted, path, token = np.zeros(B, np.int32), np.full((B, T), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        at, line = -1, []
        while True:
            p = x["p"][b, at + 1].double().cpu().numpy()
            q = x["q"][b, at + 1].double().cpu().numpy() if case["sampled"] else None
            now, drawn, found = p.copy(), q, None
            gone = 0.0                                   # draft probability of the children that were rejected
            for t in [t for t in range(T) if parent[b, t] == at]:
                c = int(tokens[b, t])
                if q is None:
                    mass = 1.0 - p[[int(tokens[b, s]) for s in range(t) if parent[b, s] == at]].sum()
                    if float(u[b, t]) * mass < p[c]:
                        found = t
                        break
                    now[c] = 0.0
                else:
                    if float(u[b, t]) * drawn[c] < now[c]:
                        found = t
                        break
                    now = np.maximum(now - drawn, 0.0)
                    now[c] = 0.0
                    now /= max(now.sum(), 1e-300)
                    gone += q[c]
                    drawn = drawn * (1.0 - gone + q[c]) / (1.0 - gone)
                    drawn[c] = 0.0
            if found is None:
                break
            line.append(found)
            at = found
        w = now if now.sum() > 0 else p
        upto = np.cumsum(w)
        accepted[b], path[b, :len(line)] = len(line), line
        token[b] = int(np.argmax(upto > float(r[b]) * upto[-1]))
    return dict(accepted=accepted, path=path, token=token)
