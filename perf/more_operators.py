"""Operators around the compressed cache, measured: rotary positions of queries and keys, attention of prompt tokens over
dense K and V with a sliding window and sink tokens per KV head, and the cache held in 8 bits (written, attended to, read back).

`run` computes the plain form (elementary torch operations) while `own` is false and makes the framework's calls while
it is true; `exact` computes the same from the definitions in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"


# ----------------------------------------------------------------------------- the cases
def listed():
    def rope(name, **kw):
        base = dict(name=name, kind="rope", batch=1, tokens=1, q_heads=32, kv_heads=8, head_dim=128, rotated=128,
                    dtype="bf16", interleaved=False, inverse=False, scaling="none", first=0, spread=1)
        base.update(kw)
        return base

    def window(name, **kw):
        base = dict(name=name, kind="window", batch=1, q_heads=32, kv_heads=8, head_dim=128, ctx=4096, tokens=4096,
                    ragged=False, window=1024, sinks=4, retrieval=2)
        base.update(kw)
        return base

    def cache(name, kind, **kw):
        base = dict(name=name, kind=kind, batch=1, q_heads=32, kv_heads=8, head_dim=128, ctx=4096, ragged=False,
                    window=1024, sinks=4, retrieval=2)
        base.update(kw)
        return base

    return [
        # one decode step of a small batch: latency is all that counts
        rope("rope_decode_8", batch=8, first=30000, spread=5000),
        # a long prompt's chunk at far positions, frequencies stretched for long contexts
        rope("rope_prompt_8k", tokens=8192, scaling="yarn", first=120000),
        # the other pairing, half of the head rotated, 32 bits, backwards (cached keys moved to other positions)
        rope("rope_back_fp32", batch=4, tokens=2001, q_heads=40, kv_heads=40, rotated=64, dtype="f32", interleaved=True,
             inverse=True, scaling="linear", first=1, spread=700000),
        # one token a sequence over dense K and V that are not compressed yet
        window("window_1_token", batch=4, ctx=32768, tokens=1, ragged=True, window=6553),
        # a chunk of a ragged batch, small heads, two queries each
        window("window_chunk_d64", q_heads=16, head_dim=64, batch=6, ctx=9001, tokens=333, ragged=True, window=2000,
               retrieval=1),
        # a prompt of the 64K-context model's shape: most heads see a window, a few everything
        window("window_prompt_16k", q_heads=40, kv_heads=40, ctx=16384, tokens=16384, window=4000, retrieval=6),
        # a long grouped-query prompt where every head sees everything
        window("window_full_32k", ctx=32768, tokens=32768, retrieval=8),
        # one user's short conversation over an 8-bit cache
        cache("cache8_decode_short", "decode8", ctx=509, window=128),
        # the 64K multi-head layer in 8 bits
        cache("cache8_decode_64k", "decode8", batch=4, q_heads=40, kv_heads=40, ctx=65536, window=13107, retrieval=6),
        # a ragged batch of a grouped-query model
        cache("cache8_decode_gqa", "decode8", batch=16, ctx=131072, ragged=True, window=16384, retrieval=1),
        # the end of a prompt: K and V quantised into the cache, then the first decode step
        cache("cache8_fill_32k", "fill8", batch=2, q_heads=32, kv_heads=32, ctx=32768, window=6553, retrieval=5),
        # a long head read back (a snapshot, or a move to another device)
        cache("cache8_read_128k", "read8", batch=2, ctx=131072, window=16384, retrieval=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "window", "window", "window", "decode8", "decode8", "fill8", "read8"])
    kv, group = rng.choice([2, 4, 8, 10, 32, 40]), rng.choice([1, 2, 4, 8])
    head_dim = rng.choice([64, 128, 128])
    if kind == "rope":
        tokens = _log_int(rng, 1, 16384)
        batch = max(1, min(_log_int(rng, 1, 64), 16384 // (tokens * max(1, kv * group // 32))))
        first = _log_int(rng, 1, 1_000_000)
        return dict(kind=kind, batch=batch, tokens=tokens, q_heads=kv * group, kv_heads=kv, head_dim=head_dim,
                    rotated=rng.choice([head_dim, head_dim, head_dim // 2, 32, head_dim // 4 + 6]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), interleaved=rng.random() < 0.4,
                    inverse=rng.random() < 0.3, scaling=rng.choice(["none", "linear", "ntk", "yarn", "banded"]),
                    first=first, spread=rng.choice([1, 1, 10000]))
    sinks, retrieval = rng.choice([0, 1, 4, 4, 17, 200]), rng.randint(0, 2)
    ctx = _log_int(rng, 1, 32768 if kind == "window" else 131072)
    width = max(1, int(ctx * rng.uniform(0.02, 0.5)))
    base = dict(kind=kind, q_heads=kv * group, kv_heads=kv, head_dim=head_dim, ctx=ctx, ragged=rng.random() < 0.5,
                window=width, sinks=sinks, retrieval=retrieval)
    if kind == "window":
        tokens = ctx if rng.random() < 0.5 else _log_int(rng, 1, ctx)
        # no more scores (the plain form computes all of them) and no more K and V rows than the largest listed cases have
        while kv > 2 and kv * group * tokens * ctx > 32 * 32768 * 32768:
            kv //= 2
        base.update(q_heads=kv * group, kv_heads=kv)
        batch = max(1, min(_log_int(rng, 1, 16), 32 * 32768 * 32768 // (kv * group * tokens * ctx), 8 * 32768 * 8 // (kv * ctx)))
        return dict(base, batch=batch, tokens=tokens)
    if kind == "read8":
        return dict(base, batch=1)
    most = 4 * 40 * 65536 if kind == "decode8" else 2 * 32 * 32768
    while kv > 2 and kv * ctx > most:
        kv //= 2
    base.update(q_heads=kv * group, kv_heads=kv)
    return dict(base, batch=max(1, min(_log_int(rng, 1, 64), most // (kv * ctx))))


# ----------------------------------------------------------------------------- inputs
def _frequencies(case):
    """Angle per position of every rotated pair, in 64 bits, and the factor on the rotated values."""
    R, kind = case["rotated"], case["scaling"]
    i, base, length, factor = np.arange(R // 2, dtype=np.float64), 10000.0, 8192.0, 4.0
    if kind == "ntk":                                    # a larger base instead of smaller positions
        base *= factor ** (R / (R - 2))
    w = base ** (-2.0 * i / R)
    if kind == "linear":
        return w / factor, 1.0
    if kind == "yarn":                                   # pairs that turn slowly are stretched, fast ones are not
        at = [R * math.log(length / (2 * math.pi * turns)) / (2 * math.log(base)) for turns in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), R - 1)
        ramp = np.clip((i - lo) / max(hi - lo, 0.001), 0, 1)
        return w / factor * ramp + w * (1 - ramp), 0.1 * math.log(factor) + 1
    if kind == "banded":                                 # the same by wavelength
        turns = length * w / (2 * math.pi)
        smooth = np.clip((turns - 1.0) / (4.0 - 1.0), 0, 1)
        return (1 - smooth) * w / factor + smooth * w, 1.0
    return w, 1.0


def _rope_inputs(case, seed):
    host, gen = random.Random(seed), torch.Generator(DEV)
    gen.manual_seed(seed)
    B, T, D = case["batch"], case["tokens"], case["head_dim"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    # one fused projection: queries and keys are column ranges of it
    rows = torch.randn(B, T, case["q_heads"] + 2 * case["kv_heads"], D, generator=gen, device=DEV, dtype=dtype)
    start = torch.tensor([case["first"] + host.randrange(case["spread"]) for _ in range(B)])
    positions = (start[:, None] + torch.arange(T)[None]).to(device=DEV, dtype=torch.int32)
    return rows, positions


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


def _window_inputs(case, seed):
    host, gen = random.Random(seed), torch.Generator(DEV)
    gen.manual_seed(seed)
    B, H, D = case["batch"], case["kv_heads"], case["head_dim"]
    lens, flags = _lengths(case, host), _retrieval(case, host)
    news = [min(n, host.randint(1, case["tokens"]) if case["ragged"] else case["tokens"]) for n in lens]
    K, V = _randn(gen, B, H, case["ctx"], D), _randn(gen, B, H, case["ctx"], D)
    K[:, :, :4] *= 4          # the first tokens of a context draw a large share of the attention
    return dict(lens=lens, news=news, flags=flags, K=K, V=V, q=_randn(gen, B, case["tokens"], case["q_heads"], D))


def _cache_inputs(case, seed):
    host, gen = random.Random(seed), torch.Generator(DEV)
    gen.manual_seed(seed)
    B, H, D = case["batch"], case["kv_heads"], case["head_dim"]
    x = dict(lens=_lengths(case, host), flags=_retrieval(case, host))
    x["K"], x["V"] = _randn(gen, B, H, case["ctx"], D), _randn(gen, B, H, case["ctx"], D)
    x["K"][:, :, :4] *= 4
    x["K"][..., 5] *= 6       # a channel that stands out, as keys have them
    x["q"] = _randn(gen, B, case["q_heads"], D)
    x["at"] = (host.randrange(B), x["flags"].index(1) if 1 in x["flags"] else host.randrange(H))
    return x


# ----------------------------------------------------------------------------- prepare
def prepare(case, seed):
    kind = case["kind"]
    if own:
        from paper_2407_15891_b200 import binding as rz
    if kind == "rope":
        rows, positions = _rope_inputs(case, seed)
        Hq, Hk = case["q_heads"], case["kv_heads"]
        s = dict(case=case, q=rows[:, :, :Hq], k=rows[:, :, Hq:Hq + Hk], positions=positions)
        s["q_out"], s["k_out"] = (torch.empty(x.shape, dtype=x.dtype, device=DEV) for x in (s["q"], s["k"]))
        if own:
            s["rz"] = rz
            s["w"], s["gain"] = rz.razor_rope_frequencies(case["rotated"], 10000.0, case["scaling"], 4.0, 8192)
        else:
            w, s["gain"] = _frequencies(case)
            s["w"] = torch.from_numpy(w).to(DEV)
        return s
    if kind == "window":
        x = _window_inputs(case, seed)
        s = dict(case=case, q=x["q"], K=x["K"], V=x["V"], out=torch.zeros_like(x["q"]))
        width = [[-1 if f else case["window"] for f in x["flags"]]] * case["batch"]
        s["ctx"], s["new"], s["width"] = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in (x["lens"], x["news"], width))
        if own:
            s["rz"] = rz
        return s
    x = _cache_inputs(case, seed)
    s = dict(case=case, q=x["q"], at=x["at"], flags=x["flags"], lens=x["lens"], windows=[case["window"]] * case["batch"])
    if own:
        cfg = rz.make_config(case["batch"], 1, case["q_heads"], case["kv_heads"], case["head_dim"], "i8", case["sinks"],
                             max(x["lens"]), 0)
        s["cache"] = rz.RazorCache(cfg, x["lens"], s["windows"], np.array(x["flags"], dtype=np.uint8))
        s["out"] = torch.empty(x["q"].shape, dtype=torch.float32, device=DEV)
        if kind != "fill8":
            s["cache"].compress(0, x["K"], x["V"], x["lens"], x["flags"], s["windows"])
    else:
        s["n"] = torch.tensor(x["lens"], device=DEV)[:, None]
        if kind != "fill8":
            s["groups"] = _plain_compress(case, x["K"], x["V"], s["n"], x["flags"])
    if kind == "fill8":
        s["K"], s["V"] = x["K"], x["V"]
    return s


# ----------------------------------------------------------------------------- run
def run(state):
    case = state["case"]
    kind = case["kind"]
    if own:
        if kind == "rope":
            state["rz"].razor_rope(state["q"], state["k"], state["w"], state["positions"], interleaved=case["interleaved"],
                                   inverse=case["inverse"], gain=state["gain"], q_out=state["q_out"], k_out=state["k_out"])
            return dict(q=state["q_out"], k=state["k_out"])
        if kind == "window":
            return state["rz"].razor_window_attention(state["q"], state["K"], state["V"], case["sinks"], state["width"],
                                                      state["new"], state["ctx"], out=state["out"])
        cache = state["cache"]
        if kind == "read8":
            got = cache.export(0, *state["at"])
            return {c: got[c] for c in ("kept_pos", "K", "V", "mean_k", "mean_v")}
        if kind == "fill8":
            cache.compress(0, state["K"], state["V"], state["lens"], state["flags"], state["windows"])
        return cache.decode(0, state["q"], out=state["out"])
    if kind == "rope":
        return _plain_rope(state)
    if kind == "window":
        return _plain_window(state)
    if kind == "read8":
        return _plain_read(state)
    groups = state["groups"] if kind == "decode8" else _plain_compress(case, state["K"], state["V"], state["n"], state["flags"])
    return _plain_decode(case, state["q"], groups)


def _plain_rope(state):
    case = state["case"]
    angle = state["positions"].double()[..., None] * state["w"]
    cos, sin = (t.float()[:, :, None] * state["gain"] for t in (angle.cos(), angle.sin()))
    if case["inverse"]:
        sin = -sin
    R = case["rotated"]
    a, b = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
    for x, y in ((state["q"], state["q_out"]), (state["k"], state["k_out"])):
        u, v = x[..., a].float(), x[..., b].float()
        y[..., a] = (u * cos - v * sin).to(y.dtype)
        y[..., b] = (v * cos + u * sin).to(y.dtype)
        y[..., R:] = x[..., R:]
    return dict(q=state["q_out"], k=state["k_out"])


def _plain_window(state):
    """All scores of as many (sequence, KV head) pairs and queries at once as 8 GB hold."""
    case, q, K, V, out = (state[x] for x in ("case", "q", "K", "V", "out"))
    B, T, Hq, D = q.shape
    H, N = K.shape[1], K.shape[2]
    G = Hq // H
    rows = max(1, min(T, (1 << 31) // (G * N)))
    pairs = max(1, (1 << 31) // (G * N * rows))
    q = q.view(B, T, H, G, D).permute(0, 2, 1, 3, 4).flatten(0, 1)                      # [B H, T, G, D]
    to = out.view(B, T, H, G, D).permute(0, 2, 1, 3, 4)
    K, V, n = K.flatten(0, 1), V.flatten(0, 1), torch.arange(N, device=DEV)
    width = state["width"].flatten()
    ctx, new = (state[x].long().repeat_interleave(H) for x in ("ctx", "new"))
    for p0 in range(0, B * H, pairs):
        p = slice(p0, p0 + pairs)
        at = torch.arange(p0, min(p0 + pairs, B * H), device=DEV)
        k, v = K[p].float(), V[p].float()
        for t0 in range(0, T, rows):
            t = torch.arange(t0, min(t0 + rows, T), device=DEV)
            m = (ctx[p] - new[p])[:, None, None] + t[None, :, None]                     # positions of the queries
            w = width[p][:, None, None]
            see = (n <= m) & ((n < case["sinks"]) | (w < 0) | (m - n < w))
            x = q[p, t0:t0 + rows].float() / math.sqrt(D)
            s = (x.flatten(1, 2) @ k.transpose(1, 2)).view(len(at), len(t), G, N)
            s.masked_fill_(~see[:, :, None], -math.inf)
            s = s.sub_(s.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
            total = s.sum(-1, keepdim=True)
            o = (s.flatten(1, 2) @ v).view(len(at), len(t), G, D) / total.clamp(min=1e-30)
            live = (t < new[p][:, None])[:, :, None, None]
            b, h = at // H, at % H
            old = to[b, h, t0:t0 + rows]
            to[b, h, t0:t0 + rows] = torch.where(live, o.to(out.dtype), old)
    return out


def _quantise(x):
    """8-bit codes of rows and their scales: the largest magnitude of a row is code 127."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    codes = (x * (torch.full_like(top, 127) / top)).round().to(torch.int8)
    return codes, top / torch.full_like(top, 127)


def _plain_compress(case, K, V, n, flags):
    """The compressed cache in plain tensors, one group for the heads that keep everything, one for the others."""
    N, W, D, sinks = case["ctx"], case["window"], case["head_dim"], case["sinks"]
    pos = torch.arange(N, device=DEV)[None]
    there = pos < n
    groups = []
    for flag in (1, 0):
        heads = [g for g, f in enumerate(flags) if f == flag]
        if not heads:
            continue
        k, v = K[:, heads], V[:, heads]
        if flag:
            groups.append((heads, _quantise(k), _quantise(v), there, pos.expand_as(there), None, None))
            continue
        kept = there & ((pos < sinks) | (pos >= n - W))
        gone = (there & ~kept).float()
        cnt = gone.sum(1)
        mean = [torch.einsum("bn,bhnd->bhd", gone, t.float()) / cnt.clamp(min=1)[:, None, None] for t in (k, v)]
        order = torch.where(kept, pos, N + pos).argsort(1)[:, :min(N, sinks + W)]
        at = order[:, None, :, None].expand(-1, len(heads), -1, D)
        groups.append((heads, _quantise(k.gather(2, at)), _quantise(v.gather(2, at)), kept.gather(1, order), order, mean, cnt))
    return groups


def _plain_decode(case, q, groups):
    B, Hq, D = q.shape
    G = Hq // case["kv_heads"]
    q = q.float().view(B, -1, G, D) / math.sqrt(D)
    out = torch.empty(B, case["kv_heads"], G, D, device=DEV)
    for heads, (kc, ks), (vc, vs), keep, _, mean, cnt in groups:
        x = q[:, heads]
        s = (x @ (kc.float() * ks).transpose(2, 3)).masked_fill(~keep[:, None, None], -math.inf)
        top = s.amax(-1, keepdim=True)
        if mean is not None:
            c = (x @ mean[0][..., None]) + cnt.log()[:, None, None, None]
            top = torch.maximum(top, c)
        s = (s - top).exp()
        num, den = s @ (vc.float() * vs), s.sum(-1, keepdim=True)
        if mean is not None:
            c = (c - top).exp()
            num, den = num + c * mean[1][:, :, None], den + c
        out[:, heads] = num / den
    return out.view(B, Hq, D)


def _plain_read(state):
    b, h = state["at"]
    for heads, (kc, ks), (vc, vs), keep, order, mean, _ in state["groups"]:
        if h in heads:
            i, kept = heads.index(h), keep[b]
            none = torch.zeros(kc.shape[-1], device=DEV)
            K, V = ((c[b, i].float() * s[b, i])[kept] for c, s in ((kc, ks), (vc, vs)))
            return dict(kept_pos=order[b][kept].int(), K=K, V=V, mean_k=none if mean is None else mean[0][b, i],
                        mean_v=none if mean is None else mean[1][b, i])


# ----------------------------------------------------------------------------- work
def work(case):
    B, H, D, G = case["batch"], case["kv_heads"], case["head_dim"], case["q_heads"] // case["kv_heads"]
    if case["kind"] == "rope":
        values = B * case["tokens"] * (H + H * G) * D
        return dict(bytes=2 * values * (2 if case["dtype"] == "bf16" else 4) + B * case["tokens"] * 4,
                    flops=3 * values * case["rotated"] / D)
    n = case["ctx"] * (0.625 if case["ragged"] else 1)                  # ragged lengths: a quarter of it to all of it
    whole = min(case["retrieval"], H)
    if case["kind"] == "window":
        T = case["tokens"] * (0.5 if case["ragged"] else 1)
        T = min(T, n)
        full = T * (n - (T - 1) / 2)                                    # (query, key) pairs of a head that sees everything
        reach = min(n, case["window"] + case["sinks"])
        short = T * reach if n - T >= reach else full - (n - reach) * (n - reach) / 2 + max(0, n - T - reach) ** 2 / 2
        rows = whole * n + (H - whole) * min(n, T + reach)
        return dict(bytes=B * (rows * 4 * D + T * H * G * 4 * D), flops=4 * D * B * G * (whole * full + (H - whole) * short))
    kept = whole * n + (H - whole) * min(n, case["sinks"] + case["window"])
    row = 2 * (D + 4)                                                   # K and V codes and their scales
    if case["kind"] == "read8":
        kept = n if whole else min(n, case["sinks"] + case["window"])
        return dict(bytes=kept * (row + 8 * D + 4), flops=kept * 2 * D)
    held = B * kept * row + B * H * G * D * 6
    if case["kind"] == "decode8":
        return dict(bytes=held, flops=B * G * kept * 4 * D)
    return dict(bytes=held + B * kept * row + B * H * n * 4 * D, flops=B * (G + 1) * kept * 4 * D + B * H * n * 2 * D)


# ----------------------------------------------------------------------------- exact
def exact(case, seed):
    kind = case["kind"]
    if kind == "rope":
        return _exact_rope(case, seed)
    if kind == "window":
        return _exact_window(case, seed)
    return _exact_cache(case, seed)


def _exact_rope(case, seed):
    rows, positions = _rope_inputs(case, seed)
    w, gain = _frequencies(case)
    R, Hq, Hk = case["rotated"], case["q_heads"], case["kv_heads"]
    turn = torch.polar(torch.full((), gain, dtype=torch.float64, device=DEV),
                       positions.double()[:, :, None, None] * torch.from_numpy(w).to(DEV))
    if case["inverse"]:
        turn = turn.conj()
    out = []
    for x in (rows[:, :, :Hq], rows[:, :, Hq:Hq + Hk]):
        y = x.double()
        pairs = y[..., :R].unflatten(-1, (R // 2, 2) if case["interleaved"] else (2, R // 2))
        if not case["interleaved"]:
            pairs = pairs.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        y[..., :R] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        out.append(y)
    return dict(q=out[0], k=out[1])


def _exact_window(case, seed):
    x = _window_inputs(case, seed)
    B, T, Hq, D = x["q"].shape
    G = Hq // case["kv_heads"]
    out = torch.zeros(B, T, Hq, D, dtype=torch.float64, device=DEV)
    for b, (n, new) in enumerate(zip(x["lens"], x["news"])):
        for t0 in range(0, new, 2048):
            t1 = min(new, t0 + 2048)
            m0, m1 = n - new + t0, n - new + t1                          # positions of these queries
            m = torch.arange(m0, m1, device=DEV)[:, None]
            for g in range(case["kv_heads"]):
                # only keys that some of these queries see
                lo = 0 if x["flags"][g] else max(0, m0 - case["window"] + 1)
                at = torch.cat([torch.arange(min(case["sinks"], lo)), torch.arange(lo, m1)]).to(DEV)
                hidden = at > m
                if not x["flags"][g]:
                    hidden |= (at >= case["sinks"]) & (at <= m - case["window"])
                K, V = x["K"][b, g, at].double(), x["V"][b, g, at].double()
                for h in range(g * G, (g + 1) * G):
                    s = (x["q"][b, t0:t1, h].double() @ K.T).div_(math.sqrt(D))
                    s[hidden] = -math.inf
                    out[b, t0:t1, h] = torch.softmax(s, -1) @ V
    return out


def _exact_cache(case, seed):
    """Attention over the values that the codes stand for; the codes themselves are whole numbers by definition."""
    x = _cache_inputs(case, seed)
    B, H, D = case["batch"], case["kv_heads"], case["head_dim"]
    G = case["q_heads"] // H

    def held(rows):
        top = rows.double().abs().amax(1, keepdim=True)
        # (127 / top and its product with a value are taken in 32 bits: that is the code's definition)
        step = (np.float32(127) / top.float().cpu().numpy()).astype(np.float32)
        codes = np.rint(rows.float().cpu().numpy() * step)
        return torch.from_numpy(codes).to(DEV).double() * (top / 127)

    def head(b, g):
        n = x["lens"][b]
        lo, hi = (n, n) if x["flags"][g] else (case["sinks"], n - case["window"])
        K, V = x["K"][b, g, :n], x["V"][b, g, :n]
        if lo >= hi:
            return list(range(n)), held(K), held(V), 0, None, None
        pos = list(range(lo)) + list(range(hi, n))
        return (pos, held(torch.cat([K[:lo], K[hi:]])), held(torch.cat([V[:lo], V[hi:]])), hi - lo,
                K[lo:hi].double().mean(0), V[lo:hi].double().mean(0))

    if case["kind"] == "read8":
        pos, K, V, gone, mk, mv = head(*x["at"])
        none = torch.zeros(D, dtype=torch.float64, device=DEV)
        return dict(kept_pos=torch.tensor(pos, dtype=torch.int32), K=K, V=V, mean_k=mk if gone else none,
                    mean_v=mv if gone else none)
    if B * sum(case["ctx"] if f else min(case["ctx"], case["sinks"] + case["window"]) for f in x["flags"]) > 4_000_000:
        return None                                                      # (rounding on the host takes too long)
    out = torch.zeros(B, H * G, D, dtype=torch.float64, device=DEV)
    for b in range(B):
        for g in range(H):
            _, K, V, gone, mk, mv = head(b, g)
            bias = torch.zeros(K.shape[0] + (gone > 0), dtype=torch.float64, device=DEV)
            if gone:
                K, V = torch.cat([K, mk[None]]), torch.cat([V, mv[None]])
                bias[-1] = math.log(gone)
            s = x["q"][b, g * G:(g + 1) * G].double() @ K.T / math.sqrt(D) + bias
            out[b, g * G:(g + 1) * G] = torch.softmax(s, -1) @ V
    return out
