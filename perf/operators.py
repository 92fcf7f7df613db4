"""Attention over resident KV caches: what is measured, its plain form, and its exact results.

A case is one call: `window` is commitkv_window_attention (new tokens attend to the resident caches of a batch of
trajectories, with a sliding window and sink tokens), `prefix` is commitkv_prefix_attention (the same for trajectories
that share a prefix).  With absolute positions pos of the cached tokens, token i is visible to a query at position p iff
    pos_i <= p  and  (window = 0  or  pos_i > p - window  or  pos_i < sinks),
    s_i = scale <q, k_i>,  lse = log sum exp s_i,  o = sum exp(s_i - lse) v_i   over the visible tokens of the prefix
and of the trajectory's own cache together; o = 0 and lse = -inf for a query that sees none.  Query head h reads KV
head h / (Hq / H).

Fields: op; dtype, d (head width), M layers, H KV heads, Hq query heads; n trajectories; W new tokens of a trajectory
(the last ones of its cache) and ctx resident tokens, W included (the largest ones when n > 1); keep (share of the
older tokens that compression kept: their positions have gaps); window, sinks; pre (prefix tokens); lse (also returned);
layout (the seed of lengths and positions, so that a case's work is fixed)."""
import math
import random

import numpy as np
import torch

own = False

RECENT = 128  # a compressed cache keeps this many of the latest tokens without gaps


def _case(name, op, n, W, ctx, dtype="bf16", d=128, M=1, H=8, Hq=32, keep=1.0, window=0, sinks=0, pre=0, lse=False,
          layout=1):
    return dict(name=name, op=op, dtype=dtype, d=d, M=M, H=H, Hq=Hq, n=n, W=W, ctx=ctx, keep=keep, window=window,
                sinks=sinks, pre=pre, lse=lse, layout=layout)


def listed():
    return [
        # the smallest: one decoded token on the one-layer fp32 reference shape, where launches and host time count
        _case("decode_tiny_f32", "window", 1, 1, 2304, "f32", 64, 1, 2, 4),
        # decoding with a sliding window and sinks, concurrent agents of very different lengths, one layer
        _case("decode_window_16", "window", 16, 1, 36896, window=4096, sinks=4, layout=2),
        # decoding over caches after their checkpoints: compressed to at most 8,192 tokens, all of them visible
        _case("decode_compressed_64", "window", 64, 1, 8192, keep=0.25, layout=3),
        # the probe window's queries of all layers, with the log-sum-exp that the page effects start from
        _case("probe_layers_32k", "window", 1, 32, 36896, M=36, lse=True, layout=4),
        # a returned observation prefilled with a sliding window
        _case("prompt_window_4k", "window", 1, 4096, 36864, window=4096, sinks=4, layout=5),
        # the same observation attending to everything: bound by arithmetic
        _case("prompt_full_4k", "window", 1, 4096, 36864, layout=6),
        # 64-wide heads, three prompts of odd lengths over compressed caches
        _case("prompt_d64_odd", "window", 3, 517, 8191, d=64, H=4, Hq=16, keep=0.5, window=1000, sinks=16, layout=7),
        # fp32 prompt, five query heads to a KV head
        _case("prompt_f32", "window", 1, 301, 3001, "f32", H=2, Hq=10, keep=0.5, layout=8),
        # four agents at the start of their turns behind a short system prompt: latency
        _case("prefix_decode_4", "prefix", 4, 1, 203, pre=2048, layout=9),
        # a full batch decoding behind the same tool descriptions
        _case("prefix_decode_64", "prefix", 64, 1, 2048, pre=16384, layout=10),
        # tool results of eight agents prefilled behind a long shared prefix, log-sum-exp as well
        _case("prefix_prompt_8", "prefix", 8, 256, 2048, pre=32768, lse=True, layout=11),
        # fp32, 64-wide heads, three speculated tokens each, a window that ends inside the prefix
        _case("prefix_f32_spec", "prefix", 6, 3, 700, "f32", 64, 1, 2, 8, pre=1501, window=1200, sinks=4, layout=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["window", "window", "prefix"])
    kind = rng.choice(["8b", "8b", "8b", "32b", "d64", "f32"])
    c = dict(op=op, dtype="bf16", d=128, M=1, H=8, Hq=32)
    if kind == "32b":
        c.update(Hq=64)
    elif kind == "d64":
        c.update(d=64, H=rng.choice([2, 4, 8]))
        c.update(Hq=c["H"] * rng.choice([1, 2, 4, 5]))
    elif kind == "f32":
        c.update(dtype="f32", d=rng.choice([64, 128]), H=rng.choice([1, 2, 4]))
        c.update(Hq=c["H"] * rng.choice([1, 2, 4, 7]))
    form = rng.choice(["decode", "decode", "spec", "probe", "prompt", "prompt"])
    small = kind == "f32"
    n, W, ctx = 1, 1, 0
    if form == "decode":
        n, ctx = _log(rng, 1, 16 if small else 64), _log(rng, 129, 6000 if small else 32768)
        ctx = min(ctx, 600000 // n)
    elif form == "spec":
        n, W, ctx = _log(rng, 1, 16), rng.randint(2, 8), _log(rng, 200, 6000 if small else 24000)
    elif form == "probe":
        W, ctx = rng.choice([8, 16, 31, 32, 64]), _log(rng, 300, 6000 if small else 32768)
        c.update(M=1 if small else rng.choice([1, 4, 12]))
    else:
        n, W = rng.choice([1, 1, 2, 3, 5]), _log(rng, 65, 500 if small else 4096)
        ctx = W + _log(rng, 1, 4000 if small else 30000)
        while n * W * ctx * c["Hq"] * c["d"] > 4096 * 34000 * 32 * 128:
            W, ctx = W // 2, ctx // 2
    c.update(n=n, W=W, ctx=ctx, keep=rng.choice([1.0, 1.0, 0.5, 0.25]), window=0, sinks=0, pre=0,
             lse=rng.random() < 0.3, layout=rng.randrange(1 << 20))
    if rng.random() < 0.5:
        c.update(window=_log(rng, 64, 8192), sinks=rng.choice([0, 4, 4, 16, 64]))
    if op == "prefix":
        c.update(pre=_log(rng, 256, 4000 if small else 24000), ctx=max(W + 1, ctx // 4))
    return c


# ------------------------------------------------------------------------------------------------ layout
def _layouts(c):
    """Per trajectory: (positions of its cached tokens, positions of its W new tokens), numpy int64."""
    rng = random.Random(c["layout"])
    out = []
    for t in range(c["n"]):
        W = c["W"] if c["n"] == 1 or c["W"] < 16 else rng.randint(c["W"] // 2, c["W"])
        S = c["ctx"] if c["n"] == 1 else rng.randint(max(W, c["ctx"] // 8), c["ctx"])
        gaps = np.ones(S, np.int64)
        old = max(0, S - max(RECENT, W))
        if c["keep"] < 1.0:
            gaps[:old] = np.random.RandomState(c["layout"] + t).geometric(c["keep"], old)
        gaps[0] = 0
        pos = c["pre"] + np.cumsum(gaps)
        out.append((pos, pos[S - W:]))
    return out


def _visible(pos, p, window, sinks):
    """(first, end) of the window's tokens and the end of the sinks for every query position p, as indices into pos."""
    end = np.searchsorted(pos, p, "right")
    if not window:
        return np.zeros_like(end), end, np.zeros_like(end)
    lo = np.searchsorted(pos, p - window, "right")
    return lo, end, np.minimum(np.searchsorted(pos, sinks, "left"), lo)


def work(case):
    c = case
    b = 2 if c["dtype"] == "bf16" else 4
    lays = _layouts(c)
    tokens = pairs = rows = 0
    prefix = np.arange(c["pre"])
    for cache in [None] + lays:  # the prefix is read once for all
        ranges = []
        for pos, p in lays if cache is None else [cache]:
            lo, end, se = _visible(prefix if cache is None else pos, p, c["window"], c["sinks"])
            pairs += int((end - lo + se).sum())
            ranges += list(zip(lo, end)) + [(0, x) for x in se]
            rows += 0 if cache is None else len(p)
        seen = np.zeros((c["pre"] if cache is None else len(cache[0])) + 1, np.int64)
        for a, e in ranges:
            if e > a:
                seen[a] += 1
                seen[e] -= 1
        tokens += int((np.cumsum(seen)[:-1] > 0).sum())
    out = rows * c["Hq"] * (2 * c["d"] * b + (4 if c["lse"] else 0))
    return {"bytes": c["M"] * (tokens * c["H"] * 2 * c["d"] * b + out) + 4 * tokens,
            "flops": 4 * c["M"] * c["Hq"] * c["d"] * pairs}


# ------------------------------------------------------------------------------------------------ inputs
def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _cache(c, gen, S, u, first):
    """K, V [M][H][S][d]: four outlier channels a KV head; the first tokens of the text gather attention."""
    M, H, d = c["M"], c["H"], c["d"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    K = _normal(gen, (M, H, S, d), dt)
    K[..., :4] *= 4
    if first:
        K[:, :, :4] += (8 * u).to(dt)
    return K, _normal(gen, (M, H, S, d), dt)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    u = torch.randn(c["d"], generator=gen, device="cuda")
    u /= u.norm()
    s = dict(case=c, prefix=None, trajs=[])
    if c["pre"]:
        K, V = _cache(c, gen, c["pre"], u, True)
        s["prefix"] = dict(K=K, V=V, pos=torch.arange(c["pre"], dtype=torch.int32, device="cuda"))
    for pos, p in _layouts(c):
        K, V = _cache(c, gen, len(pos), u, not c["pre"])
        Q = (torch.randn((c["M"], c["Hq"], len(p), c["d"]), generator=gen, device="cuda") + 4 * u).to(dt)
        s["trajs"].append(dict(K=K, V=V, pos=torch.from_numpy(pos.astype(np.int32)).cuda(), Q=Q,
                               qpos=torch.from_numpy(p.astype(np.int32)).cuda()))
    if own:
        from paper_2608_07855_gb300 import commitkv as ck
        s["shape"] = ck.make_shape(c["M"], c["H"], c["Hq"], c["d"], dt)
        trajs = [ck.TrajTensors(t["K"], t["V"], t["pos"], t["Q"], t["qpos"]) for t in s["trajs"]]
        pre = ck.TrajTensors(**{k.lower() if k != "pos" else k: v for k, v in s["prefix"].items()}) if c["pre"] else None
        s["ws"] = ck.alloc_attention_workspace(s["shape"], trajs, pre)
        rows = [t["Q"].shape[0] * t["Q"].shape[1] * t["Q"].shape[2] for t in s["trajs"]]
        s["out"] = torch.empty(sum(rows) * c["d"], dtype=dt, device="cuda")
        s["lse"] = torch.empty(sum(rows), device="cuda") if c["lse"] else None
        outs = [o.view(t["Q"].shape) for o, t in zip(s["out"].split([r * c["d"] for r in rows]), s["trajs"])]
        lses = [x.view(t["Q"].shape[:3]) for x, t in zip(s["lse"].split(rows), s["trajs"])] if c["lse"] else None
        # the batch's descriptors, kept from call to call
        s["batch"] = ck.attention_batch(s["shape"], trajs, outs, lses, prefix=pre)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _attend(K, V, pos, Q, qpos, window, sinks):
    """The definition in elementary operations, fp32: o [M][Hq][W][d] and lse [M][Hq][W]."""
    M, H, S, d = K.shape
    Hq, W = Q.shape[1:3]
    s = torch.matmul(Q.float().view(M, H, -1, d), K.float().transpose(2, 3)).view(M, Hq, W, S) / math.sqrt(d)
    p, i = qpos[:, None], pos[None, :]
    seen = (i <= p) & ((i > p - window) | (i < sinks)) if window else i <= p
    s = torch.where(seen, s, float("-inf"))
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), torch.zeros_like(m), m)
    e = torch.exp(s - m)
    l = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(M, H, -1, S), V.float()).view(M, Hq, W, d)
    return (o / torch.where(l > 0, l, torch.ones_like(l))).to(Q.dtype), (m + torch.log(l)).squeeze(-1)


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2608_07855_gb300 import commitkv as ck
        if c["pre"]:
            ck.commitkv_prefix_attention(s["shape"], s["batch"], window=c["window"], sinks=c["sinks"], workspace=s["ws"])
        else:
            ck.commitkv_window_attention(s["shape"], s["batch"], window=c["window"], sinks=c["sinks"], workspace=s["ws"])
        return {"out": s["out"], "lse": s["lse"]} if c["lse"] else {"out": s["out"]}
    P = s["prefix"]
    got = [_attend(torch.cat([P["K"], t["K"]], 2) if P else t["K"], torch.cat([P["V"], t["V"]], 2) if P else t["V"],
                   torch.cat([P["pos"], t["pos"]]) if P else t["pos"], t["Q"], t["qpos"], c["window"], c["sinks"])
           for t in s["trajs"]]
    out = torch.cat([o.reshape(-1) for o, _ in got])
    return {"out": out, "lse": torch.cat([x.reshape(-1) for _, x in got])} if c["lse"] else {"out": out}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """Every query head by itself, its scores in blocks of queries, in 64 bits."""
    if work(case)["flops"] > 8e12:
        return None
    s = prepare(case, seed)
    c, P = case, s["prefix"]
    g = c["Hq"] // c["H"]
    outs, lses = [], []
    for t in s["trajs"]:
        parts = ([P] if P else []) + [t]
        pos = torch.cat([x["pos"] for x in parts]).long()
        M, Hq, W, d = t["Q"].shape
        out = torch.zeros(M, Hq, W, d, dtype=torch.float64, device="cuda")
        lse = torch.full((M, Hq, W), float("-inf"), dtype=torch.float64, device="cuda")
        for layer in range(M):
            for kv in range(c["H"]):
                k = torch.cat([x["K"][layer, kv] for x in parts]).double()
                v = torch.cat([x["V"][layer, kv] for x in parts]).double()
                for b in range(0, W, 1024):
                    p = t["qpos"][b:b + 1024].long()[:, None]
                    hidden = pos[None, :] > p
                    if c["window"]:
                        hidden |= (pos[None, :] <= p - c["window"]) & (pos[None, :] >= c["sinks"])
                    for h in range(kv * g, kv * g + g):
                        a = t["Q"][layer, h, b:b + 1024].double() @ k.T
                        a = (a * d ** -0.5).masked_fill_(hidden, -math.inf)
                        z = torch.logsumexp(a, 1)
                        w = torch.exp(a - torch.where(z.isinf(), 0.0, z)[:, None])
                        out[layer, h, b:b + 1024] = w @ v
                        lse[layer, h, b:b + 1024] = z
        outs.append(out.reshape(-1))
        lses.append(lse.reshape(-1))
    return {"out": torch.cat(outs), "lse": torch.cat(lses)} if c["lse"] else {"out": torch.cat(outs)}
