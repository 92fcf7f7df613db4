"""Attention over resident caches by its definition in 64 bits, and how far a
result may be from it (test infrastructure: shares no code with the library)."""
import math

import numpy as np
import torch

EPS = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half a step, relative


def visible(pos, p, window, sinks):
    """[queries][tokens] truth values."""
    i = np.arange(len(pos))[None, :]
    x, p = np.asarray(pos, np.int64)[None, :], np.asarray(p, np.int64)[:, None]
    v = x <= p
    if window:
        v &= (x > p - window) | ((x < sinks) & (i < sinks))
    return v


def attention(parts, Q, qpos, window=0, sinks=0, scale=None, rounded_weights=False):
    """parts: [(K, V, pos)] whose tokens are summed over together, K and V
    [M][H][S][d]; Q [M][Hq][W][d].  Returns o, lse and the tolerances of both.

    A score is a sum of d products in fp32, in some order, scaled: off by at
    most (d + 4) 2^-24 sum |q_c k_c| scale; 2^x off by 2^-21 relative
    (the special-function unit's 2^-22 and the argument's own rounding); the
    base-2 reference and rescaling add a few 2^-22.  So a weight is off by
    ds + 2^-19 relative, ds the largest such score error of the row plus the
    rounding of scores and their maximum (2^-22 |s|), and by 2^-8 more where it
    is rounded to bf16.  o is a weighted mean: off by that times
    sum a |v| for the numerator and the sum of weights each (the latter without
    the bf16 rounding), n 2^-24 more for sums of n terms in fp32 (the tile
    kernels add 32 or more in a tree: at most 2^-17 relative for the sizes
    here), and half a step of its own."""
    M, Hq, W, d = Q.shape
    H = parts[0][0].shape[1]
    g = Hq // H
    scale = scale or d ** -0.5
    o = np.zeros((M, Hq, W, d))
    lse = np.full((M, Hq, W), -np.inf)
    tol_o, tol_l = np.zeros_like(o), np.zeros_like(lse)
    dt = Q.dtype
    see = np.concatenate([visible(p, qpos, window, sinks) for _, _, p in parts], 1)
    for l in range(M):
        for h in range(Hq):
            k = np.concatenate([x[l, h // g].double().numpy() for x, _, _ in parts])
            v = np.concatenate([x[l, h // g].double().numpy() for _, x, _ in parts])
            q = Q[l, h].double().numpy()
            for w in range(W):
                s = see[w]
                if not s.any():
                    continue
                kk, vv = k[s], v[s]
                with np.errstate(invalid="ignore", over="ignore"):
                    sc = kk @ q[w] * scale
                    m = sc.max()
                    e = np.exp(sc - m)
                    z = e.sum()
                    a = e / z
                    o[l, h, w] = a @ vv
                    lse[l, h, w] = m + np.log(z)
                    f = np.isfinite(sc)  # a score of -inf is exact
                    ds = (d + 4) * 2.0 ** -24 * (np.abs(kk[f]) @ np.abs(q[w])).max(initial=0) * scale + \
                        np.abs(sc[f]).max(initial=0) * 2.0 ** -21
                    rel = 2 * (ds + 2.0 ** -19 + 2.0 ** -17) + (2.0 ** -8 if rounded_weights else 0.0)
                    tol_o[l, h, w] = EPS[dt] * np.abs(o[l, h, w]) + (1 + EPS[dt]) * rel * (a @ np.abs(vv))
                    tol_l[l, h, w] = ds + 2.0 ** -16 + 2.0 ** -22 * abs(lse[l, h, w])
    return o, lse, tol_o, tol_l


def check(got, want, tol, what=""):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want)), what + ": NaN"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]) and not np.isinf(got[~inf]).any(), what + ": infinities"
    f = np.isfinite(want)
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want)
    bad = f & ~(off <= tol)
    if bad.any():
        at = tuple(x[0] for x in np.nonzero(bad))
        raise AssertionError("%s: %d of %d off, first at %s: %.9g, want %.9g, tolerance %.3g; largest off %.3g" % (
            what, bad.sum(), bad.size, at, got[at], want[at], tol[at], off[f].max()))


def positions(S, first=0, gaps=1.0, tail=16, seed=0):
    """Increasing positions, gapped before the last `tail` tokens; gaps = share kept."""
    step = np.ones(S, np.int64)
    n = max(0, S - tail)
    if gaps < 1.0:
        step[:n] = np.random.RandomState(seed).geometric(gaps, n)
    if S:
        step[0] = 0
    return first + np.cumsum(step)


def cache(M, H, S, d, dtype, seed, layout="dense"):
    """K and V [M][H][S][d] on the CPU in a layout: dense, tokens outermost
    (heads side by side), padded rows, or starting one element off."""
    g = torch.Generator().manual_seed(seed)

    def one():
        x = torch.randn(M, H, S, d, generator=g).to(dtype)
        return x

    return one(), one()


def place(x, layout, device="cuda"):
    """x [M][H][S][d] on the device in a layout with contiguous channels."""
    M, H, S, d = x.shape
    if layout == "dense":
        return x.to(device).contiguous()
    if layout == "tokens":  # [M][S][H][d]
        return x.to(device).transpose(1, 2).contiguous().transpose(1, 2)
    pad, off = (16, 0) if layout == "padded" else (8, 1)  # "odd": 2-byte aligned
    base = torch.full((M * H * (S + 3) * (d + pad) + off,), float("nan"), dtype=x.dtype, device=device)
    v = base[off:].view(M, H, S + 3, d + pad)[:, :, :S, :d]
    v.copy_(x.to(device))
    return v
