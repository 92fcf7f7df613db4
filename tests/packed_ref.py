"""Packed caches by their definition in 64 bits (test infrastructure: shares no
code with the library)."""
import numpy as np
import torch

from attention_ref import EPS, visible


def sigma_table():
    """The numbers that scale bytes stand for: 248 finite ones, then NaN."""
    s = [m * 2.0 ** -23 if e == 0 else (8 + m) * 2.0 ** (e - 24) for e in range(31) for m in range(8)]
    return np.array(s + [np.nan] * 8)


SIGMA = sigma_table()


def pack(x):
    """Rows [...][d] (float64, exact values of the inputs) as codes [...][d / 2] and scale bytes [...][d / 32]."""
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    a = np.abs(g).max(-1)
    mids = 3.5 * (SIGMA[1:248] + SIGMA[:247])  # seven times the middle of two neighbours, exact
    b = np.searchsorted(mids, a, "left")       # mids[b - 1] < a <= mids[b]
    at = np.minimum(b, 246)
    b = b + ((b < 247) & (mids[at] == a) & (b % 2 == 1))
    s = SIGMA[b][..., None]
    n = np.zeros(g.shape)
    for k in range(7):  # |x| past the middle between k and k + 1, which itself goes to the even one
        edge = (k + 0.5) * s
        n += np.where(s > 0, np.abs(g) > edge if k % 2 == 0 else np.abs(g) >= edge, False)
    u = (8 + np.sign(g) * n).astype(np.uint8).reshape(x.shape)
    b = np.where(bad, 255, b).astype(np.uint8)
    return u[..., 0::2] | (u[..., 1::2] << 4), b


def values(codes, scales):
    u = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1]).astype(np.float64) - 8
    return u * np.repeat(SIGMA[scales], 32, -1)


def attention(k, v, pos, Q, qpos, window=0, sinks=0, scale=None, weights=0.0, queries=0.0):
    """k, v [M][H][S][d] float64 values, Q [M][Hq][W][d] a torch tensor.  o, lse and
    the tolerances of both.

    A score: d products in fp32 sums that may be cut off instead of rounded, (d + 4)
    2^-23 sum |q_c k_c| scale; a query's element enters with `queries` of itself
    lost; the rounding of scaled scores and of their maximum 2^-21 |s|.  2^x 2^-21,
    the reference and rescaling 2^-19 in all.  A weight enters the product with
    `weights` of it lost.  Sums of n weights in fp32: 2^-17 for the sizes here.
    The output's own rounding: half a step.

    fp16 terms end at 2^-24, so what they hold is off by 2^-25 at least.  A row's
    weights stand as 2^11 and more for its largest: each may be off by 2^-36 of
    that, which shows where the largest weights meet values of zero.  Its queries'
    largest stands as 2^14 and more: an element may be off by 2^-39 of it."""
    M, Hq, W, d = Q.shape
    g = Hq // k.shape[1]
    scale = scale or d ** -0.5
    see = visible(pos, qpos, window, sinks)
    o, lse = np.zeros((M, Hq, W, d)), np.full((M, Hq, W), -np.inf)
    to, tl = np.zeros_like(o), np.zeros_like(lse)
    eps = EPS[Q.dtype]
    for l in range(M):
        for h in range(Hq):
            kk, vv, q = k[l, h // g], v[l, h // g], Q[l, h].double().cpu().numpy()
            for w in range(W):
                s = see[w]
                if not s.any():
                    continue
                with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                    sc = kk[s] @ q[w] * scale
                    m = sc.max()
                    e = np.exp(sc - m)
                    a = e / e.sum()
                    o[l, h, w] = a @ vv[s]
                    lse[l, h, w] = m + np.log(e.sum())
                    f = np.isfinite(sc)
                    top = (np.abs(kk[s][f]) @ np.abs(q[w])).max(initial=0) * scale
                    ds = ((d + 4) * 2.0 ** -23 + queries) * top + np.abs(sc[f]).max(initial=0) * 2.0 ** -21
                    ds += 2.0 ** -39 * np.abs(q[w]).max() * np.abs(kk[s][f]).sum(1).max(initial=0) * scale
                    rel = 2 * (ds + 2.0 ** -19 + 2.0 ** -17) + weights
                    to[l, h, w] = eps * np.abs(o[l, h, w]) + \
                        (1 + eps) * (rel * (a @ np.abs(vv[s])) + 2.0 ** -36 * a.max() * np.abs(vv[s]).sum(0))
                    tl[l, h, w] = ds + 2.0 ** -16 + 2.0 ** -22 * abs(lse[l, h, w])
    return o, lse, to, tl


def numbers(x):
    return x.double().cpu().numpy()


def layout(x, kind, device="cuda"):
    """A uint8 or float tensor [M][H][S][w] on the device: dense, heads side by side, rows with room behind them, or
    beginning at an odd address; what is not x's own holds bytes of 0xff (codes and scales that are NaN; float NaN)."""
    M, H, S, w = x.shape
    if kind == "dense":
        return x.to(device).contiguous()
    if kind == "tokens":
        return x.to(device).transpose(1, 2).contiguous().transpose(1, 2)
    step, off = {"padded": (64, 0), "odd": (3, 1)}[kind]
    n = M * H * (S + 3) * (w + step) + off
    base = torch.full((n * x.element_size(),), 255, dtype=torch.uint8, device=device).view(x.dtype)
    y = base[off:].view(M, H, S + 3, w + step)[:, :, :S, :w]
    y.copy_(x.to(device))
    return y
