"""How far attention may be from 64 bits in the 2-norm where operands are sums
of terms or rounded, and restatements with terms left out (test
infrastructure: shares no code with the library).

fp32, output against 64 bits, relative 2-norm over all rows of one call on
standard normal Q, K and V.  What adds up, as a root of squares:
  the terms' own loss (two tf32 terms)                     1.2e-7 (SPLIT below)
  2^x of the special-function unit (2^-22.5) and of its
  argument (|t| < 16: half a step 2^-21, times log 2,
  uniform: / sqrt 3)                                       1.6e-7 and 1.9e-7
  scores: 48 sums cut off at 2^-23 of a partial sum that
  grows to |s| of about 1 (uniform: rms 2^-23 / sqrt 3,
  half the final size: sqrt(48) 2^-23 / (2 sqrt 3))        2.4e-7
  sums of weights times values, the same over a tile      2.4e-7
together 4.5e-7; three times that is the bound, which every single missing
product of terms passes (2.2e-6 and more: test_attention_precision.py).

Log-sum-exp of size 6 to 16 with scores up to 6, absolute: half a step of the
result (2^-21), the constant log 2 (2^-25 of 8 and more: 2^-22), the logarithm of
the sum (a step of 4: 2^-22), the sum's own error (2^-22), and the scale times
1 / log 2, rounded twice (2^-23 of a score of 6: 7.2e-7): 1.9e-6 = 2^-19."""
import torch

F32_BOUND = 3 * 4.5e-7
LSE_BOUND = 2.0 ** -19


def rel(got, want):
    return float((got.double() - want).norm() / want.norm())


def tf32(x):
    """Rounded to 10 fraction bits."""
    return ((x.float().view(torch.int32) + 0x1000) & ~0x1FFF).view(torch.float32).double()


def tf32_cut(x):
    return (x.float().view(torch.int32) & ~0x1FFF).view(torch.float32).double()


def bf16(x):
    return x.float().bfloat16().double()


def two_tf32(x):
    h = tf32(x)
    return [h, tf32_cut(x - h)]


def three_bf16(x):
    a = bf16(x)
    b = bf16(x - a)
    return [a, b, bf16(x - a - b)]


def two_bf16(x):
    a = bf16(x)
    return [a, bf16(x - a)]


PAIRS = {two_tf32: [(0, 0), (0, 1), (1, 0)],
         three_bf16: [(0, 0), (0, 1), (1, 0), (1, 1), (0, 2), (2, 0)]}


def attention(Q, K, V, split=None, qk=None, pv=None, weights=None):
    """One head, everything visible, Q [w][d], K and V [s][d] in 64 bits, the
    operands as sums of terms of which the products qk and pv are taken."""
    d = Q.shape[1]
    products = lambda A, B, pairs, eq: sum(torch.einsum(eq, A[i], B[j]) for i, j in pairs)  # noqa: E731
    s = torch.einsum("wd,sd->ws", Q, K) if split is None else products(split(Q), split(K), qk, "wd,sd->ws")
    s = s * d ** -0.5
    e = torch.exp(s - s.amax(-1, keepdim=True))
    total = e.sum(-1, keepdim=True)
    if split is not None:
        o = products(split(e), split(V), pv, "ws,sd->wd")
    else:
        o = (e if weights is None else sum(weights(e))) @ V
    return o / total
