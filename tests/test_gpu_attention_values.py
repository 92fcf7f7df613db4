"""Attention over resident caches where values are not finite or scores are
very large: what is NaN, what is not, and the log-sum-exp beside it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import attention_ref as ref  # noqa: E402
from test_gpu_attention import BF, IDS, TYPES, Problem, kernels, run  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 24])
@pytest.mark.parametrize("prefix", [0, 700])
def test_log_sum_exp_beside_values_of_nan(dtype, d, W, prefix):
    """Keys of score -inf among tokens whose values are all NaN: the rows are NaN,
    their log-sum-exp is that of all visible tokens, in items of several tiles."""
    def put(k, v):
        k[:, :, 5::16, 3] = float("-inf")
        v[:, :, 2::16] = float("nan")

    def edit(p):
        k, v, pos, q, qp = p.host[0]
        q[..., 3] = q[..., 3].abs() + 0.5
        put(k, v)
        if prefix:
            put(*p.pre[:2])

    p = run(dtype=dtype, d=d, M=1, H=16, Hq=16, trajs=[(2900, W)], prefix=prefix, edit=edit)
    assert p.out[0].isnan().all() and p.lse[0].isfinite().all()


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 40, 150])
def test_values_of_nan_beside_scores_of_minus_infinity_alone(dtype, d, W):
    """A stretch of tokens that all have the score -inf, among them a NaN value:
    its channel is NaN (0 NaN), however the tokens are divided."""
    def edit(p):
        k, v, pos, q, qp = p.host[0]
        q[..., 3] = q[..., 3].abs() + 0.5
        k[:, :, :2000, 3] = float("-inf")
        v[:, :, 300, 5] = float("nan")

    p = run(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(2500, W)], edit=edit)
    assert p.out[0][..., 5].isnan().all() and p.lse[0].isfinite().all()


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 40, 150])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("prefix", [0, 200])
def test_scores_beyond_the_exponents_range(dtype, d, W, sign, prefix):
    """Finite scores of 1e10 to 1e12, far apart: all weight is on the largest; a
    NaN among them reaches the rows that see it.
    Scores are products of two small integers and powers of two, so exact; a
    weight of one times a value is off by the value's own terms and the
    output's rounding; the reference times log 2 by two roundings, 2^-23."""
    rng = np.random.RandomState(3)

    def keys(k):
        n = k.shape[2]
        k.zero_()
        k[..., 0] = torch.from_numpy(sign * 2.0 ** 16 * (1 + rng.randint(0, 200, n))).to(k.dtype)
        # one largest score of every prefix of the text
        k[:, :, 0, 0] = 2.0 ** 16 * (201 if sign > 0 else -0.25)

    def edit(p):
        for k, v, pos, q, qp in p.host:
            keys(k)
            q.zero_()
            q[..., 0] = 2.0 ** 20
        p.host[0][0][:, :, 899, 0] = float("nan")  # the last query's row
        if prefix:
            keys(p.pre[0])
            for h in p.host:  # the prefix has the largest
                h[0][..., 0] *= 2 if sign < 0 else 0.5

    p = Problem(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(900, W), (300, W)], prefix=prefix,
                edit=edit).upload()
    p.call()
    torch.cuda.synchronize()
    eps = 2.0 ** -8 if dtype == BF else 2.0 ** -20
    for i, (k, v, pos, q, qp) in enumerate(p.host):
        parts = ([tuple(p.pre)] if prefix else []) + [(k, v, pos)]
        o, l, _, _ = ref.attention(parts, q, qp)
        ref.check(p.out[i], o, eps * np.abs(o) + 1e-30, "out %d" % i)
        ref.check(p.lse[i], l, 2.0 ** -22 * np.abs(l), "lse %d" % i)
    p.guards()


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 40, 150])
@pytest.mark.parametrize("size", [2.0 ** 4, 2.0 ** 11, 2.0 ** 17])
def test_values_of_nan_beside_large_scores(dtype, d, W, size):
    """Rows that are done over for a value of NaN, seen in one channel or masked,
    with scores of 1e4 to 1e8, many of them equal: their weights fit the sum that
    they had before.  Scores are exact, and equal or far apart; beside the sums of
    up to a thousand equal weights and of their values in fp32 there are the
    roundings of weights and outputs."""
    rng = np.random.RandomState(5)

    def edit(p):
        for k, v, pos, q, qp in p.host:
            k.zero_()
            k[..., 0] = torch.from_numpy(size * (100.0 + 27 * rng.randint(0, 2, k.shape[2]))).to(k.dtype)
            q.zero_()
            q[..., 0] = 32.0 * 3
            v[:, :, -1 - W // 2, 5] = float("nan")

    p = Problem(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(900, W), (333, W)], edit=edit).upload()
    p.call(170)
    torch.cuda.synchronize()
    eps = 2.0 ** -7 if dtype == BF else 2.0 ** -17
    for i, (k, v, pos, q, qp) in enumerate(p.host):
        o, l, _, _ = ref.attention([(k, v, pos)], q, qp, 170)
        spread = ref.attention([(k, v.abs(), pos)], q, qp, 170)[0]
        ref.check(p.out[i], o, eps * spread, "out %d" % i)
        ref.check(p.lse[i], l, 2.0 ** -22 * np.abs(l) + 2.0 ** -16, "lse %d" % i)
    p.guards()


@pytest.mark.parametrize("W", [1, 40])
@pytest.mark.parametrize("size", [2.0 ** 8, 2.0 ** 12, 2.0 ** 16])
@pytest.mark.parametrize("where", ["own", "prefix"])
def test_equal_scores_in_parts_that_are_done_over_and_others(W, size, where, kernels):  # noqa: F811
    """Large equal scores in the prefix and in the cache, one of which has a key of
    score -inf, so that its parts are done over: all weigh the same.  Scores are
    127 size / 8, exact but for the rounding of scale / log 2, which is the same
    for all, and of the CUDA cores' product."""
    def keys(k, far):
        k.zero_()
        k[:, :, 7::50, 0] = 127.0 * size
        if far:
            k[:, :, 5::50, 1] = float("-inf")

    def edit(p):
        k, v, pos, q, qp = p.host[0]
        q.zero_()
        q[..., :2] = 1.0
        keys(k, where == "own")
        keys(p.pre[0], where == "prefix")

    p = Problem(dtype=torch.float32, d=64, M=1, H=1, Hq=4, trajs=[(900, W)], prefix=700, edit=edit).upload()
    p.call()
    torch.cuda.synchronize()
    k, v, pos, q, qp = p.host[0]
    parts = [tuple(p.pre), (k, v, pos)]
    o, l, _, _ = ref.attention(parts, q, qp)
    spread = ref.attention([(a, b.abs(), c) for a, b, c in parts], q, qp)[0]
    ref.check(p.out[0], o, 2.0 ** -17 * spread, "out")
    ref.check(p.lse[0], l, 2.0 ** -22 * np.abs(l), "lse")
