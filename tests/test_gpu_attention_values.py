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
