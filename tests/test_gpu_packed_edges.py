"""Packed caches where single rows, queries and weights are out of the ordinary."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_packed import IDS, TYPES, Problem, kernels  # noqa: E402,F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ queries
@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 3, 8, 40])
def test_infinite_queries_over_keys_of_one_sign(dtype, d, W, kernels):  # noqa: F811
    """Scores of -inf alone: such a row is zero with a log-sum-exp of -inf.  The tokens of the other sign, which would
    make it NaN, lie behind its window."""
    inf = float("inf")

    def edit(p):
        for c, pos, Q, qp in p.host:
            c.host["k_scale"][..., 0] = 150
            c.host["k"][..., 0] = 0xb << 4 | 0xf          # channels 0 and 1: 7 and 3,
            c.host["k"][:, :, 100:, 0] = 0x2 << 4 | 0x1   # -7 and -6 of the tokens in the windows
            Q[0, 0, :, 0] = inf                           # -inf
            Q[0, 1, W - 1, 0] = -inf                      # +inf
            Q[0, 2, :, :2] = inf                          # -inf twice
            Q[0, 3, :, 0], Q[0, 3, :, 1] = inf, -inf      # -inf and +inf

    p = Problem(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(300, W)], edit=edit).upload()
    p.call(window=150)
    torch.cuda.synchronize()
    out, lse = p.out[0][0].float().cpu().numpy(), p.lse[0][0].cpu().numpy()
    for h in (0, 2):
        assert (out[h] == 0).all() and (lse[h] == -np.inf).all()
    assert np.isnan(out[1, W - 1]).all() and np.isnan(lse[1, W - 1])
    assert np.isnan(out[3]).all() and np.isnan(lse[3]).all()
    assert np.isfinite(out[1, :W - 1]).all() and np.isfinite(lse[1, :W - 1]).all()
    p.guards()
