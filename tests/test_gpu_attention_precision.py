"""The precision that the header states, for each kernel: 2-norms against 64
bits with bounds that a missing term passes (test_attention_precision.py)."""
import pytest

torch = pytest.importorskip("torch")

import attention_ref as ref  # noqa: E402
import attention_terms as at  # noqa: E402
from test_gpu_attention import BF, F32, Problem, kernels  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def errors(p):
    """Outputs and log-sum-exps of all trajectories: got and in 64 bits."""
    p.call()
    torch.cuda.synchronize()
    got, want, lse, lse_want = [], [], [], []
    for i, (k, v, pos, q, qp) in enumerate(p.host):
        o, z, _, _ = ref.attention(([tuple(p.pre)] if p.pre else []) + [(k, v, pos)], q, qp)
        got.append(p.out[i].double().cpu().reshape(-1))
        want.append(torch.from_numpy(o).reshape(-1))
        lse.append(p.lse[i].double().cpu().reshape(-1))
        lse_want.append(torch.from_numpy(z).reshape(-1))
    p.guards()
    return [torch.cat(x) for x in (got, want, lse, lse_want)]


# (W, prefix, agents): a decoded token, a prompt, a prompt of more than one row tile, agents behind a prefix
FORMS = [(1, 0, 4), (40, 0, 1), (150, 0, 1), (1, 700, 40), (12, 700, 6)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("W,prefix,n", FORMS)
def test_fp32(d, W, prefix, n):
    """Whatever the kernel, within three times the expected error."""
    p = Problem(dtype=F32, d=d, M=1, H=2, Hq=8, trajs=[(1200 - 100 * (i % 4), W) for i in range(n)], prefix=prefix).upload()
    got, want, lse, lse_want = errors(p)
    assert at.rel(got, want) < at.F32_BOUND
    assert (lse - lse_want).abs().max() < at.LSE_BOUND


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("W,prefix,n", FORMS + [(1, 700, 4), (4, 0, 3)])
def test_bf16(d, W, prefix, n, kernels):  # noqa: F811
    """Up to 16 rows (heads of a KV head times positions) of a cache, a prefix's of
    all agents together: the output's own rounding and hardly more.  More rows:
    the weights' rounding as well, of the same size."""
    p = Problem(dtype=BF, d=d, M=1, H=2, Hq=8, trajs=[(1200 - 100 * (i % 4), W) for i in range(n)], prefix=prefix).upload()
    got, want, lse, lse_want = errors(p)
    own = at.rel(want.float().bfloat16(), want)
    few = 4 * W * (n if prefix else 1) <= 16
    assert at.rel(got, want) < (1.03 if kernels == "cuda_cores" or (few and kernels == "") else 1.6) * own
    assert (lse - lse_want).abs().max() < at.LSE_BOUND
