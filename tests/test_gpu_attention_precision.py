"""The precision that the header states, for each kernel: 2-norms against 64
bits with bounds that a missing term passes (test_attention_precision.py)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_07855_gb300 import commitkv as ck  # noqa: E402

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


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("W", [4, 24])
def test_bf16_outputs_as_row_statistics(d, W):
    """Page effects from (lse, 1, out) of bf16 caches.  With o' = o + e, |e| = x |o|
    for the row's output and A a page's attention mass, the difference that Eq. 6
    measures moves by A e / (1 - A) and its norm is divided by |o'|, so
        |R' - R| <= x (R + A / (1 - A)) / (1 - x)
    beside the call's own 2e-2 of R (its tolerance from exact statistics)."""
    M, H, Hq, S, G = 2, 2, 8, 700, 25
    P = S // G
    g = torch.Generator().manual_seed(d + W)
    K, V, Q = ((torch.randn(M, h, n, d, generator=g) * a).to(BF).cuda() for h, n, a in ((H, S, 1), (H, S, 1), (Hq, W, 2)))
    start = torch.arange(0, S, G, dtype=torch.int32, device="cuda")
    pos = torch.arange(S, dtype=torch.int32, device="cuda")
    tr = ck.TrajTensors(K, V, pos, Q, pos[S - W:].clone(), start, torch.full_like(start, G))
    shape = ck.make_shape(M, H, Hq, d, BF)
    out, lse = torch.empty_like(Q), torch.empty(Q.shape[:3], device="cuda")
    ck.commitkv_window_attention(shape, [tr], [out], [lse], workspace=ck.alloc_attention_workspace(shape, [tr]))
    one, none = torch.ones_like(lse), torch.zeros_like(lse)
    stats = torch.cat([torch.stack([lse, one, none, none], -1), out.float()], -1).contiguous()
    R = torch.zeros(P, device="cuda")
    ws = ck.alloc_workspace(shape, [tr])
    ck.commitkv_page_effects_from_stats(shape, [tr], [stats], [R], workspace=ws)
    torch.cuda.synchronize()
    assert ck.commitkv_workspace_status(ws) == ck.COMMITKV_OK

    k, v, q = K.double().repeat_interleave(Hq // H, 1), V.double().repeat_interleave(Hq // H, 1), Q.double()
    s = (q @ k.transpose(2, 3)) * d ** -0.5
    a = torch.softmax(s.masked_fill(pos[None, :] > tr.q_pos[:, None], float("-inf")), -1)
    o = a @ v
    size = o.norm(dim=-1)
    x = ((out.double() - o).norm(dim=-1) / size)[..., None]  # of each row
    pages = a.view(M, Hq, W, P, G)
    A = pages.sum(-1)
    part = torch.einsum("mhwpg,mhpgd->mhwpd", pages, v.view(M, Hq, P, G, d))
    r = (part - A[..., None] * o[..., None, :]).norm(dim=-1) / (1 - A) / size[..., None]
    rows = (0, 1, 2)
    want, more = r.amax(rows), (x * (r + A / (1 - A)) / (1 - x)).amax(rows)
    assert ((R.double() - want).abs() <= 2e-2 * want + more).all()
