"""What the attention calls of the binding refuse with tensors on the GPU, and
how they go on over many work items."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_07855_gb300 import commitkv as ck  # noqa: E402

from test_gpu_attention import BF, F32, SENT, Problem, kernels  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prefix", [0, 5])
@pytest.mark.parametrize("kw", [dict(window=-1), dict(sinks=-1), dict(window=-(1 << 32) + 3), dict(sinks=-(1 << 33)),
                                dict(window=1 << 40), dict(sinks=1 << 31)])
def test_windows_and_sinks_that_32_bits_would_change(prefix, kw):
    """Each refused, and not what its low 32 bits say; nothing is written."""
    p = Problem(dtype=BF, d=64, M=1, H=1, Hq=2, trajs=[(10, 1)], prefix=prefix).upload()
    with pytest.raises((ValueError, ck.CommitKVError)):
        p.call(**kw)
    torch.cuda.synchronize()
    assert (p.flat == SENT).all() and (p.flat_l == SENT).all()


@pytest.mark.parametrize("dtype,d,H,g,many,prefix", [
    (F32, 64, 4, 2, False, 0), (F32, 128, 4, 2, False, 0), (F32, 128, 4, 2, False, 900), (F32, 128, 2, 5, True, 0),
    (BF, 128, 2, 5, False, 0), (BF, 64, 2, 5, False, 900), (BF, 128, 4, 4, True, 0), (BF, 128, 2, 5, True, 0)])
def test_blocks_go_from_item_to_item(dtype, d, H, g, many, prefix, kernels):  # noqa: F811
    """More work items than SMs, ragged ones and empty caches among them: of fp32
    (whose widths differ in warps and barriers), and of bf16 where later items'
    queries are not copied by TMA (heads that do not divide 128 rows, more than
    32 trajectories)."""
    if kernels == "cuda_cores":
        pytest.skip("a block an item there")
    trajs = [(300, 40), (0, 20), (420, 150), (700, 9), (64, 64), (333, 33)]
    if many:
        trajs = [((37 * i) % 400 if i % 9 else 0, 5 + (11 * i) % 40) for i in range(36)]
    M = 24
    p = Problem(dtype=dtype, d=d, M=M, H=H, Hq=g * H, prefix=prefix, gaps=0.8, trajs=trajs).upload()
    for window, sinks in ((0, 0), (130, 3)):
        p.flat.fill_(SENT)
        p.flat_l.fill_(SENT)
        p.call(window, sinks)
        p.check(window, sinks, layers=[0, M - 1])
        first = p.flat.clone(), p.flat_l.clone()
        p.ws[256:].fill_(0xFF)
        p.call(window, sinks)
        torch.cuda.synchronize()
        assert torch.equal(first[0], p.flat) and torch.equal(first[1], p.flat_l)


@pytest.mark.parametrize("dtype", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,S,W", [(1, 2000, 1), (20, 2000, 100), (3, 900, 40)])
def test_a_cache_without_queries_changes_nothing(dtype, n, S, W):
    """The others' work is divided, and their results are, as without it."""
    p = Problem(dtype=dtype, d=64, M=1, H=1, Hq=4, trajs=[(S + 10 * i, W) for i in range(n)]).upload()
    p.call()
    torch.cuda.synchronize()
    want = [x.clone() for x in p.out + p.lse]
    long = 500000
    K = torch.zeros(1, 1, long, 64, dtype=dtype, device="cuda")
    rest = ck.TrajTensors(K, K, torch.arange(long, dtype=torch.int32, device="cuda"))
    ck.commitkv_window_attention(p.shape, p.trajs + [rest], out=p.out + [None], lse_out=p.lse + [None], workspace=p.ws)
    torch.cuda.synchronize()
    p.guards()
    assert all(torch.equal(a, b) for a, b in zip(want, p.out + p.lse))
