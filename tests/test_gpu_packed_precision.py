"""How far attention over packed caches is from 64 bits in the 2-norm, on every
kernel: bounds that a missing term would pass."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import packed_ref as ref  # noqa: E402
from test_gpu_packed import BF, F32, Problem  # noqa: E402

pytestmark = pytest.mark.gpu


def off(W, dtype, d, env, monkeypatch, S=1500):
    for name, value in env.items():
        monkeypatch.setenv(name, value)
    p = Problem(dtype=dtype, d=d, M=1, H=2, Hq=8, trajs=[(S, W)], gaps=0.5).upload()
    p.call()
    torch.cuda.synchronize()
    c, pos, Q, qp = p.host[0]
    k, v = c.values()
    o, _, _, _ = ref.attention(k, v, pos, Q, qp)
    got = ref.numbers(p.out[0])
    rounded = ref.numbers(torch.from_numpy(o).to(dtype))
    return [np.linalg.norm(x - o) / np.linalg.norm(o) for x in (got, rounded)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("W", [1, 4])
def test_decoded_bf16(W, d, monkeypatch):
    """The output's own rounding (e), and beside it weights of one fp16 term: each off by 2^-12 of itself at most,
    independently, so by less than 2^-12 of the output's norm in all.  bf16 weights (2^-9) would add 1e-3 and more."""
    got, e = off(W, BF, d, {}, monkeypatch)
    assert got <= np.hypot(e, 2.0 ** -12) * 1.01


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("W", [1, 2, 4])
def test_decoded_fp32(W, d, monkeypatch):
    """Two terms of queries and weights lose 2^-22 of each; sums of d and of 1,500 in fp32, cut off or rounded, some
    2^-22 more.  One term of either would be off by 1e-4."""
    got, _ = off(W, F32, d, {}, monkeypatch)
    assert got <= 2e-6


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("how", ["", "tiles", "full"])
def test_prompts_bf16(how, d, monkeypatch):
    """Weights as one fp16 term or rounded to bf16: 2^-9 of a weight at most (a step of 2^-8, half of it), beside the
    output's rounding."""
    got, e = off(40, BF, d, {"COMMITKV_ATTENTION": how} if how else {}, monkeypatch)
    assert got <= np.hypot(e, 2.0 ** -9) * 1.01


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("how", ["", "full"])
def test_prompts_fp32(how, d, monkeypatch):
    got, _ = off(40, F32, d, {"COMMITKV_ATTENTION": how} if how else {}, monkeypatch)
    assert got <= 2e-6


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_cuda_cores(dtype, monkeypatch):
    got, e = off(2, dtype, 128, {"COMMITKV_SCORING": "simt"}, monkeypatch)
    assert got <= e * 1.01 + 2e-6
