"""What the attention calls of the binding refuse with tensors on the GPU, and
how they go on over many work items."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_07855_gb300 import commitkv as ck  # noqa: E402

from test_gpu_attention import BF, SENT, Problem  # noqa: E402

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
