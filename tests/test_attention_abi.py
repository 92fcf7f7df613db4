"""The attention calls refuse bad arguments on the host, before any launch
(no GPU needed: none of these calls reaches the device)."""
import ctypes

import pytest

from paper_2608_07855_gb300 import build, commitkv as ck

OK, ARG, UNSUP, WS = 0, ck.COMMITKV_ERR_INVALID_ARG, ck.COMMITKV_ERR_UNSUPPORTED, ck.COMMITKV_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    build.build()
    return ck.load_library()


def traj(**kw):
    t = ck.Traj(0x10000, 0x20000, 25600, 12800, 128, 0x30000, 100, 0x40000, 0x50000, 8, None, None, 0)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


SHAPE = dict(layers=2, kv_heads=2, q_heads=8, head_dim=128, dtype=ck.COMMITKV_BF16, softmax_scale=0.0)


def call(lib, shape=None, t=None, n=1, prefix=None, window=0, sinks=0, out=0x60000, ws=0x90000, size=1 << 40,
         shared=False):
    s = ck.Shape(**{**SHAPE, **(shape or {})})
    arr = (ck.Traj * max(n, 1))(*[t or traj()] * max(n, 1))
    outs = (ctypes.c_void_p * max(n, 1))(*[out] * max(n, 1)) if out != "none" else None
    if shared:
        return lib.commitkv_prefix_attention(ctypes.byref(s), n, arr, ctypes.byref(prefix) if prefix else None, None,
                                             window, sinks, outs, None, ws, size, None)
    return lib.commitkv_window_attention(ctypes.byref(s), n, arr, None, window, sinks, outs, None, ws, size, None)


@pytest.mark.parametrize("shape", [dict(q_heads=7), dict(layers=0), dict(kv_heads=0), dict(dtype=3),
                                   dict(softmax_scale=-1.0), dict(softmax_scale=float("inf")),
                                   dict(softmax_scale=float("nan")), dict(layers=257), dict(head_dim=0)])
def test_bad_shapes(lib, shape):
    assert call(lib, shape) == ARG
    assert call(lib, shape, prefix=traj(), shared=True) == ARG


@pytest.mark.parametrize("d", [1, 32, 80, 96, 256])
def test_other_widths(lib, d):
    assert call(lib, dict(head_dim=d)) == UNSUP


@pytest.mark.parametrize("kw", [dict(S=-1), dict(W=-1), dict(k=None), dict(v=None), dict(pos=None), dict(q=None),
                                dict(q_pos=None), dict(stride_tok=127), dict(stride_head=-1), dict(stride_layer=-8),
                                dict(W=1 << 28)])
def test_bad_trajectories(lib, kw):
    assert call(lib, t=traj(**kw)) == ARG
    assert call(lib, t=traj(**kw), prefix=traj(), shared=True) == ARG


@pytest.mark.parametrize("kw", [dict(S=-1), dict(k=None), dict(v=None), dict(pos=None), dict(stride_tok=0)])
def test_bad_prefixes(lib, kw):
    assert call(lib, prefix=traj(**kw), shared=True) == ARG


def test_bad_calls(lib):
    for n in (0, -1, 65):
        assert call(lib, n=n) == ARG
    assert call(lib, window=-1) == ARG and call(lib, sinks=-1) == ARG
    assert call(lib, out="none") == ARG and call(lib, out=None) == ARG
    assert call(lib, shared=True) == ARG  # no prefix


def test_workspace(lib):
    for shared in (False, True):
        s, p = ck.Shape(**SHAPE), traj() if shared else None
        need = lib.commitkv_attention_workspace_size(ctypes.byref(s), 1, (ck.Traj * 1)(traj()), ctypes.byref(p) if p else None)
        assert need > 256
        for ws, size in ((None, need), (0x90000, need - 1), (0x90000, 0), (0x90010, need)):
            assert call(lib, ws=ws, size=size, prefix=p, shared=shared) == WS


def test_workspace_serves_smaller_calls(lib):
    def size(n, W, S, prefix, **kw):
        s = ck.Shape(**{**SHAPE, **kw})
        p = ctypes.byref(traj(S=S)) if prefix else None
        return lib.commitkv_attention_workspace_size(ctypes.byref(s), n, (ck.Traj * n)(*[traj(W=W, S=S)] * n), p)

    for prefix in (False, True):
        for kw in (dict(), dict(dtype=ck.COMMITKV_F32, head_dim=64), dict(kv_heads=8, q_heads=64)):
            for n in (1, 2, 63):
                for W in (0, 1, 3, 15, 64, 1000):
                    here = size(n, W, 100, prefix, **kw)
                    assert 0 < here <= size(n, W + 1, 100, prefix, **kw)
                    assert here <= size(n + 1, W, 100, prefix, **kw)
                    assert here == size(n, W, 1 << 20, prefix, **kw) == size(n, W, 0, prefix, **kw)
    assert size(1, -1, 100, False) == 0 and size(1, 1, -1, True) == 0


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    z = torch.zeros(1, 2, 10, 64)
    t = ck.TrajTensors(z, z, torch.arange(10, dtype=torch.int32), torch.zeros(1, 4, 1, 64), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        ck.commitkv_window_attention(ck.make_shape(1, 2, 4, 64, torch.float32), [t], out=[torch.zeros(1, 4, 1, 64)],
                                     workspace=torch.zeros(1 << 20, dtype=torch.uint8))
