"""Packed caches without a GPU: what the C entry points and the binding refuse
before any launch, workspace sizes, and the reference's own rounding."""
import ctypes

import numpy as np
import pytest

from paper_2608_07855_gb300 import build, commitkv as ck

ARG, UNSUP, WS = ck.COMMITKV_ERR_INVALID_ARG, ck.COMMITKV_ERR_UNSUPPORTED, ck.COMMITKV_ERR_WORKSPACE
SHAPE = dict(layers=2, kv_heads=2, q_heads=8, head_dim=128, dtype=ck.COMMITKV_BF16, softmax_scale=0.0)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return ck.load_library()


def cache(S=100, W=1, d=128, H=2, **kw):
    f = dict(k=0x10000, v=0x20000, stride_layer=H * S * d // 2, stride_head=S * d // 2, stride_tok=d // 2, k_scale=0x30000,
             v_scale=0x40000, scale_layer=H * S * d // 32, scale_head=S * d // 32, scale_tok=d // 32, pos=0x50000, S=S,
             q=0x60000, q_pos=0x70000, W=W, page_start=0x80000, page_len=0x90000, P=3)
    return ck.Packed(**{**f, **kw})


def rows(**kw):
    f = dict(k=0x10000, v=0x20000, stride_layer=2 * 10 * 128, stride_head=10 * 128, stride_tok=128, first=5, count=10)
    return ck.Rows(**{**f, **kw})


def copy(lib, c=None, r=None, n=1, name="commitkv_packed_write", **shape):
    s = ck.Shape(**{**SHAPE, **shape})
    m = max(n, 1)
    return getattr(lib, name)(ctypes.byref(s), n, (ck.Packed * m)(*[c or cache()] * m), (ck.Rows * m)(*[r or rows()] * m),
                              None, None)


def attend(lib, c=None, n=1, window=0, sinks=0, out=0xa0000, ws=0x100000, size=1 << 40, **shape):
    s = ck.Shape(**{**SHAPE, **shape})
    m = max(n, 1)
    o = None if out is None else (ctypes.c_void_p * m)(*[None if out == "none" else out] * m)
    return lib.commitkv_packed_attention(ctypes.byref(s), n, (ck.Packed * m)(*[c or cache()] * m), None, window, sinks, o,
                                         None, ws, size, None)


def compact(lib, c=None, dst=None, B=10, BN=2, cap=1, n_pending=1, ws=0x100000, size=1 << 30, idx=0x10000, n_idx=0x20000,
            fill=0x30000, retired=0x40000, **shape):
    s = ck.Shape(**{**SHAPE, **shape})
    one = lambda p: None if p is None else (ctypes.c_void_p * 1)(p)  # noqa: E731
    return lib.commitkv_packed_compact(
        ctypes.byref(s), 1, (ck.Packed * 1)(c or cache()), one(retired), one(0x50000), (ctypes.c_int32 * 1)(n_pending),
        one(0x60000), one(fill), B, BN, cap, one(idx), n_idx, None if dst is None else (ck.Packed * 1)(dst), ws, size, None)


BAD = [dict(S=-1), dict(W=-1), dict(P=-1), dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None),
       dict(stride_tok=63), dict(stride_head=-1), dict(stride_layer=-64), dict(scale_tok=3), dict(scale_head=-4),
       dict(scale_layer=-4), dict(W=1 << 28)]


@pytest.mark.parametrize("kw", BAD)
def test_bad_caches(lib, kw):
    for name in ("commitkv_packed_write", "commitkv_packed_read"):
        assert copy(lib, cache(**kw), name=name) == ARG
    assert attend(lib, cache(**kw)) == ARG
    assert compact(lib, cache(**kw)) == ARG
    s = ck.Shape(**SHAPE)
    assert lib.commitkv_packed_workspace_size(ctypes.byref(s), 1, (ck.Packed * 1)(cache(**kw))) == 0


@pytest.mark.parametrize("kw", [dict(pos=None), dict(q=None), dict(q_pos=None)])
def test_what_attention_reads_must_be_there(lib, kw):
    assert attend(lib, cache(**kw)) == ARG


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(first=-1), dict(count=-1), dict(first=91), dict(count=96),
                                dict(first=2**31 - 1, count=2**31 - 1)])
def test_bad_rows(lib, kw):
    for name in ("commitkv_packed_write", "commitkv_packed_read"):
        assert copy(lib, r=rows(**kw), name=name) == ARG


@pytest.mark.parametrize("kw", [dict(stride_layer=0), dict(stride_head=0), dict(scale_layer=0), dict(scale_head=0)])
def test_nothing_is_written_where_layers_or_heads_share_a_place(lib, kw):
    assert copy(lib, cache(**kw)) == ARG
    assert compact(lib, cache(**kw)) == ARG
    assert compact(lib, dst=cache(**kw)) == ARG


@pytest.mark.parametrize("kw", [dict(stride_layer=0), dict(stride_head=0), dict(stride_tok=0)])
def test_nothing_is_read_into_one_place(lib, kw):
    assert copy(lib, r=rows(**kw), name="commitkv_packed_read") == ARG


@pytest.mark.parametrize("kw", [dict(head_dim=96), dict(head_dim=32), dict(head_dim=256)])
def test_other_widths(lib, kw):
    assert copy(lib, **kw) == attend(lib, **kw) == compact(lib, **kw) == UNSUP


@pytest.mark.parametrize("kw", [dict(layers=0), dict(kv_heads=0), dict(q_heads=7), dict(dtype=2), dict(softmax_scale=-1.0)])
def test_bad_shapes(lib, kw):
    assert copy(lib, **kw) == attend(lib, **kw) == compact(lib, **kw) == ARG


def test_bad_calls(lib):
    for n in (0, -1, 65):
        assert copy(lib, n=n) == attend(lib, n=n) == ARG
    assert attend(lib, window=-1) == attend(lib, sinks=-1) == attend(lib, out="none") == attend(lib, out=None) == ARG
    s = ck.Shape(**SHAPE)
    c = (ck.Packed * 1)(cache())
    for name in ("commitkv_packed_write", "commitkv_packed_read"):
        assert getattr(lib, name)(ctypes.byref(s), 1, c, None, None, None) == ARG
        assert getattr(lib, name)(ctypes.byref(s), 1, None, (ck.Rows * 1)(rows()), None, None) == ARG


def test_nothing_to_do_needs_no_gpu(lib):
    assert copy(lib, r=rows(count=0)) == copy(lib, r=rows(count=0, k=None, v=None)) == ck.COMMITKV_OK
    assert attend(lib, cache(W=0)) == attend(lib, cache(W=0, q=None, q_pos=None), out="none") == ck.COMMITKV_OK


def test_workspaces(lib):
    s = ck.Shape(**SHAPE)
    for W in (1, 40):
        need = lib.commitkv_packed_workspace_size(ctypes.byref(s), 1, (ck.Packed * 1)(cache(W=W)))
        assert need > 256
        for ws, size in ((None, need), (0x90000, 1024), (0x90000, 0), (0x90010, need)):
            assert attend(lib, cache(W=W), ws=ws, size=size) == WS
    for ws, size in ((None, 1 << 20), (0x90000, 256), (0x90000, 511), (0x90010, 1 << 20)):
        assert compact(lib, ws=ws, size=size) == WS


def test_a_workspace_serves_smaller_calls(lib):
    def size(n, W, S, **kw):
        s = ck.Shape(**{**SHAPE, **kw})
        return lib.commitkv_packed_workspace_size(ctypes.byref(s), n, (ck.Packed * n)(*[cache(W=W, S=S)] * n))

    for kw in (dict(), dict(dtype=ck.COMMITKV_F32, head_dim=64), dict(kv_heads=8, q_heads=64)):
        for n in (1, 2, 63):
            for W in (0, 1, 3, 4, 5, 15, 64, 1000):
                for S in (0, 1, 100, 40000, 1 << 20):
                    here = size(n, W, S, **kw)
                    assert 0 < here <= size(n, W + 1, S, **kw)
                    assert here <= size(n + 1, W, S, **kw) and here <= size(n, W, S + 7, **kw)


def test_compact_refusals(lib):
    assert compact(lib, BN=11) == compact(lib, B=-1) == compact(lib, BN=-1) == compact(lib, cap=-1) == ARG
    assert compact(lib, n_pending=-1) == compact(lib, n_pending=100000) == ARG
    assert compact(lib, idx=None) == compact(lib, n_idx=None) == compact(lib, fill=None) == compact(lib, retired=None) == ARG
    assert compact(lib, cache(pos=None)) == ARG
    assert compact(lib, dst=cache(S=9)) == ARG  # no room for ten tokens
    assert compact(lib, dst=cache(k_scale=None)) == ARG


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    s = ck.make_shape(1, 2, 4, 64, torch.float32)
    z = lambda w: torch.zeros(1, 2, 10, w, dtype=torch.uint8)  # noqa: E731
    good = ck.PackedTensors(z(32), z(32), z(2), z(2), torch.arange(10, dtype=torch.int32))
    x = torch.zeros(1, 2, 3, 64)
    with pytest.raises(ValueError):  # on the host
        ck.commitkv_packed_write(s, [good], [x], [x], [0])
    with pytest.raises(ValueError):
        ck.packed_rows(s, [], [], [], [])
    with pytest.raises(ValueError):
        ck.commitkv_packed_attention(s, [good], out=[x], workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    # shapes and types, wherever the tensors are
    for kw in (dict(k=z(31)), dict(v=z(16)), dict(k_scale=z(4)), dict(v_scale=z(1)), dict(k=z(32).int()),
               dict(pos=torch.arange(9, dtype=torch.int32)), dict(pos=torch.arange(10)),
               dict(page_start=torch.zeros(2, dtype=torch.int32))):
        bad = ck.PackedTensors(**{**dict(k=good.k, v=good.v, k_scale=good.k_scale, v_scale=good.v_scale, pos=good.pos), **kw})
        with pytest.raises(ValueError):
            bad.desc()


def test_reference_rounds_to_the_nearest():
    """The tests' own packing: every group's scale is the nearest to a / 7, every code the nearest, both by search."""
    import packed_ref as ref

    rng = np.random.RandomState(0)
    for spread in (1.0, 3e-4, 2e-6, 900.0):
        x = (rng.randn(40, 64) * spread).astype(np.float32).astype(np.float64)
        x[0] = 0
        codes, scales = ref.pack(x)
        v = ref.values(codes, scales)
        g, s = x.reshape(-1, 32), ref.SIGMA[scales].reshape(-1)
        a = np.abs(g).max(-1)
        assert np.array_equal(np.abs(s - a / 7), np.abs(ref.SIGMA[None, :248] - a[:, None] / 7).min(1))
        levels = np.arange(-7, 8)[None, None] * s[:, None, None]
        best = np.abs(g[..., None] - levels).min(-1)
        assert np.array_equal(np.abs(v.reshape(-1, 32) - g), best)
        if spread < 100:
            assert (best <= s[:, None] / 2).all() or spread < 1e-5
    assert np.isnan(ref.values(*ref.pack(np.array([[np.inf] + [1.0] * 31])))).all()
