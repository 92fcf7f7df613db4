"""Attention over resident caches against its definition in 64 bits: types,
layouts, lengths, masks, positions with gaps, values that are not finite,
graphs, streams, and the calls around it."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_07855_gb300 import commitkv as ck  # noqa: E402

import attention_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
SENT = 12352.0  # representable in bf16


@pytest.fixture(autouse=True, params=["", "tiles", "cuda_cores"])
def kernels(request, monkeypatch):
    """Every test on the kernels that the library picks, on those of row tiles
    (which small calls would not reach), and on the CUDA cores."""
    if request.param == "tiles":
        monkeypatch.setenv("COMMITKV_ATTENTION", "tiles")
    elif request.param:
        monkeypatch.setenv("COMMITKV_SCORING", "simt")
    return request.param


class Problem:
    """Trajectories (S, W) with their data on the host, and the call on the device."""

    def __init__(self, dtype, d, M, H, Hq, trajs, gaps=1.0, prefix=0, layout="dense", seed=0, qpos=None, spread=1.0,
                 scale=0.0, edit=None):
        self.shape = ck.make_shape(M, H, Hq, d, dtype, scale)
        self.dtype, self.scale = dtype, scale
        self.pre, self.host = None, []
        g = torch.Generator().manual_seed(seed + 99)
        if prefix:
            k, v = ref.cache(M, H, prefix, d, dtype, seed + 7)
            self.pre = [k, v, ref.positions(prefix, 0, gaps, 0, seed + 5)]
        first = int(self.pre[2][-1]) + 1 if prefix else 0
        for i, (S, W) in enumerate(trajs):
            k, v = ref.cache(M, H, S, d, dtype, seed + 10 * i)
            pos = ref.positions(S, first, gaps, 16, seed + i)
            Q = (spread * torch.randn(M, Hq, W, d, generator=g)).to(dtype)
            last = int(pos[-1]) if S else first
            p = np.arange(last - W + 1, last + 1) if qpos is None else np.asarray(qpos(pos, W))
            self.host.append([k, v, pos, Q, p])
        if edit:
            edit(self)
        self.layout = layout

    def upload(self):
        i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()  # noqa: E731
        put = lambda x: ref.place(x, self.layout)  # noqa: E731
        self.trajs = [ck.TrajTensors(put(k), put(v), i32(pos), q.cuda().contiguous(), i32(p))
                      for k, v, pos, q, p in self.host]
        self.prefix = None if self.pre is None else ck.TrajTensors(put(self.pre[0]), put(self.pre[1]), i32(self.pre[2]))
        n = sum(t.q.numel() for t in self.trajs)
        # outputs side by side with values between them that must stay
        self.flat = torch.full((n + 64 * (len(self.trajs) + 1),), SENT, dtype=self.dtype, device="cuda")
        self.flat_l = torch.full((n // self.shape.head_dim + 64 * (len(self.trajs) + 1),), SENT, device="cuda")
        self.out, self.lse, a, b = [], [], 64, 64
        for t in self.trajs:
            m = t.q.numel()
            self.out.append(self.flat[a:a + m].view(t.q.shape))
            self.lse.append(self.flat_l[b:b + m // self.shape.head_dim].view(t.q.shape[:3]))
            a, b = a + m + 64, b + m // self.shape.head_dim + 64
        self.ws = ck.alloc_attention_workspace(self.shape, self.trajs, self.prefix)
        return self

    def call(self, window=0, sinks=0, lse=True, layer_mask=None, stream=None):
        f = ck.commitkv_window_attention if self.pre is None else ck.commitkv_prefix_attention
        kw = {} if self.pre is None else dict(prefix=self.prefix)
        f(self.shape, self.trajs, out=self.out, lse_out=self.lse if lse else None, window=window, sinks=sinks,
          layer_mask=layer_mask, workspace=self.ws, stream=stream, **kw)

    def check(self, window=0, sinks=0, layers=None, lse=True):
        torch.cuda.synchronize()
        assert ck.commitkv_workspace_status(self.ws) == ck.COMMITKV_OK
        for i, (k, v, pos, q, p) in enumerate(self.host):
            parts = ([tuple(self.pre)] if self.pre else []) + [(k, v, pos)]
            if layers is not None:
                parts, q = [(x[layers], y[layers], z) for x, y, z in parts], q[layers]
            if q.numel() == 0:
                continue
            o, l, to, tl = ref.attention(parts, q, p, window, sinks, self.scale, self.dtype == BF)
            pick = (lambda x: x) if layers is None else (lambda x: x[layers])
            ref.check(pick(self.out[i]), o, to, "out %d" % i)
            if lse:
                ref.check(pick(self.lse[i]), l, tl, "lse %d" % i)
        self.guards()

    def guards(self):
        for flat, step in ((self.flat, 1), (self.flat_l, self.shape.head_dim)):
            a = 0
            for t in self.trajs:
                assert (flat[a:a + 64] == SENT).all(), "written outside the outputs"
                a += 64 + t.q.numel() // step
            assert (flat[a:] == SENT).all(), "written outside the outputs"


def run(window=0, sinks=0, **kw):
    p = Problem(**kw).upload()
    p.call(window, sinks)
    p.check(window, sinks)
    return p


TYPES = [(F32, 64), (F32, 128), (BF, 64), (BF, 128)]
IDS = ["f32-64", "f32-128", "bf16-64", "bf16-128"]


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("S", [1, 2, 31, 33, 127, 128, 129, 640, 1025])
def test_single_token_lengths(dtype, d, S):
    run(dtype=dtype, d=d, M=1, H=2, Hq=8, trajs=[(S, 1)], gaps=0.5)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [2, 5, 17, 64, 65, 130])
def test_prompt_lengths(dtype, d, W):
    run(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(W + 150, W)], gaps=0.6)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("H,Hq", [(1, 1), (2, 2), (1, 3), (2, 10), (1, 16), (1, 40)])
@pytest.mark.parametrize("W", [1, 9])
def test_heads(dtype, d, H, Hq, W):
    run(dtype=dtype, d=d, M=2, H=H, Hq=Hq, trajs=[(201, W)], window=150, sinks=3)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (64, 0), (100, 5), (128, 4), (300, 200), (1000, 64),
                                          (2**31 - 1, 2**31 - 1)])
@pytest.mark.parametrize("W,gaps", [(1, 0.4), (40, 0.4), (300, 1.0)])
def test_windows(dtype, d, window, sinks, W, gaps):
    run(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(700, W), (333, W)], gaps=gaps, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
def test_ragged_batch(dtype, d):
    """Lengths from none to long ones, trajectories without queries or tokens."""
    run(dtype=dtype, d=d, M=1, H=2, Hq=4, gaps=0.7, window=200, sinks=4,
        trajs=[(0, 3), (1, 1), (500, 1), (64, 64), (300, 0), (1400, 33), (0, 0), (257, 2), (129, 129)])


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n", [1, 17, 64])
def test_many_trajectories(dtype, d, n):
    run(dtype=dtype, d=d, M=1, H=1, Hq=2, trajs=[(5 + 13 * i, 1) for i in range(n)])


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 48])
def test_rows_that_see_nothing(dtype, d, W):
    """Queries before the first token, behind the last window, in any order."""
    def qpos(pos, W):
        return np.array([1000, 3, 99, 100, 101, 5000, 100 + len(pos), 350] * 6, np.int64)[:W] if W > 1 else [3]

    def late(p):
        for t in p.host:
            t[2] += 100

    p = run(dtype=dtype, d=d, M=1, H=2, Hq=4, trajs=[(400, W)], qpos=qpos, window=120, edit=late)
    assert torch.isinf(p.lse[0][:, :, 1 if W > 1 else 0]).all() and (p.out[0][:, :, 1 if W > 1 else 0] == 0).all()
    run(dtype=dtype, d=d, M=1, H=2, Hq=4, trajs=[(400, W)], qpos=qpos, window=120, sinks=130, edit=late)
    run(dtype=dtype, d=d, M=1, H=2, Hq=4, trajs=[(400, W)], qpos=qpos, edit=late)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 24])
def test_far_positions(dtype, d, W):
    """Positions up to the largest int32."""
    def far(p):
        for t in p.host:
            move = 2**31 - 1 - int(t[2][-1])
            t[2] = t[2] + move
            t[4] = t[4] + move

    run(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(500, W)], gaps=0.5, edit=far)
    run(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(500, W)], gaps=0.5, edit=far, window=77)


@pytest.mark.parametrize("layout", ["tokens", "padded", "odd"])
@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 70])
def test_layouts(dtype, d, layout, W):
    """Tokens outermost, rows with padding (NaN behind the last token and
    channel), caches that only the CUDA cores can read."""
    run(dtype=dtype, d=d, M=2, H=2, Hq=6, trajs=[(300, W), (77, W)], layout=layout, gaps=0.5, window=111, sinks=2)


def test_offsets_beyond_32_bits():
    """Tokens more than 2^31 elements apart."""
    for dtype, d in ((BF, 128), (BF, 64), (F32, 64)):
        for W in (1, 70):
            p = Problem(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(2200, W)])
            p.upload()
            t, stride = p.trajs[0], (1 << 20) + 16
            for name in ("k", "v"):
                base = torch.empty(2200 * stride, dtype=dtype, device="cuda")
                x = base.as_strided((1, 1, 2200, d), (2200 * stride, 2200 * stride, stride, 1))
                x.copy_(getattr(t, name))
                setattr(t, name, x)
            p.call()
            p.check()
            del p, t, x, base
            torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 40, 150])
@pytest.mark.parametrize("prefix", [0, 90])
def test_masked_values_that_are_not_finite(dtype, d, W, prefix):
    """Infinities and NaN in tokens that no query, or only some, see."""
    def edit(p):
        k, v, pos, q, qp = p.host[0]
        qp -= 30  # the last 30 tokens are seen by none
        k[:, :, -30::2] = float("nan")
        v[:, :, -29::2] = float("nan")
        v[:, :, -20] = float("inf")
        if W > 10:  # a token that only the later queries see
            v[:, :, -30 - W // 2, 5] = float("inf")
            k[:, 0, -33] = float("nan")
        v[:, :, 3] = float("-inf")  # before every window
        k[:, :, 4] = float("inf")
        if prefix:
            p.pre[1][:, :, 10:20] = float("nan")

    p = run(dtype=dtype, d=d, M=1, H=2, Hq=4, trajs=[(400, W), (300, W)], window=120, sinks=2, edit=edit, prefix=prefix)
    assert torch.isfinite(p.out[0][:, :, 0]).all()


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
def test_visible_values_that_are_not_finite(dtype, d):
    """A visible NaN or infinity reaches exactly the rows that see it."""
    def edit(p):
        p.host[0][1][:, :, 150, 7] = float("inf")
        p.host[0][0][:, :, 260] = float("nan")

    p = Problem(dtype=dtype, d=d, M=1, H=1, Hq=2, trajs=[(300, 100)], edit=edit).upload()
    p.call()
    torch.cuda.synchronize()
    o = p.out[0].float()
    seen = torch.tensor(p.host[0][4] >= 260, device="cuda")
    assert torch.isnan(o[:, :, seen]).all() and torch.isnan(p.lse[0][:, :, seen]).all()
    rest = o[:, :, ~seen]
    assert torch.isinf(rest[..., 7]).all()
    rest[..., 7] = 0
    assert torch.isfinite(rest).all()


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 20])
def test_visible_keys_of_minus_infinity(dtype, d, W):
    """A visible score of -inf has weight zero; the other tokens' results stay."""
    def edit(p):
        k, v, pos, q, qp = p.host[0]
        q[..., 3] = q[..., 3].abs() + 0.5
        k[:, :, 100:140:7, 3] = float("-inf")

    run(dtype=dtype, d=d, M=1, H=2, Hq=4, trajs=[(200, W)], edit=edit)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 33])
def test_large_scores(dtype, d, W):
    """Scores of several hundred: the running maximum moves often and far."""
    run(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(900, W)], spread=30.0)
    run(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(900, W)], scale=0.7)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("prefix", [1, 17, 128, 700])
@pytest.mark.parametrize("n,W", [(1, 1), (3, 1), (9, 1), (2, 40), (40, 3)])
def test_prefix(dtype, d, prefix, n, W):
    run(dtype=dtype, d=d, M=1, H=2, Hq=8, prefix=prefix, trajs=[(W + (37 * i) % 150, W) for i in range(n)], gaps=0.6)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("window,sinks", [(50, 4), (200, 0), (400, 300), (3, 1)])
def test_prefix_with_window(dtype, d, window, sinks):
    """Windows that end inside the prefix, or before it is reached."""
    run(dtype=dtype, d=d, M=2, H=1, Hq=4, prefix=260, window=window, sinks=sinks,
        trajs=[(100, 1), (9, 3), (0, 2), (150, 0), (301, 80), (1, 1)])


def test_prefix_equals_one_cache():
    """A shared prefix and the same tokens in every cache agree within both tolerances."""
    for dtype, d in TYPES:
        p = run(dtype=dtype, d=d, M=1, H=2, Hq=4, prefix=333, trajs=[(70, 2), (20, 2)], window=90, sinks=4)
        joined = [ck.TrajTensors(torch.cat([p.prefix.k, t.k], 2), torch.cat([p.prefix.v, t.v], 2),
                                 torch.cat([p.prefix.pos, t.pos]), t.q, t.q_pos) for t in p.trajs]
        out = [torch.empty_like(t.q) for t in joined]
        ws = ck.alloc_attention_workspace(p.shape, joined)
        ck.commitkv_window_attention(p.shape, joined, out=out, window=90, sinks=4, workspace=ws)
        torch.cuda.synchronize()
        for o, (k, v, pos, q, at) in zip(out, p.host):
            want, _, tol, _ = ref.attention([tuple(p.pre), (k, v, pos)], q, at, 90, 4, rounded_weights=dtype == BF)
            ref.check(o, want, tol, "one cache")


def test_empty_prefix():
    p = run(dtype=BF, d=128, M=1, H=2, Hq=4, trajs=[(200, 5)])
    want = p.out[0].clone()
    z = torch.empty(1, 2, 0, 128, dtype=BF, device="cuda")
    pre = ck.TrajTensors(z, z, torch.empty(0, dtype=torch.int32, device="cuda"))
    p.flat.fill_(SENT)
    ck.commitkv_prefix_attention(p.shape, p.trajs, prefix=pre, out=p.out, workspace=ck.alloc_attention_workspace(
        p.shape, p.trajs, pre))
    torch.cuda.synchronize()
    assert torch.equal(want, p.out[0])


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("prefix", [0, 200])
@pytest.mark.parametrize("W", [1, 70])
def test_layer_mask(dtype, d, prefix, W):
    """Only the selected layers' rows are written; none selected: nothing."""
    p = Problem(dtype=dtype, d=d, M=4, H=1, Hq=4, trajs=[(800, W)], prefix=prefix).upload()
    p.call(layer_mask=[0, 0, 0, 0])
    torch.cuda.synchronize()
    assert (p.flat == SENT).all()
    p.call(layer_mask=[1, 0, 1, 0])
    p.check(layers=[0, 2])
    assert (p.out[0][[1, 3]] == SENT).all() and (p.lse[0][[1, 3]] == SENT).all()


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("prefix,W", [(0, 1), (0, 90), (300, 1), (300, 30)])
def test_same_bits_every_time(dtype, d, prefix, W):
    p = Problem(dtype=dtype, d=d, M=1, H=2, Hq=8, trajs=[(900, W), (55, W)], prefix=prefix).upload()
    p.call()
    torch.cuda.synchronize()
    first = p.flat.clone(), p.flat_l.clone()
    for _ in range(3):
        p.ws[256:].fill_(0xFF)  # what an earlier call left in the workspace does not matter
        p.call(lse=True)
        torch.cuda.synchronize()
        assert torch.equal(first[0], p.flat) and torch.equal(first[1], p.flat_l)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("prefix,W", [(0, 1), (0, 90), (300, 1)])
def test_graph_and_stream(dtype, d, prefix, W):
    """Captured on another stream and replayed on new data; two graphs share a workspace."""
    p = Problem(dtype=dtype, d=d, M=1, H=2, Hq=8, trajs=[(600, W), (155, W)], prefix=prefix).upload()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    p.call(stream=s)
    s.synchronize()
    graphs = []
    for window in (0, 100):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            p.call(window=window, sinks=4)
        graphs.append(g)
    new = Problem(dtype=dtype, d=d, M=1, H=2, Hq=8, trajs=[(600, W), (155, W)], prefix=prefix, seed=1000)
    for t, h in zip(p.trajs, new.host):
        t.k.copy_(h[0])
        t.v.copy_(h[1])
        t.q.copy_(h[3])
    p.host = [n[:2] + o[2:3] + n[3:4] + o[4:] for n, o in zip(new.host, p.host)]
    if prefix:
        p.prefix.k.copy_(new.pre[0])
        p.prefix.v.copy_(new.pre[1])
        p.pre = new.pre[:2] + p.pre[2:]
    for g, window in ((graphs[1], 100), (graphs[0], 0), (graphs[1], 100)):
        p.flat.fill_(SENT)
        p.flat_l.fill_(SENT)
        g.replay()
        p.check(window, 4)


def test_calls_at_once():
    """Two streams with a workspace each."""
    ps = [Problem(dtype=BF, d=128, M=1, H=2, Hq=8, trajs=[(900, W)], prefix=pre, seed=W).upload()
          for W, pre in ((1, 0), (90, 0), (1, 400), (64, 400))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    for _ in range(20):
        for p, s in zip(ps, streams):
            p.call(stream=s)
    for p in ps:
        p.check()


def test_batch_kept_while_caches_grow():
    """An AttentionBatch over buffers with room: lengths move, tokens are added in place."""
    cap, d = 700, 128
    p = Problem(dtype=BF, d=d, M=1, H=2, Hq=8, trajs=[(cap, 1), (cap, 1)], gaps=0.5).upload()
    b = ck.attention_batch(p.shape, p.trajs, p.out, p.lse)
    full = [list(h) for h in p.host]
    for bad in (-1, cap + 1):
        with pytest.raises(ValueError):
            b.set_length(0, bad)
    for S in ((1, 3), (128, 200), (129, 640), (700, 699)):
        for i, n in enumerate(S):
            b.set_length(i, n)
            p.trajs[i].q_pos.fill_(int(full[i][2][n - 1]))
            k, v, pos, q, _ = full[i]
            p.host[i] = [k[:, :, :n], v[:, :, :n], pos[:n], q, np.array([pos[n - 1]])]
        ck.commitkv_window_attention(p.shape, b, window=300, sinks=2, workspace=p.ws)
        p.check(300, 2)


def test_effects_from_attention():
    """The attention of the probe window is a valid source of row statistics:
    fp32 effects from (lse, 1, out) as from the library's own statistics."""
    from paper_2608_07855_gb300 import synth
    from paper_2608_07855_gb300.workload import DeviceTrajectory, shape_of

    cfg = synth.CONFIGS["tiny"]
    dev = DeviceTrajectory.upload(synth.make_trajectory(cfg, 0))
    shape, tr = shape_of(cfg), dev.post()
    out = torch.empty_like(tr.q)
    lse = torch.empty(tr.q.shape[:3], device="cuda")
    ck.commitkv_window_attention(shape, [tr], out=[out], lse_out=[lse], workspace=ck.alloc_attention_workspace(shape, [tr]))
    stats = torch.cat([torch.stack([lse, torch.ones_like(lse), torch.zeros_like(lse), torch.zeros_like(lse)], -1), out], -1)
    R, want = (torch.zeros(dev.P_post, device="cuda") for _ in range(2))
    ws = ck.alloc_workspace(shape, [tr])
    ck.commitkv_page_effects_from_stats(shape, [tr], [stats.contiguous()], [R], workspace=ws)
    ck.commitkv_page_effects(shape, [tr], [want], workspace=ws)
    torch.cuda.synchronize()
    assert ck.commitkv_workspace_status(ws) == ck.COMMITKV_OK
    assert ((R - want).abs() <= 1e-4 * want.abs()).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("prefix", [0, 900])
def test_many_items(d, prefix):
    """More work items than SMs, of one and of two row tiles: blocks go from item to item."""
    p = Problem(dtype=BF, d=d, M=24, H=4, Hq=8, prefix=prefix, gaps=0.8,
                trajs=[(300, 40), (420, 150), (700, 9), (64, 64), (0, 20), (333, 33)]).upload()
    for window, sinks in ((0, 0), (130, 3)):
        p.flat.fill_(SENT)
        p.flat_l.fill_(SENT)
        p.call(window, sinks)
        p.check(window, sinks, layers=[0, 13, 23])


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 64)], ids=["bf16-128", "bf16-64", "f32-64"])
def test_long_prompt_is_cut_at_its_end(dtype, d, kernels):
    """Whole waves of row tiles and a cut remainder: written and merged rows side by side."""
    W = 2600 if dtype == BF and kernels != "cuda_cores" else 700
    p = Problem(dtype=dtype, d=d, M=4, H=4, Hq=16, trajs=[(W + 300, W)]).upload()
    p.call()
    torch.cuda.synchronize()
    t = p.trajs[0]
    for l, h in ((0, 0), (3, 15), (2, 6)):
        s = (t.q[l, h].double() @ t.k[l, h // 4].double().T) * d ** -0.5
        s.masked_fill_(t.pos[None, :] > t.q_pos[:, None], -math.inf)
        want = torch.softmax(s, 1) @ t.v[l, h // 4].double()
        spread = torch.softmax(s, 1) @ t.v[l, h // 4].double().abs()
        # half a step of the output and of every weight, and fp32 sums (attention_ref.attention)
        eps = 2.0 ** -8 if dtype == BF else 2.0 ** -24
        tol = eps * want.abs() + (eps if dtype == BF else 0.0) * spread + 2.0 ** -14 * spread
        assert ((p.out[0][l, h].double() - want).abs() <= tol).all()
        assert ((p.lse[0][l, h].double() - torch.logsumexp(s, 1)).abs() <= 2.0 ** -14).all()
    p.guards()


def test_session_attends_before_and_after_a_checkpoint():
    """A session's own attention over its cache, compressed in between, and behind a shared prefix."""
    from paper_2608_07855_gb300.lifecycle import Session

    M, H, Hq, d, n = 2, 2, 8, 128, 500
    g = torch.Generator().manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g).to(BF)  # noqa: E731
    shape = ck.make_shape(M, H, Hq, d, BF)
    s = Session(shape, 32, 200, 0.5, 1000)
    k, v = rand(M, H, n, d), rand(M, H, n, d)
    first = 100  # behind a prefix of 100 tokens
    s.append(k.cuda(), v.cuda(), torch.arange(first, first + n, dtype=torch.int32, device="cuda"), [("obs", first, 300)])
    pk, pv = rand(M, H, first, d), rand(M, H, first, d)
    pre = ck.TrajTensors(pk.cuda(), pv.cuda(), torch.arange(first, dtype=torch.int32, device="cuda"))

    def look(W, window=0, sinks=0, prefix=False):
        Q = rand(M, Hq, W, d)
        p = np.arange(first + n - W, first + n)
        o, l = s.attend(Q.cuda(), torch.from_numpy(p.astype(np.int32)).cuda(), window, sinks, pre if prefix else None)
        S = s.S
        own = (s.K[:, :, :S].cpu(), s.V[:, :, :S].cpu(), s.pos[:S].cpu().numpy())
        parts = ([(pk, pv, np.arange(first))] if prefix else []) + [own]
        wo, wl, to, tl = ref.attention(parts, Q, p, window, sinks, rounded_weights=True)
        ref.check(o, wo, to, "out")
        ref.check(l, wl, tl, "lse")

    for W in (1, 40):
        look(W)
        look(W, 150, 4, True)
    s.checkpoint(torch.rand(n, generator=g).cuda())
    assert s.S == 200
    for W in (1, 40):
        look(W)
        look(W, 150, 4, True)


@pytest.mark.parametrize("d", [64, 128])
def test_prefix_beside_decoded_caches(d):
    """Many agents behind a long prefix: its kernel and that of their own
    caches overlap, eager and in a graph, and the merge waits for both."""
    n, H, Hq, pre = 64, 8, 32, 7000
    p = Problem(dtype=BF, d=d, M=1, H=H, Hq=Hq, prefix=pre, trajs=[(40 + 31 * i, 1) for i in range(n)]).upload()
    K, V, pos = p.prefix.k[0].double(), p.prefix.v[0].double(), p.prefix.pos

    def check():
        torch.cuda.synchronize()
        assert ck.commitkv_workspace_status(p.ws) == ck.COMMITKV_OK
        for i, t in enumerate(p.trajs):
            k, v = torch.cat([K, t.k[0].double()], 1), torch.cat([V, t.v[0].double()], 1)
            q = t.q[0, :, 0].double().view(H, Hq // H, d)
            s = (q @ k.transpose(1, 2)) * d ** -0.5
            a = torch.softmax(s, -1)
            want, spread = a @ v, a @ v.abs()
            # half a step of the output and of every weight, and fp32 sums (attention_ref.attention)
            tol = 2.0 ** -8 * want.abs() + 2.0 ** -8 * spread + 2.0 ** -14 * spread
            assert ((p.out[i][0, :, 0].double().view(want.shape) - want).abs() <= tol).all(), i
            assert ((p.lse[i][0, :, 0].double().view(H, -1) - torch.logsumexp(s, -1)).abs() <= 2.0 ** -14).all(), i
        p.guards()

    for _ in range(3):
        p.flat.fill_(SENT)
        p.flat_l.fill_(SENT)
        p.call()
        check()
    first = p.flat.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        p.call()
        p.call()
    for _ in range(3):
        p.flat.fill_(SENT)
        p.ws[256:].fill_(0xFF)
        g.replay()
        check()
        assert torch.equal(first, p.flat)


def test_long_prompts_and_decoded_tokens_in_one_batch():
    """Both kinds of rows are split over their tokens, each as far as it may be
    alone: their partial results fit the workspace together."""
    H, Hq, d, g = 8, 32, 64, torch.Generator().manual_seed(5)
    shape = ck.make_shape(1, H, Hq, d, BF)

    def trajectories(S, W, n):
        k, v = ref.cache(1, H, S, d, BF, S)
        dev, pos = (k.cuda(), v.cuda()), torch.arange(S, dtype=torch.int32, device="cuda")
        for _ in range(n):
            Q = torch.randn(1, Hq, W, d, generator=g).to(BF)
            yield (k, v, np.arange(S)), Q, ck.TrajTensors(*dev, pos, Q.cuda(), pos[S - W:].clone())

    every = [*trajectories(40000, 1500, 2), *trajectories(8192, 4, 40)]
    trajs = [t for _, _, t in every]
    out = [torch.full_like(t.q, float("nan")) for t in trajs]
    lse = [torch.full(t.q.shape[:3], float("nan"), device="cuda") for t in trajs]
    ws = ck.alloc_attention_workspace(shape, trajs)
    ck.commitkv_window_attention(shape, trajs, out, lse, workspace=ws)
    torch.cuda.synchronize()
    assert ck.commitkv_workspace_status(ws) == ck.COMMITKV_OK
    assert all(x.isfinite().all() for x in out + lse)
    for i in (0, 1, 2, 20, 41):
        part, Q, t = every[i]
        W, S = Q.shape[2], part[0].shape[2]
        rows = sorted({0, W // 2 + 1, W - 1})
        o, l, to, tl = ref.attention([part], Q[:, :, rows], np.array(rows) + S - W, rounded_weights=True)
        ref.check(out[i][:, :, rows], o, to, "out %d" % i)
        ref.check(lse[i][:, :, rows], l, tl, "lse %d" % i)


@pytest.mark.parametrize("dtype,W", [(BF, 1216), (F32, 608)], ids=["bf16", "f32"])
def test_values_that_are_not_finite_in_a_long_cache(dtype, W, kernels):
    """Every row of a prompt is done over by the definition, for longer than the
    tile kernels' waits last."""
    if kernels:
        pytest.skip("the kernels of row tiles, which this call takes by itself")
    H, Hq, d, S, g = 8, 32, 128, 131072, torch.Generator().manual_seed(9)
    shape = ck.make_shape(1, H, Hq, d, dtype)
    k, v = ref.cache(1, H, S, d, dtype, 4)
    v[:, :, S - W:, 0] = float("nan")
    Q, pos = torch.randn(1, Hq, W, d, generator=g).to(dtype), torch.arange(S, dtype=torch.int32)
    trajs = [ck.TrajTensors(k.cuda(), v.cuda(), pos.cuda(), Q.cuda(), pos[S - W:].cuda())]
    out, lse = [torch.empty_like(trajs[0].q)], [torch.empty(Q.shape[:3], device="cuda")]
    ws = ck.alloc_attention_workspace(shape, trajs)
    ck.commitkv_window_attention(shape, trajs, out, lse, workspace=ws)
    torch.cuda.synchronize()
    assert ck.commitkv_workspace_status(ws) == ck.COMMITKV_OK
    assert out[0][..., 0].isnan().all() and out[0][..., 1:].isfinite().all() and lse[0].isfinite().all()
    rows = [0, W - 1]
    for h in (0, H - 1):
        o, l, to, tl = ref.attention([(k[:, h:h + 1], v[:, h:h + 1], pos.numpy())], Q[:, 4 * h:4 * h + 4, rows],
                                     np.array(rows) + S - W, rounded_weights=dtype == BF)
        ref.check(out[0][:, 4 * h:4 * h + 4, rows], o, to, "out")
        ref.check(lse[0][:, 4 * h:4 * h + 4, rows], l, tl, "lse")


def test_session_attention_in_graphs():
    """Graphs of a session's attention share no workspace with one another or
    with its later calls."""
    from paper_2608_07855_gb300.lifecycle import Session

    H, Hq, d, n = 2, 8, 64, 6000
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF)  # noqa: E731
    s = Session(ck.make_shape(1, H, Hq, d, BF), 32, 200, 0.5, n)
    s.append(rand(1, H, n, d), rand(1, H, n, d), torch.arange(n, dtype=torch.int32, device="cuda"), [])
    Q = [rand(1, Hq, 1, d), rand(1, Hq, 70, d)]
    p = [torch.arange(n - q.shape[2], n, dtype=torch.int32, device="cuda") for q in Q]
    s.attend(Q[0], p[0])  # the session's own workspace, too small for the other
    graphs, outs = [], []
    for q, at in zip(Q, p):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(s.attend(q, at))
    for q in Q:
        q.copy_(rand(*q.shape))
    want = [s.attend(q, at) for q, at in zip(Q, p)]
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    again = [s.attend(q, at) for q, at in zip(Q, p)]
    torch.cuda.synchronize()
    for w, o, a in zip(want, outs, again):
        assert all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(w, o, a))


def test_windows_and_sinks_beyond_32_bits_are_refused():
    p = Problem(dtype=BF, d=64, M=1, H=1, Hq=2, trajs=[(10, 1)]).upload()
    for kw in (dict(window=1 << 32), dict(sinks=1 << 31)):
        with pytest.raises(ValueError):
            p.call(**kw)
    p.guards()
    assert (p.out[0] == SENT).all()
    p.call(window=(1 << 31) - 1, sinks=(1 << 31) - 1)
    p.check()


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("prefix", [0, 60])
def test_queries_in_any_order(dtype, d, prefix):
    """Early queries beside ones whose window is empty: the sinks go on behind
    the end of what the early ones see."""
    order = lambda pos, W: np.resize(pos[0] + np.array([2, 300, 140, -1, 5, 170, 89, 300, 0, 133]), W)  # noqa: E731
    for window, sinks in ((1, 4), (3, 40), (50, 8), (1, 200)):
        run(window, sinks, dtype=dtype, d=d, M=1, H=2, Hq=8, trajs=[(90, 4), (90, 50), (150, 10)], qpos=order,
            prefix=prefix)
