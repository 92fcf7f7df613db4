"""Packed caches against their definition in 64 bits: writing and reading rows,
attention over them, checkpoints, and all of them together."""
import dataclasses
import threading

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_07855_gb300 import commitkv as ck  # noqa: E402

import packed_ref as ref  # noqa: E402
from attention_ref import check, positions  # noqa: E402

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
TYPES = [(F32, 64), (F32, 128), (BF, 64), (BF, 128)]
IDS = ["f32-64", "f32-128", "bf16-64", "bf16-128"]
LAYOUTS = ["dense", "tokens", "padded", "odd"]
NAMES = ("k", "v", "k_scale", "v_scale")


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


def special_rows(n, d, dtype, seed):
    """[n][d]: rows of every size, ties, zeros, infinities and NaN."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, d, generator=g, dtype=torch.float64)
    for i in range(n):
        k = i % 12
        if k == 1:
            x[i] = 0
        elif k == 2:
            x[i] *= 10.0 ** (-(i % 9) - 2)  # down to numbers that fp32 holds and sigma does not
        elif k == 3:
            x[i] *= 10.0 ** (i % 6 + 1)  # saturates
        elif k == 4:  # quotients of whole and half numbers: ties of codes and of scales
            x[i] = torch.randint(-60, 61, (d,), generator=g).double() / 8
        elif k == 5:
            x[i] = torch.randint(-28, 29, (d,), generator=g).double() * 2.0 ** (i % 17 - 12) * 7 / 4
        elif k == 6:
            x[i, i % d] = float("inf") if i % 5 else float("nan")
        elif k == 7:
            x[i, ::3] = -0.0
            x[i, d // 2:] = 3.0e38
        elif k == 8:
            x[i] = 1e-39 if dtype is F32 else 0.5
        elif k == 9:
            x[i, :4] *= 40
    return x.to(dtype)


class Cache:
    """A packed cache with data on the host (codes and scales, numpy) and the device."""

    def __init__(self, M, H, S, d, layout="dense", seed=0, codes=None):
        rng = np.random.RandomState(seed)
        if codes is None:
            codes = [ref.pack(rng.randn(M, H, S, d) * (1 + 3 * (np.arange(d) % 40 == 3))) for _ in range(2)]
        self.host = {"k": codes[0][0], "v": codes[1][0], "k_scale": codes[0][1], "v_scale": codes[1][1]}
        self.layout = layout

    def upload(self, **more):
        self.dev = {n: ref.layout(torch.from_numpy(self.host[n]), self.layout) for n in NAMES}
        self.t = ck.PackedTensors(**self.dev, **more)
        return self.t

    def values(self):
        return ref.values(self.host["k"], self.host["k_scale"]), ref.values(self.host["v"], self.host["v_scale"])

    def now(self):
        return {n: self.dev[n].cpu().numpy() for n in NAMES}


def whole(x):
    """The bytes of a tensor's whole storage."""
    return torch.empty(0, dtype=torch.uint8, device=x.device).set_(x.untyped_storage())


# ------------------------------------------------------------------------------------------------ write and read
@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("src", ["dense", "tokens", "odd"])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_write(dtype, d, src, layout):
    """Codes and scales are the definition's, byte by byte; other rows and bytes between rows stay."""
    M, H, S = 2, 3, 90
    shape = ck.make_shape(M, H, 2 * H, d, dtype)
    for first, n in ((0, 90), (3, 67), (89, 1), (40, 0)):
        c = Cache(M, H, S, d, layout, seed=n)
        t = c.upload()
        x = [torch.stack([special_rows(H * n, d, dtype, 5 * l + kv).view(H, n, d) for l in range(M)]) for kv in range(2)]
        before = {name: whole(c.dev[name]).clone() for name in NAMES}
        k, v = (ref.layout(y, src) for y in x)
        if n == 0:
            k, v = (torch.empty(M, H, 0, d, dtype=dtype, device="cuda") for _ in range(2))
        ck.commitkv_packed_write(shape, [t], [k], [v], [first])
        torch.cuda.synchronize()
        got = c.now()
        for name, y in zip("kv", x):
            codes, scales = ref.pack(ref.numbers(y))
            want = {name: c.host[name].copy(), name + "_scale": c.host[name + "_scale"].copy()}
            if n:
                want[name][:, :, first:first + n] = codes
                want[name + "_scale"][:, :, first:first + n] = scales
            for key, w in want.items():
                assert np.array_equal(got[key], w), (key, first, n)
                c.dev[key].copy_(torch.from_numpy(c.host[key]).cuda())
                assert torch.equal(whole(c.dev[key]), before[key]), "written outside the rows"


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dst", LAYOUTS)
def test_read(dtype, d, layout, dst):
    """Every code with every scale byte comes back exactly."""
    M, H, S = 1, 2, 16 * 256 // (d // 32) // 2
    rng = np.random.RandomState(1)
    codes = np.zeros((M, H, S, d // 2), np.uint8)
    scales = rng.permutation(np.tile(np.arange(256, dtype=np.uint8), H * S * d // 32 // 256)).reshape(M, H, S, d // 32)
    both = rng.randint(0, 256, codes.shape).astype(np.uint8)
    c = Cache(M, H, S, d, layout, codes=[(both, scales), (both[..., ::-1].copy(), scales[..., ::-1].copy())])
    t = c.upload()
    shape = ck.make_shape(M, H, H, d, dtype)
    for first, n in ((0, S), (7, 33), (S - 1, 1)):
        k, v = (ref.layout(torch.full((M, H, n, d), 77.0, dtype=dtype), dst) for _ in range(2))
        old = [whole(x).clone() for x in (k, v)]
        ck.commitkv_packed_read(shape, [t], [k], [v], [first])
        torch.cuda.synchronize()
        for got, want, o in zip((k, v), c.values(), old):
            assert np.array_equal(ref.numbers(got), want[:, :, first:first + n], equal_nan=True)
            got.fill_(77.0)
            assert torch.equal(whole(got), o), "written outside the rows"


def test_batches_layers_and_streams():
    """Trajectories of many lengths in one call, some without rows; a layer mask; another stream; a captured call whose
    inputs change between replays."""
    M, H, d = 3, 2, 128
    shape = ck.make_shape(M, H, 8, d, BF)
    sizes = [(50, 10, 33), (1, 0, 1), (40, 40, 0), (200, 5, 190), (0, 0, 0), (64, 1, 63)] + [(9, 8, 1)] * 58
    caches = [Cache(M, H, S, d, LAYOUTS[i % 3], seed=i) for i, (S, _, _) in enumerate(sizes)]
    ts = [c.upload() for c in caches]
    new = [[torch.randn(M, H, n, d, device="cuda").to(BF) for _, _, n in sizes] for _ in range(2)]
    rows = ck.packed_rows(shape, ts, *new, [f for _, f, _ in sizes])
    back = [[torch.full_like(x, 5.0) for x in y] for y in new]
    read = ck.packed_rows(shape, ts, *back, [f for _, f, _ in sizes])

    def expect(mask):
        for c, (S, f, n), x, y, bk, bv in zip(caches, sizes, *new, *back):
            got = c.now()
            for name, z, b in (("k", x, bk), ("v", y, bv)):
                codes, scales = ref.pack(ref.numbers(z))
                for l in range(M):
                    want = c.host[name][l].copy(), c.host[name + "_scale"][l].copy()
                    if mask[l]:
                        want[0][:, f:f + n], want[1][:, f:f + n] = codes[l], scales[l]
                        assert np.array_equal(ref.numbers(b[l]), ref.values(codes[l], scales[l]))
                    else:
                        assert (b[l] == 5.0).all()
                    assert np.array_equal(got[name][l], want[0]) and np.array_equal(got[name + "_scale"][l], want[1])

    mask = [True, False, True]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ck.commitkv_packed_write(shape, rows, layer_mask=mask)
        ck.commitkv_packed_read(shape, read, layer_mask=mask)
    s.synchronize()
    expect(mask)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ck.commitkv_packed_write(shape, rows)
        ck.commitkv_packed_read(shape, read)
    for i in range(2):
        for x in new[0] + new[1]:
            x.copy_(torch.randn_like(x, dtype=torch.float32) * (i + 1))
        g.replay()
        torch.cuda.synchronize()
        expect([True] * M)
    read.set_rows(3, 7, 2)
    ck.commitkv_packed_read(shape, read)
    assert np.array_equal(ref.numbers(back[0][3].flatten()[:d]), ref.values(*ref.pack(ref.numbers(new[0][3][0, 0, 2])))[:d])
    for bad in ((3, 199, 2), (3, -1, 2), (3, 0, 191)):
        with pytest.raises(ValueError):
            read.set_rows(*bad)


def test_rows_beyond_32_bits():
    """Tokens more than 2^31 bytes and elements apart, in the cache and in the rows."""
    d, H = 128, 1
    far = (1 << 31) + 4096
    n = 3
    base = torch.zeros(2 * far + 256, dtype=torch.uint8, device="cuda")
    codes = [base[o:].as_strided((1, H, n, d // 2), (0, 0, far, 1)) for o in (0, 64)]
    scales = [torch.zeros(1, H, n, d // 32, dtype=torch.uint8, device="cuda") for _ in range(2)]
    t = ck.PackedTensors(*codes, *scales, i32(np.arange(n)))
    wide = torch.zeros(2 * far + 256, dtype=BF, device="cuda")
    k, v = (wide[o:].as_strided((1, H, n, d), (0, 0, far, 1)) for o in (0, 128))
    k.copy_(torch.randn(1, H, n, d))
    v.copy_(torch.randn(1, H, n, d))
    shape = ck.make_shape(1, H, 4, d, BF)
    ck.commitkv_packed_write(shape, [t], [k], [v], [0])
    for c, s, x in zip(codes, scales, (k, v)):
        want = ref.pack(ref.numbers(x))
        assert np.array_equal(c.cpu().numpy(), want[0]) and np.array_equal(s.cpu().numpy(), want[1])
    want = [ref.values(*ref.pack(ref.numbers(x))) for x in (k, v)]
    ck.commitkv_packed_read(shape, [t], [k], [v], [0])
    assert all(np.array_equal(ref.numbers(x), w) for x, w in zip((k, v), want))
    Q, p = torch.randn(1, 4, 1, d, device="cuda").to(BF), i32([n])
    for W in (1, 5):  # attention over the same cache
        q, p = torch.randn(1, 4, W, d, device="cuda").to(BF), i32([n] * W)
        tr = ck.PackedTensors(*codes, *scales, i32(np.arange(n)), q, p)
        out, lse = torch.empty_like(q), torch.empty(1, 4, W, device="cuda")
        ck.commitkv_packed_attention(shape, [tr], [out], [lse], workspace=ck.alloc_packed_workspace(shape, [tr]))
        o, l, to, tl = ref.attention(*want, np.arange(n), q, [n] * W, weights=2.0 ** -8)
        check(out, o, to)
        check(lse, l, tl)


# ------------------------------------------------------------------------------------------------ attention
@pytest.fixture(params=["", "tiles", "full", "cuda_cores"])
def kernels(request, monkeypatch):
    """On the kernels that the library picks; from 17 rows on, those of row tiles on the codes, and those of full-width
    caches; the CUDA cores."""
    if request.param == "cuda_cores":
        monkeypatch.setenv("COMMITKV_SCORING", "simt")
    elif request.param:
        monkeypatch.setenv("COMMITKV_ATTENTION", request.param)
    return request.param


class Problem:
    """Trajectories (S, W) with their data on the host, and the call on the device."""

    def __init__(self, dtype, d, M, H, Hq, trajs, gaps=1.0, layout="dense", seed=0, qpos=None, spread=1.0, scale=0.0,
                 edit=None):
        self.shape, self.dtype, self.scale = ck.make_shape(M, H, Hq, d, dtype, scale), dtype, scale
        g = torch.Generator().manual_seed(seed + 99)
        self.host = []
        for i, (S, W) in enumerate(trajs):
            c = Cache(M, H, S, d, layout, seed + 10 * i)
            pos = positions(S, 0, gaps, 16, seed + i)
            Q = (spread * torch.randn(M, Hq, W, d, generator=g)).to(dtype)
            last = int(pos[-1]) if S else 0
            self.host.append([c, pos, Q, np.arange(last - W + 1, last + 1) if qpos is None else np.asarray(qpos(pos, W))])
        if edit:
            edit(self)
        self.SENT = 12352.0

    def upload(self):
        self.trajs = [c.upload(pos=i32(pos), q=Q.cuda().contiguous(), q_pos=i32(p)) for c, pos, Q, p in self.host]
        sizes = [t.q.numel() for t in self.trajs]
        d = self.shape.head_dim
        # outputs side by side with values between them that must stay
        self.flat = torch.full((sum(sizes) + 64 * (len(sizes) + 1),), self.SENT, dtype=self.dtype, device="cuda")
        self.flat_l = torch.full((sum(sizes) // d + 64 * (len(sizes) + 1),), self.SENT, device="cuda")
        self.out, self.lse, a, b = [], [], 64, 64
        for t, m in zip(self.trajs, sizes):
            self.out.append(self.flat[a:a + m].view(t.q.shape))
            self.lse.append(self.flat_l[b:b + m // d].view(t.q.shape[:3]))
            a, b = a + m + 64, b + m // d + 64
        self.ws = ck.alloc_packed_workspace(self.shape, self.trajs)
        return self

    def call(self, window=0, sinks=0, lse=True, **kw):
        ck.commitkv_packed_attention(self.shape, self.trajs, out=self.out, lse_out=self.lse if lse else None, window=window,
                                     sinks=sinks, workspace=self.ws, **kw)

    def check(self, window=0, sinks=0, layers=None, lse=True):
        torch.cuda.synchronize()
        assert ck.commitkv_workspace_status(self.ws) == ck.COMMITKV_OK
        pick = slice(None) if layers is None else layers
        for i, (c, pos, Q, p) in enumerate(self.host):
            if Q.numel() == 0:
                continue
            k, v = (x[pick] for x in c.values())
            # up to 16 rows of bf16: weights as one fp16 term, 2^-12 at most; more: rounded to bf16 (2^-8 at most).
            # fp32: weights and queries as two fp16 terms (2^-22) or three bf16 ones (2^-25, and the values too)
            few = (Q.shape[1] // k.shape[1]) * Q.shape[2] <= 16
            w, q = (2.0 ** -12 if few else 2.0 ** -8, 0.0) if self.dtype == BF else (2.0 ** -21, 2.0 ** -21)
            o, l, to, tl = ref.attention(k, v, pos, Q[pick], p, window, sinks, self.scale, w, q)
            check(self.out[i][pick], o, to, "out %d" % i)
            if lse:
                check(self.lse[i][pick], l, tl, "lse %d" % i)
        self.guards()

    def guards(self):
        for flat, step in ((self.flat, 1), (self.flat_l, self.shape.head_dim)):
            a = 0
            for t in self.trajs:
                assert (flat[a:a + 64] == self.SENT).all(), "written outside the outputs"
                a += 64 + t.q.numel() // step
            assert (flat[a:] == self.SENT).all(), "written outside the outputs"


def run(window=0, sinks=0, **kw):
    p = Problem(**kw).upload()
    p.call(window, sinks)
    p.check(window, sinks)
    return p


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("S", [1, 2, 7, 31, 33, 127, 128, 129, 640, 1025])
def test_single_token_lengths(dtype, d, S, kernels):
    run(dtype=dtype, d=d, M=1, H=2, Hq=8, trajs=[(S, 1)], gaps=0.5)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [2, 3, 4, 5, 17, 65, 130])
def test_prompt_lengths(dtype, d, W, kernels):
    run(dtype=dtype, d=d, M=2, H=1, Hq=4, trajs=[(W + 150, W)], gaps=0.6)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("H,Hq", [(1, 1), (2, 2), (1, 3), (2, 10), (1, 8), (1, 9), (1, 16), (1, 40)])
@pytest.mark.parametrize("W", [1, 6])
def test_heads(dtype, d, H, Hq, W, kernels):
    run(dtype=dtype, d=d, M=2, H=H, Hq=Hq, trajs=[(201, W)], window=150, sinks=3)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (64, 0), (100, 5), (128, 4), (300, 200), (1000, 64),
                                          (2**31 - 1, 2**31 - 1)])
@pytest.mark.parametrize("W,gaps", [(1, 0.4), (4, 1.0), (40, 0.4)])
def test_windows(dtype, d, window, sinks, W, gaps, kernels):
    run(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(700, W), (333, W)], gaps=gaps, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
def test_ragged_batch(dtype, d, kernels):
    """Lengths from none to long ones, trajectories without queries or tokens."""
    run(dtype=dtype, d=d, M=1, H=2, Hq=4, gaps=0.7, window=200, sinks=4,
        trajs=[(0, 3), (1, 1), (500, 1), (64, 64), (300, 0), (1400, 33), (0, 0), (257, 2), (129, 129)])


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n", [17, 64])
def test_many_trajectories(dtype, d, n, kernels):
    run(dtype=dtype, d=d, M=1, H=1, Hq=2, trajs=[(5 + 13 * i, 1) for i in range(n)])


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 4, 48])
def test_rows_that_see_nothing(dtype, d, W, kernels):
    """Queries before the first token, behind the last window, in any order."""
    def qpos(pos, W):
        return np.array([1000, 3, 99, 100, 101, 5000, 100 + len(pos), 350] * 6, np.int64)[:W] if W > 1 else [3]

    def late(p):
        for t in p.host:
            t[1] = t[1] + 100

    p = run(dtype=dtype, d=d, M=1, H=2, Hq=4, trajs=[(400, W)], qpos=qpos, window=120, edit=late)
    assert torch.isinf(p.lse[0][:, :, 1 if W > 1 else 0]).all() and (p.out[0][:, :, 1 if W > 1 else 0] == 0).all()
    run(dtype=dtype, d=d, M=1, H=2, Hq=4, trajs=[(400, W)], qpos=qpos, window=120, sinks=130, edit=late)
    run(dtype=dtype, d=d, M=1, H=2, Hq=4, trajs=[(400, W)], qpos=qpos, edit=late)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 24])
def test_far_positions(dtype, d, W, kernels):
    """Positions up to the largest int32."""
    def far(p):
        for t in p.host:
            move = 2**31 - 1 - int(t[1][-1])
            t[1], t[3] = t[1] + move, t[3] + move

    run(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(500, W)], gaps=0.5, edit=far)
    run(dtype=dtype, d=d, M=1, H=1, Hq=4, trajs=[(500, W)], gaps=0.5, edit=far, window=77)


@pytest.mark.parametrize("layout", ["tokens", "padded", "odd"])
@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 3, 40])
def test_layouts(dtype, d, layout, W, kernels):
    """Tokens outermost, rows with room behind them (NaN scales behind the last token), odd addresses."""
    run(dtype=dtype, d=d, M=2, H=2, Hq=6, trajs=[(300, W), (77, W)], layout=layout, gaps=0.5, window=111, sinks=2)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 4, 40])
def test_scales_that_are_not_numbers(dtype, d, W, kernels):
    """NaN scales: of masked tokens they reach nothing, of visible values their 32 channels of the rows that see them, of
    visible keys the whole rows."""
    groups = d // 32

    def bad(p):
        for n, (c, pos, Q, qp) in enumerate(p.host):
            S = len(pos)
            c.host["v_scale"][0, 0, 5, 1] = 0xff       # beyond the window, and no sink
            c.host["k_scale"][0, 0, 6, 0] = 0xf8
            c.host["v_scale"][0, 0, 0, groups - 1] = 0xf9 if n else 0x20  # a sink
            c.host["v_scale"][0, 1, S - 1, 0] = 0xff   # the last token: only the last query sees it
            c.host["k_scale"][1, 0, S - 1, 1] = 0xff
            c.host["v_scale"][1, 1, S - 60, :] = 0xfc  # all of a token in the window
            c.host["k_scale"][1, 1, 2, 0] = 0xff       # the first token that is no sink

    p = run(dtype=dtype, d=d, M=2, H=2, Hq=4, trajs=[(300, W), (423, W)], window=100, sinks=2, edit=bad)
    out = p.out[0].float()
    assert torch.isfinite(out[0, :2]).all() and torch.isnan(out[0, 2:, -1, :32]).all()
    assert torch.isfinite(out[0, 2:, -1, 32:]).all() and torch.isnan(out[1, :2, -1]).all()
    if W > 1:
        assert torch.isfinite(out[0, 2:, :-1]).all() and torch.isfinite(out[1, :2, :-1]).all()
    assert torch.isnan(p.out[1].float()[0, :2, :, -32:]).all() and torch.isfinite(p.lse[1][0]).all()


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 4, 40])
def test_queries_that_are_not_numbers(dtype, d, W, kernels):
    """A NaN or infinite element of a query makes its rows NaN where a score is, and no other row."""
    def bad(p):
        for c, pos, Q, qp in p.host:
            Q[0, 0, 0, 3] = float("nan")
            Q[0, 2, W - 1, d - 1] = float("inf")
            c.host["k"][0, 1, :, d // 2 - 1] = np.arange(len(pos)) % 16 << 4 | 3  # codes of every sign for that channel

    run(dtype=dtype, d=d, M=1, H=2, Hq=4, trajs=[(200, W)], edit=bad)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 4, 30])
@pytest.mark.parametrize("size", [1e-30, 1e-4, 30.0, 1e4])
def test_queries_of_any_size(dtype, d, W, size, kernels):
    """One row's queries far from 1, the others ordinary; scores far apart."""
    def edit(p):
        for c, pos, Q, qp in p.host:
            Q[:, ::2] = (Q[:, ::2].double() * size).to(Q.dtype)

    run(dtype=dtype, d=d, M=1, H=2, Hq=4, trajs=[(333, W)], edit=edit)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("W", [1, 4, 30])
def test_values_of_any_size(dtype, d, W, kernels):
    """Scales from the smallest to the largest, zeros among them, all codes."""
    def edit(p):
        rng = np.random.RandomState(4)
        for c, pos, Q, qp in p.host:
            c.host["v_scale"][:] = rng.choice([0, 1, 2, 7, 8, 9, 100, 240, 247], c.host["v_scale"].shape)
            c.host["v"][:] = rng.randint(0, 256, c.host["v"].shape)
            c.host["k_scale"][:] = rng.choice([0, 1, 60, 130, 140], c.host["k_scale"].shape)
            c.host["k"][:] = rng.randint(0, 256, c.host["k"].shape)

    run(dtype=dtype, d=d, M=1, H=2, Hq=4, trajs=[(333, W)], edit=edit, scale=0.3)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("trajs", [[(900, 1), (2000, 4)], [(700, 60), (900, 1), (300, 200)]])
def test_same_bits_in_any_workspace_stream_and_graph(dtype, d, trajs, kernels):
    """The same call gives the same bits: what the workspace held, another stream, a captured call replayed over changed
    queries beside another captured call with a workspace of its own."""
    p = Problem(dtype=dtype, d=d, M=4, H=2, Hq=8, gaps=0.7, trajs=trajs).upload()
    p.call(600, 4)
    p.check(600, 4, layers=[0, 3])
    want = p.flat.clone(), p.flat_l.clone()
    p.ws[256:].fill_(0xff)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    p.flat.fill_(p.SENT), p.flat_l.fill_(p.SENT)
    torch.cuda.synchronize()
    p.call(600, 4, stream=s)
    s.synchronize()
    assert torch.equal(want[0], p.flat) and torch.equal(want[1], p.flat_l)
    other = Problem(dtype=dtype, d=d, M=4, H=2, Hq=8, gaps=0.7, trajs=trajs[:1], seed=3).upload()
    graphs = []
    for x in (p, other):
        x.batch = ck.attention_batch(x.shape, x.trajs, x.out, x.lse)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ck.commitkv_packed_attention(x.shape, x.batch, window=600, sinks=4, workspace=x.ws)
        graphs.append(g)
    for t, h in zip(p.trajs, p.host):
        h[2] = (h[2].float() * 0.5 + 0.1).to(dtype)
        t.q.copy_(h[2])
    for g in graphs:
        g.replay()
    p.check(600, 4, layers=[1])
    other.check(600, 4, layers=[1])
    got = p.flat.clone(), p.flat_l.clone()
    for g in graphs[::-1]:
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], p.flat) and torch.equal(got[1], p.flat_l)


def test_layer_masks_and_outputs_left_out(kernels):
    for trajs in ([(300, 1)], [(300, 40), (100, 1)]):
        p = Problem(dtype=BF, d=64, M=3, H=2, Hq=4, trajs=trajs).upload()
        p.call(layer_mask=[False, True, False], lse=False)
        p.check(layers=[1], lse=False)
        for out in p.out:
            assert (out[[0, 2]] == p.SENT).all()
        assert (p.flat_l == p.SENT).all()
        p.call(layer_mask=[False] * 3)
        p.check(layers=[1], lse=False)


def test_set_length(kernels):
    """Buffers with room: the batch says how many tokens they hold."""
    for W in (1, 20):
        p = Problem(dtype=BF, d=128, M=1, H=2, Hq=8, trajs=[(400, W)], qpos=lambda pos, W: [500] * W).upload()
        b = ck.attention_batch(p.shape, p.trajs, p.out, p.lse)
        for S in (400, 1, 0, 129):
            b.set_length(0, S)
            ck.commitkv_packed_attention(p.shape, b, workspace=p.ws)
            c, pos, Q, qp = p.host[0]
            k, v = (x[:, :, :S] for x in c.values())
            o, l, to, tl = ref.attention(k, v, pos[:S], Q, qp, weights=2.0 ** -8)
            check(p.out[0], o, to)
            check(p.lse[0], l, tl)


def test_attention_refusals():
    p = Problem(dtype=BF, d=64, M=1, H=1, Hq=2, trajs=[(10, 1)]).upload()
    full = ck.TrajTensors(*(torch.zeros(1, 1, 10, 64, dtype=BF, device="cuda") for _ in range(2)), p.trajs[0].pos, p.trajs[0].q,
                          p.trajs[0].q_pos)
    for kw in (dict(window=-1), dict(sinks=-1), dict(window=1 << 40), dict(sinks=1 << 31)):
        with pytest.raises((ValueError, ck.CommitKVError)):
            p.call(**kw)
    with pytest.raises(ValueError):
        ck.commitkv_packed_attention(p.shape, [full], p.out, workspace=p.ws)
    with pytest.raises(ValueError):
        ck.commitkv_window_attention(p.shape, p.trajs, p.out, workspace=p.ws)
    with pytest.raises(ValueError):
        ck.commitkv_packed_attention(p.shape, p.trajs + [full], p.out * 2, workspace=p.ws)
    with pytest.raises(ValueError):
        ck.attention_batch(p.shape, p.trajs, p.out, prefix=full)
    with pytest.raises(ck.CommitKVError):
        ck.commitkv_packed_attention(p.shape, p.trajs, p.out, workspace=p.ws[:512])
    t = p.trajs[0]
    for kw in (dict(q=t.q.float()), dict(pos=None), dict(k=t.k.repeat(1, 2, 1, 1), v=t.v.repeat(1, 2, 1, 1),
                                                          k_scale=t.k_scale.repeat(1, 2, 1, 1), v_scale=t.v_scale.repeat(1, 2, 1, 1))):
        bad = dataclasses.replace(t, **kw)
        with pytest.raises(ValueError):
            ck.commitkv_packed_attention(p.shape, [bad], p.out, workspace=p.ws)
    torch.cuda.synchronize()
    assert (p.flat == p.SENT).all() and (p.flat_l == p.SENT).all()


# ------------------------------------------------------------------------------------------------ checkpoints
def checkpoint(dtype, d, M, H, sizes, B, layout="dense", to="dense", place="dst", seed=0, cap=3, BN=None, pos=True):
    """A checkpoint of packed caches against commitkv_compact of their values, for the selection, and the rows moved."""
    rng = np.random.RandomState(seed)
    shape = ck.make_shape(M, H, H, d, dtype)
    caches = [Cache(M, H, S, d, layout, seed + i) for i, S in enumerate(sizes)]
    BN = B // 3 if BN is None else BN
    args = dict(retired=[], pending=[], prio=[], fill=[])
    full, packed = [], []
    for c, S in zip(caches, sizes):
        ps = np.arange(0, S, 16)
        pl = np.minimum(rng.randint(1, 17, len(ps)), S - ps)
        p = i32(np.cumsum(rng.randint(1, 4, S)))
        kw = dict(page_start=i32(ps), page_len=i32(pl))
        packed.append(c.upload(pos=p.clone(), **kw))
        x = torch.zeros(M, H, S, d, dtype=dtype, device="cuda")
        full.append(ck.TrajTensors(x, x, p, None, None, kw["page_start"], kw["page_len"]))
        args["retired"].append(torch.from_numpy((rng.rand(len(ps)) < 0.3).astype(np.uint8)).cuda())
        args["pending"].append(i32(rng.permutation(len(ps))[:5]))
        args["prio"].append(torch.from_numpy(rng.rand(len(ps)).astype(np.float32)).cuda())
        args["fill"].append(torch.from_numpy(rng.randint(0, S + 1, S).astype(np.float32)).cuda())
    call = [args["retired"], args["pending"], args["prio"], args["fill"], B, BN, cap]
    fresh = lambda: ([torch.full((max(B, 1),), -7, dtype=torch.int32, device="cuda")[:B] for _ in sizes],  # noqa: E731
                     torch.full((len(sizes),), -7, dtype=torch.int32, device="cuda"))
    idx, n = fresh()
    ck.commitkv_compact(shape, full, *call, idx, n, workspace=ck.alloc_workspace(shape, full))
    got, n2 = fresh()
    ws = ck.alloc_packed_workspace(shape, packed)
    olds = [{name: whole(c.dev[name]).clone() for name in NAMES} for c in caches]
    old_pos = [t.pos.clone() for t in packed]
    dst = None
    if place == "dst":
        targets = [Cache(M, H, max(1, min(B, S)), d, to, 77 + i) for i, S in enumerate(sizes)]
        dst = [t.upload(pos=torch.full((t.host["k"].shape[2],), -5, dtype=torch.int32, device="cuda") if pos else None)
               for t in targets]
        before = [{name: whole(t.dev[name]).clone() for name in NAMES} for t in targets]
    ck.commitkv_packed_compact(shape, packed, *call, got, n2, dst=dst, workspace=ws)
    torch.cuda.synchronize()
    assert ck.commitkv_workspace_status(ws) == ck.COMMITKV_OK
    assert torch.equal(n, n2)
    for i, (c, S) in enumerate(zip(caches, sizes)):
        m = int(n[i])
        assert torch.equal(idx[i], got[i]), "the selection"
        keep = idx[i][:m].cpu().numpy()
        into = targets[i] if dst else c
        now = into.now()
        for name in NAMES:
            assert np.array_equal(now[name][:, :, :m], c.host[name][:, :, keep]), name
        t = dst[i] if dst else packed[i]
        if t.pos is not None:
            assert np.array_equal(t.pos[:m].cpu().numpy(), old_pos[i].cpu().numpy()[keep])
        if dst:  # nothing else moved: the caches, the rows behind the retained ones, what lies between rows
            assert torch.equal(packed[i].pos, old_pos[i])
            assert all(torch.equal(whole(c.dev[name]), olds[i][name]) for name in NAMES)
            assert t.pos is None or (t.pos[m:] == -5).all()
            for name in NAMES:
                into.dev[name][:, :, :m].copy_(torch.from_numpy(into.host[name][:, :, :m]).cuda())
                assert torch.equal(whole(into.dev[name]), before[i][name])
        else:  # rows behind the retained ones keep stale values; what lies between rows stays
            assert all(np.array_equal(now[name][:, :, max(m, 1):], c.host[name][:, :, max(m, 1):]) for name in NAMES)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("place", ["dst", "in place"])
@pytest.mark.parametrize("layout,to", [("dense", "dense"), ("tokens", "padded"), ("odd", "dense"), ("padded", "odd")])
def test_checkpoints(dtype, d, place, layout, to):
    checkpoint(dtype, d, 2, 3, [500], 120, layout, to, place)
    checkpoint(dtype, d, 1, 2, [1300, 40, 700, 1], 333, layout, to, place, seed=1)


@pytest.mark.parametrize("place", ["dst", "in place"])
@pytest.mark.parametrize("S,B", [(1, 1), (100, 0), (100, 100), (100, 200), (9000, 8990), (9000, 700), (5000, 4096)])
def test_checkpoint_sizes(place, S, B):
    checkpoint(BF, 128, 1, 1, [S], B, place=place, pos=S != 100)
    checkpoint(BF, 64, 2, 1, [S, 3], B, place=place, seed=2)


@pytest.mark.parametrize("place", ["dst", "in place"])
def test_checkpoint_device_errors(place):
    """A NaN score ends the trajectory: nothing is retained, nothing moves, the workspace says so."""
    c = Cache(1, 1, 50, 64)
    t = c.upload(pos=i32(np.arange(50)))
    dst = [Cache(1, 1, 10, 64, seed=9).upload()] if place == "dst" else None
    shape = ck.make_shape(1, 1, 1, 64, BF)
    ws = ck.alloc_packed_workspace(shape, [t])
    none = torch.zeros(0, dtype=torch.uint8, device="cuda")
    fill = torch.rand(50, device="cuda")
    fill[7] = float("nan")
    idx, n = torch.zeros(10, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    ck.commitkv_packed_compact(shape, [t], [none], [None], [None], [fill], 10, 0, 0, [idx], n, dst=dst, workspace=ws)
    torch.cuda.synchronize()
    assert ck.commitkv_workspace_status(ws) == ck.COMMITKV_ERR_DEVICE_INPUT and int(n) == 0
    assert all(np.array_equal(x, c.host[name]) for name, x in c.now().items())


# ------------------------------------------------------------------------------------------------ together
def test_checkpoint_refusals():
    shape = ck.make_shape(2, 2, 4, 64, F32)
    c = ck.alloc_packed_cache(shape, 100)
    page = torch.tensor([0, 16], dtype=torch.int32, device="cuda")
    t = dataclasses.replace(c, page_start=page, page_len=torch.full_like(page, 16))
    i32 = dict(dtype=torch.int32, device="cuda")
    good = dict(cache=[t], retired=[torch.zeros(2, dtype=torch.uint8, device="cuda")], pending=[torch.ones(1, **i32)],
                pending_priority=[torch.zeros(2, device="cuda")], fill_score=[torch.zeros(100, device="cuda")], budget_B=10,
                pending_tokens_BN=0, pending_cap_pages=0, idx_out=[torch.empty(10, **i32)], n_idx_out=torch.empty(1, **i32),
                workspace=ck.alloc_packed_workspace(shape, [t]))
    ck.commitkv_packed_compact(shape, **good)
    bad = [dict(workspace=None), dict(workspace=good["workspace"].cpu()), dict(dst=[]), dict(cache=[]), dict(retired=[]),
           dict(pending=[]), dict(pending_priority=[]), dict(fill_score=[]), dict(idx_out=[]), dict(cache=[object()]),
           dict(retired=[None]), dict(retired=[good["retired"][0][:1]]), dict(retired=[good["retired"][0].int()]),
           dict(pending=[good["pending"][0].long()]), dict(pending_priority=[None]), dict(pending_priority=[good["fill_score"][0][:1]]),
           dict(fill_score=[None]), dict(fill_score=[torch.zeros(99, device="cuda")]), dict(fill_score=[torch.zeros(200, device="cuda")[::2]]),
           dict(idx_out=[torch.empty(9, **i32)]), dict(n_idx_out=torch.empty(0, **i32)), dict(n_idx_out=torch.empty(1)),
           dict(fill_score=[torch.zeros(100)]), dict(dst=[ck.alloc_packed_cache(ck.make_shape(1, 2, 4, 64, F32), 100)])]
    for kw in bad:
        with pytest.raises(ValueError):
            ck.commitkv_packed_compact(shape, **{**good, **kw})
    with pytest.raises(ck.CommitKVError):  # no room
        ck.commitkv_packed_compact(shape, **good, dst=[ck.alloc_packed_cache(shape, 9)])


@pytest.mark.parametrize("dtype", [F32, BF], ids=["f32", "bf16"])
def test_write_attend_compact_attend(dtype, kernels):
    """A prompt written and attended to, a checkpoint in place, decoded tokens after it: against a cache of the values
    themselves, which the full-width calls hold."""
    M, H, Hq, d, B = 2, 2, 8, 128, 200
    shape = ck.make_shape(M, H, Hq, d, dtype)
    cache = ck.alloc_packed_cache(shape, 600)
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    S, at = 0, 0
    for n in (300, 1, 40, 3, 1):
        new = [rand(M, H, n, d) for _ in range(2)]
        ck.commitkv_packed_write(shape, [cache], [new[0]], [new[1]], [S])
        cache.pos[S:S + n] = torch.arange(at, at + n, device="cuda", dtype=torch.int32)
        S, at = S + n, at + n
        view = lambda x: x[:, :, :S]  # noqa: E731, B023
        Q, p = rand(M, Hq, n, d), i32(np.arange(at - n, at))
        t = ck.PackedTensors(view(cache.k), view(cache.v), view(cache.k_scale), view(cache.v_scale), cache.pos[:S], Q, p)
        ws = ck.alloc_packed_workspace(shape, [t])
        out, lse = torch.empty_like(Q), torch.empty(M, Hq, n, device="cuda")
        ck.commitkv_packed_attention(shape, [t], [out], [lse], window=150, sinks=4, workspace=ws)
        k, v = (torch.empty(M, H, S, d, dtype=dtype, device="cuda") for _ in range(2))
        ck.commitkv_packed_read(shape, [t], [k], [v], [0])
        o, l, to, tl = ref.attention(ref.numbers(k), ref.numbers(v), cache.pos[:S].cpu().numpy(), Q, p.cpu().numpy(), 150, 4,
                                     weights=2.0 ** -8 if dtype == BF else 2.0 ** -21, queries=2.0 ** -21)
        check(out, o, to)
        check(lse, l, tl)
        last = [ref.values(*ref.pack(ref.numbers(x))) for x in new]
        assert all(np.array_equal(ref.numbers(x[:, :, S - n:]), y) for x, y in zip((k, v), last))
        if n == 40:
            idx, n_idx = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
            none = torch.zeros(0, dtype=torch.uint8, device="cuda")
            ck.commitkv_packed_compact(shape, [t], [none], [None], [None], [torch.rand(S, generator=g, device="cuda")], B, 0, 0,
                                       [idx], n_idx, workspace=ws)
            S = B
            kept = [torch.empty(M, H, B, d, dtype=dtype, device="cuda") for _ in range(2)]
            ck.commitkv_packed_read(shape, [cache], [kept[0]], [kept[1]], [0])
            assert all(torch.equal(x, y[:, :, idx.long()]) for x, y in zip(kept, (k, v)))


def far_cache(n, d, seed):
    """Tokens more than 2^31 bytes apart, codes and scale bytes, of one layer and head."""
    far = (1 << 31) + 4096
    base = torch.zeros((n - 1) * far + 256, dtype=torch.uint8, device="cuda")
    c = Cache(1, 1, n, d, seed=seed)
    c.dev = {}
    for name, at in zip(NAMES, (0, 64, 128, 160)):
        c.dev[name] = base[at:].as_strided((1, 1, n, c.host[name].shape[3]), (0, 0, far, 1))
        c.dev[name].copy_(torch.from_numpy(c.host[name]))
    return c


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
def test_attention_beyond_32_bits(dtype, d, kernels):
    n = 5
    c = far_cache(n, d, 3)
    shape = ck.make_shape(1, 1, 4, d, dtype)
    pos = np.arange(n)
    for W in (1, 4, 40):
        q, p = torch.randn(1, 4, W, d, device="cuda").to(dtype), [n] * W
        tr = ck.PackedTensors(**c.dev, pos=i32(pos), q=q, q_pos=i32(p))
        out, lse = torch.empty_like(q), torch.empty(1, 4, W, device="cuda")
        ck.commitkv_packed_attention(shape, [tr], [out], [lse], workspace=ck.alloc_packed_workspace(shape, [tr]))
        few = 4 * W <= 16
        w, e = (2.0 ** -12 if few else 2.0 ** -8, 0.0) if dtype == BF else (2.0 ** -21, 2.0 ** -21)
        o, l, to, tl = ref.attention(*c.values(), pos, q.cpu(), p, 0, 0, 0.0, w, e)
        check(out, o, to)
        check(lse, l, tl)


@pytest.mark.parametrize("place", ["dst", "in place"])
def test_checkpoint_beyond_32_bits(place):
    n, B = 5, 3
    c = far_cache(n, 64, 4)
    shape = ck.make_shape(1, 1, 1, 64, BF)
    none = torch.zeros(0, dtype=torch.uint8, device="cuda")
    t = ck.PackedTensors(**c.dev, pos=i32(10 + np.arange(n)))
    idx, m = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    to = far_cache(B, 64, 5) if place == "dst" else c
    dst = [ck.PackedTensors(**to.dev, pos=i32(np.zeros(B)))] if place == "dst" else None
    ck.commitkv_packed_compact(shape, [t], [none], [None], [None], [torch.tensor([1.0, 5, 2, 4, 3], device="cuda")], B, 0, 0,
                               [idx], m, dst=dst, workspace=ck.alloc_packed_workspace(shape, [t]))
    keep = idx.cpu().numpy()
    assert int(m) == B and sorted(keep) == list(keep) and len(set(keep)) == B
    now = to.now()
    assert all(np.array_equal(now[name][:, :, :B], c.host[name][:, :, keep]) for name in NAMES)
    assert np.array_equal((dst or [t])[0].pos[:B].cpu().numpy(), 10 + keep)


def test_two_threads(kernels):
    """Calls of two host threads at once, each with a stream and a workspace of its own."""
    a = Problem(dtype=BF, d=128, M=2, H=2, Hq=8, gaps=0.7, trajs=[(900, 1), (2000, 4), (500, 40)]).upload()
    b = Problem(dtype=F32, d=64, M=3, H=1, Hq=4, gaps=0.7, trajs=[(700, 60), (900, 2)], seed=3).upload()
    want = []
    for p in (a, b):
        p.call(300, 4)
        p.check(300, 4)
        want.append((p.flat.clone(), p.flat_l.clone()))
        p.flat.fill_(p.SENT), p.flat_l.fill_(p.SENT)
    torch.cuda.synchronize()
    failed = []

    def work(p, want):
        try:
            s = torch.cuda.Stream()
            for _ in range(50):
                p.call(300, 4, stream=s)
            s.synchronize()
            assert torch.equal(p.flat, want[0]) and torch.equal(p.flat_l, want[1])
        except BaseException as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=x) for x in zip((a, b), want)]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    assert not failed


def test_captured_checkpoint():
    """Append, checkpoint and read back as one graph, replayed over new rows and scores."""
    M, H, S, d, B = 2, 2, 300, 64, 50
    shape = ck.make_shape(M, H, H, d, BF)
    t, dst = ck.alloc_packed_cache(shape, S), ck.alloc_packed_cache(shape, B)
    t.pos.copy_(i32(np.arange(S)))
    k, v = (torch.randn(M, H, S, d, device="cuda").to(BF) for _ in range(2))
    got = [torch.zeros(M, H, B, d, dtype=BF, device="cuda") for _ in range(2)]
    none = torch.zeros(0, dtype=torch.uint8, device="cuda")
    fill = torch.rand(S, device="cuda")
    idx, m = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = ck.alloc_packed_workspace(shape, [t])
    write, read = ck.packed_rows(shape, [t], [k], [v], [0]), ck.packed_rows(shape, [dst], [got[0]], [got[1]], [0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ck.commitkv_packed_write(shape, write)
        ck.commitkv_packed_compact(shape, [t], [none], [None], [None], [fill], B, 0, 0, [idx], m, dst=[dst], workspace=ws)
        ck.commitkv_packed_read(shape, read)
    for seed in range(3):
        r = torch.Generator(device="cuda").manual_seed(seed)
        fill.copy_(torch.randperm(S, generator=r, device="cuda").float())
        k.copy_(torch.randn(M, H, S, d, generator=r, device="cuda"))
        v.copy_(torch.randn(M, H, S, d, generator=r, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        keep = fill.topk(B).indices.sort().values
        assert int(m) == B and torch.equal(idx, keep.int()) and torch.equal(dst.pos, keep.int())
        for x, y in zip((k, v), got):
            want = ref.values(*ref.pack(ref.numbers(x[:, :, keep].contiguous())))
            assert np.array_equal(ref.numbers(y), want)
