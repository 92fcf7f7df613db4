"""Packed caches where single rows, queries and weights are out of the ordinary."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_07855_gb300 import commitkv as ck  # noqa: E402
from paper_2608_07855_gb300.lifecycle import Session  # noqa: E402

import packed_ref as ref  # noqa: E402
from attention_ref import check  # noqa: E402
from test_gpu_packed import BF, F32, IDS, NAMES, TYPES, Problem, i32, kernels, run  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def rows_and_kernels(*Ws):
    """W positions of 4 heads to one, on each set of kernels that takes them."""
    return pytest.mark.parametrize("W,kernels", [(W, how) for W in Ws for how in
                                                 (("", "cuda_cores") if W <= 4 else ("", "tiles", "full", "cuda_cores"))],
                                   indirect=["kernels"])


# ------------------------------------------------------------------------------------------------ queries
@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@rows_and_kernels(1, 3, 8, 40)
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


# ------------------------------------------------------------------------------------------------ single tokens
def by_tokens(x):
    return x.transpose(1, 2).contiguous().transpose(1, 2)


def odd(x):
    """x with strides of single entries that mean nothing."""
    return x.as_strided(x.shape, [s if n > 1 else 7 for n, s in zip(x.shape, x.stride())])


def rand(*shape, dtype):
    return torch.randn(*shape, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("M,H", [(3, 2), (1, 2), (3, 1), (1, 1)])
def test_a_sessions_single_token_in_any_layout(dtype, d, M, H):
    """K made anew by a rotary embedding, V a view of a projection, and the other way round; all layers and one by one."""
    shape = ck.make_shape(M, H, 2 * H, d, dtype)
    pos = i32([0])
    for lay in ((odd, by_tokens), (by_tokens, odd), (lambda x: x, odd), (odd, lambda x: x),
                (by_tokens, lambda x: torch.cat([x, x, x], 2)[:, :, 1:2])):
        K, V = (f(rand(M, H, 1, d, dtype=dtype)) for f in lay)
        s = Session(shape, 16, 40, 0.2, 50, packed=True)
        s.append(K, V, pos, [], decoded=1)
        s.append(None, None, pos + 1, [], decoded=1)
        for layer in range(M):
            s.fill(layer, K[layer], V[layer])
        assert s.S == 2 and s.decoded_since == 2
        for x, codes, scales in ((K, s.packed.k, s.packed.k_scale), (V, s.packed.v, s.packed.v_scale)):
            want = ref.pack(ref.numbers(x))
            for i in range(2):
                assert np.array_equal(codes[:, :, i:i + 1].cpu().numpy(), want[0])
                assert np.array_equal(scales[:, :, i:i + 1].cpu().numpy(), want[1])


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("M,H,S", [(1, 2, 1), (2, 1, 1), (1, 1, 1), (1, 2, 5), (3, 1, 5)])
def test_strides_of_single_entries_mean_nothing(dtype, d, M, H, S):
    """Written, read, attended to and compacted, K and V alike but for such strides."""
    shape = ck.make_shape(M, H, 4 * H, d, dtype)
    c = ck.alloc_packed_cache(shape, S)
    pos = i32(np.arange(S))
    q, p = rand(M, 4 * H, 1, d, dtype=dtype), i32([S])
    t = ck.PackedTensors(c.k, odd(c.v), odd(c.k_scale), c.v_scale, pos, q, p)
    K, V = rand(M, H, S, d, dtype=dtype), odd(rand(M, H, S, d, dtype=dtype))
    ck.commitkv_packed_write(shape, [t], [K], [V], [0])
    values = []
    for x, codes, scales in ((K, t.k, t.k_scale), (V, t.v, t.v_scale)):
        want = ref.pack(ref.numbers(x))
        assert np.array_equal(codes.cpu().numpy(), want[0]) and np.array_equal(scales.cpu().numpy(), want[1])
        values.append(ref.values(*want))
    back = odd(torch.zeros_like(K)), torch.zeros_like(K)
    ck.commitkv_packed_read(shape, [t], [back[0]], [back[1]], [0])
    assert all(np.array_equal(ref.numbers(x), w) for x, w in zip(back, values))
    out, lse = torch.empty_like(q), torch.empty(M, 4 * H, 1, device="cuda")
    ws = ck.alloc_packed_workspace(shape, [t])
    ck.commitkv_packed_attention(shape, [t], [out], [lse], workspace=ws)
    few = dict(weights=2.0 ** -11) if dtype is BF else dict(weights=2.0 ** -21, queries=2.0 ** -21)
    o, l, to, tl = ref.attention(*values, np.arange(S), q, [S], **few)
    check(out, o, to)
    check(lse, l, tl)
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    to_ = ck.alloc_packed_cache(shape, S)
    dst = ck.PackedTensors(odd(to_.k), to_.v, to_.k_scale, odd(to_.v_scale), to_.pos)
    idx, n = i32(np.zeros(S)), i32([0])
    ck.commitkv_packed_compact(shape, [t], [none], [None], [None], [torch.rand(S, device="cuda")], S, 0, 0, [idx], n, [dst],
                               workspace=ws)
    assert n.item() == S and all(torch.equal(getattr(dst, a), getattr(t, a)) for a in ("k", "v", "k_scale", "v_scale", "pos"))


# ------------------------------------------------------------------------------------------------ weights
@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@rows_and_kernels(1, 4, 40)
@pytest.mark.parametrize("S", [700, 2000])
@pytest.mark.parametrize("scales", ["usual", "small", "nan"])
def test_weights_far_below_the_largest(dtype, d, W, S, scales, kernels):  # noqa: F811
    """One of 32 tokens, of values 0, has nearly all of the weight, the others 2^-31.5 or 2^-33.9 of it and positive
    values: each weight is off by 2^-36 of the largest at most, whatever scales stand beside it (some below 32, or
    some of values NaN)."""
    def edit(p):
        rng = np.random.RandomState(S + d)
        for c, pos, Q, qp in p.host:
            c.host["k_scale"][:] = c.host["v_scale"][:] = 168                        # sigma 1
            c.host["k"][:] = 0x88
            c.host["k"][..., 0] = 0x80 | rng.choice([1, 2], c.host["k"].shape[:3])  # channel 0: -7, -6
            c.host["v"][:] = 0xff
            c.host["k"][:, :, 5::32, 0], c.host["v"][:, :, 5::32] = 0x8f, 0x88      # 7; values 0
            if scales == "small":
                c.host["k_scale"][:, :, ::7, 1] = 9
                c.host["v_scale"][:, :, 5::32] = 1
            elif scales == "nan":
                c.host["v_scale"][:, :, ::31, 0] = 0xff
            Q[:] = 0
            Q[..., 0] = 1.6796875                                                    # 2^-2.423 a step of the code

    p = Problem(dtype=dtype, d=d, M=1, H=2, Hq=8, trajs=[(S, W)], edit=edit, scale=1.0).upload()
    p.call(S - 30, 6)
    p.check(S - 30, 6)
    assert (p.out[0][..., 32:].float() > 1e-9).all()
    if scales == "nan":
        assert torch.isnan(p.out[0][..., :32]).all()


# ------------------------------------------------------------------------------------------------ calls
@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@rows_and_kernels(1, 4, 40)
@pytest.mark.parametrize("spread", [6.0, 40.0])
def test_peaked_rows(dtype, d, W, spread, kernels):  # noqa: F811
    """Scores far apart: the reference is raised often, the chunks of a row differ."""
    run(dtype=dtype, d=d, M=1, H=2, Hq=8, trajs=[(1500, W), (200, W)], gaps=0.6, spread=spread)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@rows_and_kernels(1, 4, 40)
@pytest.mark.parametrize("dims", ["heads", "layers", "both"])
def test_caches_that_heads_or_layers_share(dtype, d, W, dims, kernels):  # noqa: F811
    """Strides of 0, of expanded views."""
    def cut(x):
        return x[:1 if dims != "heads" else None, :1 if dims != "layers" else None]

    def edit(p):
        for c, pos, Q, qp in p.host:
            for n in NAMES:
                c.host[n][:] = cut(c.host[n])

    p = Problem(dtype=dtype, d=d, M=2, H=2, Hq=8, trajs=[(300, W)], gaps=0.6, edit=edit).upload()
    t = p.trajs[0]
    p.trajs = [dataclasses.replace(t, **{n: cut(getattr(t, n)).expand_as(getattr(t, n)) for n in NAMES})]
    p.call(200, 3)
    p.check(200, 3)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@rows_and_kernels(1, 3, 40)
@pytest.mark.parametrize("what", ["q", "out", "both"])
def test_queries_and_outputs_at_odd_addresses(dtype, d, W, what, kernels):  # noqa: F811
    """One trajectory's stand one element off, another's do not."""
    p = Problem(dtype=dtype, d=d, M=2, H=1, Hq=4, trajs=[(500, W), (300, W)], gaps=0.6).upload()
    t, n = p.trajs[0], p.trajs[0].q.numel()
    ends = []
    if what != "out":
        q = torch.empty(n + 1, dtype=dtype, device="cuda")[1:].view(t.q.shape)
        q.copy_(t.q)
        p.trajs[0] = dataclasses.replace(t, q=q)
    if what != "q":
        x, y = torch.full((n + 2,), p.SENT, dtype=dtype, device="cuda"), torch.full((n // d + 2,), p.SENT, device="cuda")
        p.out[0], p.lse[0] = x[1:-1].view(t.q.shape), y[1:-1].view(t.q.shape[:3])
        ends = [x[0], x[-1], y[0], y[-1]]
    p.call(250, 2)
    p.check(250, 2)
    assert all(e == p.SENT for e in ends)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("W", [1, 3])
@pytest.mark.parametrize("S", [8, 1500])
@pytest.mark.parametrize("scale,least", [(1, -13), (8, -13), (31, -13), (32, -10), (40, -10), (56, -10), (80, -10)])
def test_small_values(d, W, S, scale, least):
    """fp32 sums of small values are as exact as those of values of 2^least.  An MMA adds 16 products and the sum so far,
    lined up with the largest, each cut off at 2^-23 of it or finer; a weight's two terms of w and w 2^-11.  Over all
    MMAs that is 17 (1 + 2^-11) 2^-23 2^least sum(w) at most beside the error of larger values (2e-6 in the 2-norm)."""
    def edit(p):
        for c, pos, Q, qp in p.host:
            c.host["v_scale"][:] = scale

    p = Problem(dtype=F32, d=d, M=1, H=2, Hq=8, trajs=[(S, W)], spread=3.0, edit=edit).upload()
    p.call()
    torch.cuda.synchronize()
    c, pos, Q, qp = p.host[0]
    o, _, _, _ = ref.attention(*c.values(), pos, Q, qp)
    off = ref.numbers(p.out[0]) - o
    assert np.linalg.norm(off) <= 2e-6 * np.linalg.norm(o) + 18 * 2.0 ** (least - 23) * np.sqrt(o.size)
