"""A session's own attention as a model uses it: layer by layer, on several
streams, in graphs, with device errors reported."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_07855_gb300 import commitkv as ck  # noqa: E402
from paper_2608_07855_gb300.lifecycle import Session  # noqa: E402

import attention_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("prefix", [0, 50])
def test_model_of_several_layers(dtype, prefix):
    """A small model runs through the session: a prompt, a checkpoint and decoded
    tokens, where each layer's queries, keys and values are linear in what the
    layer below put out.  Every layer's attention against 64 bits."""
    M, H, Hq, d = 3, 2, 4, 64
    g = torch.Generator(device="cuda").manual_seed(11)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    Wq, Wk, Wv = ([rand(Hq * d, h * d) / (Hq * d) ** 0.5 for _ in range(M)] for h in (Hq, H, H))
    s = Session(ck.make_shape(M, H, Hq, d, dtype), 16, 96, 0.5, 400)
    pre = None
    if prefix:
        pre = ck.TrajTensors(rand(M, H, prefix, d).to(dtype), rand(M, H, prefix, d).to(dtype), i32(np.arange(prefix)))
    at = prefix
    for n in (150, 1, 33, 1):
        x = rand(n, Hq * d)  # the new tokens
        pos = np.arange(at, at + n)
        s.append(None, None, i32(pos), [("obs", at, n)], decoded=n == 1)
        for layer in range(M):
            heads = lambda w, h: (x @ w[layer]).view(n, h, d).transpose(0, 1).to(dtype).contiguous()  # noqa: E731, B023
            s.fill(layer, heads(Wk, H), heads(Wv, H))
            Q = heads(Wq, Hq)
            o, lse = s.attend(Q, i32(pos), 120, 4, prefix=pre, layer=layer)
            assert o.shape == Q.shape and lse.shape == Q.shape[:2]
            parts = [] if pre is None else [(pre.k[layer:layer + 1].cpu(), pre.v[layer:layer + 1].cpu(), np.arange(prefix))]
            parts.append((s.K[layer:layer + 1, :, :s.S].cpu(), s.V[layer:layer + 1, :, :s.S].cpu(), s.pos[:s.S].cpu().numpy()))
            wo, wl, to, tl = ref.attention(parts, Q[None].cpu(), pos, 120, 4, rounded_weights=dtype == BF)
            ref.check(o[None], wo, to, "layer %d" % layer)
            ref.check(lse[None], wl, tl, "layer %d, lse" % layer)
            x = x + o.transpose(0, 1).reshape(n, Hq * d).float()
        at += n
        if n == 150:
            s.checkpoint(torch.rand(150, generator=g, device="cuda"))
            assert s.S == 96
            with pytest.raises(ValueError):  # the prompt's tokens have moved
                s.fill(0, torch.zeros(H, 150, d, device="cuda"), torch.zeros(H, 150, d, device="cuda"))


def test_layers_equal_one_call_over_all():
    """Layer by layer and all layers at once agree where the queries are given."""
    M, H, Hq, d, n = 3, 2, 8, 128, 300
    g = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF)  # noqa: E731
    s = Session(ck.make_shape(M, H, Hq, d, BF, 0.05), 16, 96, 0.5, 400)
    s.append(rand(M, H, n, d), rand(M, H, n, d), i32(np.arange(n)), [])
    for W in (1, 60):
        Q, p = rand(M, Hq, W, d), i32(np.arange(n - W, n))
        o, lse = s.attend(Q, p)
        for layer in range(M):
            a, b = s.attend(Q[layer], p, layer=layer)
            parts = [(s.K[layer:layer + 1, :, :n].cpu(), s.V[layer:layer + 1, :, :n].cpu(), np.arange(n))]
            wo, wl, to, tl = ref.attention(parts, Q[layer:layer + 1].cpu(), p.cpu().numpy(), scale=0.05, rounded_weights=True)
            for out, l in ((a, b), (o[layer], lse[layer])):
                ref.check(out[None], wo, to, "out")
                ref.check(l[None], wl, tl, "lse")


@pytest.fixture
def workspaces(monkeypatch):
    """The attention workspaces that a session makes."""
    made, alloc = [], ck.alloc_attention_workspace

    def record(*a, **kw):
        made.append(alloc(*a, **kw))
        return made[-1]

    monkeypatch.setattr(ck, "alloc_attention_workspace", record)
    return made


def small_session(n=400, H=2, d=64):
    g = torch.Generator(device="cuda").manual_seed(2)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF)  # noqa: E731
    s = Session(ck.make_shape(1, H, 4 * H, d, BF), 16, 96, 0.5, n)
    s.append(rand(1, H, n, d), rand(1, H, n, d), i32(np.arange(n)), [("obs", 0, n)])
    return s, rand


@pytest.mark.parametrize("how", ["eager", "replaced", "captured"])
@pytest.mark.parametrize("reader", ["check", "pre_commit", "post_commit", "fill_scores", "checkpoint", "state_dict"])
def test_device_errors_of_attention_are_raised(how, reader, workspaces):
    """A wait that ran out on an attention workspace (here the bounded barrier of
    the test entry point) is raised by what the session does next, once."""
    s, rand = small_session()
    Q, p = rand(1, 8, 1, 64), i32([399])
    if how == "captured":
        s.attend(Q, p)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = s.attend(Q, p)  # noqa: F841
        graph.replay()
    else:
        s.attend(Q, p)
    ck.commitkv_test_barrier_timeout(workspaces[-1])
    if how == "replaced":  # by a larger one
        s.attend(rand(1, 8, 100, 64), i32(np.arange(300, 400)))
        assert len(workspaces) == 2
    call = {"check": s.check, "pre_commit": lambda: s.pre_commit(Q, p), "post_commit": lambda: s.post_commit(Q, p),
            "fill_scores": lambda: s.fill_scores(Q, p), "state_dict": s.state_dict,
            "checkpoint": lambda: s.checkpoint(torch.zeros(400, device="cuda"))}[reader]
    with pytest.raises(RuntimeError, match="device status"):
        call()
    assert s.S == 400 and len(s.pages) == 25 and s.measured == []  # nothing was done
    s.attend(Q, p)
    s.check()
    call()


def test_streams_share_no_workspace(workspaces):
    """Calls on two streams at once, prompts and single tokens that are split over
    their tokens: a workspace for each stream, and the results of calls alone."""
    s, rand = small_session(n=6000)
    main = torch.cuda.current_stream()
    streams = [torch.cuda.Stream() for _ in range(2)]
    Q = [rand(1, 8, 1, 64), rand(1, 8, 70, 64)]
    p = [i32(np.arange(6000 - q.shape[2], 6000)) for q in Q]
    want = [s.attend(q, at) for q, at in zip(Q, p)]
    torch.cuda.synchronize()
    alone = len(workspaces)
    for x in streams:
        x.wait_stream(main)
    got = [[], []]
    for _ in range(20):
        for i, x in enumerate(streams):
            with torch.cuda.stream(x):
                got[i].append(s.attend(Q[i], p[i]))
    torch.cuda.synchronize()
    made = workspaces[alone:]
    assert len(made) == 2 and made[0].data_ptr() != made[1].data_ptr()
    for w, outs in zip(want, got):
        assert all(torch.equal(a, b) for o in outs for a, b in zip(o, w))
    with torch.cuda.stream(streams[0]):
        ck.commitkv_test_barrier_timeout(made[0])  # a second, which the check waits for
        s.attend(Q[0], p[0])
    with pytest.raises(RuntimeError, match="device status"):
        s.check()
    s.check()
