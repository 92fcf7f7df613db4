"""A session whose cache is held in 4 bits: it decides, compresses and attends as
a full-width session does whose keys and values are what the codes stand for."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_07855_gb300 import commitkv as ck  # noqa: E402
from paper_2608_07855_gb300.lifecycle import Session  # noqa: E402

import packed_ref as ref  # noqa: E402
from attention_ref import check  # noqa: E402

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


def rounded(x):
    """What x stands for after packing."""
    return torch.from_numpy(ref.values(*ref.pack(ref.numbers(x)))).to(x.dtype).cuda()


class Pair:
    """A packed session and a full-width one that is given the packed one's values."""

    def __init__(self, dtype, d, M=2, H=2, Hq=4, G=16, B=160, capacity=700):
        self.shape = ck.make_shape(M, H, Hq, d, dtype)
        self.dims, self.dtype = (M, H, Hq, d), dtype
        self.args = (self.shape, G, B, 0.2, capacity)
        self.packed, self.full = Session(*self.args, packed=True), Session(*self.args)
        self.g = torch.Generator(device="cuda").manual_seed(3)
        self.at = 0

    def rand(self, *s):
        return torch.randn(*s, generator=self.g, device="cuda").to(self.dtype)

    def append(self, n, events=(), decoded=0, by_layer=False, token_major=False):
        M, H, _, d = self.dims
        K, V = ((self.rand(M, n, H, d).transpose(1, 2) if token_major else self.rand(M, H, n, d)) for _ in range(2))
        K[..., :3] *= 5
        pos = i32(np.arange(self.at, self.at + n))
        ev = [(kind, self.at + b, m) for kind, b, m in events]
        for s, (k, v) in ((self.packed, (K, V)), (self.full, (rounded(K), rounded(V)))):
            if by_layer:
                s.append(None, None, pos, ev, decoded)
                for layer in range(M):
                    s.fill(layer, k[layer], v[layer])
            else:
                s.append(k, v, pos, ev, decoded)
        self.at += n

    def same(self):
        a, b = self.packed, self.full
        assert a.S == b.S and a.pages == b.pages and a.retired == b.retired and a.measured == b.measured
        assert torch.equal(a.pos[:a.S], b.pos[:b.S])
        for x, y in zip(a._values(), b._values()):
            assert torch.equal(x, y)

    def window(self, W):
        M, _, Hq, d = self.dims
        return self.rand(M, Hq, W, d), i32(np.arange(self.at - W, self.at))

    def attends(self, window=0, sinks=0, W=1):
        Q, p = self.window(W)
        k, v = (ref.numbers(x) for x in self.full._values())
        w = 2.0 ** -8 if self.dtype is BF else 2.0 ** -21
        o, l, to, tl = ref.attention(k, v, self.full.pos[:self.full.S].cpu().numpy(), Q, p.cpu().numpy(), window, sinks,
                                     weights=w, queries=2.0 ** -21)
        out, lse = self.packed.attend(Q, p, window, sinks)
        check(out, o, to)
        check(lse, l, tl)
        for layer in range(self.dims[0]):
            out, lse = self.packed.attend(Q[layer], p, window, sinks, layer=layer)
            check(out, o[layer], to[layer])
            check(lse, l[layer], tl[layer])


@pytest.mark.parametrize("dtype,d", [(F32, 64), (F32, 128), (BF, 64), (BF, 128)], ids=["f32-64", "f32-128", "bf16-64", "bf16-128"])
def test_commits_and_checkpoints(dtype, d):
    p = Pair(dtype, d)
    p.append(250, [("obs", 10, 100), ("call", 150, 60)])
    p.attends(W=20)
    for commit in range(3):
        p.append(40, [("call", 5, 30)], decoded=40, by_layer=commit == 1)
        p.same()
        Q, pos = p.window(8)
        assert torch.equal(p.packed.pre_commit(Q, pos), p.full.pre_commit(Q, pos))
        p.append(60, [("obs", 0, 60)], token_major=commit == 2)
        Q, pos = p.window(8)
        a, b = p.packed.post_commit(Q, pos), p.full.post_commit(Q, pos)
        assert torch.equal(a["R_post"], b["R_post"]) and all(a[k] == b[k] for k in ("cand", "accepted", "step_R"))
        p.same()
        p.attends(120, 4)
        p.attends(W=7)
        if commit:
            Q, pos = p.window(8)
            assert torch.equal(p.packed.fill_scores(Q, pos), p.full.fill_scores(Q, pos))
            assert torch.equal(p.packed.decode_checkpoint(Q, pos), p.full.decode_checkpoint(Q, pos))
            p.same()
            assert p.packed.S == 160
            p.attends(W=3)
    p.packed.check()


def test_saved_and_resumed(tmp_path):
    p = Pair(BF, 128)
    p.append(300, [("obs", 0, 200)])
    Q, pos = p.window(8)
    p.packed.pre_commit(Q, pos)
    torch.save(p.packed.state_dict(), tmp_path / "s")
    again = Session(*p.args, packed=True)
    again.load_state_dict(torch.load(tmp_path / "s", weights_only=False))
    fill = torch.rand(300, generator=p.g, device="cuda")
    want, got = p.packed.checkpoint(fill), again.checkpoint(fill)
    assert torch.equal(want, got) and again.pages == p.packed.pages
    assert all(torch.equal(x, y) for x, y in zip(again._values(), p.packed._values()))
    st = p.packed.state_dict()
    assert sum(st[n].numel() for n in ("k", "v", "k_scale", "v_scale")) * 2 < 0.54 * sum(
        x.numel() * x.element_size() for x in p.packed._values())
    with pytest.raises(ValueError):
        p.full.load_state_dict(st)
    with pytest.raises(ValueError):
        again.load_state_dict(p.full.state_dict())


def test_streams_and_graphs():
    """Calls on two streams, and a captured call beside an eager one, replayed as queries change."""
    p = Pair(BF, 64)
    p.append(400, [("obs", 0, 300)])
    for W in (1, 30):
        (Qa, pos), (Qb, _) = p.window(W), p.window(W)
        want = [p.packed.attend(Q, pos, 100, 2) for Q in (Qa, Qb)]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        got = []
        for s, Q in zip(streams, (Qa, Qb)):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(p.packed.attend(Q, pos, 100, 2))
        p.packed.check()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y))
        q = Qa.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out, lse = p.packed.attend(q, pos, 100, 2)
        for Q, w in ((Qb, want[1]), (Qa, want[0])):
            q.copy_(Q)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, w[0]) and torch.equal(lse, w[1])
        p.packed.check()


def test_refusals():
    p = Pair(BF, 64)
    p.append(30)
    Q, pos = p.window(1)
    k, v = p.full._values()
    with pytest.raises(ValueError):
        p.packed.attend(Q, pos, prefix=ck.TrajTensors(k, v, p.full.pos[:30]))
    with pytest.raises(ValueError):
        p.packed.append(None, p.rand(2, 2, 3, 64), i32([30, 31, 32]), [])
    with pytest.raises(ValueError):
        p.packed.append(p.rand(2, 2, 3, 32), p.rand(2, 2, 3, 32), i32([30, 31, 32]), [])
    p.same()
