"""A session filled layer by layer (CPU): the tokens of an append get each
layer's K and V as a model computes them, and nothing reads a layer before."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_07855_gb300 import commitkv as ck  # noqa: E402
from paper_2608_07855_gb300.lifecycle import Session  # noqa: E402

M, H, D = 3, 2, 64


def session():
    return Session(ck.Shape(M, H, 4, D, ck.COMMITKV_F32, 0.0), 16, 40, 0.125, capacity=100, device="cpu")


def tokens(n, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(M, H, n, D, generator=g), torch.randn(M, H, n, D, generator=g)


def test_layers_one_by_one_equal_all_at_once():
    a, b = session(), session()
    at = 0
    for n in (20, 1, 7):
        K, V = tokens(n, n)
        pos = torch.arange(at, at + n, dtype=torch.int32)
        events = [("obs", at, n)]
        a.append(K, V, pos, events, decoded=n)
        b.append(None, None, pos, events, decoded=n)
        for layer in (1, 0, 2):
            b.fill(layer, K[layer], V[layer])
        at += n
    assert a.S == b.S == 28 and a.pages == b.pages and a.decoded_since == b.decoded_since
    assert torch.equal(a.K, b.K) and torch.equal(a.V, b.V) and torch.equal(a.pos, b.pos)
    K, V = tokens(7, 50)  # the latest tokens may be written again
    a.fill(1, K[1], V[1])
    assert torch.equal(a.K[1, :, 21:28], K[1]) and torch.equal(a.K[:, :, :21], b.K[:, :, :21])


def test_unfilled_layers_are_not_read():
    s = session()
    K, V = tokens(5, 0)
    pos = torch.arange(5, dtype=torch.int32)
    s.append(None, None, pos, [])
    s.fill(0, K[0], V[0])
    q = torch.zeros(M, 4, 1, D)
    for read in (lambda: s.append(K, V, pos + 5, []), lambda: s.state_dict(), lambda: s.pre_commit(q, pos[-1:]),
                 lambda: s.post_commit(q, pos[-1:]), lambda: s.fill_scores(q, pos[-1:]),
                 lambda: s.checkpoint(torch.zeros(5)), lambda: s.attend(q, pos[-1:]),
                 lambda: s.attend(q[1], pos[-1:], layer=1)):
        with pytest.raises(ValueError, match="lack"):
            read()
    assert s.S == 5 and s.unfilled == {1, 2}


def test_bad_layers_and_shapes():
    s = session()
    K, V = tokens(5, 0)
    pos = torch.arange(5, dtype=torch.int32)
    with pytest.raises(ValueError):
        s.append(K, None, pos, [])
    assert s.S == 0
    s.append(None, None, pos, [])
    for layer, k, v in ((-1, K[0], V[0]), (M, K[0], V[0]), (0, K[0, :, :4], V[0]), (0, K, V), (0, K[0], V[0, :1])):
        with pytest.raises(ValueError):
            s.fill(layer, k, v)
    assert s.unfilled == {0, 1, 2}
    for layer in range(M):
        s.fill(layer, K[layer], V[layer])
    for layer, q in ((-1, K[0]), (M, K[0]), (0, K)):
        with pytest.raises(ValueError):
            s.attend(q, pos[-1:], layer=layer)


def test_loading_a_state_ends_the_latest_append():
    s, t = session(), session()
    K, V = tokens(5, 0)
    s.append(K, V, torch.arange(5, dtype=torch.int32), [])
    t.append(None, None, torch.arange(9, dtype=torch.int32), [])
    t.load_state_dict(s.state_dict())
    assert not t.unfilled and torch.equal(t.K[:, :, :5], K)
    with pytest.raises(ValueError):
        t.fill(0, K[0], V[0])
