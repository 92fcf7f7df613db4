"""Session.append with rows that do not fit its positions (CPU: no entry point is called)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_07855_gb300 import commitkv as ck  # noqa: E402
from paper_2608_07855_gb300.lifecycle import Session  # noqa: E402

M, H, D = 2, 3, 64


def session(packed=False):
    return Session(ck.Shape(M, H, 6, D, ck.COMMITKV_F32, 0.0), 16, 40, 0.125, capacity=20, device="cpu", packed=packed)


def rows(n):
    return torch.full((M, H, n, D), float(n))


def positions(s, n):
    return torch.arange(s.S, s.S + n, dtype=torch.int32)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("nk,nv", [(2, 2), (5, 5), (3, 2), (5, 3), (0, 0)])
def test_other_rows_than_positions_are_refused(nk, nv, packed):
    """Three positions: with fewer rows the last ones would stand for what was there before, more would be written
    behind the cache's end."""
    s = session(packed)
    if not packed:
        s.append(rows(4), rows(4), positions(s, 4), [])
    S = s.S
    with pytest.raises(ValueError if packed else RuntimeError, match="K and V" if packed else "size"):
        s.append(rows(nk), rows(nv), positions(s, 3), [("obs", S, 3)])
    assert s.S == S and not s.pages
    if not packed:
        assert (s.K[:, :, S + 3:] == 0).all() and (s.V[:, :, S + 3:] == 0).all()


def test_as_many_rows_as_positions():
    s = session()
    s.append(rows(3), rows(3), positions(s, 3), [])
    s.append(rows(1), rows(1), positions(s, 1), [])
    assert s.S == 4 and s.K[0, 0, :5, 0].tolist() == [3, 3, 3, 1, 0]


@pytest.mark.parametrize("packed", [False, True])
def test_a_refused_append_leaves_the_session_as_it_was(packed):
    """What it decoded does not count towards the checkpoint cadence either: the caller appends it again."""
    s = session(packed)
    p = torch.arange(3, dtype=torch.int32)
    for K, V, pos in ((rows(2), rows(2), p), (rows(3), rows(2), p), (rows(3), None, p),
                      (rows(21), rows(21), torch.arange(21, dtype=torch.int32))):
        with pytest.raises((ValueError, RuntimeError)):
            s.append(K, V, pos, [("obs", 0, 3)], decoded=3)
    assert (s.S, s.decoded_since, s.pages, s.tail, s.unfilled) == (0, 0, [], (0, 0), set())
    s.append(None, None, p, [("obs", 0, 3)], decoded=3)
    assert s.S == 3 and s.decoded_since == 3 and s.unfilled == {0, 1}
