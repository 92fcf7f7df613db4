"""Packed caches' bindings without a GPU: which strides count."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_07855_gb300 import commitkv as ck  # noqa: E402


@pytest.mark.parametrize("M,H,n", [(3, 2, 1), (1, 2, 1), (3, 1, 1), (1, 1, 1), (1, 2, 6), (3, 1, 6), (3, 2, 6)])
def test_strides_of_single_entries_do_not_count(M, H, n):
    x = torch.zeros(M, H, n, 64)
    for s in ((7, 7, 7), (0, 0, 0), (10**9, 10**9, 10**9)):
        y = x.as_strided(x.shape, [a if m > 1 else b for m, a, b in zip(x.shape, x.stride(), s)] + [1])
        assert ck._strides(x) == ck._strides(y)
    # what a copy in another order leaves, which torch calls contiguous all the same
    z = x.transpose(1, 2).contiguous().transpose(1, 2)
    same = ck._strides(x) == ck._strides(z)
    assert same == (n == 1 or H == 1)
    assert ck._strides(z.contiguous()) == ck._strides(x)


def test_strides_of_several_entries_count():
    x = torch.zeros(3, 4, 10, 64)
    assert ck._strides(x) == (2560, 640, 64) and ck._strides(x[:, :, ::2]) == (2560, 640, 128)
    assert ck._strides(x[:1]) == (0, 640, 64) and ck._strides(x[:, :, :1]) == (2560, 640, 64)
    assert ck._strides(x.expand(3, 4, 10, 64)[:, :, :0]) == (0, 0, 64)
