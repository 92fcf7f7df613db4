"""The bounds of attention_terms tell the kernels' arithmetic from one with a
term less (CPU: restatements of both)."""
import pytest

torch = pytest.importorskip("torch")

import attention_terms as at  # noqa: E402


def operands(d, S, seed=0, w=64):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n, d, generator=g).double() for n in (w, S, S)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("split,loss", [(at.two_tf32, 1.3e-7), (at.three_bf16, 3e-8)])
def test_a_missing_product_passes_the_bound(d, split, loss):
    Q, K, V = operands(d, 1500)
    want, all_of = at.attention(Q, K, V), at.PAIRS[split]
    assert at.rel(at.attention(Q, K, V, split, all_of, all_of), want) < loss
    for gone in all_of[1:]:
        less = [p for p in all_of if p != gone]
        assert at.rel(at.attention(Q, K, V, split, less, all_of), want) > 1.5 * at.F32_BOUND
        assert at.rel(at.attention(Q, K, V, split, all_of, less), want) > 1.5 * at.F32_BOUND


@pytest.mark.parametrize("d", [64, 128])
def test_weights_of_one_bf16_term_pass_the_roundings_bound(d):
    """Output rounding alone, with weights of two bf16 terms, and of one."""
    Q, K, V = (at.bf16(x) for x in operands(d, 1500))
    want = at.attention(Q, K, V)
    own = at.rel(at.bf16(want), want)
    two = at.rel(at.bf16(at.attention(Q, K, V, weights=at.two_bf16)), want)
    one = at.rel(at.bf16(at.attention(Q, K, V, weights=lambda e: [at.bf16(e)])), want)
    assert two < 1.03 * own and 1.25 * own < one < 1.6 * own
