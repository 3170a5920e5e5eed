"""How far a float32 attention is off whose queries, or probabilities, go into the products as two bfloat16 parts instead of three:
the threshold of the GPU's precision test lies between the two."""
import pytest
import torch


def parts(x, n):
    """Sum of n bfloat16 parts of x, each the rounding of what the others leave."""
    total, rest = torch.zeros_like(x), x.clone()
    for _ in range(n):
        p = rest.float().bfloat16().double()
        total, rest = total + p, rest - p
    return total


@pytest.mark.parametrize("d,n", [(64, 777), (128, 777), (128, 4000)])
@pytest.mark.parametrize("q_parts,p_parts,enough", [(3, 3, True), (2, 3, False), (3, 2, False)])
def test_two_parts_are_too_few(d, n, q_parts, p_parts, enough):
    g = torch.Generator().manual_seed(d + n)
    q = torch.randn(16, d, generator=g).double()
    k, v = (torch.randn(n, d, generator=g) * 2).round().div(2).double(), torch.randn(n, d, generator=g).double()
    exact = (q @ k.t() * d ** -0.5).softmax(-1) @ v
    s = parts(q, q_parts) @ k.t() * d ** -0.5
    p = (s - s.amax(-1, keepdim=True)).exp()
    got = parts(p, p_parts) @ v / p.sum(-1, keepdim=True)
    rms = ((got - exact).square().mean().sqrt() / exact.square().mean().sqrt()).item()
    assert (rms < 1e-6) == enough, rms
    if enough:
        assert rms < 1e-7
