"""Beam search where candidates of different beams are equal or near.

A row's sum of exponentials is one in fp32, off by some 2^-20 of itself at most, so that the order of candidates of different
beams says something where their scores are further apart than 1e-6 of max(1, |score|).  Candidates of one beam are in the order
of their logits, and rows of equal values have equal sums.
"""
import pytest
import torch

from test_beam import BF, F, L, check, inputs  # noqa: F401  (L: the fixture)


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
@pytest.mark.parametrize("K,V,off", [(4, 50257, 0), (8, 5001, 3), (32, 777, 1), (3, 130001, 5), (5, 9, 2), (16, 2047, 7)])
def test_equal_beams(L, io, K, V, off):
    """Beams of equal logits and scores, whose rows start at different places of a 16-byte piece: equal candidates go by the
    lower beam, then the lower token."""
    g = torch.Generator("cuda").manual_seed(V)
    one = (torch.randn((3, 1, V), generator=g, device="cuda") * 2).to(io)
    wide = torch.zeros((3 * K, V + off), device="cuda", dtype=io)
    wide[:, off:] = one.expand(3, K, V).reshape(3 * K, V)
    scores = torch.tensor([[0.0], [-3.7], [-41.3]], device="cuda").expand(3, K).contiguous()
    check(L, wide[:, off:], scores, None, -1, K)
