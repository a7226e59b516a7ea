"""Beam search where candidates of different beams are equal or near.

A row's sum of exponentials is one in fp32, off by some 2^-20 of itself at most, so that the order of candidates of different
beams says something where their scores are further apart than 1e-6 of max(1, |score|).  Candidates of one beam are in the order
of their logits, and rows of equal values have equal sums.
"""
import math

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


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
@pytest.mark.parametrize("B,K,V", [(1, 1, 1000000), (80, 8, 128256), (640, 1, 1048576)])
@pytest.mark.parametrize("low", [-5.75, -11.3125, -14.75, -16.75, -18.0])
def test_peaked_rows(L, io, B, K, V, low):
    """One word far ahead of very many equal ones, whose sum counts though each alone is lost beside it: 25 additions at most
    that round at the top's size, 2^-24 each, and what the others' own exponentials are off (2^-19 of their share)."""
    logits = torch.full((B * K, V), low, device="cuda", dtype=io)
    logits[:, V // 3] = 0.0
    scores = -20.0 * torch.arange(K, device="cuda", dtype=F).expand(B, K).contiguous()  # (a beam's first word comes before all of the next's)
    got = L.Beam(B, K, V, io=io).select(logits, scores)
    assert (got["tokens"][:, 0] == V // 3).all() and (got["parents"][:, 0] == 0).all()
    others = (V - 1) * math.exp(low)
    bound = 25 * 2.0 ** -24 + 2.0 ** -19 * others / (1 + others) + 2.0 ** -24 * math.log1p(others)
    assert (got["scores"][:, 0].double() + math.log1p(others)).abs().max() < bound
