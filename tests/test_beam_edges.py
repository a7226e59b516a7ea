"""Beam search where candidates of different beams are equal or near.

A row's sum of exponentials is one in fp32, off by some 2^-20 of itself at most, so that the order of candidates of different
beams says something where their scores are further apart than 1e-6 of max(1, |score|).  Candidates of one beam are in the order
of their logits, and rows of equal values have equal sums.
"""
import math

import pytest
import torch

import test_beam
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


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
@pytest.mark.parametrize("K,V", [(2, 128256), (8, 50257), (32, 5001)])
def test_near_beams(L, io, K, V):
    """Beams with the same words in other orders, whose scores lie four times as far apart as their sums may be off, are told
    apart."""
    g = torch.Generator("cuda").manual_seed(K)
    row = (torch.randn(V, generator=g, device="cuda") * 2).to(io)
    row[5] = 20.0  # (ahead of the others by more than all the beams' scores are apart)
    logits = torch.stack([row[torch.randperm(V, generator=g, device="cuda")] for _ in range(K)])
    order = torch.randperm(K, generator=g, device="cuda")
    scores = torch.empty((1, K), device="cuda")
    scores[0, order] = -3.0 - 12e-6 * torch.arange(K, device="cuda", dtype=F)
    got = L.Beam(1, K, V, io=io).select(logits, scores)
    assert torch.equal(got["parents"][0].long(), order)
    assert torch.equal(got["tokens"][0].long(), logits.argmax(1)[order])


@pytest.mark.gpu
def test_select_has_no_near_beams(L):
    """The cases of test_beam.py's test_select, whose order is compared as it is: no two candidates of different beams that
    are among the best lie within ten times the bound."""
    (cases,) = (m.args[1] for m in test_beam.test_select.pytestmark if m.name == "parametrize")
    for B, K, V, io, off in cases:
        logits, scores, done = inputs(B, K, V, io, V + K, off=off)
        each = torch.log_softmax(logits.double().view(B, K, V), -1) + scores.double()[..., None]
        stay = torch.full_like(each, -math.inf)
        stay[:, :, min(2, V - 1)] = scores.double()
        for c in (each, torch.where(done[..., None], stay, each)):
            best, at = c.view(B, -1).topk(min(K + 1, K * V))
            apart = (best[:, :-1] - best[:, 1:]) / best[:, :-1].abs().clamp(min=1)
            other = (at[:, :-1] // V != at[:, 1:] // V) & torch.isfinite(apart)
            assert (apart[other] > 1e-5).all(), (B, K, V)
