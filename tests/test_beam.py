"""Beam search over recurrent states against plain forms in 64 bits.

Tokens, parents, slots and moved states have to be equal.  Scores are log-probabilities rounded once to fp32 (2^-24 of
the value) from a sum of exponentials off by some 2^-22 of itself at most: 1e-6 of max(1, |score|).
"""
import ctypes
import math

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def L():
    from paper_2512_08061_gb300 import build
    build.build()
    import paper_2512_08061_gb300.luna as L
    return L


def select(logits, scores, done, end):
    """numpy, 64 bits: (scores, tokens, parents, done)."""
    B, K = scores.shape
    x = logits.reshape(B, K, -1).astype(np.float64)
    V = x.shape[-1]
    with np.errstate(all="ignore"):
        top = x.max(-1, keepdims=True)
        base = scores.astype(np.float64)[..., None] - np.log(np.exp(x - top).sum(-1, keepdims=True))
        cand = np.where(np.isfinite(base) & np.isfinite(top), base + (x - top), -np.inf)
    if done is not None:
        stay = np.full_like(cand, -np.inf)
        stay[:, :, end] = scores
        cand = np.where(done[..., None], stay, cand)
    flat = cand.reshape(B, K * V)
    at = np.argsort(-flat, axis=1, kind="stable")[:, :K]
    best = np.take_along_axis(flat, at, 1)
    parents, tokens = at // V, at % V
    ended = None if end < 0 else np.take_along_axis(done if done is not None else np.zeros((B, K), bool), parents, 1) | (tokens == end)
    return best, tokens, parents, ended


def reorder(parents, slots, pool):
    """Beam by beam."""
    pool, new = pool.copy(), slots.copy()
    for b in range(len(parents)):
        free = [slots[b][k] for k in range(len(parents[b])) if k not in parents[b]]
        seen = set()
        for k, p in enumerate(parents[b]):
            if p in seen or not 0 <= p < len(parents[b]):
                new[b][k] = free.pop(0)
                if p in seen and 0 <= slots[b][p] < len(pool) and 0 <= new[b][k] < len(pool):
                    pool[new[b][k]] = pool[slots[b][p]]
            else:
                new[b][k] = slots[b][p]
                seen.add(p)
    return new, pool


def check(L, logits, scores, done, end, beams, **kw):
    B = logits.shape[0] // beams
    p = L.Beam(B, beams, logits.shape[1], end=end, io=logits.dtype)
    got = p.select(logits, scores, done, **kw)
    want = select(logits.double().cpu().numpy(), scores.cpu().numpy(), None if done is None else done.cpu().numpy(), end)
    for name, w in zip(("tokens", "parents"), want[1:]):
        assert np.array_equal(got[name].cpu().numpy(), w), name
    if end >= 0:
        assert np.array_equal(got["done"].cpu().numpy(), want[3])
    s, w = got["scores"].double().cpu().numpy(), want[0]
    assert np.array_equal(np.isfinite(s), np.isfinite(w))
    fine = np.isfinite(w)
    assert (np.abs(s[fine] - w[fine]) <= 1e-6 * np.maximum(1, np.abs(w[fine]))).all()
    return got


def inputs(B, K, V, io, seed, spread=2.0, off=0, ended=0.2):
    g = torch.Generator("cuda").manual_seed(seed)
    wide = torch.randn((B * K, V + off), generator=g, device="cuda") * spread
    logits = wide.to(io)[:, off:]
    scores = -torch.rand((B, K), generator=g, device="cuda") * 20
    done = torch.rand((B, K), generator=g, device="cuda") < ended
    return logits, scores, done


F, BF = torch.float32, torch.bfloat16


@pytest.mark.gpu
@pytest.mark.parametrize("B,K,V,io,off", [
    (1, 1, 1, F, 0), (1, 1, 1, BF, 0), (3, 4, 1, F, 0), (2, 5, 3, F, 0), (2, 32, 7, BF, 3), (1, 4, 50257, F, 0),
    (5, 3, 1000, BF, 1), (2, 8, 8192, F, 0), (2, 8, 8193, BF, 0), (1, 32, 30001, F, 5), (64, 5, 777, BF, 7),
    (1, 1, 262144, BF, 0), (1, 7, 131072, F, 2), (150, 2, 33000, BF, 0), (3, 32, 16500, F, 0)])
def test_select(L, B, K, V, io, off):
    logits, scores, done = inputs(B, K, V, io, V + K, off=off)
    check(L, logits, scores, done, min(2, V - 1), K)
    check(L, logits, scores, None, min(2, V - 1), K)
    check(L, logits, scores, None, -1, K)


@pytest.mark.gpu
@pytest.mark.parametrize("order", ["rising", "falling", "equal", "comb"])
@pytest.mark.parametrize("K", [1, 4, 32])
def test_select_ordered_rows(L, order, K):
    """Rows whose largest values lie together, where a thread or a piece holds more than its share of them."""
    V = 40000
    x = torch.arange(V, device="cuda", dtype=F) * 1e-3
    x = {"rising": x, "falling": x.flip(0), "equal": torch.zeros_like(x), "comb": torch.where(torch.arange(V, device="cuda") % 256 == 3, x, -x)}[order]
    logits = x.repeat(2 * K, 1)
    scores = -torch.arange(2 * K, device="cuda", dtype=F).view(2, K)
    check(L, logits, scores, None, -1, K)


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
def test_select_full_pools_repeat(L, io):
    """Blocks whose room for candidates runs full again and again, at different pieces, give the same every time: whether
    it is full has to be decided alike by all warps of a block."""
    B, K, V = 32, 8, 60000
    steps = torch.linspace(0.2, 4.0, B * K, device="cuda")[:, None] * torch.arange(V, device="cuda", dtype=F) * 1e-3
    logits = (steps + torch.rand(B * K, V, device="cuda", generator=torch.Generator("cuda").manual_seed(1))).to(io)
    scores = -torch.arange(B * K, device="cuda", dtype=F).view(B, K) * 0.1
    p = L.Beam(B, K, V, io=io)
    first = p.select(logits, scores)
    for _ in range(40):
        again = p.select(logits, scores)
        assert all(torch.equal(first[name], again[name]) for name in first)
    check(L, logits, scores, None, -1, K)


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
def test_select_equal_values(L, io):
    """Equal scores go by the lower beam, then the lower token; 0 and -0 are equal."""
    logits = torch.zeros((6, 500), device="cuda", dtype=io)
    logits[:, ::3] = -0.0
    scores = torch.zeros((2, 3), device="cuda")
    got = check(L, logits, scores, None, -1, 3)
    assert got["tokens"].tolist() == [[0, 1, 2]] * 2 and got["parents"].tolist() == [[0, 0, 0]] * 2
    few = torch.randint(0, 4, (40, 3000), device="cuda").to(io)
    check(L, few, torch.zeros((5, 8), device="cuda"), None, -1, 8)


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
def test_select_masked_and_not_finite(L, io):
    """Masked words, rows without any, beams not in use, scores and logits that are no numbers."""
    inf, nan = float("inf"), float("nan")
    K, V, end = 8, 20000, 5
    logits, scores, done = inputs(6, K, V, io, 9, ended=0.3)
    logits[:, 100:] = -inf                       # a mask that leaves few words
    logits[3] = -inf                             # one that leaves none
    logits[4, 50] = nan
    logits[5, 50] = inf
    logits[6] = nan
    logits[9] = torch.finfo(io).min              # masked by the type's lowest value throughout
    logits[10, 3:] = torch.finfo(io).min
    logits[2 * K:3 * K] = -inf                   # a sequence without a word
    scores[3, 1:] = -inf                         # a first step: one beam in use
    scores[4, 2], scores[4, 3], scores[4, 4] = nan, inf, -inf
    done[3:] = False
    check(L, logits, scores, None, end, K)
    check(L, logits, scores, done, end, K)
    check(L, logits, scores, torch.ones_like(done) & (scores > -1e30) & (scores < 1e30), end, K)
    logits[:] = -inf
    check(L, logits, scores, None, -1, K)


@pytest.mark.gpu
def test_select_in_place_streams_and_graph(L):
    """Scores and ends may be updated in place; the call runs on the stream it is given and can be captured."""
    logits, scores, done = inputs(3, 4, 5000, F, 3)
    p = L.Beam(3, 4, 5000, end=1, io=F)
    want = p.select(logits, scores, done)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    there = p.select(logits, scores, done, stream=s)
    s.synchronize()
    assert all(torch.equal(there[k], want[k]) for k in want)
    run = {"scores": scores.clone(), "done": done.clone(), "tokens": torch.empty_like(want["tokens"]), "parents": torch.empty_like(want["parents"])}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p.select(logits, run["scores"], run["done"], out=run)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(run[k], want[k]) for k in want)
    g.replay()
    torch.cuda.synchronize()
    again = p.select(logits, want["scores"], want["done"])
    assert all(torch.equal(run[k], again[k]) for k in want)


@pytest.mark.gpu
@pytest.mark.parametrize("B,K,shape,dtype", [(1, 1, (3, 5), F), (1, 4, (2, 32, 64), F), (5, 3, (7,), torch.uint8), (4, 32, (33,), F),
                                             (3, 16, (4, 1000), BF), (2, 2, (1, 3), torch.uint8), (8, 5, (100001,), F)])
def test_reorder(L, B, K, shape, dtype):
    g = torch.Generator("cuda").manual_seed(B * K)
    nslots = B * K + 3
    for trial in range(4):
        parents = torch.randint(0, K, (B, K), generator=g, device="cuda", dtype=torch.int32)
        if trial == 1:
            parents = parents.sort(1, descending=True)[0].contiguous()
        elif trial == 2:
            parents = torch.full_like(parents, K - 1)
        slots = torch.randperm(nslots, generator=g, device="cuda")[:B * K].to(torch.int32).view(B, K)
        pool = torch.randint(0, 200, (nslots, *shape), generator=g, device="cuda").to(dtype)
        second = pool.flip(0).contiguous().view(torch.uint8).clone()
        want, moved = reorder(parents.cpu().numpy(), slots.cpu().numpy(), pool.float().cpu().numpy())
        _, moved2 = reorder(parents.cpu().numpy(), slots.cpu().numpy(), second.cpu().numpy())
        got = L.Beam(B, K).reorder(parents, slots, pool, second)
        assert np.array_equal(got.cpu().numpy(), want)
        assert np.array_equal(pool.float().cpu().numpy(), moved) and np.array_equal(second.cpu().numpy(), moved2)
        assert torch.equal(L.Beam(B, K).reorder(parents, slots), got)


@pytest.mark.gpu
def test_reorder_idle(L):
    """Slots outside the pool and parents outside the beams move nothing and write nowhere."""
    parents = torch.tensor([[0, 0, 7, 0], [1, 1, 1, -1]], dtype=torch.int32, device="cuda")
    slots = torch.tensor([[0, 9, 2, -1], [-4, 3, 5, 6]], dtype=torch.int32, device="cuda")
    pool = torch.arange(8, device="cuda", dtype=F).view(8, 1).repeat(1, 40).contiguous()
    want, moved = reorder(parents.cpu().numpy(), slots.cpu().numpy(), pool.cpu().numpy())
    assert np.array_equal(L.Beam(2, 4).reorder(parents, slots, pool).cpu().numpy(), want)
    assert np.array_equal(pool.cpu().numpy(), moved)


@pytest.mark.gpu
def test_search_over_a_delta_layer(L):
    """A search as it runs: tokens through a layer of the gated delta rule, logits by a linear layer, the best beams,
    their states; against the same search in 64 bits that keeps each beam's states by itself.  (fp32 throughout;
    candidates nearer to each other than 1e-3 would make the order a matter of rounding: there are none.)"""
    B, K, H, d, V, end, steps = 3, 4, 2, 32, 97, 0, 12
    g = torch.Generator("cuda").manual_seed(2)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    embed, W, head = rn(V, 24), rn(3 * H * d, 24) / 5, rn(V, H * d) / 2
    lg, bt = -torch.rand((V, H), generator=g, device="cuda"), torch.rand((V, H), generator=g, device="cuda")
    delta, beam = L.Delta(B * K, H, 1, d, d, io=F), L.Beam(B, K, V, end=end, io=F)
    into, out_of = L.Linear(B * K, 3 * H * d, 24, io=F), L.Linear(B * K, V, H * d, io=F)
    slots = torch.randperm(B * K + 5, generator=g, device="cuda")[:B * K].to(torch.int32).view(B, K)
    pool = torch.full((B * K + 5, H, d, d), float("nan"), device="cuda")
    pool[slots.long()] = 0.0
    tokens = torch.full((B, K), 1, dtype=torch.int32, device="cuda")
    scores = torch.tensor([[0.0] + [-math.inf] * (K - 1)] * B, device="cuda")
    done = torch.zeros((B, K), dtype=torch.bool, device="cuda")
    S = np.zeros((B * K, H, d, d))
    w = {k: v.double().cpu().numpy() for k, v in (("embed", embed), ("W", W), ("head", head), ("lg", lg), ("bt", bt))}
    rt, rs, rd = np.full(B * K, 1), scores.double().cpu().numpy(), np.zeros((B, K), bool)
    for step in range(steps):
        t = tokens.view(-1).long()
        y = into.forward(embed[t], W).view(B * K, 3, H, d)
        q, k = (torch.nn.functional.normalize(y[:, i], dim=-1) for i in (0, 1))
        o = delta.step(q, k, y[:, 2], lg[t], bt[t], pool, slots.view(-1))
        best = beam.select(out_of.forward(o.view(B * K, H * d), head), scores, done)
        slots = beam.reorder(best["parents"], slots, pool)
        scores, tokens, done = best["scores"], best["tokens"], best["done"]

        y = (w["embed"][rt] @ w["W"].T).reshape(B * K, 3, H, d)
        q, k = (y[:, i] / np.linalg.norm(y[:, i], axis=-1, keepdims=True) for i in (0, 1))
        old = np.exp(w["lg"][rt])[..., None, None] * S
        u = w["bt"][rt][..., None] * (y[:, 2] - np.einsum("bhd,bhde->bhe", k, old))
        S = old + k[..., None] * u[..., None, :]
        o = np.einsum("bhd,bhde->bhe", q, S) * d ** -0.5
        rs, tok, par, rd = select(o.reshape(B * K, -1) @ w["head"].T, rs, rd, end)
        S = S.reshape(B, K, H, d, d)[np.arange(B)[:, None], par].reshape(B * K, H, d, d)
        rt = tok.reshape(-1)
        assert np.array_equal(tokens.cpu().numpy().reshape(-1), rt), step
        assert np.array_equal(best["parents"].cpu().numpy(), par), step
        assert np.array_equal(done.cpu().numpy(), rd), step
        assert np.allclose(scores.cpu().numpy(), rs, rtol=1e-5, atol=1e-5), step
    live = pool[slots.long()].double().cpu().numpy().reshape(S.shape)
    assert np.linalg.norm(live - S) < 1e-5 * np.linalg.norm(S)


def test_refusals(L):
    lib, P = L._lib, ctypes.c_void_p

    def size(bd):
        return lib.luna_beam_workspace_size(ctypes.byref(bd), ctypes.byref(ctypes.c_size_t()))

    def sel(bd, logits=256, scores=256, done=None, out=256, ended=None, ws=256, nbytes=1 << 40):
        return lib.luna_beam_select(ctypes.byref(bd), P(logits), P(scores), P(done), P(out), P(256), P(256), P(ended), P(ws), nbytes, None)

    def order(bd, parents=256, slots=512, nslots=4, pool=256, nbytes=64, new=1024):
        return lib.luna_beam_reorder(ctypes.byref(bd), P(parents), P(slots), nslots, P(pool), nbytes, P(new), None)

    ok = dict(B=2, K=4, V=100, end=3)
    assert size(L.beam_desc(**ok)) == 0
    for bad in (dict(ok, B=-1), dict(ok, K=0), dict(ok, V=-1), dict(ok, end=100), dict(ok, end=-2), dict(ok, io=5)):
        assert size(L.beam_desc(**bad)) == 1, bad
    for bad in (dict(ok, K=33), dict(ok, V=(1 << 24) + 1), dict(ok, B=1 << 15)):
        assert size(L.beam_desc(**bad)) == 2, bad
    bd = L.beam_desc(**ok)
    assert sel(bd, logits=0) == 1 and sel(bd, scores=0) == 1 and sel(bd, out=0) == 1 and sel(bd, ws=0) == 1 and sel(bd, ws=64) == 1
    assert sel(bd, nbytes=256) == 3 and sel(L.beam_desc(2, 4)) == 1
    bd.ld = 99
    assert sel(bd) == 1
    bd = L.beam_desc(**dict(ok, end=-1))
    assert sel(bd, done=256) == 1 and sel(bd, ended=256) == 1
    bd = L.beam_desc(2, 4)
    assert order(bd, parents=0) == 1 and order(bd, slots=0) == 1 and order(bd, new=0) == 1 and order(bd, new=512) == 1 and order(bd, new=256) == 1
    assert order(bd, pool=0) == 1 and order(bd, nslots=-1) == 1 and order(bd, nbytes=(1 << 40) + 1) == 1
    none = L.beam_desc(0, 4, 100)
    assert sel(none, logits=0, scores=0, out=0, ws=0, nbytes=0) == 0 and order(none, parents=0, slots=0, new=0) == 0


def test_binding_checks(L):
    p = L.Beam(2, 3, 10, end=1, io=torch.float32, device="cpu")
    x, s, done = torch.zeros(6, 10), torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.bool)
    for bad, error in (((x[:5], s), ValueError), ((x.double(), s), TypeError), ((x, s.double()), TypeError), ((x, s, done.int()), TypeError),
                       ((x.t().contiguous().t(), s), ValueError), ((x, s.t().contiguous().t()), ValueError), ((x, s[:1]), ValueError)):
        with pytest.raises(error):
            p.select(*bad)
    with pytest.raises(ValueError):
        p.select(x, s, out={"scores": s})
    parents, slots = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32)
    for bad, error in (((parents.long(), slots), TypeError), ((parents, slots[:1]), ValueError), ((parents, slots, torch.zeros(8, 4).t()), ValueError),
                       ((parents, slots, torch.zeros(())), ValueError)):
        with pytest.raises(error):
            p.reorder(*bad)
