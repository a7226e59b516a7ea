"""Linear attention with a decay for each head against its recurrence in 64 bits, token by token.

Tolerances (relative 2-norms), from the number formats: a bf16 output carries its own rounding
(2^-9 at most, 1.7e-3 in the root mean square over a binade) and those of the scores and the state
that enter its products, so sqrt(3) * 1.7e-3 = 2.9e-3, taken as 4e-3; an fp32 output or state sums
at most a few thousand terms rounded at 2^-24, so under sqrt(4096) * 6e-8 = 4e-6, taken as 1e-5.
"""
import ctypes
import os

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TOL = {torch.float32: 1e-5, torch.bfloat16: 4e-3}


@pytest.fixture(scope="module")
def L():
    from paper_2512_08061_gb300 import build
    build.build()
    import paper_2512_08061_gb300.luna as L
    return L


def recurrence(q, k, v, log_decay, scale, lengths=None, S0=None, dO=None, dS1=None):
    """fp64 numpy, heads of k and v already repeated: O, S1 and with dO the gradients."""
    B, H, n, d = q.shape
    dv = v.shape[-1]
    lam = np.exp(log_decay)[None, :, None, None]
    lens = np.full(B, n) if lengths is None else np.clip(lengths, 0, n)
    S = np.zeros((B, H, d, dv)) if S0 is None else S0.copy()
    q, k, v = (np.where((np.arange(n) < lens[:, None])[:, None, :, None], x, 0.0) for x in (q, k, v))
    O, before = np.zeros((B, H, n, dv)), np.zeros((n, B, H, d, dv)) if dO is not None else None
    for t in range(n):
        on = (t < lens)[:, None, None, None]
        S = np.where(on, lam * S + k[:, :, t, :, None] * v[:, :, t, None, :], S)
        O[:, :, t] = np.where(on[..., 0], scale * np.einsum("bhd,bhde->bhe", q[:, :, t], S), 0.0)
        if dO is not None:
            before[t] = S
    if dO is None:
        return {"O": O, "S1": S}
    R = np.zeros((B, H, d, dv)) if dS1 is None else dS1.copy()
    g = {"dQ": np.zeros((B, H, n, d)), "dK": np.zeros((B, H, n, d)), "dV": np.zeros((B, H, n, dv))}
    for t in range(n - 1, -1, -1):
        on = (t < lens)[:, None, None, None]
        do = np.where(on[..., 0], dO[:, :, t], 0.0)
        g["dQ"][:, :, t] = scale * np.einsum("bhde,bhe->bhd", before[t], do)
        now = R + scale * q[:, :, t, :, None] * do[:, :, None, :]
        g["dK"][:, :, t] = np.where(on[..., 0], np.einsum("bhde,bhe->bhd", now, v[:, :, t]), 0.0)
        g["dV"][:, :, t] = np.where(on[..., 0], np.einsum("bhde,bhd->bhe", now, k[:, :, t]), 0.0)
        R = np.where(on, lam * now, R)
    return {"O": O, "S1": S, **g, "dS0": R}


def f64(t):
    return t.double().cpu().numpy()


def rel(a, r):
    a = f64(a)
    assert np.isfinite(a).all()
    return np.linalg.norm(a - r) / max(np.linalg.norm(r), 1e-30)


def inputs(B, H, Hkv, n, d, dv, io, layout, seed, state):
    g = torch.Generator("cuda").manual_seed(seed)

    def rn(heads, w):
        x = torch.randn((B, n, heads, w), generator=g, device="cuda").to(io)
        if layout == "tokens":      # heads next to each other within a token
            return x.transpose(1, 2)
        if layout == "wide":        # views into a wider row, as of a fused projection
            y = torch.full((B, n, heads * w + 24), float("nan"), device="cuda", dtype=io)
            y[..., 16:16 + heads * w] = x.flatten(2)
            return y[..., 16:16 + heads * w].unflatten(2, (heads, w)).transpose(1, 2)
        return x.transpose(1, 2).contiguous()

    rate = torch.logspace(-3, -0.3, H, device="cuda")
    S = torch.randn((B, H, d, dv), generator=g, device="cuda") if state else None
    dS = torch.randn((B, H, d, dv), generator=g, device="cuda") if state else None
    return rn(H, d), rn(Hkv, d), rn(Hkv, dv), rn(H, dv), -rate, S, dS


def check_all(L, B, H, Hkv, n, d, dv, io, layout, lengths, state, log_decay=None, nan_padding=False):
    Q, K, V, dO, ld, S0, dS1 = inputs(B, H, Hkv, n, d, dv, io, layout, 7 * n + d, state)
    ld = ld if log_decay is None else torch.tensor(log_decay, device="cuda", dtype=torch.float32)
    lens = None if lengths is None else torch.tensor(lengths, device="cuda", dtype=torch.int32)
    ref_in = [f64(x) for x in (Q, K, V, dO)]
    if nan_padding:
        for b, m in enumerate(lengths):
            for x in (Q, K, V, dO):
                x[b, :, max(0, m):] = float("nan")
    G = H // Hkv
    rq, rk, rv, rg = ref_in
    ref = recurrence(rq, rk.repeat(G, 1), rv.repeat(G, 1), f64(ld), d ** -0.5, lengths and np.array(lengths),
                     None if S0 is None else f64(S0), rg, None if dS1 is None else f64(dS1))
    for x in ("dK", "dV"):
        ref[x] = ref[x].reshape(B, Hkv, G, n, -1).sum(2)
    p = L.Decay(B, H, n, d, dv, Hkv=Hkv, io=io, backward=True)
    O, S1 = p.forward(Q, K, V, ld, lens, S0, want_state=True)
    g = p.backward(Q, K, V, dO, ld, lens, S0, dS1)
    assert L.luna_device_status(p.ws) == 0
    got = {"O": O, "S1": S1, **g}
    for name, t in got.items():
        assert rel(t, ref[name]) < TOL[t.dtype], name
    if lengths is not None:
        for b, m in enumerate(lengths):
            for name in ("O", "dQ", "dK", "dV"):
                assert not got[name][b, :, max(0, min(n, m)):].any(), name
    again = p.backward(Q, K, V, dO, ld, lens, S0, dS1)
    for name in g:
        assert torch.equal(g[name], again[name]), name


F, BF = torch.float32, torch.bfloat16
CASES = [  # B, H, Hkv, n, d, dv, io, layout, lengths, state
    (1, 1, 1, 1, 1, 1, F, "heads", None, False),
    (2, 3, 3, 33, 7, 5, F, "tokens", [33, 0], True),
    (1, 2, 1, 300, 40, 72, F, "wide", None, True),
    (2, 4, 2, 515, 64, 64, F, "heads", [515, 257], False),
    (1, 1, 1, 1, 64, 64, BF, "heads", None, True),
    (2, 2, 2, 127, 64, 64, BF, "tokens", [127, 1], False),
    (1, 2, 2, 128, 128, 128, BF, "heads", None, True),
    (3, 2, 1, 129, 128, 64, BF, "wide", [129, 128, 0], True),
    (1, 3, 1, 700, 32, 128, BF, "tokens", [641], True),
    (2, 6, 3, 1025, 128, 128, BF, "tokens", [1025, 300], True),
    (1, 2, 2, 260, 40, 24, BF, "heads", None, False),
    (1, 2, 1, 200, 33, 50, BF, "tokens", [199], True),     # widths that no 16-byte access covers
    (1, 2, 2, 520, 8, 120, BF, "wide", None, False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,Hkv,n,d,dv,io,layout,lengths,state", CASES)
def test_prompts_and_gradients(L, B, H, Hkv, n, d, dv, io, layout, lengths, state):
    check_all(L, B, H, Hkv, n, d, dv, io, layout, lengths, state)


@pytest.mark.gpu
@pytest.mark.parametrize("H,Hkv,n,d,dv", [(8, 8, 1024, 128, 128), (8, 2, 900, 128, 64), (6, 6, 1100, 64, 64), (12, 4, 700, 32, 64)])
def test_many_heads_of_many_chunks(L, H, Hkv, n, d, dv):
    """Every SM at work on pieces of many chunks (few heads are cut into pieces of one or two), against the
    fp32 form of the same call on the same values: both within the bf16 tolerance of the definition."""
    B = 40
    Q, K, V, dO, ld, _, _ = inputs(B, H, Hkv, n, d, dv, BF, "tokens", 21, False)
    lens = torch.randint(n // 2, n + 1, (B,), device="cuda", dtype=torch.int32)
    p, f = L.Decay(B, H, n, d, dv, Hkv=Hkv, io=BF, backward=True), L.Decay(B, H, n, d, dv, Hkv=Hkv, io=F, backward=True)
    wide = [x.float() for x in (Q, K, V, dO)]
    want, S = f.forward(*wide[:3], ld, lens, want_state=True)
    grads = f.backward(*wide, ld, lens)
    for _ in range(3):
        got, S1 = p.forward(Q, K, V, ld, lens, want_state=True)
        pairs = {"O": (got, want), "S1": (S1, S), "O without state": (p.forward(Q, K, V, ld, lens), want)}
        pairs.update({k: (v, grads[k]) for k, v in p.backward(Q, K, V, dO, ld, lens).items()})
        assert L.luna_device_status(p.ws) == 0
        for name, (a, b) in pairs.items():
            by_head = (a.double() - b).flatten(2).norm(dim=2) / b.double().flatten(2).norm(dim=2)
            assert by_head.max() < TOL[a.dtype], name


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
def test_padding_may_hold_anything(L, io):
    """NaN in rows at and past the length reaches no output; lengths outside [0, n] are clamped."""
    check_all(L, 3, 2, 2, 300, 64, 64, io, "heads", [299, 130, 0], True, nan_padding=True)
    check_all(L, 2, 2, 2, 300, 64, 64, io, "heads", [-5, 1000], True)


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
def test_extreme_decays(L, io):
    """lambda = 0 (each token sees itself alone), 1 (no decay), tiny, and beyond the range of exp."""
    check_all(L, 1, 6, 6, 400, 64, 64, io, "heads", None, False, [-float("inf"), 0.0, -1e-6, -30.0, -200.0, -3e38])


@pytest.mark.gpu
def test_unaligned_views(L):
    """bf16 tensors one element off a 16-byte boundary take the CUDA-core form and give the same values."""
    B, H, n, d = 1, 2, 200, 64
    Q, K, V, dO, ld, S0, _ = inputs(B, H, H, n, d, d, BF, "heads", 3, True)
    odd = []
    for x in (Q, K, V):
        y = torch.empty(x.numel() + 1, dtype=BF, device="cuda")[1:].view(x.shape)
        odd.append(y.copy_(x))
    p = L.Decay(B, H, n, d, d, io=BF)
    a = p.forward(Q, K, V, ld, None, S0)
    b = p.forward(*odd, ld, None, S0)
    assert (a.double() - b.double()).norm() < TOL[BF] * a.double().norm()


@pytest.mark.gpu
@pytest.mark.parametrize("io,d,dv,H,Hkv", [(F, 13, 70, 4, 2), (BF, 64, 64, 3, 3), (BF, 128, 128, 4, 1), (BF, 33, 6, 2, 2)])
def test_tokens_continue_a_prompt(L, io, d, dv, H, Hkv):
    """A prompt in two pieces, then single tokens, give the rows of the whole prompt."""
    B, n = 2, 150
    Q, K, V, _, ld, S0, _ = inputs(B, H, Hkv, n, d, dv, io, "tokens", 11, True)
    cut, steps = 77, 9
    G = H // Hkv
    ref = recurrence(f64(Q), f64(K).repeat(G, 1), f64(V).repeat(G, 1), f64(ld), d ** -0.5, None, f64(S0))
    state = S0.clone()
    out = []
    for a, b in ((0, cut), (cut, n - steps)):
        p = L.Decay(B, H, b - a, d, dv, Hkv=Hkv, io=io)
        o, state = p.forward(Q[:, :, a:b], K[:, :, a:b], V[:, :, a:b], ld, None, state, want_state=True)
        out.append(o)
    pool = torch.full((5, H, d, dv), float("nan"), device="cuda")
    slots = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    pool[slots.long()] = state
    p = L.Decay(B, H, 1, d, dv, Hkv=Hkv, io=io)
    for t in range(n - steps, n):
        out.append(p.step(Q[:, :, t], K[:, :, t], V[:, :, t], ld, pool, slots).unsqueeze(2))
    assert rel(torch.cat(out, 2), ref["O"]) < TOL[io]
    assert rel(pool[slots.long()], ref["S1"]) < TOL[F]
    assert torch.isnan(pool[[0, 2, 4]]).all()


@pytest.mark.gpu
def test_idle_slots(L):
    """A slot outside the pool leaves every state alone and gives zeros."""
    B, H, d = 3, 2, 32
    p = L.Decay(B, H, 1, d, d, io=BF)
    pool = torch.ones((2, H, d, d), device="cuda")
    q = torch.ones((B, H, d), device="cuda", dtype=BF)
    slots = torch.tensor([-1, 2, 1], dtype=torch.int32, device="cuda")
    o = p.step(q, q, q, torch.zeros(H, device="cuda"), pool, slots)
    assert not o[:2].any() and o[2].any()
    assert (pool[0] == 1).all() and (pool[1] == 2).all()


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["Q", "K", "V", "S0"])
def test_gradients_against_differences(L, which):
    """The outputs are linear in each of Q, K, V, S0 alone, so a central difference of any width is exact."""
    B, H, n, d, dv = 1, 2, 270, 24, 40
    Q, K, V, dO, ld, S0, dS1 = inputs(B, H, H, n, d, dv, F, "heads", 5, True)
    p = L.Decay(B, H, n, d, dv, io=F, backward=True)
    g = p.backward(Q, K, V, dO, ld, None, S0, dS1)["d" + which]
    x = {"Q": Q, "K": K, "V": V, "S0": S0}
    step = torch.randn_like(x[which])
    loss = []
    for sign in (1, -1):
        y = dict(x)
        y[which] = x[which] + sign * step
        O, S1 = p.forward(y["Q"], y["K"], y["V"], ld, None, y["S0"], want_state=True)
        loss.append((O.double() * dO).sum() + (S1.double() * dS1).sum())
    by_formula = (g.double() * step).sum()
    size = (g.double() * step).norm() * 10
    assert abs((loss[0] - loss[1]) / 2 - by_formula) < 1e-4 * size


@pytest.mark.gpu
def test_other_stream_and_graph(L):
    """The calls run on the stream they are given, and can be captured."""
    Q, K, V, _, ld, S0, _ = inputs(2, 4, 4, 600, 64, 64, BF, "tokens", 2, True)
    p = L.Decay(2, 4, 600, 64, 64, io=BF)
    want, S1 = p.forward(Q, K, V, ld, None, S0, want_state=True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    O, S = torch.zeros_like(want), torch.zeros_like(S1)
    with torch.cuda.stream(s):
        p.forward(Q, K, V, ld, None, S0, want_state=True, O=O, S1=S)
    s.synchronize()
    assert torch.equal(O, want) and torch.equal(S, S1)
    O.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p.forward(Q, K, V, ld, None, S0, want_state=True, O=O, S1=S)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(O, want)


def test_refusals(L):
    """Bad descriptors, strides, pointers and sizes are refused before any launch."""
    lib, P = L._lib, ctypes.c_void_p

    def size(dd):
        return lib.luna_decay_workspace_size(ctypes.byref(dd), 0, ctypes.byref(ctypes.c_size_t()))

    def fwd(dd, ld=256, q=256, o=256, ws=256, nbytes=1 << 40):
        return lib.luna_decay_fwd(ctypes.byref(dd), P(ld), P(q), P(256), P(256), None, None, P(o), None, P(ws), nbytes, None)

    ok = dict(B=2, H=4, n=100, d=64, dv=64)
    assert size(L.decay_desc(**ok)) == 0
    for bad in (dict(ok, B=-1), dict(ok, d=0), dict(ok, Hkv=3), dict(ok, Hkv=0), dict(ok, io=7), dict(ok, scale=float("nan"))):
        assert size(L.decay_desc(**bad)) == 1, bad
    for bad in (dict(ok, d=129), dict(ok, dv=200), dict(ok, n=(1 << 24) + 1), dict(ok, B=1 << 23)):
        assert size(L.decay_desc(**bad)) == 2, bad
    dd = L.decay_desc(**ok)
    assert fwd(dd, ld=0) == 1 and fwd(dd, q=0) == 1 and fwd(dd, o=0) == 1 and fwd(dd, ws=0) == 1 and fwd(dd, ws=128) == 1
    assert fwd(dd, nbytes=64) == 3
    for s in ((64 * 99, 64 * 100, 64), (64 * 400, 64 * 100, 63), (0, 64 * 100, 64), (64 * 400, 1, 64)):  # overlapping outputs
        dd.o = L.Strides(*s)
        assert fwd(dd) == 1, s
    dd.o = L.Strides(0, 0, 0)
    dd.q = L.Strides(-64, 1, 1)
    assert fwd(dd) == 1
    # gradients and the step
    dd = L.decay_desc(**ok)
    assert lib.luna_decay_bwd(ctypes.byref(dd), P(256), P(256), P(256), P(256), None, None, None, None, P(256), P(256),
                              P(256), None, P(256), 1 << 40, None) == 1
    dd.gk = L.Strides(64, 64, 64)
    assert lib.luna_decay_bwd(ctypes.byref(dd), P(256), P(256), P(256), P(256), P(256), None, None, None, P(256), P(256),
                              P(256), None, P(256), 1 << 40, None) == 1
    assert lib.luna_decay_step(ctypes.byref(dd), P(256), P(256), P(256), P(256), None, 1, P(256), P(256), None) == 1
    assert lib.luna_decay_step(ctypes.byref(dd), P(256), P(256), P(256), P(256), None, 2, None, P(256), None) == 1
    # empty problems are no-ops
    for z in (dict(ok, B=0), dict(ok, H=0, Hkv=0)):
        dd = L.decay_desc(**z)
        assert lib.luna_decay_fwd(ctypes.byref(dd), None, None, None, None, None, None, None, None, None, 0, None) == 0
    dd = L.decay_desc(**dict(ok, n=0))
    assert lib.luna_decay_fwd(ctypes.byref(dd), None, None, None, None, None, None, None, None, None, 0, None) == 0


def test_binding_checks():
    """The class refuses shapes, types and layouts that the call could not tell apart."""
    from paper_2512_08061_gb300 import build
    build.build()
    import paper_2512_08061_gb300.luna as L
    p = L.Decay(2, 2, 8, 16, 16, io=torch.float32, device="cpu")
    x = torch.zeros(2, 2, 8, 16)
    ld = torch.zeros(2)
    with pytest.raises(ValueError):
        p.forward(x[:, :, :7], x, x, ld)
    with pytest.raises(TypeError):
        p.forward(x.double(), x, x, ld)
    with pytest.raises(ValueError):
        p.forward(x, x.transpose(2, 3).contiguous().transpose(2, 3), x, ld)
    with pytest.raises(ValueError):
        p.forward(x, x[:1, :1, :1].expand(2, 2, 8, 16), x, ld)
    with pytest.raises(ValueError):
        p.forward(x, x, x, torch.zeros(3))
    with pytest.raises(ValueError):
        p.forward(x, x, x, ld, None, torch.zeros(2, 2, 16, 16).transpose(2, 3))
    with pytest.raises(TypeError):
        p.forward(x, x, x, ld, torch.zeros(2, dtype=torch.int64))
