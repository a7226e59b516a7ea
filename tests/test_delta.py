"""The gated delta rule against its recurrence in 64 bits, token by token.

Tolerances (relative 2-norms), from the number formats.  A bf16 output carries its own rounding (2^-9 of a value at
most, 1.7e-3 in the root mean square over a binade) and those of the two operands of the product it comes from:
sqrt(3) * 1.7e-3 = 2.9e-3, taken as 4e-3.  The gates' bf16 gradients are sums of such products in which parts of
either sign meet (twice their norm at most over these inputs): 6e-3.  fp32 outputs and states sum at most a few
thousand terms rounded at 2^-24, under sqrt(4096) * 6e-8 = 4e-6 (states of the bf16 form come from operands in two
terms, off by less than that): 1e-5; the gates' fp32 gradients twice that.
"""
import ctypes
import os

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F, BF = torch.float32, torch.bfloat16
TOL = {F: 1e-5, BF: 4e-3}
GATE_TOL = {F: 2e-5, BF: 6e-3}


def tol(name, dtype):
    return (GATE_TOL if name in ("dlog_decay", "dbeta") else TOL)[dtype]


@pytest.fixture(scope="module")
def L():
    from paper_2512_08061_gb300 import build
    build.build()
    import paper_2512_08061_gb300.luna as L
    return L


def recurrence(q, k, v, g, beta, scale, lengths=None, S0=None, dO=None, dS1=None):
    """fp64 numpy, heads of q and k already repeated: O, S1 and with dO the gradients."""
    B, H, n, d = q.shape
    dv = v.shape[-1]
    lens = np.full(B, n) if lengths is None else np.clip(lengths, 0, n)
    live = (np.arange(n) < lens[:, None])[:, None, :]
    q, k, v = (np.where(live[..., None], x, 0.0) for x in (q, k, v))
    a, beta = np.exp(np.where(live, g, 0.0)), np.where(live, beta, 0.0)
    S = np.zeros((B, H, d, dv)) if S0 is None else S0.copy()
    O, states = np.zeros((B, H, n, dv)), [S]
    for t in range(n):
        old = a[:, :, t, None, None] * S
        u = beta[:, :, t, None] * (v[:, :, t] - np.einsum("bhd,bhde->bhe", k[:, :, t], old))
        S = old + k[:, :, t, :, None] * u[:, :, None, :]   # (a row behind the end: a = 1, u = 0)
        O[:, :, t] = scale * np.einsum("bhd,bhde->bhe", q[:, :, t], S)
        if dO is not None:
            states.append(S)
    out = {"O": O, "S1": S}
    if dO is None:
        return out
    dO = np.where(live[..., None], dO, 0.0)
    R = np.zeros((B, H, d, dv)) if dS1 is None else dS1.copy()
    dQ, dK, dV = np.zeros((B, H, n, d)), np.zeros((B, H, n, d)), np.zeros((B, H, n, dv))
    dg, db = np.zeros((B, H, n)), np.zeros((B, H, n))
    for t in range(n - 1, -1, -1):
        b = beta[:, :, t, None]
        old = a[:, :, t, None, None] * states[t]
        err = v[:, :, t] - np.einsum("bhd,bhde->bhe", k[:, :, t], old)
        dQ[:, :, t] = scale * np.einsum("bhde,bhe->bhd", states[t + 1], dO[:, :, t])
        R = R + scale * q[:, :, t, :, None] * dO[:, :, t, None, :]
        du = np.einsum("bhd,bhde->bhe", k[:, :, t], R)
        dV[:, :, t] = b * du
        db[:, :, t] = (du * err).sum(-1)
        dK[:, :, t] = np.einsum("bhde,bhe->bhd", R, b * err) - np.einsum("bhde,bhe->bhd", old, b * du)
        R = R - k[:, :, t, :, None] * (b * du)[:, :, None, :]
        dg[:, :, t] = (R * old).sum((-1, -2))
        R = a[:, :, t, None, None] * R
    on = live[..., None]
    out |= {"dQ": np.where(on, dQ, 0), "dK": np.where(on, dK, 0), "dV": np.where(on, dV, 0), "dlog_decay": np.where(live, dg, 0),
            "dbeta": np.where(live, db, 0), "dS0": R}
    return out


def f64(t):
    return t.double().cpu().numpy()


def rel(a, r):
    a = f64(a)
    assert np.isfinite(a).all()
    return np.linalg.norm(a - r) / max(np.linalg.norm(r), 1e-30)


def inputs(B, H, Hk, n, d, dv, io, layout, seed, state):
    g = torch.Generator("cuda").manual_seed(seed)

    def rn(heads, w, unit=False):
        x = torch.randn((B, n, heads, w), generator=g, device="cuda")
        x = (x / x.norm(dim=-1, keepdim=True).clamp(min=1e-20) if unit else x).to(io)
        if layout == "tokens":      # heads next to each other within a token
            return x.transpose(1, 2)
        if layout == "wide":        # views into a wider row, as of a fused projection
            y = torch.full((B, n, heads * w + 24), float("nan"), device="cuda", dtype=io)
            y[..., 16:16 + heads * w] = x.flatten(2)
            return y[..., 16:16 + heads * w].unflatten(2, (heads, w)).transpose(1, 2)
        return x.transpose(1, 2).contiguous()

    def gates(x):
        return x.to(io) if layout == "heads" else x.transpose(1, 2).contiguous().to(io).transpose(1, 2)

    rate = torch.logspace(-3, -0.3, H, device="cuda").view(1, H, 1)
    lg = gates(-rate * 2 * torch.rand((B, H, n), generator=g, device="cuda"))
    beta = gates(torch.rand((B, H, n), generator=g, device="cuda"))
    S = torch.randn((B, H, d, dv), generator=g, device="cuda") if state else None
    dS = torch.randn((B, H, d, dv), generator=g, device="cuda") if state else None
    return rn(Hk, d, True), rn(Hk, d, True), rn(H, dv), rn(H, dv), lg, beta, S, dS


def check_all(L, B, H, Hk, n, d, dv, io, layout, lengths, state, gates=None, nan_padding=False, beta=None):
    Q, K, V, dO, lg, bt, S0, dS1 = inputs(B, H, Hk, n, d, dv, io, layout, 7 * n + d, state)
    if gates is not None:
        lg.copy_(gates(lg))
    if beta is not None:
        bt.copy_(beta(bt))
    lens = None if lengths is None else torch.tensor(lengths, device="cuda", dtype=torch.int32)
    rq, rk, rv, rg, ra, rb = (f64(x) for x in (Q, K, V, dO, lg, bt))
    if nan_padding:
        for b, m in enumerate(lengths):
            for x in (Q, K, V, dO, lg, bt):
                x[b, :, max(0, m):] = float("nan")
    G = H // Hk
    ref = recurrence(rq.repeat(G, 1), rk.repeat(G, 1), rv, ra, rb, d ** -0.5, lengths and np.array(lengths),
                     None if S0 is None else f64(S0), rg, None if dS1 is None else f64(dS1))
    for x in ("dQ", "dK"):
        ref[x] = ref[x].reshape(B, Hk, G, n, -1).sum(2)
    p = L.Delta(B, H, n, d, dv, Hk=Hk, io=io, backward=True)
    O, S1 = p.forward(Q, K, V, lg, bt, lens, S0, want_state=True)
    assert L.luna_device_status(p.ws) == 0
    g = p.backward(Q, K, V, dO, lg, bt, lens, S0, dS1)
    assert L.luna_device_status(p.ws) == 0
    got = {"O": O, "S1": S1, **g}
    off = {name: rel(t, ref[name]) for name, t in got.items()}
    assert all(off[name] < tol(name, t.dtype) for name, t in got.items()), off
    if lengths is not None:
        for b, m in enumerate(lengths):
            for name in set(got) - {"S1", "dS0"}:
                assert not got[name][b, :, max(0, min(n, m)):].any(), name
    again = p.backward(Q, K, V, dO, lg, bt, lens, S0, dS1)
    for name in g:
        assert torch.equal(g[name], again[name]), name
    assert torch.equal(p.forward(Q, K, V, lg, bt, lens, S0), O)


CASES = [  # B, H, Hk, n, d, dv, io, layout, lengths, state
    (1, 1, 1, 1, 1, 1, F, "heads", None, False),
    (2, 3, 3, 33, 7, 5, F, "tokens", [33, 0], True),
    (1, 2, 1, 300, 40, 72, F, "wide", None, True),
    (2, 4, 2, 515, 64, 64, F, "heads", [515, 257], False),
    (3, 2, 2, 130, 128, 128, F, "tokens", [64, 65, 128], True),
    (1, 1, 1, 1, 64, 64, BF, "heads", None, True),
    (2, 2, 2, 127, 64, 64, BF, "tokens", [127, 1], False),
    (1, 2, 2, 128, 128, 128, BF, "heads", None, True),
    (3, 2, 1, 129, 128, 64, BF, "wide", [129, 128, 0], True),
    (1, 3, 1, 700, 32, 128, BF, "tokens", [641], True),
    (2, 6, 3, 1025, 128, 128, BF, "tokens", [1025, 300], True),
    (1, 2, 2, 260, 40, 24, BF, "heads", None, False),
    (1, 2, 1, 200, 33, 50, BF, "tokens", [199], True),     # widths that no 16-byte access covers
    (1, 2, 2, 520, 8, 120, BF, "wide", None, False),
    (4, 2, 2, 66, 64, 128, BF, "heads", [63, 64, 65, 66], True),
    (2, 4, 2, 150, 61, 61, BF, "wide", [150, 77], True),
    (1, 2, 2, 90, 5, 128, BF, "heads", None, True),
    (1, 2, 1, 200, 127, 7, BF, "tokens", None, False),
    (3, 5, 5, 70, 72, 88, BF, "tokens", [70, 3, 64], True),
    (2, 2, 2, 400, 96, 17, F, "tokens", [400, 190], True),
    (8, 24, 24, 70, 72, 40, F, "tokens", [70, 1, 64, 65, 0, 17, 16, 33], True),  # (more columns than the SMs hold in small blocks)
    (10, 16, 8, 40, 20, 50, F, "heads", None, False),
    (10, 16, 16, 37, 64, 64, F, "wide", [37, 36, 32, 31, 17, 16, 15, 2, 1, 0], True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,Hk,n,d,dv,io,layout,lengths,state", CASES)
def test_prompts_and_gradients(L, B, H, Hk, n, d, dv, io, layout, lengths, state):
    check_all(L, B, H, Hk, n, d, dv, io, layout, lengths, state)


def test_formulas_against_differences():
    """The reference's gradients are those of its outputs: central differences in 64 bits, whose error at steps of
    1e-5 is some 1e-10 of the third derivative and 1e-16 / 1e-5 of the loss."""
    r = np.random.default_rng(3)
    B, H, n, d, dv = 2, 2, 9, 5, 4
    x = {"q": r.normal(size=(B, H, n, d)), "k": r.normal(size=(B, H, n, d)) * d ** -0.5, "v": r.normal(size=(B, H, n, dv)),
         "g": -r.random((B, H, n)), "beta": r.random((B, H, n)), "S0": r.normal(size=(B, H, d, dv))}
    dO, dS1, lens = r.normal(size=(B, H, n, dv)), r.normal(size=(B, H, d, dv)), np.array([9, 6])
    grads = recurrence(**x, scale=0.4, lengths=lens, dO=dO, dS1=dS1)
    on = (np.arange(n) < lens[:, None])[:, None, :, None]

    def loss(y):
        out = recurrence(**y, scale=0.4, lengths=lens)
        return (out["O"] * dO * on).sum() + (out["S1"] * dS1).sum()

    for name, grad in (("q", "dQ"), ("k", "dK"), ("v", "dV"), ("g", "dlog_decay"), ("beta", "dbeta"), ("S0", "dS0")):
        step = r.normal(size=x[name].shape)
        diff = (loss({**x, name: x[name] + 1e-5 * step}) - loss({**x, name: x[name] - 1e-5 * step})) / 2e-5
        want = (grads[grad] * step).sum()
        assert abs(diff - want) < 1e-7 * np.linalg.norm(grads[grad]), name


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["Q", "V", "S0"])
def test_gradients_against_differences(L, which):
    """The outputs are linear in each of Q, V, S0 alone, so a central difference of any width is exact: the fp32
    outputs' 1e-5 of the loss's terms, taken as 1e-4 of their root sum of squares."""
    B, H, n, d, dv = 1, 2, 270, 24, 40
    Q, K, V, dO, lg, bt, S0, dS1 = inputs(B, H, H, n, d, dv, F, "heads", 5, True)
    p = L.Delta(B, H, n, d, dv, io=F, backward=True)
    g = p.backward(Q, K, V, dO, lg, bt, None, S0, dS1)["d" + which]
    x = {"Q": Q, "V": V, "S0": S0}
    step = torch.randn_like(x[which])
    loss = []
    for sign in (1, -1):
        y = dict(x)
        y[which] = x[which] + sign * step
        O, S1 = p.forward(y["Q"], K, y["V"], lg, bt, None, y["S0"], want_state=True)
        loss.append((O.double() * dO).sum() + (S1.double() * dS1).sum())
    by_formula = (g.double() * step).sum()
    size = (g.double() * step).norm() * 10
    assert abs((loss[0] - loss[1]) / 2 - by_formula) < 1e-4 * size


@pytest.mark.gpu
@pytest.mark.parametrize("H,Hk,n,d,dv", [(8, 8, 1024, 128, 128), (8, 2, 900, 128, 64), (6, 6, 1100, 64, 64), (12, 4, 700, 32, 64)])
def test_many_heads_of_many_chunks(L, H, Hk, n, d, dv):
    """Every SM at work, against the fp32 form of the same call on the same values, head by head."""
    B = 24
    Q, K, V, dO, lg, bt, _, _ = inputs(B, H, Hk, n, d, dv, BF, "tokens", 21, False)
    lens = torch.randint(n // 2, n + 1, (B,), device="cuda", dtype=torch.int32)
    p, f = (L.Delta(B, H, n, d, dv, Hk=Hk, io=io, backward=True) for io in (BF, F))
    wide = [x.float() for x in (Q, K, V, dO, lg, bt)]
    want, S = f.forward(*wide[:3], *wide[4:], lens, want_state=True)
    grads = f.backward(*wide, lens)
    for _ in range(3):
        got, S1 = p.forward(Q, K, V, lg, bt, lens, want_state=True)
        pairs = {"O": (got, want), "S1": (S1, S)}
        pairs.update({k: (v, grads[k]) for k, v in p.backward(Q, K, V, dO, lg, bt, lens).items()})
        for name, (a, b) in pairs.items():
            by_head = (a.double() - b).flatten(2).norm(dim=2) / b.double().flatten(2).norm(dim=2)
            assert by_head.max() < tol(name, a.dtype), name


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
def test_padding_may_hold_anything(L, io):
    """NaN in rows at and past the length reaches no output; lengths outside [0, n] are clamped."""
    check_all(L, 3, 2, 2, 300, 64, 64, io, "heads", [299, 130, 0], True, nan_padding=True)
    check_all(L, 2, 2, 2, 300, 64, 64, io, "heads", [-5, 1000], True)


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
@pytest.mark.parametrize("which", ["Q", "K", "V", "dO"])
def test_rows_of_different_size(L, io, which):
    """Rows of one tensor 2^-12 to 1 times as large as their neighbours.  What is proportional to a row (O to Q's, dQ to
    dO's) is within the tolerance with that factor divided out, and everything within it as a whole.  (A row's error over
    its own value has no bound: q_i . k_j may be as near to 0 as it likes, and the rounding of its terms is not.)"""
    B, H, n, d = 1, 2, 200, 64
    Q, K, V, dO, lg, bt, S0, dS1 = inputs(B, H, H, n, d, d, io, "tokens", 17, which != "V")
    x = {"Q": Q, "K": K, "V": V, "dO": dO}
    g = torch.Generator("cuda").manual_seed(3)
    size = 2.0 ** -torch.randint(0, 13, (B, H, n, 1), generator=g, device="cuda")
    x[which].mul_(size)
    ref = recurrence(*(f64(t) for t in (Q, K, V, lg, bt)), d ** -0.5, None, None if S0 is None else f64(S0), f64(dO),
                     None if dS1 is None else f64(dS1))
    p = L.Delta(B, H, n, d, d, io=io, backward=True)
    got = {"O": p.forward(Q, K, V, lg, bt, None, S0), **p.backward(Q, K, V, dO, lg, bt, None, S0, dS1)}
    for name, t in got.items():
        assert rel(t, ref[name]) < tol(name, t.dtype), name
    own = {"Q": "O", "dO": "dQ"}.get(which)
    if own:
        assert rel(got[own].float() / size, ref[own] / f64(size)) < TOL[io]


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1, 2, 3, 4, 5])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_not_finite(L, which, value):
    """A value that is not finite shows in its row's outputs or gradients, and stays in its sequence and head."""
    B, H, n, d = 2, 2, 150, 64
    x = list(inputs(B, H, H, n, d, d, BF, "tokens", 6, False)[:6])  # Q, K, V, dO, gates, betas
    p = L.Delta(B, H, n, d, d, io=BF, backward=True)

    def run():
        return {"O": p.forward(x[0], x[1], x[2], x[4], x[5]), **p.backward(x[0], x[1], x[2], x[3], x[4], x[5])}

    want = run()
    x[which][1, 0, 70].view(-1)[0] = value
    got = run()
    for name in got:
        for b, h in ((0, 0), (0, 1), (1, 1)):
            assert torch.equal(got[name][b, h], want[name][b, h]), name
    assert any(not torch.isfinite(got[name][1, 0, 70].float()).all() for name in got)
    assert L.luna_device_status(p.ws) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
@pytest.mark.parametrize("case", ["none", "reset", "far", "all"])
def test_extreme_gates(L, io, case):
    """No forgetting; a state that starts anew at some tokens (a gate of -inf, its gradient 0) between slow ones;
    gates far below what exp resolves; every token for itself."""
    def gates(lg):
        x = lg.clone()
        if case == "none":
            x.zero_()
        elif case == "reset":
            x[:, :, ::7] = -float("inf")
        elif case == "far":
            x[:, :, 5::11] = -1e30
            x[:, :, 3::11] = -90.0
        else:
            x.fill_(-float("inf"))
        return x

    check_all(L, 1, 4, 4, 400, 64, 64, io, "heads", None, True, gates)


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
@pytest.mark.parametrize("value", [0.0, 1.0, 1.75])
def test_extreme_betas(L, io, value):
    """Nothing is written; a value is replaced; more than replaced, so that the state changes sign along the key."""
    check_all(L, 1, 2, 2, 200, 64, 64, io, "tokens", None, True, beta=lambda b: torch.full_like(b, value))


@pytest.mark.gpu
def test_unaligned_views(L):
    """bf16 tensors one element off a 16-byte boundary give the same values."""
    B, H, n, d = 1, 2, 200, 64
    Q, K, V, dO, lg, bt, S0, _ = inputs(B, H, H, n, d, d, BF, "heads", 3, True)
    odd = []
    for x in (Q, K, V, dO):
        y = torch.empty(x.numel() + 1, dtype=BF, device="cuda")[1:].view(x.shape)
        odd.append(y.copy_(x))
    p = L.Delta(B, H, n, d, d, io=BF, backward=True)
    a, b = p.forward(Q, K, V, lg, bt, None, S0), p.forward(*odd[:3], lg, bt, None, S0)
    assert (a.double() - b.double()).norm() < TOL[BF] * a.double().norm()
    a, b = p.backward(Q, K, V, dO, lg, bt, None, S0), p.backward(*odd, lg, bt, None, S0)
    for name in a:
        assert (a[name].double() - b[name].double()).norm() < tol(name, a[name].dtype) * a[name].double().norm(), name


@pytest.mark.gpu
def test_repeated_inputs(L):
    """Inputs that repeat along a dimension (stride 0) are read as what they stand for."""
    B, H, n, d = 3, 4, 100, 64
    Q, K, V, dO, lg, bt, _, _ = inputs(1, H, 1, n, d, d, BF, "heads", 4, False)
    wide = [x.expand(B, *x.shape[1:]) for x in (Q, K, V, dO, lg[:, :1].expand(1, H, n), bt[:, :, :1].expand(1, H, n))]
    dense = [x.contiguous() for x in wide]
    p = L.Delta(B, H, n, d, d, Hk=1, io=BF, backward=True)
    out = {"d" + k: torch.empty_like(x) for k, x in zip(("Q", "K", "V", "O", "log_decay", "beta"), dense)}
    assert torch.equal(p.forward(*wide[:3], *wide[4:], O=torch.empty_like(dense[2])), p.forward(*dense[:3], *dense[4:]))
    a, b = p.backward(*wide, out=out), p.backward(*dense)
    for name in b:
        assert torch.equal(a[name], b[name]), name


@pytest.mark.gpu
@pytest.mark.parametrize("io,d,dv,H,Hk", [(F, 13, 70, 4, 2), (BF, 64, 64, 3, 3), (BF, 128, 128, 4, 1), (BF, 33, 6, 2, 2)])
def test_tokens_continue_a_prompt(L, io, d, dv, H, Hk):
    """A prompt in two pieces, then single tokens, give the rows of the whole prompt."""
    B, n = 2, 150
    Q, K, V, _, lg, bt, S0, _ = inputs(B, H, Hk, n, d, dv, io, "tokens", 11, True)
    cut, steps = 77, 9
    G = H // Hk
    ref = recurrence(f64(Q).repeat(G, 1), f64(K).repeat(G, 1), f64(V), f64(lg), f64(bt), d ** -0.5, None, f64(S0))
    state = S0.clone()
    out = []
    for a, b in ((0, cut), (cut, n - steps)):
        p = L.Delta(B, H, b - a, d, dv, Hk=Hk, io=io)
        o, state = p.forward(*(x[:, :, a:b] for x in (Q, K, V, lg, bt)), None, state, want_state=True, S1=state)
        out.append(o)
    pool = torch.full((5, H, d, dv), float("nan"), device="cuda")
    slots = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    pool[slots.long()] = state
    p = L.Delta(B, H, 1, d, dv, Hk=Hk, io=io)
    for t in range(n - steps, n):
        out.append(p.step(*(x[:, :, t] for x in (Q, K, V, lg, bt)), pool, slots).unsqueeze(2))
    assert rel(torch.cat(out, 2), ref["O"]) < TOL[io]
    assert rel(pool[slots.long()], ref["S1"]) < TOL[F]
    assert torch.isnan(pool[[0, 2, 4]]).all()


@pytest.mark.gpu
def test_slow_gates_over_many_tokens(L):
    """20000 tokens with keys of one sign under slow gates, in one call and one by one: errors of one sign would add up."""
    H, n, d = 5, 20000, 16
    g = torch.Generator("cuda").manual_seed(8)
    rates = torch.tensor([-1e-6, -1e-5, -1e-4, -1e-3, -0.49], device="cuda")
    q, v = (torch.rand((1, H, n, d), generator=g, device="cuda") for _ in range(2))
    k = torch.rand((1, H, n, d), generator=g, device="cuda")
    k = k / k.norm(dim=-1, keepdim=True)
    lg, bt = rates.view(1, H, 1).expand(1, H, n).contiguous(), torch.full((1, H, n), 1e-3, device="cuda")
    want = recurrence(*(f64(x) for x in (q, k, v, lg, bt)), d ** -0.5)
    _, prompt = L.Delta(1, H, n, d, d, io=F).forward(q, k, v, lg, bt, want_state=True)
    p, state, o = L.Delta(1, H, 1, d, d, io=F), torch.zeros((1, H, d, d), device="cuda"), None
    for t in range(n):
        o = p.step(q[:, :, t], k[:, :, t], v[:, :, t], lg[:, :, t], bt[:, :, t], state, o=o)
    for got in (prompt, state):
        off = np.linalg.norm((f64(got) - want["S1"])[0].reshape(H, -1), axis=1) / np.linalg.norm(want["S1"][0].reshape(H, -1), axis=1)
        assert (off < TOL[F]).all(), off


@pytest.mark.gpu
def test_idle_slots(L):
    """A slot outside the pool leaves every state alone and gives zeros."""
    B, H, d = 3, 2, 32
    p = L.Delta(B, H, 1, d, d, io=BF)
    pool = torch.ones((2, H, d, d), device="cuda")
    q = torch.ones((B, H, d), device="cuda", dtype=BF)
    slots = torch.tensor([-1, 2, 1], dtype=torch.int32, device="cuda")
    gate = torch.zeros((B, H), device="cuda", dtype=BF)
    o = p.step(q, q, q, gate, gate + 1, pool, slots)
    assert not o[:2].any() and o[2].any()
    assert (pool[0] == 1).all() and (pool[1] == 1 + (1 - d)).all()


@pytest.mark.gpu
def test_other_stream_and_graph(L):
    """The calls run on the stream they are given, and can be captured, forward and backward."""
    Q, K, V, dO, lg, bt, S0, _ = inputs(2, 4, 4, 600, 64, 64, BF, "tokens", 2, True)
    p = L.Delta(2, 4, 600, 64, 64, io=BF, backward=True)
    want, S1 = p.forward(Q, K, V, lg, bt, None, S0, want_state=True)
    grads = p.backward(Q, K, V, dO, lg, bt, None, S0)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    O, S = torch.zeros_like(want), torch.zeros_like(S1)
    with torch.cuda.stream(s):
        p.forward(Q, K, V, lg, bt, None, S0, want_state=True, O=O, S1=S)
    p.forward(Q, K, V, lg, bt, None, S0, stream=s)
    s.synchronize()
    assert torch.equal(O, want) and torch.equal(S, S1)
    O.zero_()
    out = {k: torch.zeros_like(v) for k, v in grads.items()}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p.forward(Q, K, V, lg, bt, None, S0, want_state=True, O=O, S1=S)
        p.backward(Q, K, V, dO, lg, bt, None, S0, out=out)
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(O, want)
    for name in grads:
        assert torch.equal(out[name], grads[name]), name


@pytest.mark.gpu
def test_memory_of_a_call_on_another_stream(L):
    """What a call on a stream allocates is that stream's: not handed out on the current one while the call may run."""
    B, H, n, d = 2, 32, 1024, 128
    io = dict(device="cuda", dtype=BF)
    x, gate = torch.randn((B, H, n, d), **io), torch.full((B, H, n), -0.1, **io)
    k = torch.nn.functional.normalize(x, dim=-1)
    s = torch.cuda.Stream()
    p = L.Delta(B, H, n, d, d, backward=True)
    want = p.forward(k, k, x, gate, -gate)
    torch.cuda.synchronize()
    for call in (lambda: (p.forward(k, k, x, gate, -gate, stream=s),), lambda: tuple(p.backward(k, k, x, x, gate, -gate, stream=s).values())[:3]):
        out = call()
        there = {t.data_ptr(): (t.shape, t.dtype) for t in out}
        del out
        mine = [torch.empty(shape, dtype=dtype, device="cuda") for shape, dtype in there.values()]
        assert not any(t.data_ptr() in there for t in mine)
        del mine
    torch.cuda.synchronize()
    assert torch.equal(p.forward(k, k, x, gate, -gate), want)


@pytest.mark.gpu
def test_two_plans_at_once(L):
    """Two plans on two streams, and a captured call replayed beside them, keep out of each other's memory."""
    a = inputs(2, 4, 4, 900, 64, 64, BF, "tokens", 2, True)
    b = inputs(2, 4, 2, 700, 128, 64, BF, "tokens", 3, True)
    plans = [L.Delta(2, 4, 900, 64, 64, backward=True), L.Delta(2, 4, 700, 128, 64, Hk=2, backward=True), L.Delta(2, 4, 900, 64, 64)]
    call = lambda p, x: p.backward(x[0], x[1], x[2], x[3], x[4], x[5], None, x[6], x[7])  # noqa: E731
    want = [call(plans[0], a), call(plans[1], b), plans[2].forward(a[0], a[1], a[2], a[4], a[5], None, a[6])]
    O = torch.empty_like(want[2])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        plans[2].forward(a[0], a[1], a[2], a[4], a[5], None, a[6], O=O)
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        O.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            x = call(plans[0], a)
        with torch.cuda.stream(t):
            y = call(plans[1], b)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x[k], want[0][k]) for k in x) and all(torch.equal(y[k], want[1][k]) for k in y)
        assert torch.equal(O, want[2])


@pytest.mark.gpu
def test_empty(L):
    """No tokens: the states pass through."""
    p = L.Delta(2, 2, 0, 16, 16, io=F, backward=True)
    x, gate = torch.zeros((2, 2, 0, 16), device="cuda"), torch.zeros((2, 2, 0), device="cuda")
    S0 = torch.randn((2, 2, 16, 16), device="cuda")
    _, S1 = p.forward(x, x, x, gate, gate, None, S0, want_state=True)
    assert torch.equal(S0, S1)
    assert torch.equal(p.backward(x, x, x, x, gate, gate, None, S0, S1)["dS0"], S1)


def test_refusals(L):
    """Bad descriptors, strides, pointers and sizes are refused before any launch."""
    lib, P = L._lib, ctypes.c_void_p

    def size(dd):
        return lib.luna_delta_workspace_size(ctypes.byref(dd), 1, ctypes.byref(ctypes.c_size_t()))

    def fwd(dd, ld=256, bt=256, q=256, o=256, ws=256, nbytes=1 << 50):
        return lib.luna_delta_fwd(ctypes.byref(dd), P(ld), P(bt), P(q), P(256), P(256), None, None, P(o), None, P(ws), nbytes, None)

    def bwd(dd, dO=256, dg=256, db=256, nbytes=1 << 50):
        return lib.luna_delta_bwd(ctypes.byref(dd), *[P(256)] * 5, P(dO), None, None, None, *[P(256)] * 3, P(dg), P(db), None,
                                  P(256), nbytes, None)

    ok = dict(B=2, H=4, n=100, d=64, dv=64)
    assert size(L.delta_desc(**ok)) == 0
    for bad in (dict(ok, B=-1), dict(ok, d=0), dict(ok, Hk=3), dict(ok, Hk=0), dict(ok, io=7), dict(ok, scale=float("nan"))):
        assert size(L.delta_desc(**bad)) == 1, bad
    for bad in (dict(ok, d=129), dict(ok, dv=200), dict(ok, n=(1 << 24) + 1), dict(ok, B=1 << 23), dict(ok, B=1 << 12, n=1 << 24)):
        assert size(L.delta_desc(**bad)) == 2, bad
    dd = L.delta_desc(**ok)
    assert fwd(dd, ld=0) == 1 and fwd(dd, bt=0) == 1 and fwd(dd, q=0) == 1 and fwd(dd, o=0) == 1
    assert fwd(dd, ws=0) == 1 and fwd(dd, ws=128) == 1 and fwd(dd, nbytes=64) == 3
    for s in ((64 * 99, 64 * 100, 64), (64 * 400, 64 * 100, 63), (0, 64 * 100, 64), (64 * 400, 1, 64)):  # overlapping outputs
        dd.o = L.Strides(*s)
        assert fwd(dd) == 1, s
    dd.o = L.Strides(0, 0, 0)
    for field in ("q", "g", "beta"):
        setattr(dd, field, L.Strides(-64, 1, 1))
        assert fwd(dd) == 1
        setattr(dd, field, L.Strides(0, 0, 0))
    # gradients and the step
    assert bwd(dd, dO=0) == 1 and bwd(dd, dg=0) == 1 and bwd(dd, db=0) == 1 and bwd(dd, nbytes=256) == 3
    for field, s in (("gk", (64, 64, 64)), ("gg", (100, 0, 1)), ("gbeta", (400, 99, 1))):
        dd = L.delta_desc(**ok)
        setattr(dd, field, L.Strides(*s))
        assert bwd(dd) == 1, field
    dd = L.delta_desc(**ok)
    step = [ctypes.byref(dd)] + [P(256)] * 5
    assert lib.luna_delta_step(*step, None, 1, P(256), P(256), None) == 1
    assert lib.luna_delta_step(*step, None, 2, None, P(256), None) == 1
    assert lib.luna_delta_step(*step, P(256), -1, P(256), P(256), None) == 1
    # empty problems are no-ops
    for z in (dict(ok, B=0), dict(ok, H=0, Hk=0), dict(ok, n=0)):
        dd = L.delta_desc(**z)
        assert lib.luna_delta_fwd(ctypes.byref(dd), *[None] * 10, 0, None) == 0
        assert lib.luna_delta_bwd(ctypes.byref(dd), *[None] * 16, 0, None) == 0


def test_binding_checks(L):
    """The class refuses shapes, types and layouts that the call could not tell apart."""
    p = L.Delta(2, 2, 8, 16, 16, io=torch.float32, device="cpu", backward=True)
    x, gate = torch.zeros(2, 2, 8, 16), torch.zeros(2, 2, 8)
    for bad, error in (
        ((x[:, :, :7], x, x, gate, gate), ValueError),
        ((x.double(), x, x, gate, gate), TypeError),
        ((x, x.transpose(2, 3).contiguous().transpose(2, 3), x, gate, gate), ValueError),
        ((x, x[:1, :1, :1].expand(2, 2, 8, 16), x, gate, gate), ValueError),
        ((x, x, x, gate[:, :, :7], gate), ValueError),
        ((x, x, x, gate.bfloat16(), gate), TypeError),
        ((x, x, x, gate, gate[:1, :1, :1].expand(2, 2, 8)), ValueError),
        ((x, x, x, gate, gate, torch.zeros(2, dtype=torch.int64)), TypeError),
        ((x, x, x, gate, gate, None, torch.zeros(2, 2, 16, 16).transpose(2, 3)), ValueError),
    ):
        with pytest.raises(error):
            p.forward(*bad)
    with pytest.raises(ValueError):
        p.backward(x, x, x, x[:, :1], gate, gate)
    with pytest.raises(ValueError):
        p.step(x[:, :, 0], x[:, :, 0], x[:, :, 0], gate[:, :, 0], gate, torch.zeros(2, 2, 16, 16))
