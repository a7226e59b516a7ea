"""The gated delta rule where its parts are of very different size: chunks without queries, keys or gradients, strong
gates; and forms of the chain that only many heads reach.

Tolerances are those of test_delta.py, taken chunk by chunk or head by head instead of over whole tensors: they come
from the rounding of single values and of the operands of a product, which is the same for any 64 rows.
"""
import numpy as np
import pytest
import torch

from test_delta import BF, F, GATE_TOL, L, TOL, f64, inputs, recurrence, tol  # noqa: F401  (L: the fixture)


def by(parts, got, want):
    """Largest relative error of the parts that a tensor's rows are cut into by `parts`, on the heads' axis or the rows'."""
    got = f64(got)
    assert np.isfinite(got).all()
    worst = 0.0
    for at in parts:
        off, size = np.linalg.norm(got[at] - want[at]), np.linalg.norm(want[at])
        worst = max(worst, off / size if size else (0.0 if not off else np.inf))
    return worst


def chunks(n):
    return [np.s_[:, :, t:t + 64] for t in range(0, n, 64)]


def heads(H):
    return [np.s_[:, h] for h in range(H)]


def gradients(L, x, Hk, lens=None):
    """O, S1 and the gradients of the call, and of the recurrence in 64 bits."""
    Q, K, V, dO, lg, bt, S0, dS1 = x
    B, H, n, dv = V.shape
    d, G = Q.shape[-1], H // Hk
    ref = recurrence(f64(Q).repeat(G, 1), f64(K).repeat(G, 1), f64(V), f64(lg), f64(bt), d ** -0.5, lens,
                     None if S0 is None else f64(S0), f64(dO), None if dS1 is None else f64(dS1))
    for name in ("dQ", "dK"):
        ref[name] = ref[name].reshape(B, Hk, G, n, d).sum(2)
    p = L.Delta(B, H, n, d, dv, Hk=Hk, io=V.dtype, backward=True)
    lengths = None if lens is None else torch.tensor(lens, device="cuda", dtype=torch.int32)
    O, S1 = p.forward(Q, K, V, lg, bt, lengths, S0, want_state=True)
    got = {"O": O, "S1": S1, **p.backward(Q, K, V, dO, lg, bt, lengths, S0, dS1)}
    assert L.luna_device_status(p.ws) == 0
    return got, ref


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("which,size", [("Q", 0.0), ("Q", 2.0 ** -40), ("K", 0.0), ("K", 2.0 ** -40), ("V", 0.0), ("dO", 0.0), ("dO", 2.0 ** -40)])
@pytest.mark.parametrize("where", ["all", "chunk"])
@pytest.mark.parametrize("state", [True, False])
def test_chunks_of_nothing_or_little(L, io, d, which, size, where, state):
    """Queries, keys, values or output gradients that are zero, or far smaller than all others, throughout or in one chunk:
    what does not hang on them keeps its values.  (A zero key still reads nothing and writes nothing; a zero query still
    has a gradient.)"""
    H, Hk, n = 4, 2, 200
    x = list(inputs(1, H, Hk, n, d, 64, io, "tokens", 31, state))
    t = x[("Q", "K", "V", "dO").index(which)]
    (t if where == "all" else t[:, :, 64:128]).mul_(size)
    got, ref = gradients(L, x, Hk)
    for name, t in got.items():
        parts = [np.s_[:]] if name in ("S1", "dS0") else chunks(n)
        assert by(parts, t, ref[name]) < tol(name, t.dtype), name


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
@pytest.mark.parametrize("d,dv,lens", [(64, 64, None), (128, 128, [200, 77]), (40, 24, None)])
def test_strong_gates(L, io, d, dv, lens):
    """Gates that forget nearly everything at every token: their gradients are as small as exp(gate), and as exact."""
    rates = [-3.0, -5.0, -8.0, -12.0, -30.0]
    H, n, B = len(rates), 200, 2
    x = list(inputs(B, H, H, n, d, dv, io, "heads", 13, True))
    x[4] = torch.tensor(rates, device="cuda").view(1, H, 1).expand(B, H, n).to(io).contiguous()
    got, ref = gradients(L, x, H, lens and np.array(lens))
    for name, t in got.items():
        if name != "dS0" and name != "S1":  # (a state behind 200 such tokens is 0 but for the last of them)
            assert by(heads(H), t, ref[name]) < tol(name, t.dtype), name


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
def test_gates_strong_and_weak(L, io):
    """A strong gate at every fifth token among weak ones, and gates that grow from 0 to -20 along the sequence: the
    gradients of the strong ones on their own."""
    H, n, d = 2, 250, 64
    x = list(inputs(1, H, H, n, d, d, io, "heads", 19, True))
    x[4][:, 0, ::5] = -9.0
    x[4][:, 1] = -torch.linspace(0, 20, n, device="cuda").to(io)
    got, ref = gradients(L, x, H)
    parts = [np.s_[:, 0, ::5], np.s_[:, 0, 1::5], *(np.s_[:, 1, t:t + 50] for t in range(0, n, 50))]
    assert by(parts, got["dlog_decay"], ref["dlog_decay"]) < GATE_TOL[io]


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
def test_zero_keys_under_gates(L, io):
    """Where a chunk's keys are zero and it has no output gradients, a key's gradient is that of the state behind the chunk
    times what the gates leave of the row: row by row, down to exp(-16)."""
    H, n, d = 2, 192, 64
    x = list(inputs(1, H, H, n, d, d, io, "tokens", 37, True))
    for t in (x[1], x[3]):
        t[:, :, 64:128] = 0
    x[4][:, :, 64:128] = -0.25
    got, ref = gradients(L, x, H)
    rows = [np.s_[:, h, t:t + 1] for h in range(H) for t in range(64, 128)]
    assert by(rows, got["dK"], ref["dK"]) < TOL[io]
    assert by(rows, got["dQ"], 0 * ref["dQ"]) == 0.0


@pytest.mark.gpu
@pytest.mark.parametrize("H,Hk,n,d,dv", [(8, 8, 330, 61, 61), (8, 4, 330, 127, 127), (8, 8, 330, 64, 128), (8, 8, 200, 127, 20), (8, 2, 200, 64, 32)])
def test_many_heads_of_any_width(L, H, Hk, n, d, dv):
    """Rows that do not start on 16-byte boundaries, and 128 columns of a state of 64, with every SM at work: against the
    fp32 form of the same call on the same values, head by head."""
    B = 24
    Q, K, V, dO, lg, bt, S0, dS1 = inputs(B, H, Hk, n, d, dv, BF, "tokens", 23, True)
    lens = torch.randint(n // 2, n + 1, (B,), device="cuda", dtype=torch.int32, generator=torch.Generator("cuda").manual_seed(1))
    p, f = (L.Delta(B, H, n, d, dv, Hk=Hk, io=io, backward=True) for io in (BF, F))
    wide = [x.float() for x in (Q, K, V, dO, lg, bt)]
    want, S = f.forward(*wide[:3], *wide[4:], lens, S0, want_state=True)
    grads = f.backward(*wide, lens, S0, dS1)
    got, S1 = p.forward(Q, K, V, lg, bt, lens, S0, want_state=True)
    pairs = {"O": (got, want), "S1": (S1, S)}
    pairs.update({k: (v, grads[k]) for k, v in p.backward(Q, K, V, dO, lg, bt, lens, S0, dS1).items()})
    assert L.luna_device_status(p.ws) == 0
    for name, (a, b) in pairs.items():
        by_head = (a.double() - b).flatten(2).norm(dim=2) / b.double().flatten(2).norm(dim=2)
        assert by_head.max() < tol(name, a.dtype), name


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,n,d,dv", [(1, 2, 200, 64, 64), (24, 8, 150, 64, 128)])
def test_unaligned_views_to_the_bit(L, B, H, n, d, dv):
    """bf16 tensors one element off a 16-byte boundary give the same bits: rows are read and written in other pieces, the
    sums are the same."""
    Q, K, V, dO, lg, bt, S0, dS1 = inputs(B, H, H, n, d, dv, BF, "heads", 3, True)
    odd = [torch.empty(x.numel() + 1, dtype=BF, device="cuda")[1:].view(x.shape).copy_(x) for x in (Q, K, V, dO)]
    p = L.Delta(B, H, n, d, dv, io=BF, backward=True)
    assert torch.equal(p.forward(Q, K, V, lg, bt, None, S0), p.forward(*odd[:3], lg, bt, None, S0))
    a, b = p.backward(Q, K, V, dO, lg, bt, None, S0, dS1), p.backward(*odd, lg, bt, None, S0, dS1)
    for name in a:
        assert torch.equal(a[name], b[name]), name


@pytest.mark.gpu
@pytest.mark.parametrize("d", [16, 128])
def test_slow_gates_over_many_bf16_tokens(L, d):
    """As test_slow_gates_over_many_tokens, on bf16 tensors: the final state of 20000 tokens under slow gates."""
    H, n = 5, 20000
    g = torch.Generator("cuda").manual_seed(8)
    rates = torch.tensor([-1e-6, -1e-5, -1e-4, -1e-3, -0.49], device="cuda")
    q, v = (torch.rand((1, H, n, 16), generator=g, device="cuda").to(BF) for _ in range(2))
    k = torch.rand((1, H, n, d), generator=g, device="cuda")
    k = (k / k.norm(dim=-1, keepdim=True)).to(BF)
    q = q if d == 16 else k
    lg, bt = rates.view(1, H, 1).expand(1, H, n).to(BF).contiguous(), torch.full((1, H, n), 1e-3, device="cuda").to(BF)
    want = recurrence(*(f64(x) for x in (q, k, v, lg, bt)), d ** -0.5)
    _, prompt = L.Delta(1, H, n, d, 16, io=BF).forward(q, k, v, lg, bt, want_state=True)
    p, state, o = L.Delta(1, H, 1, d, 16, io=BF), torch.zeros((1, H, d, 16), device="cuda"), None
    for t in range(n):
        o = p.step(q[:, :, t], k[:, :, t], v[:, :, t], lg[:, :, t], bt[:, :, t], state, o=o)
    for got in (prompt, state):
        assert by(heads(H), got, want["S1"]) < TOL[F]


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1, 2, 3, 4, 5])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_not_finite_fp32(L, which, value):
    """A value that is not finite shows in its row's outputs or gradients, and stays in its sequence and head."""
    B, H, n, d = 2, 2, 150, 64
    x = list(inputs(B, H, H, n, d, d, F, "tokens", 6, False)[:6])  # Q, K, V, dO, gates, betas
    p = L.Delta(B, H, n, d, d, io=F, backward=True)

    def run():
        return {"O": p.forward(x[0], x[1], x[2], x[4], x[5]), **p.backward(x[0], x[1], x[2], x[3], x[4], x[5])}

    want = run()
    x[which][1, 0, 70].view(-1)[0] = value
    got = run()
    for name in got:
        for b, h in ((0, 0), (0, 1), (1, 1)):
            assert torch.equal(got[name][b, h], want[name][b, h]), name
    assert any(not torch.isfinite(got[name][1, 0, 70].float()).all() for name in got)
