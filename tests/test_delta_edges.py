"""The gated delta rule where its parts are of very different size: chunks without queries, keys or gradients, strong gates.

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
