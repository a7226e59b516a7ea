"""Linear attention with decay over very many tokens."""
import pytest
import torch

from test_decay import BF, F, TOL


@pytest.fixture(scope="module")
def L():
    from paper_2512_08061_gb300 import build
    build.build()
    import paper_2512_08061_gb300.luna as L
    return L


RATES = [-1e-7, -1e-6, -3e-6, -1e-5, -1e-4, -1e-3, -1e-2, -0.49, -0.51, 0.0, -float("inf")]


def final_state(k, v, ld):
    """sum_j lambda^{n - 1 - j} k_j v_j^T in 64 bits."""
    n = k.shape[2]
    gone = n - 1 - torch.arange(n, device="cuda", dtype=torch.float64)
    w = torch.exp(torch.where(gone == 0, 0.0, ld.double()[:, None] * gone))
    return torch.einsum("hn,hnd,hne->hde", w, k[0].double(), v[0].double())


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F, BF])
def test_slow_decays_over_many_tokens(L, io):
    """20000 single tokens, and the same tokens as a prompt: the states of slow decays as near to the definition as
    sums of that many rounded terms are (the tolerance of states; keys and values of one sign, so that errors of one
    sign would add up)."""
    H, n, d = len(RATES), 20000, 16
    g = torch.Generator("cuda").manual_seed(8)
    q, k, v = (torch.rand((1, H, n, d), generator=g, device="cuda").to(io) for _ in range(3))
    ld = torch.tensor(RATES, device="cuda")
    want = final_state(k, v, ld)
    _, prompt = L.Decay(1, H, n, d, d, io=io).forward(q, k, v, ld, want_state=True)
    p = L.Decay(1, H, 1, d, d, io=io)
    state, o = torch.zeros((1, H, d, d), device="cuda"), None
    for t in range(n):
        o = p.step(q[:, :, t], k[:, :, t], v[:, :, t], ld, state, o=o)
    for got in (prompt, state):
        off = (got[0].double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
        assert (off < TOL[F]).all(), off
    out = d ** -0.5 * torch.einsum("hd,hde->he", q[0, :, -1].double(), want)
    off = (o[0].double() - out).norm(dim=1) / out.norm(dim=1)
    assert (off < TOL[io]).all(), off
