"""Linear layers far from the middle of their range: activations' tails, and sums over very many rows."""
import pytest
import torch

from test_linear import F, TOL, matrix


@pytest.fixture(scope="module")
def L():
    from paper_2512_08061_gb300 import build
    build.build()
    import paper_2512_08061_gb300.luna as L
    return L


def gelu(z):
    """In 64 bits with the lower tail whole (torch.special.ndtr is 1 + erf, which at -8 has lost it in 64 bits too)."""
    return 0.5 * z * torch.erfc(-z * 0.5 ** 0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(64, 96, 32), (20, 300, 64), (1025, 520, 1100)])
@pytest.mark.parametrize("shift", [-4.0, -5.5, -8.0])
def test_gelu_below_zero_in_fp32(L, m, n, k, shift):
    """Pre-activations all well below zero: the distribution function's lower tail has fp32 accuracy.  Its relative
    error is about |z| times that of z (some 3e-7 absolute) and z^2 2^-23 for the argument's rounding: 1e-5 holds
    to z = -8."""
    g = torch.Generator("cuda").manual_seed(m)
    x, W, dY = matrix(g, m, k, F, 0), matrix(g, n, k, F, 0, 0.1 * k ** -0.5), matrix(g, m, n, F, 0)
    b = torch.full((n,), shift, device="cuda")
    p = L.Linear(m, n, k, "gelu", F, backward=True)
    Y, Z = p.forward(x, W, b, save_z=True)
    got = {"Y": Y, **p.backward(x, W, dY, Z)}
    z = Z.double().requires_grad_()
    y = gelu(z)
    y.backward(dY.double())
    for name, v in (("Y", y.detach()), ("dX", z.grad @ W.double()), ("dW", z.grad.t() @ x.double())):
        assert (got[name].double() - v).norm() < TOL[F] * v.norm(), name
