"""Linear layers far from the middle of their range: activations' tails, and sums over very many rows."""
import pytest
import torch

from test_linear import BF, F, TOL, matrix


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


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_fp32_activations_element_by_element(L, act):
    """A layer of one weight of 1: its pre-activations are the inputs and its input gradients the slopes, both to
    fp32 accuracy of each value.  Bounds by CUDA's stated errors, in units of 2^-23 of a value or, for a slope, of
    its two terms: SiLU at most 2 for expf, 1 for the sum, 2 for the quotient, 1 a product: 7, taken as 8.  GELU
    4 for erfcf and 2 for expf, 2 for the products and z^2 / 2 for the rounding of z^2 and of z / sqrt 2 (at most
    2^-23 of it, and the tail's logarithm is -z^2 / 2, to twice that with the density's): z^2 + 8."""
    unit = 2.0 ** -23
    x = torch.linspace(-12.5 if act == "gelu" else -86.0, 30.0, 4099, device="cuda").view(-1, 1)
    W = torch.ones((1, 1), device="cuda")
    p = L.Linear(x.shape[0], 1, 1, act, F, backward=True)
    Y, Z = p.forward(x, W, save_z=True)
    assert torch.equal(Z, x)
    got = p.backward(x, W, torch.ones_like(x), Z)["dX"].double()
    z = x.double()
    if act == "gelu":
        terms = [0.5 * torch.erfc(-z * 0.5 ** 0.5), z * torch.exp(-0.5 * z * z) * (2 * torch.pi) ** -0.5]
        bound = (z * z + 8) * unit
        value = z * terms[0]
    else:
        s, rest = 1 / (1 + torch.exp(-z)), 1 / (1 + torch.exp(z))
        terms, bound, value = [s, z * s * rest], 8 * unit, z * s
    tiny = 2.0 ** -126  # (below it fp32 has fewer bits)
    assert ((Y.double() - value).abs() <= bound * value.abs() + tiny).all()
    assert ((got - sum(terms)).abs() <= bound * sum(t.abs() for t in terms) + tiny).all()


@pytest.mark.gpu
def test_fp32_silu_ends(L):
    """Down to the smallest normal result, and at the infinities."""
    x = torch.tensor([[-87.5], [-89.0], [-90.5], [-1e30], [1e30], [float("inf")], [float("nan")], [0.0]], device="cuda")
    W = torch.ones((1, 1), device="cuda")
    y = L.Linear(8, 1, 1, "silu", F).forward(x, W).double()
    want = x.double() * torch.sigmoid(x.double())
    assert ((y - want)[:3].abs() <= 8 * 2.0 ** -23 * want[:3].abs() + 100 * 2.0 ** -149).all() and (y[:3] < 0).all()
    assert y[3] == 0 and y[4] == x[4] and y[5] == float("inf") and y[6].isnan() and y[7] == 0


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,direction", [((1 << 20) + 37, 1600, 1600, "dW"), (131100, 40, 20000, "dW"), (20, 20000, 131136, "Y"),
                                             (300, 16000, 70000, "Y"), (100, 40000, 70000, "Y")])
def test_long_sums_of_positive_products(L, m, n, k, direction):
    """Tensor cores cut their fp32 additions off, which on sums of one sign adds up: 1024 additions of 16 products
    lose at most 2^-13, and then the sum is joined with the others in rounded additions.  With the value's own
    rounding (half a unit of eight bits: 2^-8 at most) every value is within 2^-8 + 2^-13."""
    g = torch.Generator("cuda").manual_seed(6)

    def positive(rows, cols):
        t = torch.empty((rows, cols), device="cuda", dtype=BF)
        for a in range(0, rows, 1 << 16):
            t[a:a + (1 << 16)] = torch.rand(t[a:a + (1 << 16)].shape, generator=g, device="cuda") * 0.5 + 0.5
        return t

    p = L.Linear(m, n, k, "none", BF, backward=direction == "dW")
    x = positive(m, k)
    want = 0.0
    if direction == "dW":
        dY, W = positive(m, n), torch.empty((n, k), device="cuda", dtype=BF)
        got = p.backward(x, W, dY, out={"dW": W})["dW"][:16]
        for a in range(0, m, 1 << 16):
            want = want + dY[a:a + (1 << 16), :16].double().t() @ x[a:a + (1 << 16)].double()
    else:
        W = positive(n, k)
        got = p.forward(x, W)[:16]
        for a in range(0, k, 1 << 12):
            want = want + x[:16, a:a + (1 << 12)].double() @ W[:, a:a + (1 << 12)].double().t()
    assert L.luna_device_status(p.ws) == 0
    assert ((got.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -13) * want).all()


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(2, 3680, 128), (64, 96, 200), (33, 131, 77), (64, 512, 512), (7, 64, 4096)])
def test_gradients_of_few_rows_round_once(L, m, n, k):
    """Layers of few rows keep dz to 2^-17 in its products: a gradient carries half a unit of its own eight bits
    (2^-8 at most) and 2^-17 of its terms' size, with 1e-4 of that for fp32 sums and bf16-grade slopes.  Views off
    their boundaries, and an infinity, which has no second term."""
    g = torch.Generator("cuda").manual_seed(m * n + k)
    x, W, dY = matrix(g, m, k, BF, 0), matrix(g, n, k, BF, 0, k ** -0.5), matrix(g, m, n, BF, 0)
    Z = matrix(g, m, n, BF, 0)
    p = L.Linear(m, n, k, "silu", BF, backward=True)
    got = p.backward(x, W, dY, Z)
    z = Z.double().requires_grad_()
    (z * torch.sigmoid(z)).backward(dY.double())
    for name, v, size in (("dX", z.grad @ W.double(), z.grad.abs() @ W.double().abs()),
                          ("dW", z.grad.t() @ x.double(), z.grad.abs().t() @ x.double().abs())):
        assert ((got[name].double() - v).abs() <= 2.0 ** -8 * v.abs() + 1e-4 * size).all(), name

    def odd(t):
        return torch.empty(t.numel() + 1, dtype=BF, device="cuda")[1:].view(t.shape).copy_(t)

    again = p.backward(odd(x), odd(W), odd(dY), odd(Z))
    assert all(torch.equal(got[name], again[name]) for name in got)
    dY[1, 3] = float("inf")
    W = W.abs() + 0.125
    dX = p.backward(x, W, dY, Z.abs())["dX"]
    assert (dX[1] == float("inf")).all() and torch.isfinite(dX[0]).all() and torch.isfinite(dX[2:]).all()
    assert L.luna_device_status(p.ws) == 0
