"""Linear layers with their epilogue, against the formulas in 64 bits.

Tolerances (relative 2-norms): a bf16 output carries one rounding (1.7e-3 in the root mean square over
a binade), and a gradient through an activation also those of the kept z and of dz: sqrt(3) * 1.7e-3 =
2.9e-3, taken as 4e-3; an fp32 output sums up to 16384 terms rounded at 2^-24: under 8e-6, taken as 1e-5.
"""
import ctypes

import pytest
import torch

TOL = {torch.float32: 1e-5, torch.bfloat16: 4e-3}
F, BF = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def L():
    from paper_2512_08061_gb300 import build
    build.build()
    import paper_2512_08061_gb300.luna as L
    return L


def act_of(z, act):
    return {"none": lambda u: u, "relu": torch.relu, "gelu": lambda u: u * torch.special.ndtr(u),
            "silu": lambda u: u * torch.sigmoid(u)}[act](z)


CASES = [  # m, n, k, act, bias, residual, io, pad (elements between rows beyond their width)
    (1, 1, 1, "none", True, True, F, 0),
    (5, 7, 3, "gelu", True, True, F, 0),
    (130, 257, 129, "silu", True, False, F, 3),
    (33, 64, 4000, "none", False, True, F, 0),
    (1, 512, 1024, "none", True, True, BF, 0),
    (4, 1000, 776, "silu", True, False, BF, 0),
    (8, 130, 40, "gelu", False, True, BF, 8),
    (9, 256, 512, "relu", True, True, BF, 0),
    (31, 1032, 320, "gelu", True, True, BF, 0),
    (64, 128, 8192, "none", True, False, BF, 0),
    (65, 96, 64, "relu", True, False, BF, 0),
    (128, 256, 64, "none", False, False, BF, 0),
    (129, 264, 72, "gelu", True, True, BF, 24),
    (300, 520, 1000, "silu", True, True, BF, 0),
    (1000, 768, 768, "gelu", True, True, BF, 0),
    (2049, 2304, 264, "none", True, True, BF, 16),
    (77, 201, 51, "gelu", True, True, BF, 1),      # nothing aligned
    (513, 40, 2000, "relu", False, True, BF, 0),
    (5000, 16, 16, "silu", True, False, BF, 0),
    (3, 9000, 24, "none", True, True, BF, 0),
]


def matrix(g, rows, cols, io, pad, scale=1.0):
    x = (torch.randn((rows, cols), generator=g, device="cuda") * scale).to(io)
    if not pad:
        return x
    y = torch.full((rows, cols + pad), float("nan"), dtype=io, device="cuda")
    y[:, :cols] = x
    return y[:, :cols]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,act,bias,res,io,pad", CASES)
def test_values_and_gradients(L, m, n, k, act, bias, res, io, pad):
    g = torch.Generator("cuda").manual_seed(m + n + k)
    x, W = matrix(g, m, k, io, pad), matrix(g, n, k, io, pad, k ** -0.5)
    b = torch.randn(n, generator=g, device="cuda").to(io) if bias else None
    r, dY = matrix(g, m, n, io, pad) if res else None, matrix(g, m, n, io, pad)
    leaf = [t.double().requires_grad_() if t is not None else None for t in (x, W, b)]
    z = leaf[0] @ leaf[1].t() + (leaf[2] if bias else 0.0)
    y = act_of(z, act) + (r.double() if res else 0.0)
    y.backward(dY.double())
    want = {"Y": y, "Z": z, "dX": leaf[0].grad, "dW": leaf[1].grad}
    p = L.Linear(m, n, k, act, io, backward=True)
    Y, Z = p.forward(x, W, b, r, save_z=True)
    assert torch.equal(p.forward(x, W, b, r), Y)
    got = {"Y": Y, "Z": Z, **p.backward(x, W, dY, Z, bias=bias)}
    if bias:
        want["db"] = leaf[2].grad
    assert L.luna_device_status(p.ws) == 0
    for name, v in want.items():
        v = v.detach()
        assert torch.isfinite(got[name]).all(), name
        assert (got[name].double() - v).norm() < TOL[io] * v.norm(), name
    again = p.backward(x, W, dY, Z, bias=bias)
    assert all(torch.equal(got[k], again[k]) for k in again)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(300, 256, 512), (6, 256, 512), (40, 264, 520)])
def test_views_residual_in_place_and_offsets(L, m, n, k):
    """Columns of a wider matrix in and out, the residual overwritten, and matrices off a 16-byte boundary."""
    g = torch.Generator("cuda").manual_seed(3)
    x, W = matrix(g, m, k, BF, 0), matrix(g, n, k, BF, 0, k ** -0.5)
    r = matrix(g, m, n, BF, 0)
    p = L.Linear(m, n, k, "gelu", BF)
    want = p.forward(x, W, None, r)
    wide = torch.zeros((m, n + 64), dtype=BF, device="cuda")
    p.forward(x, W, None, r, Y=wide[:, 32:32 + n])
    assert torch.equal(wide[:, 32:32 + n], want) and not wide[:, :32].any() and not wide[:, 32 + n:].any()
    keep = r.clone()
    assert torch.equal(p.forward(x, W, None, keep, Y=keep), want)

    def odd(t):
        return torch.empty(t.numel() + 1, dtype=BF, device="cuda")[1:].view(t.shape).copy_(t)

    got = p.forward(odd(x), odd(W), None, odd(r), Y=odd(r))
    assert (got.double() - want.double()).norm() < TOL[BF] * want.double().norm()


@pytest.mark.gpu
def test_gradients_against_differences(L):
    """Y is linear in X and in W, so a central difference of any width is exact without an activation."""
    m, n, k = 37, 50, 29
    g = torch.Generator("cuda").manual_seed(4)
    x, W, dY = matrix(g, m, k, F, 0), matrix(g, n, k, F, 0), matrix(g, m, n, F, 0)
    b = torch.randn(n, generator=g, device="cuda")
    p = L.Linear(m, n, k, "none", F, backward=True)
    back = p.backward(x, W, dY, bias=True)
    for name, t in (("dX", x), ("dW", W), ("db", b)):
        by = torch.randn(t.shape, generator=g, device="cuda")
        loss = []
        for sign in (1, -1):
            u = [t2 + sign * by if t2 is t else t2 for t2 in (x, W, b)]
            loss.append((p.forward(*u).double() * dY).sum())
        want = (back[name].double() * by).sum()
        assert abs((loss[0] - loss[1]) / 2 - want) < 1e-4 * (back[name].double() * by).norm() * 10


@pytest.mark.gpu
def test_other_stream_and_graph(L):
    g = torch.Generator("cuda").manual_seed(5)
    x, W = matrix(g, 200, 512, BF, 0), matrix(g, 300, 512, BF, 0)
    p = L.Linear(200, 300, 512, "relu", BF)
    want = p.forward(x, W)
    torch.cuda.synchronize()
    s, Y = torch.cuda.Stream(), torch.zeros_like(want)
    with torch.cuda.stream(s):
        p.forward(x, W, Y=Y)
    s.synchronize()
    assert torch.equal(Y, want)
    Y.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.forward(x, W, Y=Y)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(Y, want)


@pytest.mark.gpu
def test_nothing_to_sum(L):
    """k = 0 leaves bias and residual; m = 0 gives gradients of zero."""
    b = torch.randn(6, device="cuda")
    p = L.Linear(4, 6, 0, "none", F, backward=True)
    x, W = torch.empty((4, 0), device="cuda"), torch.empty((6, 0), device="cuda")
    assert torch.equal(p.forward(x, W, b), b.expand(4, 6))
    dY = torch.randn(4, 6, device="cuda")
    assert torch.allclose(p.backward(x, W, dY, bias=True)["db"], dY.sum(0))
    p = L.Linear(0, 6, 5, "none", F, backward=True)
    back = p.backward(torch.empty((0, 5), device="cuda"), torch.ones((6, 5), device="cuda"), torch.empty((0, 6), device="cuda"), bias=True)
    assert not back["dW"].any() and not back["db"].any()


def test_refusals(L):
    lib, P = L._lib, ctypes.c_void_p

    def size(ld):
        return lib.luna_linear_workspace_size(ctypes.byref(ld), 1, ctypes.byref(ctypes.c_size_t()))

    ok = dict(m=4, n=8, k=16)
    assert size(L.linear_desc(**ok)) == 0
    for bad in (dict(ok, m=-1), dict(ok, n=-1), dict(ok, k=-1), dict(ok, io=3)):
        assert size(L.linear_desc(**bad)) == 1, bad
    for bad in (dict(ok, m=(1 << 23) + 1), dict(ok, n=(1 << 20) + 1), dict(ok, k=(1 << 20) + 1)):
        assert size(L.linear_desc(**bad)) == 2, bad
    for field, v in (("ldx", 15), ("ldw", 15), ("ldy", 7), ("ldr", 7), ("ldz", 7), ("lddy", 7), ("lddx", 15), ("act", 8)):
        ld = L.linear_desc(**ok)
        setattr(ld, field, v)
        assert size(ld) == 1, field
    ld, x = L.linear_desc(**ok), 256

    def fwd(*p, ws=256, nbytes=1 << 40):
        return lib.luna_linear_fwd(ctypes.byref(ld), *(P(q) for q in p), P(ws), nbytes, None)

    assert fwd(0, x, 0, 0, x, 0) == 1 and fwd(x, 0, 0, 0, x, 0) == 1 and fwd(x, x, 0, 0, 0, 0) == 1
    assert fwd(x, x, 0, 0, x, 0, ws=0) == 1 and fwd(x, x, 0, 0, x, 0, ws=16) == 1 and fwd(x, x, 0, 0, x, 0, nbytes=8) == 3

    def bwd(ld, *p, ws=256, nbytes=1 << 40):
        return lib.luna_linear_bwd(ctypes.byref(ld), *(P(q) for q in p), P(ws), nbytes, None)

    #              X  W  Z  dY dX dW db
    assert bwd(ld, x, x, 0, 0, x, x, x) == 1 and bwd(ld, 0, x, 0, x, x, x, x) == 1 and bwd(ld, x, 0, 0, x, x, x, x) == 1
    assert bwd(L.linear_desc(**ok, act="gelu"), x, x, 0, x, x, x, x) == 1  # the activation's gradient needs z
    assert bwd(ld, x, x, 0, x, x, x, x, nbytes=100) == 3
    for z in (dict(ok, m=0), dict(ok, n=0)):
        e = L.linear_desc(**z)
        assert lib.luna_linear_fwd(ctypes.byref(e), None, None, None, None, None, None, None, 0, None) == 0
    p = L.Linear(4, 8, 16, io=F, device="cpu")
    with pytest.raises(ValueError):
        p.forward(torch.zeros(4, 15), torch.zeros(8, 16))
    with pytest.raises(ValueError):
        p.forward(torch.zeros(16, 4).t(), torch.zeros(8, 16))
    with pytest.raises(TypeError):
        p.forward(torch.zeros(4, 16, dtype=BF), torch.zeros(8, 16))


PLANES = [  # m, n, k, act, bias, residual, pad: fp32 products large enough for tensor cores
    (700, 650, 577, "none", True, True, 0),
    (1025, 520, 1100, "gelu", True, True, 4),
    (2000, 1032, 320, "silu", False, True, 3),
    (48, 4096, 4096, "relu", True, False, 0),
    (20, 6000, 2051, "none", False, True, 0),
    (4100, 264, 256, "none", True, False, 0),
    (513, 515, 5000, "none", False, False, 1),
]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,act,bias,res,pad", PLANES)
def test_wide_products_in_fp32(L, m, n, k, act, bias, res, pad):
    """Three bf16 planes carry an fp32 value whole, and sums of 256 products lose about 3e-7 before they
    are joined in fp32: without an activation 1e-6 holds, with signs mixed or not."""
    g = torch.Generator("cuda").manual_seed(m + n + k)
    x, W = matrix(g, m, k, F, pad), matrix(g, n, k, F, pad, k ** -0.5)
    if not res:
        x, W = x.abs(), W.abs()
    b = torch.randn(n, generator=g, device="cuda") if bias else None
    r, dY = matrix(g, m, n, F, pad) if res else None, matrix(g, m, n, F, pad)
    leaf = [t.double().requires_grad_() if t is not None else None for t in (x, W, b)]
    z = leaf[0] @ leaf[1].t() + (leaf[2] if bias else 0.0)
    y = act_of(z, act) + (r.double() if res else 0.0)
    y.backward(dY.double())
    p = L.Linear(m, n, k, act, F, backward=True)
    Y, Z = p.forward(x, W, b, r, save_z=True)
    got = {"Y": Y, "Z": Z, **p.backward(x, W, dY, Z, bias=bias)}
    assert L.luna_device_status(p.ws) == 0
    for name, v in {"Y": y, "Z": z, "dX": leaf[0].grad, "dW": leaf[1].grad}.items():
        v = v.detach()
        assert (got[name].double() - v).norm() < (1e-6 if act == "none" else TOL[F]) * v.norm(), name
    if res:
        keep = r.clone()
        assert torch.equal(p.forward(x, W, b, keep, Y=keep), Y)


@pytest.mark.gpu
def test_wide_products_with_infinities_and_large_values(L):
    """An infinity times a finite value is an infinity of its sign, a NaN stays in its row, and values near
    the largest one are values."""
    m, n, k = 640, 768, 700
    g = torch.Generator("cuda").manual_seed(9)
    x, W = matrix(g, m, k, F, 0), matrix(g, n, k, F, 0).sign() * 0.5
    r = matrix(g, m, n, F, 0)
    p = L.Linear(m, n, k, "none", F)
    clean = p.forward(x, W, None, r)
    x[3, 5], x[10, 699], x[600, 0] = float("inf"), float("-inf"), float("nan")
    keep = r.clone()
    y = p.forward(x, W, None, keep, Y=keep)
    assert torch.equal(y[3], float("inf") * W[:, 5]) and torch.equal(y[10], float("-inf") * W[:, 699])
    assert y[600].isnan().all()
    rest = [i for i in range(m) if i not in (3, 10, 600)]
    assert (y[rest].double() - clean[rest].double()).norm() < 1e-5 * clean[rest].double().norm()
    x = torch.zeros((m, k), device="cuda")
    x[:, 7] = torch.finfo(F).max
    assert torch.equal(p.forward(x, W), x[:, 7:8] * W[:, 7])
    assert L.luna_device_status(p.ws) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,act", [(5, 1, 300, "gelu"), (40, 3, 129, "silu"), (1, 60, 2048, "gelu"), (130, 31, 77, "relu"),
                                       (20, 16, 4096, "silu")])
def test_small_gradients_round_once(L, m, n, k, act):
    """The gradients of a small layer carry the rounding of their own bf16 values alone (half a unit in the
    last of eight bits: at most 2^-8 of each) and what fp32 sums and slopes lose."""
    g = torch.Generator("cuda").manual_seed(m * n + k)
    x, W, dY = matrix(g, m, k, BF, 0), matrix(g, n, k, BF, 0, k ** -0.5), matrix(g, m, n, BF, 0)
    p = L.Linear(m, n, k, act, BF, backward=True)
    _, Z = p.forward(x, W, save_z=True)
    got = p.backward(x, W, dY, Z)
    z = Z.double().requires_grad_()
    act_of(z, act).backward(dY.double())
    for name, v, size in (("dX", z.grad @ W.double(), z.grad.abs() @ W.double().abs()),
                          ("dW", z.grad.t() @ x.double(), z.grad.abs().t() @ x.double().abs())):
        err = (got[name].double() - v).abs()
        assert (err <= 2.0 ** -8 * v.abs() + 1e-4 * size).all(), name
    assert L.luna_device_status(p.ws) == 0
