"""The norms before and after a block with its gate and residual scale, against their formulas in 64 bits.

Tolerances (relative 2-norms): a bf16 output carries one rounding (1.7e-3 in the root mean square),
taken as 2.5e-3; fp32 outputs and weight gradients sum up to 16384 columns or a few thousand rows of
terms rounded at 2^-24 with approximate roots and exponentials (a few 2^-22), taken as 1e-5.
"""
import ctypes

import pytest
import torch

TOL = {torch.float32: 1e-5, torch.bfloat16: 2.5e-3}
F, BF = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def L():
    from paper_2512_08061_gb300 import build
    build.build()
    import paper_2512_08061_gb300.luna as L
    return L


def norm(z, groups, kind, eps, w, b):
    z = z.unflatten(-1, (groups, -1))
    if kind == "layer":
        z = z - z.mean(-1, keepdim=True)
    z = (z / (z.square().mean(-1, keepdim=True) + eps).sqrt()).flatten(-2) * w
    return z if b is None else z + b


def formula(t, groups, kind, gate, alpha, eps):
    """x', h from a dict of 64-bit leaves."""
    if t["y"] is None:
        x = t["x"]
    else:
        u = norm(t["y"], groups, kind, eps, t["w_post"], t["b_post"]) if t["w_post"] is not None else t["y"]
        if gate != "none":
            u = u * torch.sigmoid(t["gate"]) * (t["gate"] if gate == "silu" else 1.0)
        x = alpha * u + (t["x"] if t["x"] is not None else 0.0)
    return x, norm(x, 1, kind, eps, t["w_pre"], t["b_pre"]) if t["w_pre"] is not None else None


CASES = [  # rows, cols, groups, kind, gate, parts (x residual, p post, q pre, b biases, y no block output), io
    (1, 1, 1, "rms", "none", "xpq", F),
    (3, 5, 5, "rms", "silu", "xpqb", F),
    (7, 96, 3, "layer", "sigmoid", "xpqb", F),
    (50, 771, 3, "layer", "silu", "xpqb", F),
    (33, 2048, 16, "rms", "silu", "xpq", BF),
    (9, 4096, 32, "layer", "silu", "xpqb", BF),
    (300, 64, 1, "rms", "none", "xq", BF),
    (300, 256, 4, "rms", "sigmoid", "pb", BF),
    (17, 8192, 8, "rms", "silu", "xpq", BF),
    (5, 16384, 1, "layer", "silu", "xpqb", BF),
    (5, 16384, 128, "layer", "silu", "xpqb", F),
    (21, 6000, 6, "layer", "silu", "xpq", F),
    (6, 4099, 1, "rms", "silu", "xpq", BF),
    (4, 12321, 3, "layer", "none", "xpqb", F),
    (40, 768, 12, "layer", "none", "qyb", BF),
    (40, 100, 1, "rms", "none", "qy", F),
    (11, 384, 4, "layer", "none", "xp", F),     # 96 columns a group: not a power of two of vectors
    (2500, 24, 3, "layer", "silu", "pq", BF),
    (1000, 333, 9, "rms", "sigmoid", "x", BF),  # no norm at all: gate and residual alone
]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,groups,kind,gate,parts,io", CASES)
def test_values_and_gradients(L, rows, cols, groups, kind, gate, parts, io):
    g = torch.Generator("cuda").manual_seed(rows + cols)
    alpha, eps = 0.7, 1e-5

    def rn(*shape, dtype=io):
        return (torch.randn(shape, generator=g, device="cuda") * 1.5 + 0.3).to(dtype)

    def wide(t):  # rows of a wider matrix
        y = torch.full((rows, cols + 8), float("nan"), dtype=io, device="cuda")
        y[:, :cols] = t
        return y[:, :cols]

    has_y = "y" not in parts
    t = {"x": wide(rn(rows, cols)) if "x" in parts or not has_y else None, "y": rn(rows, cols) if has_y else None,
         "gate": wide(rn(rows, cols)) if gate != "none" else None}
    for w, on in (("post", "p" in parts), ("pre", "q" in parts)):
        t["w_" + w] = rn(cols, dtype=F) if on else None
        t["b_" + w] = rn(cols, dtype=F) if on and "b" in parts else None
    leaf = {k: None if v is None else v.double().requires_grad_() for k, v in t.items()}
    x, h = formula(leaf, groups, kind, gate, alpha, eps)
    want = {"H": h} if h is not None else {}
    if h is None or (t["x"] is not None and has_y):
        want["X"] = x
    dX = rn(rows, cols) if "X" in want else None
    dH = rn(rows, cols) if h is not None else None
    sum((want[k] * d.double()).sum() for k, d in (("X", dX), ("H", dH)) if d is not None).backward()

    p = L.BlockNorm(rows, cols, groups, kind, gate, alpha, eps, io, backward=True)
    got = p.forward(t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"], t["b_post"], t["b_pre"])
    assert set(got) == set(want)
    back = p.backward(t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"], dX, dH, t["b_post"], t["b_pre"])
    names = {"x": "dx", "y": "dy", "gate": "dgate", "w_post": "dw_post", "w_pre": "dw_pre", "b_post": "db_post",
             "b_pre": "db_pre"}
    want.update({names[k]: v.grad for k, v in leaf.items() if v is not None})
    got.update(back)
    assert set(got) == set(want)
    for k, v in want.items():
        v = v.detach()
        # a gradient that cancels (a group of one or two columns) is measured against its terms' size
        size = max(v.norm().item(), 1e-3 * (v.numel() ** 0.5))
        assert torch.isfinite(got[k]).all()
        assert (got[k].double() - v).norm().item() < TOL[got[k].dtype] * size, k
    again = p.backward(t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"], dX, dH, t["b_post"], t["b_pre"])
    assert all(torch.equal(back[k], again[k]) for k in back)


@pytest.mark.gpu
def test_unaligned_rows(L):
    """Rows off a 16-byte boundary, and leading dimensions that no vector divides, give the same values."""
    rows, cols = 20, 512
    p = L.BlockNorm(rows, cols, 4, "rms", "silu", 0.5, io=BF)
    x, y, g = (torch.randn(rows, cols, device="cuda").to(BF) for _ in range(3))
    w = torch.randn(cols, device="cuda")
    a = p.forward(x, y, g, w, w)

    def odd(t):
        buf = torch.empty(rows * (cols + 3) + 1, dtype=BF, device="cuda")[1:].view(rows, cols + 3)[:, :cols]
        return buf.copy_(t)

    b = p.forward(odd(x), odd(y), odd(g), w, w)
    for k in a:
        assert (a[k].double() - b[k].double()).norm() <= TOL[BF] * a[k].double().norm()


@pytest.mark.gpu
def test_in_place(L):
    """x' and h may overwrite x and y."""
    rows, cols = 64, 1024
    p = L.BlockNorm(rows, cols, 8, "rms", "silu", 0.5, io=BF)
    x, y, g = (torch.randn(rows, cols, device="cuda").to(BF) for _ in range(3))
    w = torch.randn(cols, device="cuda")
    want = p.forward(x, y, g, w, w)
    got = p.forward(x, y, g, w, w, X=x, H=y)
    assert got["X"] is x and torch.equal(x, want["X"]) and torch.equal(y, want["H"])


@pytest.mark.gpu
@pytest.mark.parametrize("kind,gate", [("rms", "silu"), ("layer", "sigmoid")])
def test_gradients_against_differences(L, kind, gate):
    """Central differences of the 32-bit forward: their own error is about step^2 for the curvature and
    2^-24 / step of the outputs' size for the rounding; 1e-2 keeps both under 2e-4 of the terms' size."""
    rows, cols, step = 6, 48, 1e-2
    g = torch.Generator("cuda").manual_seed(1)
    t = {k: torch.randn((rows, cols), generator=g, device="cuda") for k in ("x", "y", "gate")}
    t.update({k: torch.randn(cols, generator=g, device="cuda") for k in ("w_post", "w_pre", "b_post", "b_pre")})
    dX, dH = (torch.randn((rows, cols), generator=g, device="cuda") for _ in range(2))
    p = L.BlockNorm(rows, cols, 3, kind, gate, 0.5, 1e-2, F, backward=True)
    args = ("x", "y", "gate", "w_post", "w_pre", "b_post", "b_pre")
    back = p.backward(*(t[k] for k in args[:5]), dX, dH, t["b_post"], t["b_pre"])
    for k in args:
        by = torch.randn(t[k].shape, generator=g, device="cuda")
        loss = []
        for sign in (1, -1):
            u = dict(t)
            u[k] = t[k] + sign * step * by
            o = p.forward(*(u[j] for j in args))
            loss.append((o["X"].double() * dX).sum() + (o["H"].double() * dH).sum())
        formula_d = (back["d" + k].double() * by).sum()
        size = (back["d" + k].double() * by).norm() * 10
        assert abs((loss[0] - loss[1]) / (2 * step) - formula_d) < 1e-2 * size, k


def test_refusals(L):
    lib, P = L._lib, ctypes.c_void_p

    def size(nd):
        return lib.luna_norm_workspace_size(ctypes.byref(nd), ctypes.byref(ctypes.c_size_t()))

    def fwd(nd, *ptrs):
        return lib.luna_norm_fwd(ctypes.byref(nd), *(P(p) for p in ptrs), None)

    ok = dict(rows=4, cols=64, groups=4)
    assert size(L.norm_desc(**ok)) == 0
    for bad in (dict(ok, rows=-1), dict(ok, cols=0), dict(ok, groups=0), dict(ok, groups=3), dict(ok, eps=-1.0),
                dict(ok, eps=float("inf")), dict(ok, res_scale=float("nan")), dict(ok, io=5)):
        assert size(L.norm_desc(**bad)) == 1, bad
    assert size(L.norm_desc(4, 16385)) == 2
    nd = L.norm_desc(**ok)
    nd.ldy = 63
    assert size(nd) == 1
    for field in ("kind", "gate"):
        nd = L.norm_desc(**ok)
        setattr(nd, field, 9)
        assert size(nd) == 1
    nd, x = L.norm_desc(**ok), 256
    #             x  y  gate wpost bpost wpre bpre X  H
    assert fwd(nd, 0, 0, 0, 0, 0, x, 0, x, x) == 1     # nothing to norm
    assert fwd(nd, x, 0, 0, x, 0, x, 0, x, x) == 1     # a post-norm without a block output
    assert fwd(nd, x, x, 0, 0, x, x, 0, x, x) == 1     # a bias without its norm
    assert fwd(nd, x, x, 0, x, 0, x, 0, x, 0) == 1     # h asked for, nowhere to go
    assert fwd(nd, x, x, 0, x, 0, 0, 0, 0, x) == 1     # x' has nowhere to go
    assert fwd(L.norm_desc(**ok, gate="silu"), x, x, 0, x, 0, x, 0, x, x) == 1  # no gate
    assert fwd(L.norm_desc(0, 64), 0, 0, 0, 0, 0, 0, 0, 0, 0) == 0

    def bwd(nd, *ptrs, ws=256, nbytes=1 << 40):
        return lib.luna_norm_bwd(ctypes.byref(nd), *(P(p) for p in ptrs), P(ws), nbytes, None)

    #             x  y  gate wpost bpost wpre dX dH dx dy dg dwpost dbpost dwpre dbpre
    assert bwd(nd, x, x, 0, x, 0, x, x, 0, x, x, 0, x, 0, x, 0) == 1   # no dH
    assert bwd(nd, x, x, 0, x, 0, 0, 0, 0, x, x, 0, x, 0, 0, 0) == 1   # no dX
    assert bwd(nd, x, x, 0, x, 0, x, x, x, 0, x, 0, x, 0, x, 0) == 1   # no dx
    assert bwd(nd, x, x, 0, x, 0, 0, x, 0, x, x, 0, x, 0, x, 0) == 1   # a gradient of a weight that is not there
    assert bwd(nd, x, x, 0, x, 0, x, x, x, x, x, 0, x, 0, x, 0, ws=0) == 1
    assert bwd(nd, x, x, 0, x, 0, x, x, x, x, x, 0, x, 0, x, 0, nbytes=100) == 3
    p = L.BlockNorm(4, 8, io=F, device="cpu")
    with pytest.raises(ValueError):
        p.forward(torch.zeros(4, 7), torch.zeros(4, 8), w_pre=torch.zeros(8))
    with pytest.raises(ValueError):
        p.forward(torch.zeros(8, 4).t(), torch.zeros(4, 8), w_pre=torch.zeros(8))
    with pytest.raises(TypeError):
        p.forward(torch.zeros(4, 8), torch.zeros(4, 8), w_pre=torch.zeros(8, dtype=BF))


WIDE = [  # more rows than blocks, and rows that a block walks in passes
    (700, 7094, 1, "rms", "none", "xpq", F),
    (310, 5001, 3, "layer", "silu", "xpqb", F),
    (305, 5001, 3, "rms", "sigmoid", "xpq", BF),
    (400, 8140, 4, "rms", "none", "pq", BF),
    (330, 8192, 16, "layer", "silu", "xpqb", BF),
    (320, 16384, 16, "rms", "silu", "xpqb", F),
    (306, 9000, 250, "layer", "sigmoid", "xpqb", BF),  # groups of 36, in pieces of several to a warp
    (200, 16001, 1, "layer", "none", "qyb", F),
    (199, 4400, 1, "layer", "silu", "xp", F),
    (198, 6000, 5, "rms", "silu", "x", BF),
]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,groups,kind,gate,parts,io", WIDE)
def test_wide_rows(L, rows, cols, groups, kind, gate, parts, io):
    test_values_and_gradients(L, rows, cols, groups, kind, gate, parts, io)


@pytest.mark.gpu
@pytest.mark.parametrize("cols,groups", [(6000, 4), (6001, 1)])
def test_wide_rows_in_place(L, cols, groups):
    g = torch.Generator("cuda").manual_seed(12)
    x, y, gate, dX, dH = (torch.randn((320, cols), generator=g, device="cuda") for _ in range(5))
    wq, wp = torch.randn(cols, generator=g, device="cuda"), torch.randn(cols, generator=g, device="cuda")
    p = L.BlockNorm(320, cols, groups=groups, gate="silu", io=F, backward=True)
    f = p.forward(x, y, gate, wp, wq)
    want = p.backward(x, y, gate, wp, wq, dX, dH)
    out = {"dx": dX.clone(), "dy": y.clone(), "dgate": gate.clone()}
    got = p.backward(x, out["dy"], out["dgate"], wp, wq, out["dx"], dH, out=out)
    assert all(torch.equal(got[k], want[k]) for k in ("dx", "dy", "dgate"))
    a, b = x.clone(), y.clone()
    p.forward(a, b, gate, wp, wq, X=a, H=b)
    assert torch.equal(a, f["X"]) and torch.equal(b, f["H"])
