"""The norms around a block where their statistics are extreme or their launch shapes leave threads idle.

Tolerances (relative 2-norms) as in test_block_norm.py: a bf16 output carries one rounding (1.7e-3 in the root
mean square), taken as 2.5e-3; fp32 values sum terms rounded at 2^-24, taken as 1e-5.
"""
import pytest
import torch

from test_block_norm import BF, F, TOL, formula


@pytest.fixture(scope="module")
def L():
    from paper_2512_08061_gb300 import build
    build.build()
    import paper_2512_08061_gb300.luna as L
    return L


def leaves(rows, cols, io, seed, gate=True):
    g = torch.Generator("cuda").manual_seed(seed)

    def rn(*shape, dtype=io):
        return (torch.randn(shape, generator=g, device="cuda") * 1.5 + 0.3).to(dtype)

    t = {"x": rn(rows, cols), "y": rn(rows, cols), "gate": rn(rows, cols) if gate else None}
    t.update({k: rn(cols, dtype=F) for k in ("w_post", "b_post", "w_pre", "b_pre")})
    return t, rn(rows, cols), rn(rows, cols)


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [0.0, 1e-30])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("cols,groups,io", [(40, 5, F), (96, 3, F), (1152, 9, BF), (1008, 2, BF), (771, 3, F), (1544, 8, F),
                                            (2056, 257, BF)])
def test_no_eps(L, cols, groups, io, kind, eps):
    """eps = 0, or too small to matter, is the bare formula on rows that vary: rows that leave threads without a
    vector, groups within a warp and through shared memory."""
    for rows, gate in ((11, "silu"), (300, "none")):
        t, dX, dH = leaves(rows, cols, io, cols + rows, gate != "none")
        leaf = {k: None if v is None else v.double().requires_grad_() for k, v in t.items()}
        x, h = formula(leaf, groups, kind, gate, 0.7, eps)
        ((x * dX.double()).sum() + (h * dH.double()).sum()).backward()
        p = L.BlockNorm(rows, cols, groups, kind, gate, 0.7, eps, io, backward=True)
        got = p.forward(t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"], t["b_post"], t["b_pre"])
        got.update(p.backward(t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"], dX, dH, t["b_post"], t["b_pre"]))
        want = {"X": x, "H": h, **{"d" + k: v.grad for k, v in leaf.items() if v is not None}}
        assert set(got) == set(want)
        for k, v in want.items():
            v = v.detach()
            assert torch.isfinite(got[k]).all(), k
            assert (got[k].double() - v).norm() < TOL[got[k].dtype] * v.norm(), k


@pytest.mark.gpu
@pytest.mark.parametrize("cols,groups,io", [(512, 4, F), (2048, 1, BF)])
def test_rows_of_absent_matrices(L, cols, groups, io):
    """A leading dimension of a matrix that the call does not have changes nothing: equal bits (the form for rows
    off their boundaries sums in another order)."""
    t, _, dH = leaves(64, cols, io, 5, gate=False)
    p = L.BlockNorm(64, cols, groups, "rms", "none", 0.5, io=io, backward=True)
    odd = torch.randn((64, cols + 1), device="cuda").to(io)[:, :cols]

    def call(x, dX):
        return {**p.forward(x, t["y"], None, t["w_post"], t["w_pre"]),
                **p.backward(x, t["y"], None, t["w_post"], t["w_pre"], dX, dH)}

    want = call(None, None)
    call(odd, odd)
    got = call(None, None)
    assert set(got) == set(want) and all(torch.equal(got[k], want[k]) for k in want)
    # the same of a descriptor's own fields
    nd = L.norm_desc(64, cols, groups, res_scale=0.5, io=L._DTYPES[io])
    nd.ldx = nd.ldgate = nd.ldX = cols + 1
    h = torch.empty_like(t["y"])
    L.luna_norm_fwd(nd, None, t["y"], None, t["w_post"], None, t["w_pre"], None, None, h)
    assert torch.equal(h, want["H"])


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("gate", ["none", "sigmoid", "silu"])
def test_gradients_against_extrapolated_differences(L, kind, gate):
    """Central differences of the 32-bit forward at steps of 1e-2 and 2e-2, extrapolated: what is left of the
    curvature is under 3e-7 of the terms' norm (in 64 bits, over 20 draws of this problem), and 576 outputs rounded at
    some 1.5 2^-24 leave about sqrt(576) 9e-8 / 2e-2 * 5/3 = 2e-4 beside terms of a norm of 10 and more: 1e-3."""
    rows, cols, step = 6, 48, 1e-2
    g = torch.Generator("cuda").manual_seed(2)
    t = {k: torch.randn((rows, cols), generator=g, device="cuda") for k in ("x", "y", "gate")}
    t.update({k: torch.randn(cols, generator=g, device="cuda") for k in ("w_post", "w_pre", "b_post", "b_pre")})
    dX, dH = (torch.randn((rows, cols), generator=g, device="cuda") for _ in range(2))
    if gate == "none":
        t["gate"] = None
    p = L.BlockNorm(rows, cols, 3, kind, gate, 0.5, 1e-2, F, backward=True)
    args = ("x", "y", "gate", "w_post", "w_pre", "b_post", "b_pre")
    back = p.backward(*(t[k] for k in args[:5]), dX, dH, t["b_post"], t["b_pre"])
    for k in args:
        if t[k] is None:
            continue
        by = torch.randn(t[k].shape, generator=g, device="cuda")
        slope = []
        for h in (step, 2 * step):
            loss = []
            for sign in (1, -1):
                o = p.forward(*(t[j] + sign * h * by if j == k else t[j] for j in args))
                loss.append((o["X"].double() * dX).sum() + (o["H"].double() * dH).sum())
            slope.append((loss[0] - loss[1]) / (2 * h))
        terms = back["d" + k].double() * by
        assert abs((4 * slope[0] - slope[1]) / 3 - terms.sum()) < 1e-3 * terms.norm(), k
