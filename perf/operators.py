"""Measured cases of the operators of a block of linear attention with decay.

Three operators make up the block, forward and backward, for prompts and for single tokens:

  decay    o_i = scale * q_i^T S_i,  S_i = lambda_h S_{i-1} + k_i v_i^T   (a decay lambda_h for each head)
  norm     the norms after and before a block with its gate and residual scale:
           x' = x + alpha * norm(y) w_post * act(gate),   h = norm(x') w_pre
  linear   y = act(x W^T + b) + r

`run` computes them in elementary torch operations (own = False) or through the framework's calls (own = True).
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one user's next token: the long-context head shape, all latency
        {"name": "decay step one", "op": "decay_step", "B": 1, "H": 32, "Hkv": 32, "d": 128, "dv": 128, "slots": 1, "io": "bf16"},
        # the serving batch: 64 live sequences in a pool of 96 slots
        {"name": "decay step batch", "op": "decay_step", "B": 64, "H": 32, "Hkv": 32, "d": 128, "dv": 128, "slots": 96, "io": "bf16"},
        # prompts of a padded batch of short texts, their states kept for the tokens that follow
        {"name": "decay prompts short", "op": "decay_fwd", "B": 32, "H": 12, "Hkv": 12, "n": 512, "d": 64, "dv": 64, "least": 200, "state": False, "io": "bf16"},
        # one long prompt with shared keys and values, continued from an earlier state
        {"name": "decay prompt long", "op": "decay_fwd", "B": 1, "H": 32, "Hkv": 8, "n": 65536, "d": 128, "dv": 128, "least": 65536, "state": True, "io": "bf16"},
        # a training step on padded sequences
        {"name": "decay train", "op": "decay_train", "B": 8, "H": 16, "Hkv": 16, "n": 4096, "d": 128, "dv": 128, "least": 2048, "state": False, "io": "bf16"},
        # a small model trained in 32 bits, at odd sizes, with a state carried between pieces of text
        {"name": "decay train odd f32", "op": "decay_train", "B": 2, "H": 6, "Hkv": 3, "n": 1571, "d": 40, "dv": 72, "least": 1, "state": True, "io": "f32"},
        # between two blocks of a decoder, one token of each of four sequences
        {"name": "norm step", "op": "norm_fwd", "rows": 4, "cols": 4096, "groups": 32, "kind": "rms", "gate": "silu", "res": True, "post": True, "pre": True, "io": "bf16"},
        # between two blocks in training, forward and backward
        {"name": "norm train", "op": "norm_train", "rows": 32768, "cols": 2048, "groups": 16, "kind": "rms", "gate": "silu", "res": True, "post": True, "pre": True, "io": "bf16"},
        # the same in 32 bits with means taken out and an odd width
        {"name": "norm train odd f32", "op": "norm_train", "rows": 3152, "cols": 771, "groups": 3, "kind": "layer", "gate": "sigmoid", "res": True, "post": True, "pre": True, "io": "f32"},
        # the projection of a single token: the weight's bytes
        {"name": "linear step", "op": "linear_fwd", "m": 1, "n": 8192, "k": 4096, "act": "none", "bias": True, "res": False, "io": "bf16"},
        # the projection of a long prompt with its residual, the largest product
        {"name": "linear prompt", "op": "linear_fwd", "m": 65536, "n": 4096, "k": 4096, "act": "none", "bias": True, "res": True, "io": "bf16"},
        # a feed-forward layer's training step over a ragged number of rows
        {"name": "linear train", "op": "linear_train", "m": 16333, "n": 4096, "k": 1024, "act": "gelu", "bias": True, "res": False, "io": "bf16"},
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(["decay_step", "decay_fwd", "decay_train", "norm_fwd", "norm_train", "linear_fwd", "linear_train"])
    io = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op.startswith("decay"):
        d = rng.choice([32, 64, 128, 128, 8 * rng.randint(2, 16), rng.randint(5, 128)])
        dv = rng.choice([d, d, 64, rng.randint(5, 128)])
        hkv = rng.choice([1, 2, 3, 4, 8, 16])
        h = hkv * rng.choice([1, 1, 2, 3, 4])
        if op == "decay_step":
            b = _log(rng, 1, 64)
            return {"op": op, "B": b, "H": h, "Hkv": hkv, "d": d, "dv": dv, "slots": b + rng.randint(0, 8), "io": io}
        n = _log(rng, 1, 32768 if op == "decay_fwd" else 8192)
        b = max(1, min(_log(rng, 1, 32), (1 << (20 if op == "decay_fwd" else 18)) // (n * h)))
        return {"op": op, "B": b, "H": h, "Hkv": hkv, "n": n, "d": d, "dv": dv, "least": rng.randint(0, n), "state": rng.random() < 0.5, "io": io}
    if op.startswith("norm"):
        groups = rng.choice([1, 1, 4, 12, 16])
        cols = groups * rng.randint(8, 8192 // groups)
        rows = max(1, min(_log(rng, 1, 40000), (1 << 26) // cols))
        post = rng.random() < 0.7
        return {"op": op, "rows": rows, "cols": cols, "groups": groups, "kind": rng.choice(["rms", "rms", "layer"]), "gate": rng.choice(["none", "sigmoid", "silu"]),
                "res": rng.random() < 0.7, "post": post, "pre": not post or rng.random() < 0.6, "io": io}
    n, k = (rng.choice([x, 8 * max(1, x // 8), 64 * max(1, x // 64)]) for x in (_log(rng, 16, 8192), _log(rng, 16, 8192)))
    most = (1 << 38) if io == "bf16" else (1 << 35)
    m = _log(rng, 1, max(1, min(40000, most // (n * k))))
    return {"op": op, "m": m, "n": n, "k": k, "act": rng.choice(["none", "relu", "gelu", "silu"]), "bias": rng.random() < 0.7, "res": rng.random() < 0.5, "io": io}


def work(c):
    e = 2 if c["io"] == "bf16" else 4
    if c["op"].startswith("decay"):
        B, H, Hkv, d, dv = c["B"], c["H"], c["Hkv"], c["d"], c["dv"]
        S = B * H * d * dv
        if c["op"] == "decay_step":
            return {"bytes": 8 * S + e * B * (H + Hkv) * (d + dv), "flops": 5 * S}
        used = (c["least"] + c["n"]) / 2 / c["n"]  # the rows that lengths leave, on the average
        rows = B * c["n"] * used
        fwd = e * (rows * (H * d + Hkv * (d + dv)) + B * c["n"] * H * dv) + 4 * S * (1 + c["state"])
        if c["op"] == "decay_fwd":
            return {"bytes": fwd, "flops": 4 * rows * H * d * dv}
        bwd = e * (rows * (H + Hkv) * (d + dv) + B * c["n"] * (H * d + Hkv * (d + dv))) + 12 * S * c["state"]
        return {"bytes": fwd + bwd, "flops": 14 * rows * H * d * dv}
    if c["op"].startswith("norm"):
        N = c["rows"] * c["cols"]
        reads, writes = 1 + c["res"] + (c["gate"] != "none"), (c["res"] or not c["pre"]) + c["pre"]
        moved = reads + writes
        if c["op"] == "norm_train":
            moved += reads + writes + reads  # the inputs again, the gradients of both outputs, the gradients of the inputs
        return {"bytes": e * N * moved + 8 * c["cols"], "flops": (12 if c["op"] == "norm_fwd" else 40) * N}
    m, n, k = c["m"], c["n"], c["k"]
    b = e * (m * k + n * k + m * n * (1 + c["res"]))
    if c["op"] == "linear_fwd":
        return {"bytes": b, "flops": 2 * m * n * k}
    return {"bytes": 2 * b + e * (m * n if c["act"] != "none" else 0), "flops": 6 * m * n * k}


# ---------------------------------------------------------------------------------------------------------------------
# inputs


def prepare(c, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    io = DT[c["io"]]

    def rn(*shape, s=1.0, dtype=io):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(s).to(dtype)

    if c["op"].startswith("decay"):
        B, H, Hkv, d, dv = c["B"], c["H"], c["Hkv"], c["d"], c["dv"]
        # decays from a half a token to a thousandth, spread over the heads
        rate = 0.5 * 500.0 ** -torch.rand(H, generator=g, device="cuda")
        s = {"case": c, "log_decay": -rate}
        if c["op"] == "decay_step":
            s |= {"q": rn(B, H, d), "k": rn(B, Hkv, d), "v": rn(B, Hkv, dv), "S": rn(c["slots"], H, d, dv, dtype=torch.float32)}
            s["slots"] = torch.randperm(c["slots"], generator=g, device="cuda")[:B].to(torch.int32)
        else:
            n = c["n"]
            # the heads lie next to each other within a token, as a projection leaves them
            s |= {"q": rn(B, n, H, d).transpose(1, 2), "k": rn(B, n, Hkv, d).transpose(1, 2), "v": rn(B, n, Hkv, dv).transpose(1, 2)}
            s["lengths"] = torch.randint(c["least"], n + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            s["S0"] = rn(B, H, d, dv, dtype=torch.float32) if c["state"] else None
            if c["op"] == "decay_train":
                s["dO"] = rn(B, n, H, dv).transpose(1, 2)
                s["dS1"] = rn(B, H, d, dv, s=0.1, dtype=torch.float32) if c["state"] else None
    elif c["op"].startswith("norm"):
        R, C = c["rows"], c["cols"]
        s = {"case": c}
        s["x"] = rn(R, C) if c["res"] else None
        s["y"] = rn(R, C, s=2.0)
        s["gate"] = rn(R, C) if c["gate"] != "none" else None
        s["w_post"], s["w_pre"] = (1 + rn(C, s=0.1, dtype=torch.float32) if c[w] else None for w in ("post", "pre"))
        layer = c["kind"] == "layer"
        s["b_post"], s["b_pre"] = (rn(C, s=0.1, dtype=torch.float32) if c[w] and layer else None for w in ("post", "pre"))
        if c["op"] == "norm_train":
            s["dX"] = rn(R, C) if c["res"] or not c["pre"] else None
            s["dH"] = rn(R, C) if c["pre"] else None
    else:
        m, n, k = c["m"], c["n"], c["k"]
        s = {"case": c, "x": rn(m, k), "W": rn(n, k, s=k ** -0.5), "b": rn(n, s=0.1) if c["bias"] else None, "r": rn(m, n) if c["res"] else None}
        if c["op"] == "linear_train":
            s["dY"] = rn(m, n)
    if own:
        import paper_2512_08061_gb300.luna as L
        train = c["op"].endswith("train")
        if c["op"].startswith("decay"):
            s["plan"] = L.Decay(c["B"], c["H"], c.get("n", 1), c["d"], c["dv"], Hkv=c["Hkv"], io=io, backward=train)
        elif c["op"].startswith("norm"):
            s["plan"] = L.BlockNorm(c["rows"], c["cols"], groups=c["groups"], kind=c["kind"], gate=c["gate"], res_scale=ALPHA, eps=EPS, io=io, backward=train)
        else:
            s["plan"] = L.Linear(c["m"], c["n"], c["k"], act=c["act"], io=io, backward=train)
    return s


ALPHA, EPS = 0.5, 1e-6


# ---------------------------------------------------------------------------------------------------------------------
# the framework's calls


def _run_own(s):
    c, p = s["case"], s["plan"]
    if c["op"] == "decay_step":
        return {"o": p.step(s["q"], s["k"], s["v"], s["log_decay"], s["S"], s["slots"]), "S": s["S"]}
    if c["op"].startswith("decay"):
        O, S1 = p.forward(s["q"], s["k"], s["v"], s["log_decay"], s["lengths"], s["S0"], want_state=True)
        out = {"O": O, "S1": S1}
        if c["op"] == "decay_train":
            out |= p.backward(s["q"], s["k"], s["v"], s["dO"], s["log_decay"], s["lengths"], s["S0"], s["dS1"])
        return out
    if c["op"].startswith("norm"):
        out = p.forward(s["x"], s["y"], s["gate"], s["w_post"], s["w_pre"], s["b_post"], s["b_pre"])
        if c["op"] == "norm_train":
            out |= p.backward(s["x"], s["y"], s["gate"], s["w_post"], s["w_pre"], s["dX"], s["dH"], s["b_post"], s["b_pre"])
        return out
    if c["op"] == "linear_fwd":
        return {"Y": p.forward(s["x"], s["W"], s["b"], s["r"])}
    Y, Z = p.forward(s["x"], s["W"], s["b"], s["r"], save_z=True)
    return {"Y": Y} | p.backward(s["x"], s["W"], s["dY"], Z, bias=s["b"] is not None)


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms, in 32 bits


def _mix(a, b, c, g):
    """out_i = sum_{j <= i} exp(g (i - j)) (a_i . b_j) c_j, in pieces of the rows; a, b, c: (B, H, n, *), g: (H,)."""
    B, H, n, _ = a.shape
    C = 128 if n <= 8192 else 256
    m = -(-n // C)
    a, b, c = (torch.nn.functional.pad(x, (0, 0, 0, m * C - n)).view(B, H, m, C, -1) for x in (a, b, c))
    i = torch.arange(C, device=a.device, dtype=torch.float32)
    u = torch.arange(m, device=a.device, dtype=torch.float32)
    g = g.view(H, 1, 1)
    inside = torch.where(i[:, None] >= i, torch.exp(g * (i[:, None] - i).clamp(min=0)), 0.0)          # (H, C, C)
    across = torch.where(u[:, None] > u, torch.exp(g * C * (u[:, None] - u - 1).clamp(min=0)), 0.0)  # (H, m, m)
    out = (a @ b.transpose(-1, -2) * inside[:, None]) @ c
    pieces = (b * torch.exp(g * (C - 1 - i)[:, None])[:, None]).transpose(-1, -2) @ c
    before = (across @ pieces.flatten(3)).view(pieces.shape)
    out = out + (a * torch.exp(g * (i + 1)[:, None])[:, None]) @ before
    return out.reshape(B, H, m * C, -1)[:, :, :n]


def _run_decay(s):
    c = s["case"]
    io, H, Hkv, n = DT[c["io"]], c["H"], c["Hkv"], c["n"]
    g, scale = s["log_decay"], c["d"] ** -0.5
    t = torch.arange(n, device=g.device, dtype=torch.float32)
    length = s["lengths"].view(-1, 1, 1, 1)
    live = t.view(1, 1, n, 1) < length
    q = torch.where(live, s["q"].float(), 0.0) * scale
    k, v = (torch.where(live, s[x].float(), 0.0).repeat_interleave(H // Hkv, 1) for x in ("k", "v"))
    left = torch.where(live, torch.exp(g.view(H, 1, 1) * (length - 1 - t.view(n, 1)).clamp(min=0)), 0.0)  # (B, H, n, 1)
    past = torch.exp(g.view(H, 1, 1) * (t + 1).view(n, 1))                                               # (H, n, 1)
    whole = torch.exp(g.view(1, H, 1, 1) * length)
    O, S1 = _mix(q, k, v, g), (k * left).transpose(-1, -2) @ v
    if s["S0"] is not None:
        O, S1 = O + (q * past) @ s["S0"], S1 + whole * s["S0"]
    out = {"O": torch.where(live, O, 0.0).to(io), "S1": S1}
    if c["op"] == "decay_fwd":
        return out
    dO = torch.where(live, s["dO"].float(), 0.0)
    dQ = _mix(dO, v, k, g)
    dV = _mix(k.flip(2), q.flip(2), dO.flip(2), g).flip(2)
    dK = _mix(v.flip(2), dO.flip(2), q.flip(2), g).flip(2)
    if s["S0"] is not None:
        dQ = dQ + (dO * past) @ s["S0"].transpose(-1, -2)
        dV = dV + (k * left) @ s["dS1"]
        dK = dK + (v * left) @ s["dS1"].transpose(-1, -2)
        out["dS0"] = whole * s["dS1"] + (q * past).transpose(-1, -2) @ dO
    dK, dV = (x.reshape(c["B"], Hkv, H // Hkv, n, -1).sum(2) for x in (dK, dV))
    return out | {"dQ": torch.where(live, dQ * scale, 0.0).to(io), "dK": torch.where(live, dK, 0.0).to(io), "dV": torch.where(live, dV, 0.0).to(io)}


def _run_step(s):
    c, at = s["case"], s["slots"].long()
    G = c["H"] // c["Hkv"]
    q, k, v = s["q"].float(), s["k"].float().repeat_interleave(G, 1), s["v"].float().repeat_interleave(G, 1)
    S = s["S"][at] * torch.exp(s["log_decay"]).view(-1, 1, 1) + k[..., None] * v[..., None, :]
    s["S"][at] = S
    return {"o": ((q * c["d"] ** -0.5)[..., None, :] @ S)[..., 0, :].to(q.dtype if c["io"] == "f32" else torch.bfloat16), "S": s["S"]}


def _hat(x, groups, layer):
    """x with each group's mean (layer) taken out and its root mean square divided out, and 1 / that root."""
    x = x.unflatten(-1, (groups, -1))
    if layer:
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _hat_grad(d, xhat, r, groups, layer):
    """The gradient of _hat's input from d, that of its output."""
    d = d.unflatten(-1, (groups, -1))
    d = d - xhat * (d * xhat).mean(-1, keepdim=True) - (d.mean(-1, keepdim=True) if layer else 0.0)
    return (d * r).flatten(-2)


def _run_norm(s):
    c, io = s["case"], DT[s["case"]["io"]]
    layer, G = c["kind"] == "layer", c["groups"]
    y = u = s["y"].float()
    if c["post"]:
        yhat, yr = _hat(y, G, layer)
        u = yhat.flatten(-2) * s["w_post"] + (s["b_post"] if layer else 0.0)
    gate = s["gate"].float() if c["gate"] != "none" else None
    sig = torch.sigmoid(gate) if gate is not None else None
    act = None if gate is None else sig if c["gate"] == "sigmoid" else gate * sig
    x = ALPHA * (u if act is None else u * act)
    x = x + s["x"].float() if c["res"] else x
    out = {}
    if c["res"] or not c["pre"]:
        out["X"] = x.to(io)
    if c["pre"]:
        xhat, xr = _hat(x, 1, layer)
        out["H"] = (xhat.flatten(-2) * s["w_pre"] + (s["b_pre"] if layer else 0.0)).to(io)
    if c["op"] == "norm_fwd":
        return out
    d = s["dX"].float() if s["dX"] is not None else 0.0
    if c["pre"]:
        dh = s["dH"].float()
        out["dw_pre"] = (dh * xhat.flatten(-2)).sum(0)
        if layer:
            out["db_pre"] = dh.sum(0)
        d = d + _hat_grad(dh * s["w_pre"], xhat, xr, 1, layer)
    if c["res"]:
        out["dx"] = d.to(io)
    d = d * ALPHA
    if act is not None:
        slope = sig * (1 - sig) if c["gate"] == "sigmoid" else sig * (1 + gate * (1 - sig))
        out["dgate"] = (d * u * slope).to(io)
        d = d * act
    if c["post"]:
        out["dw_post"] = (d * yhat.flatten(-2)).sum(0)
        if layer:
            out["db_post"] = d.sum(0)
        d = _hat_grad(d * s["w_post"], yhat, yr, G, layer)
    return out | {"dy": d.to(io)}


def _act(z, act):
    """act(z) and its slope."""
    if act == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if act == "gelu":
        phi = 0.5 * (1 + torch.erf(z * 0.5 ** 0.5))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if act == "silu":
        sig = torch.sigmoid(z)
        return z * sig, sig * (1 + z * (1 - sig))
    return z, None


def _run_linear(s):
    c, io = s["case"], DT[s["case"]["io"]]
    x, W = s["x"].float(), s["W"].float()
    z = x @ W.t()
    z = z + s["b"].float() if c["bias"] else z
    y, slope = _act(z, c["act"])
    out = {"Y": (y + s["r"].float() if c["res"] else y).to(io)}
    if c["op"] == "linear_train":
        dz = s["dY"].float()
        dz = dz if slope is None else dz * slope
        out |= {"dX": (dz @ W).to(io), "dW": (dz.t() @ x).to(io)}
        if c["bias"]:
            out["db"] = dz.sum(0).to(io)
    return out


def run(s):
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    return _run_step(s) if op == "decay_step" else {"decay": _run_decay, "norm": _run_norm, "linear": _run_linear}[op.split("_")[0]](s)


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits


def _exact_decay(s):
    """Token by token: the state decays, takes in k v^T and is read by q; the gradients walk the same recurrence back."""
    c = s["case"]
    B, H, Hkv, n, d, dv = (c[x] for x in ("B", "H", "Hkv", "n", "d", "dv"))
    f = dict(device="cuda", dtype=torch.float64)
    lam = torch.exp(s["log_decay"].double()).view(1, H, 1, 1)
    scale = d ** -0.5

    def rows(x, heads):  # (n, B, H, width), 64 bits, a head of keys and values repeated for its queries
        return x.double().repeat_interleave(H // heads, 1).permute(2, 0, 1, 3)

    q, k, v = rows(s["q"], H) * scale, rows(s["k"], Hkv), rows(s["v"], Hkv)
    on = torch.arange(n, device="cuda")[:, None] < s["lengths"][None, :]
    S = s["S0"].double().clone() if s["S0"] is not None else torch.zeros(B, H, d, dv, **f)
    O = torch.zeros(n, B, H, dv, **f)
    train = c["op"] == "decay_train"
    dQ = torch.zeros(n, B, H, d, **f) if train else None
    do = rows(s["dO"], H) if train else None
    for t in range(n):
        w = on[t].view(B, 1, 1, 1)
        S = torch.where(w, S * lam + k[t].unsqueeze(-1) * v[t].unsqueeze(-2), S)
        O[t] = torch.where(w[..., 0], (q[t].unsqueeze(-2) @ S).squeeze(-2), 0.0)
        if train:
            dQ[t] = torch.where(w[..., 0], scale * (S @ do[t].unsqueeze(-1)).squeeze(-1), 0.0)
    out = {"O": O.permute(1, 2, 0, 3), "S1": S}
    if train:
        R = s["dS1"].double().clone() if s["dS1"] is not None else torch.zeros(B, H, d, dv, **f)
        dK, dV = torch.zeros(n, B, H, d, **f), torch.zeros(n, B, H, dv, **f)
        for t in range(n - 1, -1, -1):
            w = on[t].view(B, 1, 1, 1)
            now = R + q[t].unsqueeze(-1) * do[t].unsqueeze(-2)
            dK[t] = torch.where(w[..., 0], (now @ v[t].unsqueeze(-1)).squeeze(-1), 0.0)
            dV[t] = torch.where(w[..., 0], (k[t].unsqueeze(-2) @ now).squeeze(-2), 0.0)
            R = torch.where(w, now * lam, R)
        share = lambda x: x.permute(1, 2, 0, 3).unflatten(1, (Hkv, H // Hkv)).sum(2)  # noqa: E731
        out |= {"dQ": dQ.permute(1, 2, 0, 3), "dK": share(dK), "dV": share(dV)}
        if s["S0"] is not None:
            out["dS0"] = R
    return out


def _exact_step(s):
    c, at, G = s["case"], s["slots"].long(), s["case"]["H"] // s["case"]["Hkv"]
    S = s["S"].double()
    q, k, v = s["q"].double(), s["k"].double().repeat_interleave(G, 1), s["v"].double().repeat_interleave(G, 1)
    S[at] = torch.einsum("bhde,h->bhde", S[at], s["log_decay"].double().exp()) + torch.einsum("bhd,bhe->bhde", k, v)
    return {"o": torch.einsum("bhd,bhde->bhe", q, S[at]) / math.sqrt(c["d"]), "S": S}


def _exact_norm(s):
    """The forward formula; the gradients from torch's differentiation of it in 64 bits."""
    c = s["case"]
    R, C = c["rows"], c["cols"]
    leaf = {x: s[x].double().requires_grad_() if s.get(x) is not None else None for x in ("x", "y", "gate", "w_post", "w_pre", "b_post", "b_pre")}

    def norm(z, groups, w, b):
        z = z.reshape(R, groups, C // groups)
        if c["kind"] == "layer":
            z = z - z.sum(-1, keepdim=True) / (C // groups)
        z = z / torch.sqrt((z ** 2).sum(-1, keepdim=True) / (C // groups) + EPS)
        z = z.reshape(R, C) * w
        return z if b is None else z + b

    t = norm(leaf["y"], c["groups"], leaf["w_post"], leaf["b_post"]) if c["post"] else leaf["y"]
    if c["gate"] != "none":
        t = t / (1 + torch.exp(-leaf["gate"])) * (leaf["gate"] if c["gate"] == "silu" else 1.0)
    x = ALPHA * t + (leaf["x"] if c["res"] else 0.0)
    out, back = {}, []
    if c["res"] or not c["pre"]:
        out["X"] = x
    if c["pre"]:
        out["H"] = norm(x, 1, leaf["w_pre"], leaf["b_pre"])
    if c["op"] == "norm_train":
        back = [(out[o] * s[d].double()).sum() for o, d in (("X", "dX"), ("H", "dH")) if s[d] is not None]
        sum(back).backward()
        names = {"x": "dx", "y": "dy", "gate": "dgate", "w_post": "dw_post", "w_pre": "dw_pre", "b_post": "db_post", "b_pre": "db_pre"}
        out |= {names[a]: v.grad for a, v in leaf.items() if v is not None}
    return {a: v.detach() for a, v in out.items()}


def _exact_linear(s):
    c = s["case"]
    if 2 * c["m"] * c["n"] * c["k"] * (3 if c["op"] == "linear_train" else 1) > 4e12:
        return None
    train = c["op"] == "linear_train"
    x, W, b = (s[a].double().requires_grad_(train) if s[a] is not None else None for a in ("x", "W", "b"))
    z = torch.einsum("mk,nk->mn", x, W)
    z = z if b is None else z + b
    y = {"none": lambda u: u, "relu": torch.relu, "gelu": lambda u: u * torch.special.ndtr(u), "silu": lambda u: u / (1 + torch.exp(-u))}[c["act"]](z)
    out = {"Y": y if s["r"] is None else y + s["r"].double()}
    if train:
        out["Y"].backward(s["dY"].double())
        out |= {"dX": x.grad, "dW": W.grad} | ({"db": b.grad} if b is not None else {})
    return {a: v.detach() for a, v in out.items()}


def exact(c, seed):
    global own
    was, own = own, False
    s = prepare(c, seed)
    own = was
    if c["op"] == "decay_step":
        return _exact_step(s)
    return {"decay": _exact_decay, "norm": _exact_norm, "linear": _exact_linear}[c["op"].split("_")[0]](s)
