"""Measured cases of the gated delta rule and of beam search over recurrent states.

Three operators, for training, for prompts and for single tokens:

  delta    S_t = a_t (S_{t-1} - b_t k_t (k_t^T S_{t-1})) + b_t k_t v_t^T,  o_t = scale S_t^T q_t,  a_t = exp(g_t):
           linear attention whose state forgets by a gate of each token and writes the difference to what it holds
  select   the `beams` best continuations of each sequence over its beams and the vocabulary
  reorder  the recurrent states follow their beams: a beam that goes on keeps its slot, further children of a beam get
           copies in the slots of beams that ended

`run` computes them in elementary torch operations (own = False) or through the framework's calls (own = True).
"""
import math

import torch

own = False

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
C = 64  # rows of a chunk of the plain form


def listed():
    return [
        # one user's next token at the long-context head shape: all latency
        {"name": "delta step one", "op": "delta_step", "B": 1, "H": 32, "Hk": 16, "d": 128, "dv": 128, "slots": 1, "io": "bf16"},
        # a serving batch: 64 live sequences in a pool of 96 slots
        {"name": "delta step batch", "op": "delta_step", "B": 64, "H": 32, "Hk": 32, "d": 128, "dv": 128, "slots": 96, "io": "bf16"},
        # prompts of a padded batch of short texts, their states kept for the tokens that follow
        {"name": "delta prompts short", "op": "delta_fwd", "B": 32, "H": 12, "Hk": 12, "n": 512, "d": 64, "dv": 64, "least": 200, "state": False, "io": "bf16"},
        # one long prompt whose queries and keys serve two value heads each, continued from an earlier state
        {"name": "delta prompt long", "op": "delta_fwd", "B": 1, "H": 32, "Hk": 16, "n": 32768, "d": 128, "dv": 128, "least": 32768, "state": True, "io": "bf16"},
        # a training step on padded sequences
        {"name": "delta train", "op": "delta_train", "B": 8, "H": 16, "Hk": 16, "n": 4096, "d": 128, "dv": 128, "least": 2048, "state": False, "io": "bf16"},
        # a training step with shared queries and keys at the narrow head shape, pieces of text that carry a state
        {"name": "delta train shared", "op": "delta_train", "B": 4, "H": 12, "Hk": 4, "n": 2000, "d": 64, "dv": 64, "least": 1, "state": True, "io": "bf16"},
        # a small model trained in 32 bits, at odd sizes
        {"name": "delta train odd f32", "op": "delta_train", "B": 2, "H": 6, "Hk": 3, "n": 1571, "d": 40, "dv": 72, "least": 1, "state": True, "io": "f32"},
        # one user's search step
        {"name": "select one", "op": "select", "B": 1, "K": 4, "V": 50257, "io": "f32"},
        # a batch of searches, a large vocabulary
        {"name": "select batch", "op": "select", "B": 32, "K": 8, "V": 128256, "io": "bf16"},
        # a wide search over a small vocabulary, as of speech
        {"name": "select wide", "op": "select", "B": 16, "K": 32, "V": 5001, "io": "f32"},
        # the states of one user's beams
        {"name": "reorder one", "op": "reorder", "B": 1, "K": 4, "slots": 4, "H": 32, "d": 128, "dv": 128},
        # the states of a batch's beams, in a pool that other requests share
        {"name": "reorder batch", "op": "reorder", "B": 32, "K": 8, "slots": 300, "H": 32, "d": 128, "dv": 128},
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(["delta_step", "delta_fwd", "delta_fwd", "delta_train", "delta_train", "select", "select", "reorder"])
    io = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "select":
        K, V = rng.choice([1, 2, 3, 4, 5, 8, 16, rng.randint(1, 32)]), _log(rng, 100, 262144)
        B = max(1, min(_log(rng, 1, 64), (1 << 25) // (K * V)))
        return {"op": op, "B": B, "K": K, "V": V, "io": rng.choice(["bf16", "f32"])}
    hk = rng.choice([1, 2, 3, 4, 8, 16])
    h = hk * rng.choice([1, 1, 2, 3, 4])
    d = rng.choice([32, 64, 128, 128, 8 * rng.randint(2, 16), rng.randint(5, 128)])
    dv = rng.choice([d, d, 64, rng.randint(5, 128)])
    if op == "reorder":
        K, B = rng.randint(2, 16), _log(rng, 1, 32)
        B = max(1, min(B, (1 << 27) // (K * h * d * dv)))
        return {"op": op, "B": B, "K": K, "slots": B * K + rng.randint(0, 9), "H": h, "d": d, "dv": dv}
    if op == "delta_step":
        b = _log(rng, 1, 64)
        return {"op": op, "B": b, "H": h, "Hk": hk, "d": d, "dv": dv, "slots": b + rng.randint(0, 8), "io": io}
    n = _log(rng, 1, 32768 if op == "delta_fwd" else 8192)
    b = max(1, min(_log(rng, 1, 32), (1 << (20 if op == "delta_fwd" else 18)) // (n * h)))
    return {"op": op, "B": b, "H": h, "Hk": hk, "n": n, "d": d, "dv": dv, "least": rng.randint(0, n), "state": rng.random() < 0.5, "io": io}


def work(c):
    if c["op"] == "select":
        N = c["B"] * c["K"] * c["V"]
        return {"bytes": (2 if c["io"] == "bf16" else 4) * N + 18 * c["B"] * c["K"], "flops": 4 * N}
    if c["op"] == "reorder":
        # the parents are drawn at random: a beam is nobody's parent with (1 - 1/K)^K, and that many states are copied
        moved = c["B"] * c["K"] * (1 - 1 / c["K"]) ** c["K"]
        return {"bytes": 8 * moved * c["H"] * c["d"] * c["dv"] + 12 * c["B"] * c["K"], "flops": 0}
    e = 2 if c["io"] == "bf16" else 4
    B, H, Hk, d, dv = c["B"], c["H"], c["Hk"], c["d"], c["dv"]
    S = B * H * d * dv
    if c["op"] == "delta_step":
        return {"bytes": 8 * S + e * B * (2 * H * dv + 2 * Hk * d + 2 * H), "flops": 7 * S}
    used = (c["least"] + c["n"]) / 2 / c["n"]  # the rows that lengths leave, on the average
    rows = B * c["n"] * used
    fwd = e * (rows * (2 * Hk * d + H * (dv + 2)) + B * c["n"] * H * dv) + 4 * S * (1 + c["state"])
    if c["op"] == "delta_fwd":
        return {"bytes": fwd, "flops": 6 * rows * H * d * dv}
    bwd = e * (rows * (2 * Hk * d + H * (2 * dv + 2)) + B * c["n"] * (2 * Hk * d + H * (dv + 2))) + 12 * S * c["state"]
    return {"bytes": fwd + bwd, "flops": 18 * rows * H * d * dv}


# ---------------------------------------------------------------------------------------------------------------------
# inputs


def prepare(c, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    io = DT[c.get("io", "f32")]

    def rn(*shape, s=1.0, dtype=torch.float32):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(s).to(dtype)

    s = {"case": c}
    if c["op"] == "select":
        B, K, V = c["B"], c["K"], c["V"]
        # a few words far ahead of the rest; running log-probabilities of beams that have gone some way together
        s["logits"] = rn(B * K, V, s=2.0).to(io)
        s["scores"] = (-torch.rand((B, 1), generator=g, device=DEV) * 20 - torch.rand((B, K), generator=g, device=DEV) * 4).sort(-1, descending=True)[0].contiguous()
        s["done"] = torch.rand((B, K), generator=g, device=DEV) < 0.1
    elif c["op"] == "reorder":
        B, K = c["B"], c["K"]
        s["parents"] = torch.randint(0, K, (B, K), generator=g, device=DEV, dtype=torch.int32)
        s["slots"] = torch.randperm(c["slots"], generator=g, device=DEV)[:B * K].to(torch.int32).view(B, K)
        s["S"] = rn(c["slots"], c["H"], c["d"], c["dv"])
    else:
        B, H, Hk, d, dv, n = c["B"], c["H"], c["Hk"], c["d"], c["dv"], c.get("n", 1)

        def unit(x):
            return (x / x.norm(dim=-1, keepdim=True)).to(io)

        # queries and keys of length one; the heads lie next to each other within a token, as a projection leaves them
        q, k, v = unit(rn(B, n, Hk, d)), unit(rn(B, n, Hk, d)), rn(B, n, H, dv, dtype=io)
        # gates: forgetting from half a token's to a thousandth, spread over the heads, more or less at each token
        rate = 0.5 * 500.0 ** -torch.rand(H, generator=g, device=DEV)
        gate = (-rate * 2 * torch.rand((B, n, H), generator=g, device=DEV)).to(io)
        beta = torch.sigmoid(rn(B, n, H)).to(io)
        if c["op"] == "delta_step":
            s |= {"q": q[:, 0], "k": k[:, 0], "v": v[:, 0], "g": gate[:, 0], "b": beta[:, 0], "S": rn(c["slots"], H, d, dv)}
            s["slots"] = torch.randperm(c["slots"], generator=g, device=DEV)[:B].to(torch.int32)
        else:
            s |= {"q": q.transpose(1, 2), "k": k.transpose(1, 2), "v": v.transpose(1, 2), "g": gate.transpose(1, 2), "b": beta.transpose(1, 2)}
            s["lengths"] = torch.randint(c["least"], n + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
            s["S0"] = rn(B, H, d, dv) if c["state"] else None
            if c["op"] == "delta_train":
                s["dO"] = rn(B, n, H, dv, dtype=io).transpose(1, 2)
                s["dS1"] = rn(B, H, d, dv, s=0.1) if c["state"] else None
    if own:
        import paper_2512_08061_gb300.luna as L
        if c["op"] == "select":
            s["plan"] = L.Beam(c["B"], c["K"], c["V"], end=END, io=io)
        elif c["op"] == "reorder":
            s["plan"] = L.Beam(c["B"], c["K"])
        else:
            s["plan"] = L.Delta(c["B"], c["H"], c.get("n", 1), c["d"], c["dv"], Hk=c["Hk"], io=io, backward=c["op"] == "delta_train")
    return s


END = 2  # the token that ends a sequence


# ---------------------------------------------------------------------------------------------------------------------
# the framework's calls


def _run_own(s):
    c, p = s["case"], s["plan"]
    if c["op"] == "select":
        return p.select(s["logits"], s["scores"], s["done"])
    if c["op"] == "reorder":
        return {"slots": p.reorder(s["parents"], s["slots"], s["S"]), "S": s["S"]}
    if c["op"] == "delta_step":
        return {"o": p.step(s["q"], s["k"], s["v"], s["g"], s["b"], s["S"], s["slots"]), "S": s["S"]}
    O, S1 = p.forward(s["q"], s["k"], s["v"], s["g"], s["b"], s["lengths"], s["S0"], want_state=True)
    out = {"O": O, "S1": S1}
    if c["op"] == "delta_train":
        out |= p.backward(s["q"], s["k"], s["v"], s["dO"], s["g"], s["b"], s["lengths"], s["S0"], s["dS1"])
    return out


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms, in 32 bits


def _run_delta(s):
    """Chunk by chunk.  With G_i the sum of a chunk's gates to row i, S the state before the chunk and
    T = (1 + tril(diag(b) (K K^T * exp(G_i - G_j)), -1))^-1, the rows that a chunk writes are
    U = T diag(b) (V - diag(exp G) K S); the gradients are those of these products."""
    c = s["case"]
    io, H, Hk, n, B = DT[c["io"]], c["H"], c["Hk"], c["n"], c["B"]
    m, scale = -(-n // C), c["d"] ** -0.5
    live = torch.arange(n, device=DEV) < s["lengths"].view(-1, 1, 1)

    def cut(x, heads):  # (B, H, m, C, width), rows past a sequence's end zero
        x = x.float().repeat_interleave(H // heads, 1)
        x = torch.where(live if x.dim() == 3 else live[..., None], x, 0.0)
        pad = (0, m * C - n) if x.dim() == 3 else (0, 0, 0, m * C - n)
        x = torch.nn.functional.pad(x, pad)
        return x.view(B, H, m, C) if x.dim() == 3 else x.view(B, H, m, C, -1)

    q, k, v, g, b = (cut(s[x], h) for x, h in (("q", Hk), ("k", Hk), ("v", H), ("g", H), ("b", H)))
    b = b[..., None]
    G = g.double().cumsum(-1)
    gap = (G[..., :, None] - G[..., None, :]).tril_().exp_().float()          # exp(G_i - G_j) where i >= j
    past, left = G.exp().float()[..., None], (G[..., -1:] - G).exp().float()[..., None]
    whole = past[..., -1:, :]
    A = ((k @ k.transpose(-1, -2)) * gap).tril(-1) * b
    T, at = torch.eye(C, device=DEV).expand_as(A), torch.arange(C, device=DEV)
    for w in (1, 2, 4, 8, 16, 32):  # inverses of diagonal blocks of w rows become those of 2 w rows
        low = (at[:, None] // (2 * w) == at // (2 * w)) & (at[:, None] // w != at // w)
        T = T - T @ (A * low) @ T
    del A
    ends = (k * left).transpose(-1, -2)
    S = torch.zeros(B, H, c["d"], c["dv"], device=DEV) if s["S0"] is None else s["S0"]
    U, before = torch.empty_like(v), torch.empty(B, H, m + 1, c["d"], c["dv"], device=DEV)
    for i in range(m):
        before[:, :, i] = S
        U[:, :, i] = T[:, :, i] @ (b[:, :, i] * (v[:, :, i] - past[:, :, i] * (k[:, :, i] @ S)))
        S = whole[:, :, i] * S + ends[:, :, i] @ U[:, :, i]
    before[:, :, m] = S
    P = (q @ k.transpose(-1, -2)).mul_(gap).tril_()
    O = scale * ((q * past) @ before[:, :, :m] + P @ U)

    def rows(x, heads=H):  # back to (B, heads, n, width) in the tensors' type, shared heads summed
        return x.reshape(B, heads, H // heads, m * C, -1).sum(2)[:, :, :n].to(io)

    out = {"O": rows(O), "S1": S}
    if c["op"] == "delta_fwd":
        return out
    dO = cut(s["dO"], H)
    dU, dX, after = P.transpose(-1, -2) @ dO * scale, torch.empty_like(v), torch.empty_like(before)
    ends, starts, reads = k * left, scale * (q * past).transpose(-1, -2), (k * past * b).transpose(-1, -2)
    T = T.transpose(-1, -2)
    R = torch.zeros_like(S) if s["dS1"] is None else s["dS1"]
    after[:, :, m] = R
    for i in range(m - 1, -1, -1):
        dX[:, :, i] = T[:, :, i] @ (dU[:, :, i] + ends[:, :, i] @ R)
        R = whole[:, :, i] * R + starts[:, :, i] @ dO[:, :, i] - reads[:, :, i] @ dX[:, :, i]
        after[:, :, i] = R
    P = (dO @ U.transpose(-1, -2)).mul_(gap).tril_().mul_(scale)
    W = (dX @ U.transpose(-1, -2)).mul_(gap).tril_(-1)
    St = before[:, :, :m].transpose(-1, -2)
    dQ = scale * past * (dO @ St) + P @ k
    Z = past * (dX @ St) + W @ k
    dKw = left * (U @ after[:, :, 1:].transpose(-1, -2)) + P.transpose(-1, -2) @ q - W.transpose(-1, -2) @ (b * k)
    db = (dX * v).sum(-1) - (k * Z).sum(-1)
    dG = (q * dQ).sum(-1) - (b * k * Z).sum(-1) - (k * dKw).sum(-1)
    dg = dG.flip(-1).cumsum(-1).flip(-1) + (before[:, :, 1:] * after[:, :, 1:]).sum((-1, -2))[..., None]
    if s["S0"] is not None:
        out["dS0"] = R
    dg, db = (torch.where(live, x.reshape(B, H, m * C)[:, :, :n], 0.0).to(io) for x in (dg, db))
    return out | {"dQ": rows(dQ, Hk), "dK": rows(dKw - b * Z, Hk), "dV": rows(b * dX), "dlog_decay": dg, "dbeta": db}


def _run_step(s):
    c, at = s["case"], s["slots"].long()
    share = c["H"] // c["Hk"]
    q, k, v = s["q"].float().repeat_interleave(share, 1), s["k"].float().repeat_interleave(share, 1), s["v"].float()
    S = s["S"][at] * torch.exp(s["g"].float())[..., None, None]
    u = s["b"].float()[..., None] * (v - (k[..., None, :] @ S)[..., 0, :])
    S = S + k[..., None] * u[..., None, :]
    s["S"][at] = S
    return {"o": ((q * c["d"] ** -0.5)[..., None, :] @ S)[..., 0, :].to(s["q"].dtype), "S": s["S"]}


def _run_select(s):
    """Scores in 64 bits, so that near ones stay in their order; equal ones go by their place, beam before token."""
    c = s["case"]
    B, K, V = c["B"], c["K"], c["V"]
    x = s["logits"].double().view(B, K, V)
    top = x.amax(-1, keepdim=True)
    base = s["scores"].double()[..., None] - top - torch.log(torch.exp(x - top).sum(-1, keepdim=True))
    all_ = torch.where(torch.isfinite(base), base + x, -math.inf)
    ends = torch.arange(V, device=DEV) == END
    all_ = torch.where(s["done"][..., None], torch.where(ends, s["scores"].double()[..., None], -math.inf), all_)
    value, place = all_.view(B, K * V).sort(dim=-1, descending=True, stable=True)
    value, place = value[:, :K], place[:, :K]
    parents, tokens = place // V, place % V
    return {"scores": value.float(), "tokens": tokens.int(), "parents": parents.int(), "done": s["done"].gather(1, parents) | (tokens == END)}


def _run_reorder(s):
    c = s["case"]
    K, parents = c["K"], s["parents"].long()
    j = torch.arange(K, device=DEV)
    same = parents[:, :, None] == parents[:, None, :]
    first = ~(same & (j[:, None] > j)).any(-1)                     # the first child of its parent keeps its slot
    lost = ~(parents[:, None, :] == j[:, None]).any(-1)             # beams without a child, whose slots are free
    nth = (~first).long().cumsum(-1) - 1                            # the others take the free slots in order
    free = torch.where(lost, j, K).sort(-1)[0].clamp(max=K - 1)
    slots = torch.where(first, s["slots"].gather(1, parents), s["slots"].gather(1, free.gather(1, nth.clamp(min=0))))
    moved = s["S"][s["slots"].gather(1, parents).long()]
    s["S"][slots.long()] = moved
    return {"slots": slots, "S": s["S"]}


def run(s):
    if own:
        return _run_own(s)
    return {"delta_step": _run_step, "delta_fwd": _run_delta, "delta_train": _run_delta, "select": _run_select, "reorder": _run_reorder}[s["case"]["op"]](s)


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits


def _exact_delta(s):
    """Token by token, as the recurrence is written; the gradients walk it back, with the states between every 64th
    token computed again."""
    c = s["case"]
    B, H, Hk, n, d, dv = (c[x] for x in ("B", "H", "Hk", "n", "d", "dv"))
    f = dict(device=DEV, dtype=torch.float64)

    def rows(x, heads):  # (n, B, H, width)
        return x.double().repeat_interleave(H // heads, 1).movedim(2, 0)

    q, k, v = rows(s["q"], Hk) * d ** -0.5, rows(s["k"], Hk), rows(s["v"], H)
    a, b = rows(s["g"], H).exp(), rows(s["b"], H)
    on = torch.arange(n, device=DEV)[:, None] < s["lengths"][None, :]
    on = on.view(n, B, 1, 1)

    def read(x, S):  # x^T S
        return (x.unsqueeze(-2) @ S).squeeze(-2)

    def write(S, t):
        faded = a[t].view(B, H, 1, 1) * S
        wrote = b[t].unsqueeze(-1) * (v[t] - read(k[t], faded))
        return torch.where(on[t].unsqueeze(-1), faded + k[t].unsqueeze(-1) * wrote.unsqueeze(-2), S)

    S = s["S0"].double().clone() if s["S0"] is not None else torch.zeros(B, H, d, dv, **f)
    O, kept, train = torch.zeros(n, B, H, dv, **f), [], c["op"] == "delta_train"
    for t in range(n):
        if train and t % 64 == 0:
            kept.append(S)
        S = write(S, t)
        O[t] = torch.where(on[t], read(q[t], S), 0.0)
    out = {"O": O.permute(1, 2, 0, 3), "S1": S}
    if not train:
        return out
    do = rows(s["dO"], H)
    R = s["dS1"].double().clone() if s["dS1"] is not None else torch.zeros(B, H, d, dv, **f)
    dQ, dK, dV = (torch.zeros(n, B, H, w, **f) for w in (d, d, dv))
    dg, db = torch.zeros(n, B, H, **f), torch.zeros(n, B, H, **f)
    for start in range((n - 1) // 64 * 64, -1, -64):
        states = [kept.pop()]
        for t in range(start, min(n, start + 64)):
            states.append(write(states[-1], t))
        for t in range(min(n, start + 64) - 1, start - 1, -1):
            was, now = states[t - start], states[t - start + 1]
            w = on[t]
            dQ[t] = torch.where(w, d ** -0.5 * (now @ do[t].unsqueeze(-1)).squeeze(-1), 0.0)
            R_ = R + q[t].unsqueeze(-1) * do[t].unsqueeze(-2)       # of the state after the token
            faded = a[t].view(B, H, 1, 1) * was
            err = v[t] - read(k[t], faded)
            du = read(k[t], R_)                                     # of u = b err
            derr = b[t].unsqueeze(-1) * du
            dV[t] = torch.where(w, derr, 0.0)
            db[t] = torch.where(w[..., 0], (du * err).sum(-1), 0.0)
            dK[t] = torch.where(w, (R_ @ (b[t].unsqueeze(-1) * err).unsqueeze(-1)).squeeze(-1) - (faded @ derr.unsqueeze(-1)).squeeze(-1), 0.0)
            dfaded = R_ - k[t].unsqueeze(-1) * derr.unsqueeze(-2)
            dg[t] = torch.where(w[..., 0], (dfaded * faded).sum((-1, -2)), 0.0)
            R = torch.where(w.unsqueeze(-1), a[t].view(B, H, 1, 1) * dfaded, R)
    share = lambda x: x.permute(1, 2, 0, 3).unflatten(1, (Hk, H // Hk)).sum(2)  # noqa: E731
    out |= {"dQ": share(dQ), "dK": share(dK), "dV": dV.permute(1, 2, 0, 3), "dlog_decay": dg.permute(1, 2, 0), "dbeta": db.permute(1, 2, 0)}
    if s["S0"] is not None:
        out["dS0"] = R
    return out


def _exact_step(s):
    c, at, share = s["case"], s["slots"].long(), s["case"]["H"] // s["case"]["Hk"]
    S = s["S"].double()
    q, k, v = s["q"].double().repeat_interleave(share, 1), s["k"].double().repeat_interleave(share, 1), s["v"].double()
    old = torch.einsum("bhde,bh->bhde", S[at], s["g"].double().exp())
    err = v - torch.einsum("bhd,bhde->bhe", k, old)
    S[at] = old + torch.einsum("bh,bhd,bhe->bhde", s["b"].double(), k, err)
    return {"o": torch.einsum("bhd,bhde->bhe", q, S[at]) / math.sqrt(c["d"]), "S": S}


def _exact_select(s):
    c = s["case"]
    B, K, V = c["B"], c["K"], c["V"]
    p = torch.log_softmax(s["logits"].double(), -1).view(B, K, V) + s["scores"].double()[:, :, None]
    stay = torch.full_like(p, -math.inf)
    stay[:, :, END] = s["scores"].double()
    p = torch.where(s["done"][:, :, None], stay, p)
    return {"scores": p.reshape(B, K * V).topk(K)[0], "tokens": None, "parents": None, "done": None}


def _exact_reorder(s):
    """Beam by beam on the host."""
    c, S = s["case"], s["S"].double()
    parents, slots = s["parents"].tolist(), s["slots"].tolist()
    for b in range(c["B"]):
        free = [slots[b][k] for k in range(c["K"]) if k not in parents[b]]
        seen = set()
        for p in parents[b]:
            if p in seen:
                S[free.pop(0)] = S[slots[b][p]]
            seen.add(p)
    return {"slots": None, "S": S}


def exact(c, seed):
    global own
    was, own = own, False
    s = prepare(c, seed)
    own = was
    return {"delta_step": _exact_step, "delta_fwd": _exact_delta, "delta_train": _exact_delta, "select": _exact_select, "reorder": _exact_reorder}[c["op"]](s)
