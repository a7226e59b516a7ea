"""A stack of decayed linear-attention blocks, trained and served with the library's own kernels.

One block, on x (B, n, width) with H heads of width d:

    h = norm(x) w_in                                   luna_norm_fwd (for a later block: with the one before)
    q, k, v, g = split(h W_qkvg^T + b)                 luna_linear_fwd
    o = decayed attention of q, k, v                   luna_decay_fwd (prompts) or luna_decay_step (tokens)
    u = norm(o) over each head, times silu(g)          luna_norm_fwd, groups = H
    x <- x + u W_out^T                                 luna_linear_fwd with the residual in its epilogue
    h = norm(x) w_mlp;  x <- x + gelu(h W_up^T) W_down^T

Run it: python -m paper_2512_08061_gb300.examples.decay_block
It takes some training steps on a synthetic next-token task, then continues a prompt token by token and
compares that with the prompt form.  Random weights and data; needs the built library and a GPU.
"""
from __future__ import annotations

import torch

import paper_2512_08061_gb300.luna as L


class DecayBlock:
    """One block for a fixed batch and length (length 1 for serving single tokens).  Weights are shared by
    passing the same dict to blocks of other lengths."""

    def __init__(self, B, n, width, H, d, ffn, io=torch.bfloat16, device="cuda", training=True):
        self.B, self.n, self.width, self.H, self.d, self.io = B, n, width, H, d, io
        rows, inner = B * n, H * d
        new = dict(io=io, device=device, backward=training)
        self.norm_in = L.BlockNorm(rows, width, **new)
        self.qkvg = L.Linear(rows, 4 * inner, width, **new)
        self.attn = L.Decay(B, H, n, d, d, **new)
        self.norm_heads = L.BlockNorm(rows, inner, groups=H, gate="silu", **new)
        self.out = L.Linear(rows, width, inner, **new)
        self.norm_mlp = L.BlockNorm(rows, width, **new)
        self.up = L.Linear(rows, ffn, width, act="gelu", **new)
        self.down = L.Linear(rows, width, ffn, **new)

    @staticmethod
    def weights(width, H, d, ffn, io=torch.bfloat16, device="cuda", seed=0):
        g = torch.Generator(device).manual_seed(seed)

        def mat(n, k):
            return (torch.randn((n, k), generator=g, device=device) * k ** -0.5).to(io)

        one = dict(device=device, dtype=torch.float32)
        inner = H * d
        # decays from 1 - 2^-1 to 1 - 2^-8 over the heads
        rates = torch.log1p(-2.0 ** -torch.linspace(1, 8, H, device=device))
        return {"w_in": torch.ones(width, **one), "qkvg": mat(4 * inner, width), "b_qkvg": torch.zeros(4 * inner, device=device, dtype=io),
                "log_decay": rates, "w_heads": torch.ones(inner, **one), "out": mat(width, inner), "w_mlp": torch.ones(width, **one),
                "up": mat(ffn, width), "b_up": torch.zeros(ffn, device=device, dtype=io), "down": mat(width, ffn)}

    def _split(self, y):
        """Views of the projection's columns: q, k, v as (B, H, n, d), g as (B * n, H * d)."""
        inner = self.H * self.d
        parts = [y[:, i * inner:(i + 1) * inner] for i in range(4)]
        heads = [p.unflatten(0, (self.B, self.n)).unflatten(2, (self.H, self.d)).transpose(1, 2) for p in parts[:3]]
        return (*heads, parts[3])

    def _rows(self, t):
        """(B, H, n, d) laid out token by token -> (B * n, H * d)."""
        return t.transpose(1, 2).reshape(self.B * self.n, self.H * self.d)

    def forward(self, x, w, lengths=None, state=None):
        """x: (B * n, width) -> the block's output, the states after it, and what backward needs."""
        h = self.norm_in.forward(x, None, w_pre=w["w_in"])["H"]
        y = self.qkvg.forward(h, w["qkvg"], w["b_qkvg"])
        q, k, v, g = self._split(y)
        o = torch.empty((self.B, self.n, self.H, self.d), dtype=self.io, device=x.device).transpose(1, 2)
        o, after = self.attn.forward(q, k, v, w["log_decay"], lengths, state, want_state=True, O=o)
        u = self.norm_heads.forward(None, self._rows(o), g, w_post=w["w_heads"])["X"]
        x1 = self.out.forward(u, w["out"], None, x)
        h2 = self.norm_mlp.forward(x1, None, w_pre=w["w_mlp"])["H"]
        a, z = self.up.forward(h2, w["up"], w["b_up"], save_z=True)
        x2 = self.down.forward(a, w["down"], None, x1)
        return x2, after, (x, h, y, o, u, x1, h2, a, z, lengths, state)

    def backward(self, dx2, w, kept):
        """The gradient of x and of every weight (decays are constants)."""
        x, h, y, o, u, x1, h2, a, z, lengths, state = kept
        q, k, v, g = self._split(y)
        grads = {}
        b = self.down.backward(a, w["down"], dx2)
        grads["down"] = b["dW"]
        b = self.up.backward(h2, w["up"], b["dX"], z, bias=True)
        grads["up"], grads["b_up"] = b["dW"], b["db"]
        b = self.norm_mlp.backward(x1, None, None, None, w["w_mlp"], dx2, b["dX"])  # dx2: the residual past the MLP
        dx1, grads["w_mlp"] = b["dx"], b["dw_pre"]
        b = self.out.backward(u, w["out"], dx1)
        grads["out"] = b["dW"]
        dy = torch.empty_like(y)  # the projection's gradient, filled part by part through views
        dq, dk, dv, dg = self._split(dy)
        do = torch.empty_like(o)
        flat = do.transpose(1, 2).view(self.B * self.n, self.H * self.d)
        n = self.norm_heads.backward(None, self._rows(o), g, w["w_heads"], None, b["dX"], None,
                                     out={"dy": flat, "dgate": dg, "dw_post": torch.empty_like(w["w_heads"])})
        grads["w_heads"] = n["dw_post"]
        self.attn.backward(q, k, v, do, w["log_decay"], lengths, state, None, out={"dQ": dq, "dK": dk, "dV": dv})
        b = self.qkvg.backward(h, w["qkvg"], dy, bias=True)
        grads["qkvg"], grads["b_qkvg"] = b["dW"], b["db"]
        b = self.norm_in.backward(x, None, None, None, w["w_in"], dx1, b["dX"])
        grads["w_in"] = b["dw_pre"]
        return b["dx"], grads

    def step(self, x, w, pool, slots=None):
        """One token of each sequence: x (B, width), advancing the states of the pool in place."""
        h = self.norm_in.forward(x, None, w_pre=w["w_in"])["H"]
        y = self.qkvg.forward(h, w["qkvg"], w["b_qkvg"]).view(self.B, 4, self.H, self.d)
        o = self.attn.step(y[:, 0], y[:, 1], y[:, 2], w["log_decay"], pool, slots)
        u = self.norm_heads.forward(None, o.flatten(1), y[:, 3].flatten(1), w_post=w["w_heads"])["X"]
        x1 = self.out.forward(u, w["out"], None, x)
        h2 = self.norm_mlp.forward(x1, None, w_pre=w["w_mlp"])["H"]
        return self.down.forward(self.up.forward(h2, w["up"], w["b_up"]), w["down"], None, x1)


def main(steps=30, B=4, n=256, width=256, H=4, d=64, ffn=512, vocab=64, device="cuda"):
    """Trains one block to name the token `gap` places back, then serves it.  Returns (first loss, last loss,
    relative difference between the served tokens and the prompt form)."""
    g = torch.Generator(device).manual_seed(1)
    w = DecayBlock.weights(width, H, d, ffn, device=device)
    embed = torch.randn((vocab, width), generator=g, device=device) * 0.5
    head = torch.randn((vocab, width), generator=g, device=device) * width ** -0.5
    block = DecayBlock(B, n, width, H, d, ffn, device=device)
    logits_of = L.Linear(B * n, vocab, width, device=device, backward=True)
    gap, rate, momentum, first = 1, 0.5, 0.9, None
    w["head"] = head.to(torch.bfloat16)
    master = {k: v.float() for k, v in w.items()}
    speed = {k: torch.zeros_like(v) for k, v in master.items()}
    for it in range(steps):
        ids = torch.randint(0, vocab, (B, n), generator=g, device=device)
        target = torch.roll(ids, gap, 1).reshape(-1)
        x = embed[ids].reshape(B * n, width).to(torch.bfloat16)
        y, _, kept = block.forward(x, w)
        logits = logits_of.forward(y, w["head"]).float()
        p = torch.softmax(logits, -1)
        valid = (torch.arange(n, device=device) >= gap).repeat(B)
        loss = -torch.log(p[torch.arange(B * n, device=device), target])[valid].mean()
        p[torch.arange(B * n, device=device), target] -= 1.0
        dlogits = (p * valid[:, None] / valid.sum()).to(torch.bfloat16)
        b = logits_of.backward(y, w["head"], dlogits)
        _, grads = block.backward(b["dX"], w, kept)
        grads["head"] = b["dW"]
        for k, v in grads.items():  # stochastic gradient descent with momentum on 32-bit copies
            speed[k] = momentum * speed[k] + v.float()
            master[k] -= rate * speed[k]
            w[k] = master[k].to(w[k].dtype)
        first = loss.item() if first is None else first
    last = loss.item()

    # serving: a prompt of n - 8 tokens, then the last eight one at a time
    cut = n - 8
    whole, _, _ = block.forward(x, w)
    prompt = DecayBlock(B, cut, width, H, d, ffn, device=device, training=False)
    xs = x.view(B, n, width)
    _, state, _ = prompt.forward(xs[:, :cut].reshape(B * cut, width), w)
    token = DecayBlock(B, 1, width, H, d, ffn, device=device, training=False)
    served = torch.stack([token.step(xs[:, t].contiguous(), w, state) for t in range(cut, n)], 1)
    want = whole.view(B, n, width)[:, cut:].float()
    off = ((served.float() - want).norm() / want.norm()).item()
    return first, last, off


if __name__ == "__main__":
    a, b, off = main()
    print(f"loss {a:.3f} -> {b:.3f}; served tokens against the prompt form: {off:.2e}")
