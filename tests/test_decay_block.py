"""The example block: its forward and gradients against the same block in 64 bits, training and serving.

Tolerance (relative 2-norm): some ten bf16 roundings of 1.7e-3 follow one another on the way to any of the
values, independent of each other: sqrt(10) * 1.7e-3 = 5.4e-3, doubled for the gradients' way back: 1.1e-2,
taken as 2e-2."""
import pytest
import torch


@pytest.fixture(scope="module")
def ex():
    from paper_2512_08061_gb300 import build
    build.build()
    from paper_2512_08061_gb300.examples import decay_block
    return decay_block


def plain(x, w, B, n, H, d):
    def norm(z, groups=1):
        z = z.unflatten(-1, (groups, -1))
        return (z / (z.square().mean(-1, keepdim=True) + 1e-6).sqrt()).flatten(-2)

    inner = H * d
    y = (norm(x) * w["w_in"]) @ w["qkvg"].t() + w["b_qkvg"]
    q, k, v = (y[:, i * inner:(i + 1) * inner].view(B, n, H, d).transpose(1, 2) for i in range(3))
    i = torch.arange(n, device=x.device)
    decay = torch.where(i[:, None] >= i, torch.exp(w["log_decay"].view(H, 1, 1) * (i[:, None] - i).clamp(min=0)), 0.0)
    o = (((q @ k.transpose(-1, -2)) * d ** -0.5 * decay) @ v).transpose(1, 2).reshape(B * n, inner)
    g = y[:, 3 * inner:]
    x = x + (norm(o, H) * w["w_heads"] * g * torch.sigmoid(g)) @ w["out"].t()
    z = (norm(x) * w["w_mlp"]) @ w["up"].t() + w["b_up"]
    return x + (z * torch.special.ndtr(z)) @ w["down"].t()


@pytest.mark.gpu
def test_block_and_its_gradients(ex):
    B, n, width, H, d, ffn = 2, 300, 256, 4, 64, 384
    w = ex.DecayBlock.weights(width, H, d, ffn, seed=3)
    block = ex.DecayBlock(B, n, width, H, d, ffn)
    g = torch.Generator("cuda").manual_seed(2)
    x, dy = (torch.randn((B * n, width), generator=g, device="cuda").bfloat16() for _ in range(2))
    y, _, kept = block.forward(x, w)
    dx, grads = block.backward(dy, w, kept)
    leaf = {k: v.double().requires_grad_() for k, v in w.items()}
    xd = x.double().requires_grad_()
    want = plain(xd, leaf, B, n, H, d)
    want.backward(dy.double())
    got = {"y": (y, want.detach()), "dx": (dx, xd.grad), **{k: (v, leaf[k].grad) for k, v in grads.items()}}
    assert set(grads) == set(w) - {"log_decay"}
    for name, (a, b) in got.items():
        assert ((a.double() - b).norm() / b.norm()).item() < 2e-2, name


@pytest.mark.gpu
def test_trains_and_serves(ex):
    """The loss falls, and single tokens continue a prompt as the prompt form does."""
    first, last, off = ex.main(steps=20)
    assert last < 0.9 * first
    assert off < 2e-2
