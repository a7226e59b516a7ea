"""What the classes of the decayed linear-attention block take and own, beyond what their operators' tests check."""
import types

import pytest
import torch


@pytest.fixture(scope="module")
def L():
    from paper_2512_08061_gb300 import build
    build.build()
    import paper_2512_08061_gb300.luna as L
    return L


def test_a_device_has_its_number(L, monkeypatch):
    """A plan for "cuda" is one for the GPU that was current when it was made, and refuses tensors of another."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 2)
    p = L.BlockNorm(4, 8, io=torch.float32, device="cuda")
    assert p.device == torch.device("cuda", 2)
    there, elsewhere = (types.SimpleNamespace(shape=(4, 8), dtype=torch.float32, device=torch.device("cuda", i)) for i in (2, 0))
    L._want("x", there, (4, 8), torch.float32, p.device)
    with pytest.raises(ValueError):
        L._want("x", elsewhere, (4, 8), torch.float32, p.device)
    assert L.BlockNorm(4, 8, device="cpu").device == torch.device("cpu")
    assert L.BlockNorm(4, 8, device="cuda:1").device == torch.device("cuda", 1)


def test_decay_workspace_is_what_the_call_uses(L):
    """One piece a head keeps no states of pieces; shared heads keep their gradients, one for each query head."""
    size = L.luna_decay_workspace_size
    for n, d, io in ((100, 128, L.LUNA_BF16), (64, 128, L.LUNA_F32), (100, 40, L.LUNA_BF16)):
        one = L.decay_desc(64, 32, n, d, d, io=io)
        assert size(one, False) <= 256 and size(one, True) <= 256
        shared = L.decay_desc(64, 32, n, d, d, Hkv=8, io=io)
        assert size(shared, False) <= 256 and size(shared, True) == 256 + 64 * 32 * n * d * 4
    long = L.decay_desc(1, 2, 1 << 16, 128, 128)
    state = 2 * 128 * 128 * 4
    assert size(long, False) > 2 * 2 * state and size(long, True) > 3 * 2 * state


def test_linear_workspace_is_what_the_call_uses(L):
    """Partial products are kept for products that may be cut along their depth alone."""
    size, F, BF = L.luna_linear_workspace_size, L.LUNA_F32, L.LUNA_BF16
    for m, n, k, io in ((65536, 4096, 4096, BF), (1, 8192, 4096, BF), (8, 8192, 4096, BF), (32, 512, 4096, F), (1 << 20, 512, 64, BF)):
        assert size(L.linear_desc(m, n, k, io=io), False) <= 256, (m, n, k, io)
    # dX and dW of a large layer: the bias gradient's sums over 256 rows, and dz where there is an activation
    assert size(L.linear_desc(65536, 4096, 4096, io=BF), True) == 256 + 256 * 4096 * 4
    assert size(L.linear_desc(65536, 4096, 4096, "gelu", io=BF), True) == 256 + 256 * 4096 * 4 + 65536 * 4096 * 2
    # few tiles and a depth to cut
    assert 256 < size(L.linear_desc(128, 128, 8192, io=BF), False) <= 256 + 128 * 128 * 4 * 32


def test_grids_are_the_devices(L):
    """Grids that stay for all rows, and with them the weight gradients' partial sums, go by the device's SMs."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count if torch.cuda.is_available() else 148  # (as the library's own default)
    for cols, io in ((4096, L.LUNA_BF16), (16384, L.LUNA_F32), (5001, L.LUNA_BF16)):
        size = L.luna_norm_workspace_size(L.norm_desc(1 << 20, cols, io=io))
        sums = size // (16 * cols) // sms * sms * 16 * cols  # (four arrays of fp32 a block)
        assert sums > 0 and size == (sums + 255) // 256 * 256


@pytest.mark.gpu
def test_memory_of_a_call_on_another_stream(L):
    """What a call on a stream allocates is that stream's, and the workspace outlives what is queued there: neither
    is handed out on the current stream while the call may still run.  (Sizes over 10 MB have blocks of their own,
    which the allocator otherwise hands out again at once.)"""
    io = dict(device="cuda", dtype=torch.bfloat16)
    s = torch.cuda.Stream()
    x, W = torch.randn((4096, 1024), **io), torch.randn((4096, 1024), **io)
    q = torch.randn((2, 32, 1024, 128), **io)
    rates = torch.full((32,), -0.1, device="cuda")
    w = torch.ones(4096, device="cuda")
    li = L.Linear(4096, 4096, 1024, "gelu", backward=True)
    at = L.Decay(2, 32, 1024, 128, 128, backward=True)
    nm = L.BlockNorm(4096, 4096, backward=True)
    want, z = li.forward(x, W, save_z=True)
    torch.cuda.synchronize()
    calls = {
        "linear": lambda: li.forward(x, W, save_z=True, stream=s),
        "linear gradients": lambda: tuple(li.backward(x, W, want, z, stream=s).values())[:2],
        "decay": lambda: at.forward(q, q, q, rates, stream=s),
        "decay gradients": lambda: tuple(at.backward(q, q, q, q, rates, stream=s).values()),
        "norm": lambda: tuple(nm.forward(None, want, None, w, w, stream=s).values()),
        "norm gradients": lambda: (nm.backward(None, want, None, w, None, want, None, stream=s)["dy"],),
    }
    for name, call in calls.items():
        out = call()
        out = out if isinstance(out, tuple) else (out,)
        there = {t.data_ptr(): (t.shape, t.dtype) for t in out}
        del out
        mine = [torch.empty(shape, dtype=dtype, device="cuda") for shape, dtype in there.values()]
        assert not any(t.data_ptr() in there for t in mine), name
        del mine
    torch.cuda.synchronize()
    again = li.forward(x, W, stream=s)
    s.synchronize()
    assert torch.equal(again, want)
    del again
    # the workspace of a plan that is gone
    torch.cuda.synchronize()
    size, there = li.ws.numel(), li.ws.data_ptr()
    assert size > 11 << 20
    with torch.cuda.stream(s):
        torch.cuda._sleep(100_000_000)  # (some 50 ms of the stream's time)
    li.backward(x, W, want, z, stream=s)
    del li
    assert torch.empty(size, dtype=torch.uint8, device="cuda").data_ptr() != there
    torch.cuda.synchronize()
