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
