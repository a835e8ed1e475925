"""The autograd functions of the sequence operators: what they refuse and what they take, on a stand-in of the library (CPU) and on the library (GPU)."""
import pytest
import torch

from paper_2107_01460_amd import memory
from memory_stand_in import StandIn


@pytest.fixture(params=["stand-in", pytest.param("library", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "library":
        return "cuda"
    monkeypatch.setattr(memory, "B", StandIn)
    return "cpu"


def inputs(device, T=5, B=4, H=4, Hk=2, D=8):
    g = torch.Generator().manual_seed(3)
    new = lambda *s: torch.randn(s, generator=g).to(device)
    return new(T, B, H, D), new(T, B, Hk, D), new(T, B, Hk, D), torch.linspace(0.7, 0.99, H).to(device)


def functions(device):
    """(name, call on the tensors that it differentiates, those tensors)"""
    q, k, v, decay = inputs(device)
    table = StandIn.rotary_table(9, 8).to(device)
    positions = torch.arange(5, dtype=torch.int32, device=device)[:, None].repeat(1, 2)
    w, b = torch.rand(8, device=device) + 0.5, torch.rand(8, device=device)
    return [("attention", lambda q, k, v: memory.Attend.apply(q, k, v, decay, None, None, 0.5)[0], (q, k, v)),
            ("norm", lambda x, w, b: memory.LayerNorm.apply(x, w, b, 1e-5), (q, w, b)),
            ("rotation", lambda q, k: torch.cat([y.flatten() for y in memory.Rotate.apply(q, k, table, positions)]), (q, k))]


def test_second_derivatives_are_refused(device):
    """They would need gradients of the gradients' kernels; without an error their terms would be missing."""
    for name, f, args in functions(device):
        args = [a.requires_grad_() for a in args]
        out = f(*args)
        grads = torch.autograd.grad((out ** 2).sum(), args, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            sum((g ** 2).sum() for g in grads).backward()
