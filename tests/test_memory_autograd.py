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


def gradients(f, args, layout):
    """Of a sum (its gradient is an expanded number) or of a product with a transposed tensor, at inputs laid out as asked."""
    args = [layout(a.detach()).requires_grad_() for a in args]
    out = f(*args)
    weight = torch.linspace(-1, 1, out.numel(), device=out.device).reshape(out.shape[::-1]).permute(*range(out.dim() - 1, -1, -1))
    both = torch.autograd.grad(out.sum(), args, retain_graph=True) + torch.autograd.grad((out * weight).sum(), args)
    return [out.detach(), *both]


def test_gradients_and_inputs_of_any_strides(device):
    """An expanded or transposed gradient, an input whose last dimension is not contiguous: as with contiguous ones."""
    cases = functions(device)
    cases.append(("norm of a matrix", lambda x, w, b: memory.LayerNorm.apply(x, w, b, 1e-5), (torch.randn(7, 8, device=device), *cases[1][2][1:])))
    q, k = cases[2][2]
    table, positions = StandIn.rotary_table(9, 8).to(device), torch.zeros((5, 2), dtype=torch.int32, device=device)
    cases.append(("rotation of queries", lambda q, k: memory.Rotate.apply(q, k, table, positions)[0], (q, k)))

    decay, state = inputs(device)[3], torch.randn(4, 4, 8, 8, device=device)
    cases.append(("attention from a state", lambda q, k, v, s: memory.Attend.apply(q, k, v, decay, s, None, 0.5)[1], (*cases[0][2], state)))

    def turned(x):   # the same values, the last dimension not contiguous
        return x if x.dim() < 2 else x.transpose(0, -1).contiguous().transpose(0, -1)
    for name, f, args in cases:
        plain = gradients(f, args, lambda x: x.clone())
        for x, y in zip(plain, gradients(f, args, turned)):
            assert x.shape == y.shape and torch.equal(x, y), name
        want = gradients(f, [a.double() for a in args], lambda x: x.clone()) if device == "cpu" else None
        for x, y in zip(plain, want or plain):
            assert float((x - y).abs().max()) <= 1e-5 * float(y.abs().max()) + 1e-6, name


def test_rows_of_the_norm_that_are_expanded(device):
    """One row for all: x is read in place, its gradient is the sum."""
    x = torch.randn(1, 8, device=device).requires_grad_()
    out = memory.LayerNorm.apply(x.expand(6, 8), None, None, 1e-5)
    weight = torch.randn(6, 8, device=device)
    got, = torch.autograd.grad((out * weight).sum(), x)
    want, = torch.autograd.grad((torch.nn.functional.layer_norm(x.expand(6, 8), (8,)) * weight).sum(), x)
    # values of order one, sums of eight and six of them: 1e-5 leaves room for a hundred roundings of 2^-24
    assert float((got - want).abs().max()) <= 1e-5 * float(want.abs().max()) + 1e-5
