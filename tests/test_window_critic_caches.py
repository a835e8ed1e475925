"""A window's state whose keys and values do not begin at the sixteen bytes that the library asks of a cache, for any width of heads and number of sequences: on a
stand-in that asks the same (CPU) and on the library (GPU)."""
import pytest
import torch

from paper_2107_01460_amd import memory
from window_stand_in import StandIn

F32, BF16 = torch.float32, torch.bfloat16


def _aligned(cache):
    for x in cache or ():
        if x.data_ptr() % 16 or not x.is_contiguous():
            raise StandIn.MarlError("marl error -2: a cache lies at sixteen bytes")


class Strict(StandIn):
    """The stand-in with the library's demands of a cache"""

    @staticmethod
    def window_attention(*a, cache=None, next_cache=None, **kw):
        _aligned(cache)
        _aligned(next_cache)
        StandIn.window_attention(*a, cache=cache, next_cache=next_cache, **kw)

    @staticmethod
    def window_attention_backward(*a, cache=None, **kw):
        _aligned(cache)
        StandIn.window_attention_backward(*a, cache=cache, **kw)

    @staticmethod
    def window_attention_step(q, k, v, cache, *a, **kw):
        _aligned(cache)
        StandIn.window_attention_step(q, k, v, cache, *a, **kw)


@pytest.fixture(params=["stand-in", pytest.param("library", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "library":
        return "cuda"
    monkeypatch.setattr(memory, "B", Strict)
    return "cpu"


def made(device, dtype, dim, window, sinks, heads=2, kv_heads=1):
    torch.manual_seed(3)
    c = memory.MemoryCritic(6, width=heads * dim, heads=heads, kv_heads=kv_heads, layers=2, max_episode=40, dtype=dtype, device=device, window=window, sinks=sinks)
    g = torch.Generator().manual_seed(5)
    with torch.no_grad():
        for p in c.parameters():
            p.copy_(torch.randn(p.shape, generator=g) / p.shape[-1] ** 0.5)
    return c


def placed(x, offset):
    """The same values, `offset` elements into memory of their own"""
    flat = torch.zeros(x.numel() + 64, dtype=x.dtype, device=x.device)
    y = flat[offset: offset + x.numel()].view(x.shape)
    y.copy_(x)
    return y


# (dtype, head width, window, first steps, sequences): halves that begin 2 to 14 bytes behind sixteen, and one that does not
CASES = [(BF16, 12, 4, 1, 1), (BF16, 7, 5, 0, 1), (BF16, 9, 3, 0, 3), (BF16, 2, 1, 0, 1), (F32, 5, 3, 2, 1), (F32, 7, 3, 0, 1), (F32, 2, 1, 0, 3), (F32, 8, 4, 1, 2)]


@pytest.mark.parametrize("dtype,dim,window,sinks,B", CASES)
def test_rollouts_gradients_and_steps(device, dtype, dim, window, sinks, B):
    """From the critic's own state, from copies of it and from slices of a larger one: the same results, bit for bit."""
    c, T = made(device, dtype, dim, window, sinks), 9
    g = torch.Generator().manual_seed(1)
    obs = torch.randn(T, B, 6, generator=g).to(device)
    start = torch.arange(T, dtype=torch.int32, device=device)[:, None].repeat(1, B)
    on = start + T
    values, state = c(obs, start, None, c.initial_state(B))       # the critic's own state, whose contents the rollout gives
    assert all(s.shape == i.shape == (2, B, 1, sinks + window, dim) for s, i in zip(state, c.initial_state(B)))
    wide = [torch.cat([s[:, :1], s], 1)[:, 1:] for s in state]    # a slice behind another sequence's
    results = []
    for made_of in (lambda s: s, lambda s: s.clone(), lambda s: s.contiguous(), lambda s: placed(s, 1), lambda s: placed(s, 16 // s.element_size()), None):
        own = [x if made_of is None else made_of(x) for x in (wide if made_of is None else state)]
        before = [x.clone() for x in own]
        c.zero_grad()
        whole, after = c(obs, on, None, own)
        whole.sum().backward()
        assert all(torch.equal(x, y) for x, y in zip(own, before))                    # a rollout leaves its state alone
        acting = [x.clone() for x in own] if made_of is None else [made_of(x.clone()) for x in own]
        steps = torch.stack([c.step(obs[t], on[t], acting) for t in range(T)])
        results.append([whole.detach(), *after, *acting, steps, *[p.grad.clone() for p in c.parameters()]])
        bound = (1e-4 if dtype == F32 else 12 * 2.0 ** -8) * max(float(whole.detach().abs().max()), 1.0)      # some twelve roundings of an activation one after another
        assert float((steps - whole.detach()).abs().max()) <= bound
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))


def test_a_step_writes_into_the_state_that_it_was_given(device):
    c = made(device, BF16, 12, 4, 1)
    state = [torch.zeros(2, 1, 1, 5, 12, dtype=BF16, device=device) for _ in range(2)]     # halves 120 bytes apart
    c.step(torch.ones(1, 6, device=device), torch.zeros(1, dtype=torch.int32, device=device), state)
    for s in state:
        assert s[:, :, :, 0].any(dim=-1).all() and not s[:, :, :, 1:].any()
