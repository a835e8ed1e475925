"""Rollouts of no steps and of no environments through the critic with a memory."""
import pytest
import torch

from paper_2107_01460_amd import memory
from memory_stand_in import StandIn


def test_positions_of_no_steps():
    for T, n in ((0, 3), (0, 0), (4, 0)):
        at = memory.episode_positions(torch.zeros((T, n), dtype=torch.uint8), torch.arange(n))
        assert at.shape == (T, n) and at.dtype == torch.int32


@pytest.fixture(params=["stand-in", pytest.param("library", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "library":
        return "cuda"
    monkeypatch.setattr(memory, "B", StandIn)
    return "cpu"


@pytest.mark.parametrize("T,envs", [(0, 3), (4, 0)])
def test_critic(device, T, envs):
    if envs == 0 and device == "cpu":
        pytest.skip("the stand-in divides sequences among environments")
    c = memory.MemoryCritic(8, width=16, heads=2, layers=1, max_episode=20, device=device)
    done = torch.zeros((T, envs), dtype=torch.uint8, device=device)
    state = [torch.rand_like(s) for s in c.initial_state(2 * envs)]
    values, after = c(torch.zeros((T, 2 * envs, 8), device=device), memory.episode_positions(done, torch.zeros(envs, device=device)), done, state)
    assert values.shape == (T, 2 * envs) and all(torch.equal(a, s) for a, s in zip(after, state))
    values.sum().backward()
    assert all(p.grad is None or not p.grad.any() for p in c.parameters())
