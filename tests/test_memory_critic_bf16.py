"""The critic with a memory in bf16: single steps against whole rollouts, and its gradients.  The bounds come from bf16's rounding alone, and mistakes planted in
a stand-in of the library on the CPU pass them by, so that a test here that passes says something."""
import pytest
import torch

from paper_2107_01460_amd import memory
from memory_stand_in import StandIn
from test_gpu_memory_critic import plain

T, ENVS, AGENTS, OBS = 24, 6, 2, 27
ROUNDINGS = 12      # of an activation on its way through two layers, each 2^-8 of a value at most


def critic(device, dtype):
    torch.manual_seed(7)
    made = memory.MemoryCritic(OBS, width=48, heads=4, kv_heads=2, layers=2, max_episode=40, dtype=dtype, device="cpu")
    return made.to(device)


def rollout(device):
    g = torch.Generator().manual_seed(11)
    obs = torch.randn(T, ENVS * AGENTS, OBS, generator=g)
    done = (torch.rand(T, ENVS, generator=g) < 0.1).to(torch.uint8)
    done[7, 0] = done[11, 1] = 1
    ret = torch.randn(T, ENVS * AGENTS, generator=g)
    state = [torch.randn(ENVS * AGENTS, 4, 12, 12, generator=g) for _ in range(2)]
    positions = memory.episode_positions(done, torch.tensor([0, 3, 1, 0, 9, 2]))
    return obs.to(device), positions.to(device), done.to(device), [s.to(device) for s in state], ret.to(device)


def stepwise(c, obs, positions, done, state):
    s = [x.clone() for x in state]
    return torch.stack([c.step(obs[t], positions[t], s, done[t - 1] if t else None) for t in range(T)])


def bound_of_values(values):
    return ROUNDINGS * 2.0 ** -8 * float(values.abs().max())


def gradients(c, obs, positions, done, state, ret):
    values, _ = c(obs, positions, done, state)
    (values * ret).sum().backward()
    return {k: p.grad.double().cpu() for k, p in c.named_parameters()}


def reference():
    """Gradients in 64 bits"""
    c = critic("cpu", torch.float32)
    obs, positions, done, state, ret = rollout("cpu")
    params = {k: v.detach().double().requires_grad_() for k, v in c.named_parameters()}
    (plain(c, params, obs, positions, done, state) * ret.double()).sum().backward()
    return {k: v.grad for k, v in params.items()}


def excess(got, want, yardstick):
    """Largest error of a parameter's gradient, in units of what is allowed: twice the error of the stand-in, which rounds in the same places with other
    luck, and four roundings of the gradient itself.  (What the state in front of the first step contributes is less than that.)"""
    error = lambda a, k: float((a[k] - want[k]).norm())
    return max(error(got, k) / (2 * error(yardstick, k) + 4 * 2.0 ** -8 * float(want[k].norm()) + 1e-12) for k in want)


# ---- on the stand-in: what is right passes, what is wrong does not ------------------------------------------------------------
@pytest.fixture
def stand_in(monkeypatch):
    monkeypatch.setattr(memory, "B", StandIn)


def test_bounds_tell_mistakes_in_values(stand_in):
    obs, positions, done, state, _ = rollout("cpu")
    c = critic("cpu", torch.bfloat16)
    with torch.no_grad():
        whole = c(obs, positions, done, state)[0]
        bound = bound_of_values(whole)
        far = lambda other: float((whole - other).abs().max())
        assert far(stepwise(c, obs, positions, done, state)) <= bound
        assert far(stepwise(c, obs, positions, done, [torch.zeros_like(s) for s in state])) > bound              # no state
        assert far(stepwise(c, obs, positions, torch.zeros_like(done), state)) > bound                              # no flags
        assert far(stepwise(c, obs, torch.zeros_like(positions), done, state)) > bound                              # no positions
        assert far(torch.stack([c.step(obs[t], positions[t], [s.clone() for s in state], done[t - 1] if t else None) for t in range(T)])) > bound  # a state that stays
        for h in range(4):                                                                                          # one head's decay
            right = float(c.decay[h])
            c.decay[h] = right + (0.15 if right < 0.8 else -0.15)
            assert far(stepwise(c, obs, positions, done, state)) > bound, h
            c.decay[h] = right


def test_bounds_tell_mistakes_in_gradients(stand_in, monkeypatch):
    want = reference()
    yardstick = gradients(critic("cpu", torch.bfloat16), *rollout("cpu"))

    def wrong(change):
        class Wrong(StandIn):
            @staticmethod
            def linear_attention_backward(*a, **kw):
                StandIn.linear_attention_backward(*a, **change(kw))
        monkeypatch.setattr(memory, "B", Wrong)
        return excess(gradients(critic("cpu", torch.bfloat16), *rollout("cpu")), want, yardstick)
    assert wrong(lambda kw: kw) <= 1.0
    assert wrong(lambda kw: {**kw, "done": None}) > 1.0
    assert wrong(lambda kw: {**kw, "scale": 1.25 * kw["scale"]}) > 1.0


# ---- on the library -----------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
def test_steps_agree_with_whole_rollouts():
    obs, positions, done, state, _ = rollout("cuda")
    c = critic("cuda", torch.bfloat16)
    with torch.no_grad():
        whole = c(obs, positions, done, state)[0]
        difference = float((whole - stepwise(c, obs, positions, done, state)).abs().max())
    assert difference <= bound_of_values(whole), difference


@pytest.mark.gpu
def test_gradients(monkeypatch):
    want = reference_on_the_stand_in(monkeypatch, reference)
    yardstick = reference_on_the_stand_in(monkeypatch, lambda: gradients(critic("cpu", torch.bfloat16), *rollout("cpu")))
    got = gradients(critic("cuda", torch.bfloat16), *rollout("cuda"))
    assert excess(got, want, yardstick) <= 1.0


def reference_on_the_stand_in(monkeypatch, f):
    with monkeypatch.context() as m:
        m.setattr(memory, "B", StandIn)
        return f()
