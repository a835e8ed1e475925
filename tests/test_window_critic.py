"""The critic that looks back over a window: whole rollouts, single steps and gradients, on a stand-in of the library (CPU) and on the library (GPU), in fp32 and bf16."""
import math
import os
import sys

import pytest
import torch

import window_oracle as O
from paper_2107_01460_amd import memory
from window_stand_in import StandIn

T, ENVS, AGENTS, OBS, WINDOW, SINKS = 24, 6, 2, 27, 5, 2
ROUNDINGS = 12      # of an activation on its way through two layers, each 2^-8 of a value at most


@pytest.fixture(params=["stand-in", pytest.param("library", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "library":
        return "cuda"
    monkeypatch.setattr(memory, "B", StandIn)
    return "cpu"


def critic(device, dtype, monkeypatch=None):
    torch.manual_seed(7)
    made = memory.MemoryCritic(OBS, width=48, heads=4, kv_heads=2, layers=2, max_episode=60, dtype=dtype, device=device, window=WINDOW, sinks=SINKS)
    g = torch.Generator().manual_seed(5)
    with torch.no_grad():
        for p in made.parameters():
            p.copy_(torch.randn(p.shape, generator=g) / math.sqrt(p.shape[-1]) + (1.0 if p.dim() == 1 and p.shape[0] in (12, 48) else 0.0))
    return made


def rollout(device, dtype=torch.float32):
    g = torch.Generator().manual_seed(11)
    obs = torch.randn(T, ENVS * AGENTS, OBS, generator=g)
    done = (torch.rand(T, ENVS, generator=g) < 0.1).to(torch.uint8)
    ret = torch.randn(T, ENVS * AGENTS, generator=g)
    state = [torch.randn(2, ENVS * AGENTS, 2, SINKS + WINDOW, 12, generator=g).to(dtype) for _ in range(2)]
    positions = memory.episode_positions(done, torch.tensor([0, 3, 1, 0, 19, 7]))
    positions[-3:, 2] = -1        # a recording that ends early
    return obs.to(device), positions.to(device), [s.to(device) for s in state], ret.to(device)


def plain(c, params, obs, positions, state):
    """The critic's formulas in 64 bits, with gradients by torch."""
    p = lambda name: params[name]
    norm = lambda x, w, b: torch.nn.functional.layer_norm(x, (x.shape[-1],), w, b, 1e-5)
    lin = lambda x, name: x @ p(name + ".weight").t() + p(name + ".bias")
    at = positions.long().repeat_interleave(AGENTS, 1)
    H, Hk, D = c.heads, c.kv_heads, c.dim

    def turned(x, w):
        u = x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w
        return torch.where((at >= 0)[:, :, None, None], O._turn(u, c.table, at, D // 2 * 2, False, False), 0.0)
    x = lin(obs.double(), "embed")
    for l in range(len(c.layers)):
        m = f"layers.{l}."
        qkv = lin(norm(x, p(m + "norm_w"), p(m + "norm_b")), m + "qkv").unflatten(-1, (H + 2 * Hk, D))
        q, k, v = turned(qkv[:, :, :H], p(m + "q_norm")), turned(qkv[:, :, H:H + Hk], p(m + "k_norm")), qkv[:, :, H + Hk:]
        seen, K = O.columns(k, state[l][0], at, c.window, c.sinks)
        _, V = O.columns(v, state[l][1], at, c.window, c.sinks)
        K, V, seen = K.repeat_interleave(H // Hk, 1), V.repeat_interleave(H // Hk, 1), seen.permute(1, 0, 2)[:, None]
        score = torch.matmul(q.permute(1, 2, 0, 3), K.transpose(2, 3)) / math.sqrt(D)
        out = torch.matmul(torch.softmax(torch.where(seen, score, -1e300), -1) * seen, V).permute(2, 0, 1, 3)
        x = x + lin(out.flatten(-2), m + "out")
        x = x + lin(torch.nn.functional.gelu(lin(norm(x, p(m + "norm2_w"), p(m + "norm2_b")), m + "up")), m + "down")
    return lin(norm(x, p("norm_w"), p("norm_b")), "value").squeeze(-1)


def held(positions):
    """[T][B] rows that hold a step"""
    return (positions >= 0).repeat_interleave(AGENTS, 1)


def stepwise(c, obs, positions, state):
    s = [x.clone() for x in state]
    return torch.stack([c.step(obs[t], positions[t], s) for t in range(T)]), s


def test_values_and_gradients_against_plain_torch(device):
    c = critic(device, torch.float32)
    obs, positions, state, ret = rollout(device)
    ret = ret * held(positions)
    values, _ = c(obs, positions, None, state)
    (values * ret).sum().backward()
    params = {k: v.detach().double().requires_grad_() for k, v in c.named_parameters()}
    want = plain(c, params, obs, positions, state)
    (want * ret.double()).sum().backward()
    # fp32 throughout, some ten products and norms deep, each within a few 2^-24 of its scale: 1e-4 of the largest value leaves room for a hundred such steps
    on = held(positions)
    assert float((values - want).detach().abs()[on].max()) <= 1e-4 * float(want.detach().abs().max())
    for k, v in c.named_parameters():
        g = params[k].grad
        assert float((v.grad - g).abs().max()) <= 1e-4 * float(g.abs().max()) + 1e-7, k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_steps_agree_with_whole_rollouts(device, dtype):
    c = critic(device, dtype)
    obs, positions, state, _ = rollout(device, dtype)
    on = held(positions)
    with torch.no_grad():
        whole, after = c(obs, positions, None, state)
        steps, acted = stepwise(c, obs, positions, state)
        bound = (1e-4 if dtype == torch.float32 else ROUNDINGS * 2.0 ** -8) * float(whole[on].abs().max())
        far = lambda other: float((whole - other)[on].abs().max())
        assert far(steps) <= bound
        if dtype == torch.float32:   # mistakes pass the bound by
            assert far(stepwise(c, obs, positions, [torch.zeros_like(s) for s in state])[0]) > bound             # no state
            assert far(stepwise(c, obs, positions.clamp(max=0), state)[0]) > bound                                 # no positions
            c.sinks, c.window = SINKS - 1, WINDOW + 1                                                             # one first step less
            assert far(stepwise(c, obs, positions, state)[0]) > bound
            c.sinks, c.window = SINKS, WINDOW
        # in two calls, the state handed on
        first, between = c(obs[:9], positions[:9].contiguous(), None, state)
        second, _ = c(obs[9:], positions[9:].contiguous(), None, between)
        assert far(torch.cat([first, second])) <= bound


def test_gradients_in_bf16(monkeypatch, device):
    """Against 64 bits: no more than twice the stand-in's error, which rounds in the same places with other luck, and four roundings of the gradient."""
    def gradients(c, where):
        obs, positions, state, ret = rollout(where, torch.bfloat16)
        values, _ = c(obs, positions, None, state)
        (values * ret * held(positions)).sum().backward()
        return {k: p.grad.double().cpu() for k, p in c.named_parameters()}
    got = gradients(critic(device, torch.bfloat16), device)
    with monkeypatch.context() as m:
        m.setattr(memory, "B", StandIn)
        yardstick = gradients(critic("cpu", torch.bfloat16), "cpu")
        c = critic("cpu", torch.float32)
        obs, positions, state, ret = rollout("cpu", torch.bfloat16)
        params = {k: v.detach().double().requires_grad_() for k, v in c.named_parameters()}
        (plain(c, params, obs, positions, state) * ret.double() * held(positions)).sum().backward()
    for k, v in params.items():
        error = lambda a: float((a[k] - v.grad).norm())
        assert error(got) <= 2 * error(yardstick) + 4 * 2.0 ** -8 * float(v.grad.norm()) + 1e-12, k


def test_second_derivatives_are_refused(device):
    g = torch.Generator().manual_seed(3)
    new = lambda *s: torch.randn(s, generator=g).to(device).requires_grad_()
    q, k, v, w = new(5, 4, 4, 8), new(5, 4, 2, 8), new(5, 4, 2, 8), new(8)
    table = StandIn.rotary_table(9, 8).to(device)
    positions = torch.arange(5, dtype=torch.int32, device=device)[:, None].repeat(1, 2)
    for f, args in ((lambda: memory.AttendWindow.apply(q, k, v, None, positions, 3, 1, 0.5)[0], (q, k, v)),
                    (lambda: torch.cat([y.flatten() for y in memory.NormRotate.apply(q, k, w, w, table, positions, 1e-6)]), (q, k, w))):
        grads = torch.autograd.grad((f() ** 2).sum(), args, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            sum((x ** 2).sum() for x in grads).backward()


def test_gradients_and_inputs_of_any_strides(device):
    """An expanded or transposed gradient, an input whose last dimension is not contiguous: as with contiguous ones."""
    g = torch.Generator().manual_seed(4)
    new = lambda *s: torch.randn(s, generator=g).to(device)
    q, k, v, w = new(5, 4, 4, 8), new(5, 4, 2, 8), new(5, 4, 2, 8), new(8)
    table = StandIn.rotary_table(9, 8).to(device)
    positions = torch.arange(5, dtype=torch.int32, device=device)[:, None].repeat(1, 2)

    def gradients(f, args):
        args = [a.detach().requires_grad_() for a in args]
        out = f(*args)
        weight = torch.linspace(-1, 1, out.numel(), device=out.device).reshape(out.shape[::-1]).permute(*range(out.dim() - 1, -1, -1))
        return [out.detach(), *torch.autograd.grad(out.sum(), args, retain_graph=True), *torch.autograd.grad((out * weight).sum(), args)]
    for f, args in ((lambda q, k, v: memory.AttendWindow.apply(q, k, v, None, positions, 3, 1, 0.5)[0], (q, k, v)),
                    (lambda q, k, w: memory.NormRotate.apply(q, k, w, w, table, positions, 1e-6)[0], (q, k, w)),
                    (lambda q, k, w: memory.NormRotate.apply(q, k, w, w, table, positions, 1e-6)[1], (q, k, w))):
        plain = gradients(f, [a.clone() for a in args])
        for x, y in zip(plain, gradients(f, [a if a.dim() < 2 else a.transpose(0, -1).contiguous().transpose(0, -1) for a in args])):
            assert x.shape == y.shape and torch.equal(x, y)


def test_a_step_on_the_state_of_a_pending_gradient(device):
    """It writes into the state, which the gradient still needs."""
    c = critic(device, torch.float32)
    obs, positions, state, _ = rollout(device)
    values, _ = c(obs, positions, None, state)
    c.step(obs[0], positions[0], [s.clone() for s in state])
    values.sum().backward()
    if device == "cuda":   # (the stand-in's writes go past autograd)
        values, _ = c(obs, positions, None, state)
        c.step(obs[0], positions[0], state)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            values.sum().backward()


@pytest.mark.parametrize("steps,envs", [(0, 3), (4, 0)])
def test_no_steps_no_environments(device, steps, envs):
    if envs == 0 and device == "cpu":
        pytest.skip("the stand-in divides sequences among environments")
    c = memory.MemoryCritic(8, width=16, heads=2, layers=1, max_episode=20, device=device, window=4, sinks=1)
    state = [torch.rand_like(s) for s in c.initial_state(2 * envs)]
    values, after = c(torch.zeros((steps, 2 * envs, 8), device=device), torch.zeros((steps, envs), dtype=torch.int32, device=device), None, state)
    assert values.shape == (steps, 2 * envs) and all(a.shape == s.shape for a, s in zip(after, state))
    assert steps or all(torch.equal(a, s) for a, s in zip(after, state))
    values.sum().backward()
    assert all(p.grad is None or not p.grad.any() for p in c.parameters())


@pytest.mark.parametrize("window,sinks", [(0, 0), (-1, 2), (4, -1), (1 << 30, 1), (None, 1)])
def test_windows_that_are_refused(monkeypatch, window, sinks):
    monkeypatch.setattr(memory, "B", StandIn)
    with pytest.raises(StandIn.MarlError, match="window"):
        memory.MemoryCritic(8, width=16, heads=2, layers=1, device="cpu", window=window, sinks=sinks)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,bound", [(torch.float32, 1e-3), (torch.bfloat16, 0.25)], ids=["f32", "bf16"])
def test_example_runs(dtype, bound):
    """bf16: activations are rounded after every product, about twelve in a row, at 2^-8 each of values of order one."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import memory_critic
    first, last, difference = memory_critic.run(envs=64, steps=40, iterations=4, dtype=dtype, say=lambda s: print(s, flush=True), window=8, sinks=2)
    assert math.isfinite(first) and math.isfinite(last) and difference < bound
