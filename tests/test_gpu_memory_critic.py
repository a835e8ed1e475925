"""The critic with a memory: whole rollouts against single steps and against a plain torch model in 64 bits, and the example that trains one."""
import math
import os
import sys

import pytest
import torch

import memory_oracle as O


def test_positions_in_episodes():
    from paper_2107_01460_amd.memory import episode_positions
    done = torch.tensor([[0, 1, 0], [0, 0, 1], [1, 0, 1], [0, 0, 0]], dtype=torch.uint8)
    first = torch.tensor([5, 0, 3])
    want = torch.tensor([[5, 0, 3], [6, 0, 4], [7, 1, 0], [0, 2, 0]], dtype=torch.int32)
    assert torch.equal(episode_positions(done, first), want)
    assert torch.equal(episode_positions(done[:1], first), want[:1])


def plain(c, params, obs, positions, done, state):
    """The critic's formulas in 64 bits, with gradients by torch."""
    norm = lambda x, w, b: torch.nn.functional.layer_norm(x, (x.shape[-1],), w, b, 1e-5)
    p = lambda name: params[name]
    lin = lambda x, name: x @ p(name + ".weight").t() + p(name + ".bias")
    T, n, H, Hk, D = obs.shape[0], obs.shape[1], c.heads, c.kv_heads, c.dim
    agents = n // done.shape[1]
    at = c.table.double()[positions.long().repeat_interleave(agents, 1)][:, :, None]
    cos, sin = at[..., :D // 2], at[..., D // 2:]
    turn = lambda x: torch.cat([x[..., :D // 2] * cos - x[..., D // 2:] * sin, x[..., :D // 2] * sin + x[..., D // 2:] * cos], -1)
    alive = 1 - done.double().repeat_interleave(agents, 1)
    x = lin(obs.double(), "embed")
    for l in range(len(c.layers)):
        m = f"layers.{l}."
        qkv = lin(norm(x, p(m + "norm_w"), p(m + "norm_b")), m + "qkv").unflatten(-1, (H + 2 * Hk, D))
        q, k, v = turn(qkv[:, :, :H]), turn(qkv[:, :, H:H + Hk]), qkv[:, :, H + Hk:]
        k, v = k.repeat_interleave(H // Hk, 2), v.repeat_interleave(H // Hk, 2)
        S, out = state[l].double(), []
        for t in range(T):
            S = c.decay.double()[None, :, None, None] * S + k[t][..., None] * v[t][:, :, None]
            out.append((q[t][..., None] * S).sum(2) / math.sqrt(D))
            S = S * alive[t][:, None, None, None]
        x = x + lin(norm(torch.stack(out), None, None).flatten(-2), m + "out")
        x = x + lin(torch.nn.functional.gelu(lin(norm(x, p(m + "norm2_w"), p(m + "norm2_b")), m + "up")), m + "down")
    return lin(norm(x, p("norm_w"), p("norm_b")), "value").squeeze(-1)


@pytest.mark.gpu
def test_values_and_gradients_against_plain_torch():
    import paper_2107_01460_amd as M
    torch.manual_seed(1)
    c = M.MemoryCritic(27, width=48, heads=4, kv_heads=2, layers=2, max_episode=30)
    T, envs, agents = 21, 5, 2
    obs, ret = torch.randn(T, envs * agents, 27, device="cuda"), torch.randn(T, envs * agents, device="cuda")
    done = (torch.rand(T, envs, device="cuda") < 0.1).to(torch.uint8)
    positions = M.episode_positions(done, torch.tensor([0, 3, 1, 0, 9], device="cuda"))
    state = [torch.randn_like(s) for s in c.initial_state(envs * agents)]
    values, _ = c(obs, positions, done, state)
    (values * ret).sum().backward()
    params = {k: v.detach().double().requires_grad_() for k, v in c.named_parameters()}
    want = plain(c, params, obs, positions, done, state)
    (want * ret.double()).sum().backward()
    # fp32 throughout, some ten products and norms deep: each within a few 2^-24 of its scale, a norm of a head's small output (widths of 12) up to ten
    # times that; 1e-4 of the tensor's largest value leaves room for twenty such steps
    assert float((values - want).abs().max()) <= 1e-4 * float(want.abs().max())
    for k, v in c.named_parameters():
        g = params[k].grad
        assert float((v.grad - g).abs().max()) <= 1e-4 * float(g.abs().max()) + 1e-7, k


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,bound", [(torch.float32, 1e-3), (torch.bfloat16, 0.25)], ids=["f32", "bf16"])
def test_example_learns_and_steps_agree(dtype, bound):
    """bf16: activations are rounded after every product, about twelve in a row, at 2^-8 each of values of order one."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import memory_critic
    first, last, difference = memory_critic.run(envs=64, steps=40, iterations=25, dtype=dtype, say=lambda s: print(s, flush=True))
    assert last < 0.8 * first and difference < bound
