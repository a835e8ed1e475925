"""A critic with a memory, fitted to the returns of rollouts, then used step by step as an acting loop would.

    python examples/memory_critic.py [--envs 256] [--steps 64] [--iterations 30] [--bf16]

Environments are rolled out by the library (random-initialised policy), advantages and returns come from marl_compute_gae; the critic learns the
returns from whole rollouts (linear attention, rotary positions and layer norms with their gradients) and then values the same rollout one
step at a time from its states.
"""
import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch

import paper_2107_01460_amd as M
import workloads as W
from paper_2107_01460_amd.trainer import init_params


def run(envs=256, steps=64, iterations=30, dtype=torch.float32, seed=0, say=print):
    """(loss of the first iteration, of the last, largest difference between whole and stepwise values)"""
    cfg = W.scaled(W.CONFIGS[1], n_envs=envs, rollout_len=steps, n_minibatches=1)
    sizes = M.query_sizes(cfg)
    state, traj = M.EnvState(cfg), M.Traj(cfg)
    params, ws = init_params(cfg, seed).cuda(), M.alloc_workspace(sizes.rollout_workspace_bytes)
    M.env_reset(cfg, state)
    torch.manual_seed(seed)
    critic = M.MemoryCritic(sizes.obs_dim, width=128, heads=4, kv_heads=2, max_episode=cfg["episode_cap"], dtype=dtype)
    optimiser = torch.optim.Adam(critic.parameters(), lr=1e-3)
    memory = critic.initial_state(envs * cfg["n_agents"])
    losses = []
    for it in range(iterations):
        first = state.t_in_ep.clone()
        before = [s.clone() for s in memory]
        M.rollout(cfg, state, params, traj, it * steps, ws)
        M.compute_gae(cfg, traj)
        obs = traj.obs[:steps].flatten(1, 2)
        positions = M.episode_positions(traj.done, first)
        values, memory = critic(obs, positions, traj.done, before)
        memory = [s.detach() for s in memory]   # the next rollout goes on from here
        loss = (values - traj.ret.flatten(1)).square().mean()
        optimiser.zero_grad()
        loss.backward()
        optimiser.step()
        losses.append(loss.detach())
        if it % 10 == 0 or it == iterations - 1:
            say(f"iteration {it}: mean squared error {losses[-1].item():.5f}")
    # the last rollout again, with the fitted critic: whole, and one step after another
    with torch.no_grad():
        whole, after = critic(obs, positions, traj.done, before)
    acting = [s.clone() for s in before]
    stepwise = torch.stack([critic.step(obs[t], positions[t], acting, traj.done[t - 1] if t else None) for t in range(steps)])
    difference = float((whole - stepwise).abs().max())
    say(f"values of whole rollouts and of single steps differ by {difference:.2e} at most")
    return losses[0].item(), losses[-1].item(), difference


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--envs", type=int, default=256)
    p.add_argument("--steps", type=int, default=64)
    p.add_argument("--iterations", type=int, default=30)
    p.add_argument("--bf16", action="store_true")
    a = p.parse_args()
    run(a.envs, a.steps, a.iterations, torch.bfloat16 if a.bf16 else torch.float32)
