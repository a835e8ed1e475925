"""MI355X-native fused multi-agent PPO training step (IPPO / MAPPO on a grid-foraging world).

Everything is computed by hand-written HIP kernels in libmarl_gfx950.so (C ABI in include/marl.h);
this package only marshals arguments.  PyTorch is used for device memory and streams.
"""
from . import binding  # noqa: F401
from .binding import (  # noqa: F401
    Config, EnvState, Traj, MarlError, lib, make_config, query_sizes, env_reset, observe, env_step,
    policy_forward, sample_actions, rollout, rollout_static, compute_gae, ppo_update, status_string, alloc_workspace,
    timing_enable, timing_read, KERNEL_CLASSES, EvalStats, evaluate, RecState, rollout_recurrent, ppo_update_recurrent, train_step, alloc_counters,
    linear_attention, linear_attention_backward, linear_attention_step, linear_attention_workspace, layer_norm, layer_norm_backward,
    layer_norm_workspace, rotary, rotary_table,
)
from .trainer import Trainer  # noqa: F401,E402
from .memory import MemoryCritic, episode_positions  # noqa: F401,E402
