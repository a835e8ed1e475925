"""A critic with a memory on top of the sequence operators: what an agent saw earlier in its episode counts for the value of a step.

The memory is linear attention with a decay for each head, on queries and keys turned by rotary positions (the step in the episode), between
layer norms.  It has two forms with the same parameters: ``forward`` takes whole rollouts, [T][B][D] observations with the done flags of a
trajectory, and has gradients; ``step`` takes one step of every sequence and a state of constant size, as an acting loop does.  The norms, the
rotation and the attention run in the library's kernels; the projections between them are plain products of torch.  The kernels have first derivatives;
asking for a second raises.

B sequences are the agents of all environments, an environment's side by side, as in the trajectory arrays.
"""
import math

import torch
from torch.autograd.function import once_differentiable

from . import binding as B


def _rows(x):
    """x with its last dimension contiguous, as the kernels read it: x itself but for transposed tensors and expanded numbers."""
    return x if x.shape[-1] <= 1 or x.stride(-1) == 1 else x.contiguous()


class Attend(torch.autograd.Function):
    """(out, next_state) = linear attention of q, k, v [T][B][heads][D]; gradients of q, k, v and the state."""

    @staticmethod
    def forward(ctx, q, k, v, decay, state, done, scale):
        q, k, v, state = _rows(q), _rows(k), _rows(v), None if state is None else state.contiguous()
        T, n, H, Dk = q.shape
        out = torch.empty((T, n, H, v.shape[3]), dtype=q.dtype, device=q.device)
        next_state = torch.empty((n, H, Dk, v.shape[3]), dtype=torch.float32, device=q.device)
        B.linear_attention(q, k, v, decay, out, B.alloc_workspace(B.linear_attention_workspace(q, k, v)), state=state, next_state=next_state, done=done,
                           scale=scale)
        ctx.save_for_backward(q, k, v, decay, state, done)
        ctx.scale = scale
        return out, next_state

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, dnext_state):
        q, k, v, decay, state, done = ctx.saved_tensors
        dq, dk, dv = (torch.empty_like(x, memory_format=torch.contiguous_format) for x in (q, k, v))
        dstate = None if state is None else torch.empty_like(state)
        B.linear_attention_backward(q, k, v, decay, dout.contiguous(), dq, dk, dv, B.alloc_workspace(B.linear_attention_workspace(q, k, v, backward=True)),
                                    state=state, dnext_state=dnext_state.contiguous(), dstate=dstate, done=done, scale=ctx.scale)
        return dq, dk, dv, None, dstate, None, None


class LayerNorm(torch.autograd.Function):
    """Layer norm over the last dimension; weight and bias may be None."""

    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        rows = _rows(x.reshape(-1, x.shape[-1]))
        out = torch.empty_like(rows)
        mean, rstd = (torch.empty(rows.shape[0], dtype=torch.float32, device=x.device) for _ in range(2))
        B.layer_norm(rows, weight, bias, out, mean, rstd, eps)
        ctx.save_for_backward(rows, weight, mean, rstd)
        ctx.has_bias = bias is not None
        return out.reshape(x.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        rows, weight, mean, rstd = ctx.saved_tensors
        dx = torch.empty_like(rows)
        dw = None if weight is None else torch.empty_like(weight)
        db = torch.empty(rows.shape[1], dtype=torch.float32, device=rows.device) if ctx.has_bias else None
        B.layer_norm_backward(_rows(dout.reshape(rows.shape)), rows, weight, mean, rstd, dx, dw, db, B.alloc_workspace(B.layer_norm_workspace(*rows.shape)))
        return dx.reshape(dout.shape), dw, db, None


class Rotate(torch.autograd.Function):
    """Rotary positions on q and k [T][B][heads][D]; the gradient turns back."""

    @staticmethod
    def forward(ctx, q, k, table, positions):
        ctx.save_for_backward(table, positions)
        q_out, k_out = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k))
        B.rotary(_rows(q), _rows(k), table, q_out, k_out, positions=positions)
        return q_out, k_out

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        table, positions = ctx.saved_tensors
        q_out, k_out = torch.empty_like(dq, memory_format=torch.contiguous_format), torch.empty_like(dk, memory_format=torch.contiguous_format)
        B.rotary(_rows(dq), _rows(dk), table, q_out, k_out, positions=positions, inverse=True)
        return q_out, k_out, None, None


def episode_positions(done, first):
    """[T][N] int32 step in its episode of every step of a rollout: `first` [N] at step 0, 0 behind a step whose done is nonzero."""
    T = done.shape[0]
    t = torch.arange(T, device=done.device, dtype=torch.int64)[:, None]
    starts = torch.zeros((T, done.shape[1]), dtype=torch.int64, device=done.device)   # the last step that began an episode, -first before any did
    if T == 0:
        return starts.int()
    starts[0] = -first.long()
    starts[1:] = torch.where(done[:-1] != 0, t[1:], starts[0])
    return (t - starts.cummax(0).values).int()


class MemoryCritic(torch.nn.Module):
    """Value of every step from the steps of its episode up to it.

    width: of the residual stream (a multiple of heads).  horizon: the heads' decays are 1 - 1 / h with h from 4 to it, in equal ratios."""

    def __init__(self, obs_dim, width=64, heads=4, kv_heads=None, layers=2, max_episode=1024, horizon=256, dtype=torch.float32, device="cuda"):
        super().__init__()
        kv_heads = heads if kv_heads is None else kv_heads
        if width % heads or heads % kv_heads:
            raise B.MarlError("width is a multiple of heads, heads of kv_heads")
        if not 2 <= width // heads <= 128:
            raise B.MarlError(f"heads of {width // heads}: 2 to 128")
        device = torch.device(device)
        if device.type == "cuda" and device.index not in (None, torch.cuda.current_device()):
            raise B.MarlError(f"{device} is not the current GPU, where the kernels run (torch.cuda.set_device)")
        self.heads, self.kv_heads, self.dim, self.dtype = heads, kv_heads, width // heads, dtype
        h = 4.0 * (horizon / 4.0) ** (torch.arange(heads, dtype=torch.float64) / max(heads - 1, 1))
        self.register_buffer("decay", (1 - 1 / h).float().to(device))
        self.register_buffer("table", B.rotary_table(max_episode + 1, self.dim // 2 * 2))
        lin = lambda i, o: torch.nn.Linear(i, o, device=device)
        ones = lambda: torch.nn.Parameter(torch.ones(width, device=device))
        zeros = lambda: torch.nn.Parameter(torch.zeros(width, device=device))
        self.embed = lin(obs_dim, width)
        self.layers = torch.nn.ModuleList()
        for _ in range(layers):
            m = torch.nn.Module()
            m.norm_w, m.norm_b, m.norm2_w, m.norm2_b = ones(), zeros(), ones(), zeros()
            m.qkv = lin(width, (heads + 2 * kv_heads) * self.dim)
            m.out, m.up, m.down = lin(width, width), lin(width, 2 * width), lin(2 * width, width)
            self.layers.append(m)
        self.norm_w, self.norm_b = ones(), zeros()
        self.value = lin(width, 1)

    def _product(self, layer, x):
        return torch.nn.functional.linear(x, layer.weight.to(self.dtype), layer.bias.to(self.dtype))

    def initial_state(self, sequences):
        """One state per layer, all zero."""
        shape = (sequences, self.heads, self.dim, self.dim)
        return [torch.zeros(shape, dtype=torch.float32, device=self.decay.device) for _ in self.layers]

    def _heads(self, m, y):
        """q, k, v as views of one product's columns."""
        qkv = self._product(m.qkv, y)
        qkv = qkv.unflatten(-1, (self.heads + 2 * self.kv_heads, self.dim))
        return qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=-2)

    def _rest(self, m, x, out):
        """Behind the memory: each head normed by itself, then the layer's own two products."""
        out = LayerNorm.apply(out, None, None, 1e-5).flatten(-2)
        x = x + self._product(m.out, out)
        y = LayerNorm.apply(x, m.norm2_w, m.norm2_b, 1e-5)
        return x + self._product(m.down, torch.nn.functional.gelu(self._product(m.up, y)))

    def forward(self, obs, positions, done=None, state=None):
        """Values [T][B] fp32 and the states behind the last step, from obs [T][B][D], positions and done [T][environments]."""
        x = self._product(self.embed, obs.to(self.dtype))
        after = []
        for n, m in enumerate(self.layers):
            q, k, v = self._heads(m, LayerNorm.apply(x, m.norm_w, m.norm_b, 1e-5))
            q, k = Rotate.apply(q, k, self.table, positions)
            out, s = Attend.apply(q, k, v, self.decay, None if state is None else state[n], done, 1 / math.sqrt(self.dim))
            after.append(s)
            x = self._rest(m, x, out)
        return self._product(self.value, LayerNorm.apply(x, self.norm_w, self.norm_b, 1e-5)).squeeze(-1).float(), after

    @torch.no_grad()
    def step(self, obs, positions, state, done=None):
        """Values [B] of one step, obs [B][D]; the states are updated in place.  positions [environments]; done: of the step before."""
        x = self._product(self.embed, obs.to(self.dtype))
        for n, m in enumerate(self.layers):
            q, k, v = self._heads(m, LayerNorm.apply(x, m.norm_w, m.norm_b, 1e-5))
            q, k = Rotate.apply(q[None], k[None], self.table, positions[None])
            out = torch.empty((*q.shape[1:3], self.dim), dtype=self.dtype, device=x.device)
            B.linear_attention_step(q[0], k[0], v, self.decay, state[n], out, done=done, scale=1 / math.sqrt(self.dim))
            x = self._rest(m, x, out)
        return self._product(self.value, LayerNorm.apply(x, self.norm_w, self.norm_b, 1e-5)).squeeze(-1).float()
