"""A critic with a memory on top of the sequence operators: what an agent saw earlier in its episode counts for the value of a step.

The memory is linear attention with a decay for each head, on queries and keys turned by rotary positions (the step in the episode), between
layer norms; or, with ``window``, attention over the last steps of the episode and its first ones, on queries and keys normed by head and turned.  It has two
forms with the same parameters: ``forward`` takes whole rollouts, [T][B][D] observations with the done flags of a
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


class NormRotate(torch.autograd.Function):
    """Each head of q and k [T][B][heads][D] normed by the root of its mean square, weighted, and turned by its position."""

    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, table, positions, eps):
        q, k = _rows(q), _rows(k)
        q_out, k_out = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k))
        B.norm_rotary(q, k, q_weight, k_weight, table, q_out, k_out, eps=eps, positions=positions)
        ctx.save_for_backward(q, k, q_weight, k_weight, table, positions)
        ctx.eps = eps
        return q_out, k_out

    @staticmethod
    @once_differentiable
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight, table, positions = ctx.saved_tensors
        dq, dk = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k))
        dqw, dkw = torch.empty_like(q_weight), torch.empty_like(k_weight)
        B.norm_rotary_backward(_rows(dq_out), _rows(dk_out), q, k, q_weight, k_weight, table, dq, dk, dqw, dkw, B.alloc_workspace(B.norm_rotary_workspace(q, k)),
                               eps=ctx.eps, positions=positions)
        return dq, dk, dqw, dkw, None, None, None


def _zero_state(shape, dtype, device):
    """A window's state [2][B][kv heads][slots][D] of zeros: keys and values, each at the sixteen bytes that the library asks of a cache."""
    strides = [math.prod(shape[n + 1:]) for n in range(len(shape))]
    strides[0] += -strides[0] % (16 // dtype.itemsize)
    return torch.empty_strided(shape, strides, dtype=dtype, device=device).zero_()


def _halves(state):
    """(keys, values) of a window's state as the library takes them: the state's own memory, or a copy where a caller's copy or slice of a state lies at other bytes."""
    return tuple(x if x.is_contiguous() and x.data_ptr() % 16 == 0 else x.clone(memory_format=torch.contiguous_format) for x in (state[0], state[1]))


class AttendWindow(torch.autograd.Function):
    """(out, state behind it) of attention over the last `window` steps and the first `sinks` of an episode; gradients of q, k, v.  state
    [2][B][kv heads][sinks + window][D]: the cache's keys and values, constants of the gradient, or None where every episode begins in the call."""

    @staticmethod
    def forward(ctx, q, k, v, state, positions, window, sinks, scale):
        q, k, v = _rows(q), _rows(k), _rows(v)
        T, n, H, D = q.shape
        out = torch.empty((T, n, H, D), dtype=q.dtype, device=q.device)
        lse = torch.empty((n, H, T), dtype=torch.float32, device=q.device)
        after = _zero_state((2, n, k.shape[2], sinks + window, D), q.dtype, q.device)     # the call leaves slots that hold no step as they were
        B.window_attention(q, k, v, out, window, sinks, lse=lse, positions=positions, cache=None if state is None else _halves(state),
                           next_cache=(after[0], after[1]), scale=scale)
        ctx.save_for_backward(q, k, v, out, lse, state, positions)
        ctx.looks = window, sinks, scale
        ctx.mark_non_differentiable(after)
        return out, after

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, _):
        q, k, v, out, lse, state, positions = ctx.saved_tensors
        window, sinks, scale = ctx.looks
        dq, dk, dv = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k, v))
        B.window_attention_backward(q, k, v, out, lse, _rows(dout), dq, dk, dv, window, sinks, positions=positions, cache=None if state is None else _halves(state),
                                    scale=scale, workspace=B.alloc_workspace(B.window_attention_workspace(q, k, v, window, sinks, kind="backward")))
        return dq, dk, dv, None, None, None, None, None


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

    width: of the residual stream (a multiple of heads).  horizon: the heads' decays are 1 - 1 / h with h from 4 to it, in equal ratios.

    window: attention over that many last steps, the present one among them, and the episode's first `sinks`, in place of a state with decays.  A state then holds
    those steps' keys and values, and positions alone tell what it holds: the step in its episode, also of the first step of a call, and 0 where one begins."""

    def __init__(self, obs_dim, width=64, heads=4, kv_heads=None, layers=2, max_episode=1024, horizon=256, dtype=torch.float32, device="cuda", window=None, sinks=0):
        super().__init__()
        kv_heads = heads if kv_heads is None else kv_heads
        if width % heads or heads % kv_heads:
            raise B.MarlError("width is a multiple of heads, heads of kv_heads")
        if not 2 <= width // heads <= 128:
            raise B.MarlError(f"heads of {width // heads}: 2 to 128")
        if window is None and sinks or window is not None and (window < 1 or sinks < 0 or window + sinks > 1 << 30):
            raise B.MarlError("window is 1 or more, sinks 0 or more (with a window), together 2^30 at most")
        device = torch.device(device)
        if device.type == "cuda" and device.index not in (None, torch.cuda.current_device()):
            raise B.MarlError(f"{device} is not the current GPU, where the kernels run (torch.cuda.set_device)")
        self.heads, self.kv_heads, self.dim, self.dtype, self.window, self.sinks = heads, kv_heads, width // heads, dtype, window, sinks
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
            if window is not None:
                m.q_norm, m.k_norm = (torch.nn.Parameter(torch.ones(self.dim, device=device)) for _ in range(2))
            self.layers.append(m)
        self.norm_w, self.norm_b = ones(), zeros()
        self.value = lin(width, 1)

    def _product(self, layer, x):
        return torch.nn.functional.linear(x, layer.weight.to(self.dtype), layer.bias.to(self.dtype))

    def initial_state(self, sequences):
        """One state per layer, all zero: [B][heads][D][D] fp32, or with a window [2][B][kv heads][sinks + window][D] keys and values."""
        device = self.decay.device
        if self.window is not None:
            return [_zero_state((2, sequences, self.kv_heads, self.sinks + self.window, self.dim), self.dtype, device) for _ in self.layers]
        return [torch.zeros((sequences, self.heads, self.dim, self.dim), dtype=torch.float32, device=device) for _ in self.layers]

    def _heads(self, m, y):
        """q, k, v as views of one product's columns."""
        qkv = self._product(m.qkv, y)
        qkv = qkv.unflatten(-1, (self.heads + 2 * self.kv_heads, self.dim))
        return qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=-2)

    def _rest(self, m, x, out):
        """Behind the memory: each head normed by itself (a window's outputs are means of values already), then the layer's own two products."""
        if self.window is None:
            out = LayerNorm.apply(out, None, None, 1e-5)
        x = x + self._product(m.out, out.flatten(-2))
        y = LayerNorm.apply(x, m.norm2_w, m.norm2_b, 1e-5)
        return x + self._product(m.down, torch.nn.functional.gelu(self._product(m.up, y)))

    def forward(self, obs, positions, done=None, state=None):
        """Values [T][B] fp32 and the states behind the last step, from obs [T][B][D], positions and done [T][environments] (a window goes by positions alone: negative
        ones, of rows behind a recording's end, take no part)."""
        x = self._product(self.embed, obs.to(self.dtype))
        after = []
        for n, m in enumerate(self.layers):
            q, k, v = self._heads(m, LayerNorm.apply(x, m.norm_w, m.norm_b, 1e-5))
            if self.window is None:
                q, k = Rotate.apply(q, k, self.table, positions)
                out, s = Attend.apply(q, k, v, self.decay, None if state is None else state[n], done, 1 / math.sqrt(self.dim))
            else:
                q, k = NormRotate.apply(q, k, m.q_norm, m.k_norm, self.table, positions, 1e-6)
                out, s = AttendWindow.apply(q, k, v, None if state is None else state[n], positions, self.window, self.sinks, 1 / math.sqrt(self.dim))
            after.append(s)
            x = self._rest(m, x, out)
        return self._product(self.value, LayerNorm.apply(x, self.norm_w, self.norm_b, 1e-5)).squeeze(-1).float(), after

    @torch.no_grad()
    def step(self, obs, positions, state, done=None):
        """Values [B] of one step, obs [B][D]; the states are updated in place.  positions [environments]; done: of the step before."""
        x = self._product(self.embed, obs.to(self.dtype))
        for n, m in enumerate(self.layers):
            q, k, v = self._heads(m, LayerNorm.apply(x, m.norm_w, m.norm_b, 1e-5))
            out = torch.empty((*q.shape[:2], self.dim), dtype=self.dtype, device=x.device)
            if self.window is None:
                q, k = Rotate.apply(q[None], k[None], self.table, positions[None])
                B.linear_attention_step(q[0], k[0], v, self.decay, state[n], out, done=done, scale=1 / math.sqrt(self.dim))
            else:
                q, k = NormRotate.apply(q[None], k[None], m.q_norm, m.k_norm, self.table, positions[None], 1e-6)
                need = B.window_attention_workspace(q, k, v[None], self.window, self.sinks, kind="step")
                cache = _halves(state[n])
                B.window_attention_step(q[0], k[0], v, cache, positions, out, self.window, self.sinks, scale=1 / math.sqrt(self.dim),
                                        workspace=B.alloc_workspace(need) if need else None)
                for own, used in zip(state[n], cache):
                    if own.data_ptr() != used.data_ptr():
                        own.copy_(used)
            x = self._rest(m, x, out)
        return self._product(self.value, LayerNorm.apply(x, self.norm_w, self.norm_b, 1e-5)).squeeze(-1).float()
