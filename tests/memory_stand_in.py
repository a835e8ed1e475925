"""The sequence operators' entry points in plain torch on the CPU, with the library's contract: outputs are filled in place, a last dimension that is not
contiguous is refused.  What memory.py makes of them can be tested without a GPU."""
import torch

import memory_oracle as O
from paper_2107_01460_amd.binding import MarlError


def _contiguous_rows(*tensors):
    for t in tensors:
        if t is not None and t.shape[-1] > 1 and t.stride(-1) != 1:
            raise MarlError("marl error -3: the last dimension is contiguous")


def _fill(out, value):
    if out is not None:
        out.detach().copy_(value)


def _positions(positions, first_position, T, n):
    if positions is None:
        return (first_position + torch.arange(T))[:, None].expand(T, n)
    return positions.repeat_interleave(n // positions.shape[1], 1)


class StandIn:
    MarlError = MarlError

    @staticmethod
    def alloc_workspace(nbytes, device="cuda"):
        return None

    @staticmethod
    def linear_attention_workspace(q, k, v, backward=False):
        return 0

    @staticmethod
    def layer_norm_workspace(rows, width):
        return 0

    @staticmethod
    def linear_attention(q, k, v, decay, out, workspace=None, state=None, next_state=None, done=None, scale=1.0, stream=None):
        _contiguous_rows(q, k, v, out)
        o, s = O.attend(q.detach(), k.detach(), v.detach(), decay, None if state is None else state.detach(), done, scale)
        _fill(out, o)
        _fill(next_state, s)

    @staticmethod
    def linear_attention_backward(q, k, v, decay, dout, dq, dk, dv, workspace=None, state=None, dnext_state=None, dstate=None, done=None, scale=1.0, stream=None):
        _contiguous_rows(q, k, v, dout, dq, dk, dv)
        got = O.attend_backward(q.detach(), k.detach(), v.detach(), decay, dout.detach(), None if state is None else state.detach(),
                                None if dnext_state is None else dnext_state.detach(), done, scale)
        for t, g in zip((dq, dk, dv, dstate), got):
            _fill(t, g)

    @staticmethod
    def linear_attention_step(q, k, v, decay, state, out, next_state=None, done=None, scale=1.0, stream=None):
        _contiguous_rows(q, k, v, out)
        S = state.detach()
        if done is not None:
            S = O._keep(O._alive(done[None], S.shape[0], 1)[0], S)
        o, s = O.attend(q.detach()[None], k.detach()[None], v.detach()[None], decay, S, None, scale)
        _fill(out, o[0])
        (state if next_state is None else next_state).detach().copy_(s)

    @staticmethod
    def layer_norm(x, weight, bias, out, mean=None, rstd=None, eps=1e-5, stream=None):
        _contiguous_rows(x, out)
        d = lambda t: None if t is None else t.detach()
        for t, v in zip((out, mean, rstd), O.layer_norm(d(x), d(weight), d(bias), eps)):
            _fill(t, v)

    @staticmethod
    def layer_norm_backward(dout, x, weight, mean, rstd, dx, dweight=None, dbias=None, workspace=None, stream=None):
        _contiguous_rows(dout, x, dx)
        dy, r = dout.detach().double(), rstd.double()[:, None]
        h = (x.detach().double() - mean.double()[:, None]) * r
        u = dy if weight is None else dy * weight.detach().double()
        _fill(dx, r * (u - u.mean(1, keepdim=True) - h * (u * h).mean(1, keepdim=True)))
        _fill(dweight, (dy * h).sum(0))
        _fill(dbias, dy.sum(0))

    @staticmethod
    def rotary_table(n_positions, rotary_dim, **kw):
        f = 10000.0 ** (-2.0 * torch.arange(rotary_dim // 2, dtype=torch.float64) / rotary_dim)
        angle = torch.arange(n_positions, dtype=torch.float64)[:, None] * f
        return torch.cat([angle.cos(), angle.sin()], 1).float()

    @staticmethod
    def rotary(q, k, table, q_out, k_out, positions=None, first_position=0, interleaved=False, inverse=False, stream=None):
        _contiguous_rows(q, k, q_out, k_out)
        at = _positions(positions, first_position, *q.shape[:2])
        for x, y in ((q, q_out), (k, k_out)):
            if x is not None:
                _fill(y, O.rotate(x.detach(), table, at, interleaved, inverse))
