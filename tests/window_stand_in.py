"""The entry points of window attention and of norm with rotation in plain torch on the CPU, with the library's contract; see memory_stand_in.py."""
import torch

import window_oracle as O
from memory_stand_in import StandIn as Memory, _contiguous_rows, _fill


def _plain(*tensors):
    return [None if t is None else t.detach() for t in tensors]


def _at(positions, first, T, n):
    return O.positions_of(positions, first, T, n, "cpu")


class StandIn(Memory):
    @staticmethod
    def norm_rotary(q, k, q_weight, k_weight, table, q_out, k_out, eps=1e-6, positions=None, first_position=0, interleaved=False, stream=None):
        _contiguous_rows(q, k, q_out, k_out)
        at = _at(positions, first_position, *q.shape[:2])
        for x, w, y in ((q, q_weight, q_out), (k, k_weight, k_out)):
            if x is not None:
                _fill(y, O.norm_rotary(*_plain(x, w), table, at, eps, interleaved)[0])

    @staticmethod
    def norm_rotary_workspace(q, k):
        return 0

    @staticmethod
    def norm_rotary_backward(dq_out, dk_out, q, k, q_weight, k_weight, table, dq, dk, dq_weight=None, dk_weight=None, workspace=None, eps=1e-6, positions=None,
                             first_position=0, interleaved=False, stream=None):
        _contiguous_rows(dq_out, dk_out, q, k, dq, dk)
        at = _at(positions, first_position, *q.shape[:2])
        for dy, x, w, dx, dw in ((dq_out, q, q_weight, dq, dq_weight), (dk_out, k, k_weight, dk, dk_weight)):
            if x is not None:
                (gx, _), (gw, _) = O.norm_rotary_backward(*_plain(dy, x, w), table, at, eps, interleaved)
                _fill(dx, gx)
                _fill(dw, gw)

    @staticmethod
    def window_attention_workspace(q, k, v, window, sinks=0, kind="forward"):
        return 0

    @staticmethod
    def window_attention(q, k, v, out, window, sinks=0, lse=None, positions=None, first_position=0, cache=None, next_cache=None, scale=1.0, workspace=None, stream=None):
        _contiguous_rows(q, k, v, out)
        q, k, v = _plain(q, k, v)
        old = None if cache is None else _plain(*cache)
        T, n = q.shape[:2]
        if T:
            o, _, s, _ = O.Attention(q, k, v, window, sinks, positions, first_position, old, scale).forward(v.shape[3])
            _fill(out, torch.where(torch.isinf(s).permute(2, 0, 1)[..., None], 0.0, o))
            _fill(lse, s)
        if next_cache is not None:
            for i, x in enumerate((k, v)):
                into = next_cache[i].detach()
                _fill(into, old[i] if T == 0 and old else O.next_cache(x, None if old is None else old[i], into, positions, first_position, window, sinks) if T else into)

    @staticmethod
    def window_attention_backward(q, k, v, out, lse, dout, dq, dk, dv, window, sinks=0, positions=None, first_position=0, cache=None, scale=1.0, workspace=None, stream=None):
        _contiguous_rows(q, k, v, out, dout, dq, dk, dv)
        q, k, v, out, lse, dout = _plain(q, k, v, out, lse, dout)
        if q.shape[0] == 0:
            return
        got = O.Attention(q, k, v, window, sinks, positions, first_position, None if cache is None else _plain(*cache), scale).backward(out, lse, dout)
        for t, (g, _) in zip((dq, dk, dv), got):
            _fill(t, g)

    @staticmethod
    def window_attention_step(q, k, v, cache, positions, out, window, sinks=0, scale=1.0, workspace=None, stream=None):
        _contiguous_rows(q, k, v, out)
        StandIn.window_attention(q[None], k[None], v[None], out[None], window, sinks, positions=positions[None], cache=cache, next_cache=cache, scale=scale)
