"""Plain 64-bit forms of the sequence operators, step by step and from their definitions, and the error bounds that the tests use."""
import torch


def _alive(done, B, T):
    """[T][B] factors 1 - done of each sequence."""
    if done is None:
        return None
    return 1.0 - (done != 0).double().repeat_interleave(B // done.shape[1], 1)


def _share(q, k):
    return torch.arange(q.shape[2], device=q.device) // (q.shape[2] // k.shape[2])


def _keep(alive, S):
    return S if alive is None else torch.where(alive[:, None, None, None] != 0, S, torch.zeros_like(S))


def attend(q, k, v, decay, state=None, done=None, scale=1.0):
    """out [T][B][H][Dv], next_state"""
    q, k, v, g = q.double(), k.double(), v.double(), decay.double()[None, :, None, None]
    T, B, H, Dk = q.shape
    share, alive = _share(q, k), _alive(done, B, T)
    S = torch.zeros((B, H, Dk, v.shape[3]), dtype=torch.float64, device=q.device) if state is None else state.double()
    out = []
    for t in range(T):
        S = g * S + k[t][:, share, :, None] * v[t][:, share, None, :]
        out.append(scale * (q[t][..., None] * S).sum(2))
        S = _keep(None if alive is None else alive[t], S)
    return (torch.stack(out) if T else q.new_zeros((0, B, H, v.shape[3]))), S


def attend_backward(q, k, v, decay, dout, state=None, dnext=None, done=None, scale=1.0):
    """dq, dk, dv, dstate"""
    q, k, v, do, g = q.double(), k.double(), v.double(), dout.double(), decay.double()[None, :, None, None]
    T, B, H, Dk = q.shape
    Hk, Dv = v.shape[2:]
    share, alive = _share(q, k), _alive(done, B, T)
    zero = torch.zeros((B, H, Dk, Dv), dtype=torch.float64, device=q.device)
    S = zero if state is None else state.double()
    dq = torch.empty_like(q)
    for t in range(T):
        S = g * S + k[t][:, share, :, None] * v[t][:, share, None, :]
        dq[t] = scale * (S * do[t][:, :, None, :]).sum(3)
        S = _keep(None if alive is None else alive[t], S)
    R = zero if dnext is None else dnext.double()
    dk, dv = torch.empty_like(k), torch.empty_like(v)
    for t in reversed(range(T)):
        R = _keep(None if alive is None else alive[t], R)
        R = R + scale * q[t][..., None] * do[t][:, :, None, :]
        dk[t] = (R * v[t][:, share, None, :]).sum(3).unflatten(1, (Hk, H // Hk)).sum(2)
        dv[t] = (R * k[t][:, share, :, None]).sum(2).unflatten(1, (Hk, H // Hk)).sum(2)
        R = g * R
    return dq, dk, dv, R


def layer_norm(x, weight, bias, eps):
    x = x.double()
    mean = x.mean(1)
    rstd = (x.var(1, unbiased=False) + eps) ** -0.5
    y = (x - mean[:, None]) * rstd[:, None]
    return (y if weight is None else y * weight.double()) + (0.0 if bias is None else bias.double()), mean, rstd


def rotate(x, table, positions, interleaved, inverse):
    """positions [T][B]"""
    R = table.shape[1]
    at = table.double()[positions.long()][:, :, None]
    c, s = at[..., : R // 2], at[..., R // 2:] * (-1.0 if inverse else 1.0)
    y = x.double().clone()
    one, two = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    a, b = y[..., one].clone(), y[..., two].clone()
    y[..., one], y[..., two] = a * c - b * s, a * s + b * c
    return y


# ---- bounds --------------------------------------------------------------------------------------------------------------
# A result is a sum of terms; `size` is the same sum over the terms' magnitudes.  In fp32 every term passes at most one rounding for each
# addition it takes part in and a few for its factors (a power of the decay: at most ten), so the error is below
# (additions + 40) 2^-24 size.
U32, U16 = 2.0 ** -24, 2.0 ** -8


def within(got, ref, size, additions, bf16=False, parts=0.0):
    """bf16: rounded once to eight bits; parts: what operands lose when they are split into parts, relative to size."""
    ref, size = ref.double(), size.double()
    bound = ((additions + 40) * U32 + parts) * size + 1e-37
    if bf16:
        bound = bound * (1 + U16) + U16 * ref.abs()
    worst = ((got.double() - ref).abs() / bound)
    worst = float(worst.max()) if worst.numel() else 0.0
    assert worst <= 1.0, worst
    return worst
