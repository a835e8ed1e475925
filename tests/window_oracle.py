"""Plain 64-bit forms of attention over a window with first steps and of the norm of heads with rotation, from their definitions, and the errors that the kernels may
have: sums of roundings, each at most half a step (2^-24 relative in fp32, 2^-8 in bf16)."""
import math

import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8


def positions_of(positions, first, T, B, device):
    if positions is None:
        return (first + torch.arange(T, device=device))[:, None].expand(T, B).long()
    return positions.long().repeat_interleave(B // positions.shape[1], 1)


def slot_step(slot, n, window, sinks):
    """The step that a slot holds once n steps have gone by, or -1."""
    if slot < sinks:
        return slot if slot < n else -1
    held = [e for e in range(max(sinks, n - window), n) if sinks + (e - sinks) % window == slot]
    return held[0] if held else -1


def columns(k, cache, at, window, sinks):
    """([T][B][columns] what each row sees, [B][Hk][columns][D] the columns in 64 bits): the cache's slots, then the call's steps."""
    T, B = at.shape
    i = torch.arange(T, device=k.device)[:, None, None]
    j = torch.arange(T, device=k.device)[None, None]
    p = at[:, :, None]
    begun = i - p
    seen = (p >= 0) & (j >= begun) & (j <= i) & ((i - j < window) | (j - begun < sinks))
    cols = k.double().permute(1, 2, 0, 3)
    if cache is not None:
        slots = window + sinks
        e = torch.tensor([[slot_step(s, int(at[0, b].clamp(min=0)), window, sinks) for s in range(slots)] for b in range(B)], device=k.device)[None]
        seen = torch.cat([(p >= 0) & (e >= 0) & (begun < 0) & ((p - e < window) | (e < sinks)), seen], 2)
        cols = torch.cat([cache.double(), cols], 2)
    return seen, cols


class Attention:
    """out, lse and the bounds of their errors; dq, dk, dv and theirs.  Columns that a row does not see are taken out of every sum."""

    def __init__(self, q, k, v, window, sinks, positions=None, first=0, cache=None, scale=1.0):
        T, B, H, Dk = q.shape
        self.shape, self.scale, self.bf16 = (T, B, H), scale, q.dtype == torch.bfloat16
        self.group = H // k.shape[2]
        at = positions_of(positions, first, T, B, q.device)
        seen, K = columns(k, None if cache is None else cache[0], at, window, sinks)
        _, V = columns(v, None if cache is None else cache[1], at, window, sinks)
        self.cached = K.shape[2] - T
        self.K, self.V = (x.repeat_interleave(self.group, 1) for x in (K, V))                # [B][H][columns][D]
        self.seen = seen.permute(1, 0, 2)[:, None]                                           # [B][1][T][columns]
        self.Q = q.double().permute(1, 2, 0, 3)
        dot = lambda a, b: torch.matmul(a, b.transpose(2, 3).contiguous())
        self.s = torch.where(self.seen, dot(self.Q, self.K) * scale, -math.inf)
        size = torch.where(self.seen, dot(self.Q.abs(), self.K.abs()) * abs(scale), 0.0)
        # a score: Dk products and additions, its two factors; an exponent of two, of the size of the score, is rounded a few times on the way
        self.es = (Dk + 12) * U32 * size.amax(3, keepdim=True)
        self.lse = torch.logsumexp(self.s, 3)
        self.dot = dot

    def forward(self, v_dim):
        n = self.seen.sum(3, keepdim=True).double()
        P = torch.where(self.seen, torch.exp(self.s - self.lse[..., None]), 0.0)
        out, size = torch.matmul(P, self.V), torch.matmul(P, self.V.abs())
        # weights and their sum: both with the scores' error and the exponential's, the sum with one rounding for each term too
        bound = (2 * self.es + (2 * n + 40) * U32 + (U16 if self.bf16 else 0)) * size
        if self.bf16:
            bound = bound * (1 + U16) + U16 * out.abs()
        lse_bound = self.es[..., 0] + (n[..., 0] + 40) * U32 + 8 * U32 * torch.where(torch.isfinite(self.lse), self.lse.abs(), 0.0)
        back = lambda x: x.permute(2, 0, 1, 3)
        return back(out), back(bound), self.lse, lse_bound

    def backward(self, out, lse, dout):
        T, B, H = self.shape
        hf = lambda x: x.double().permute(1, 2, 0, 3)
        O, D, L = hf(out), hf(dout), lse.double()[..., None]
        seen, Dv = self.seen, O.shape[3]
        P = torch.where(seen, torch.exp(self.s - L), 0.0)
        gap = torch.where(seen, self.dot(D, self.V) - (D * O).sum(3, keepdim=True), 0.0)
        S = P * gap
        # what a weight may be off, relatively, and a gap
        top = torch.where(seen, self.s.abs(), 0.0).amax(3, keepdim=True)
        eP = self.es + 8 * U32 * (top + torch.where(torch.isfinite(L), L.abs(), 0.0)) + 8 * U32
        eG = (Dv + 8) * U32 * self.dot(D.abs(), self.V.abs()) + (Dv + 40) * U32 * (D * O).abs().sum(3, keepdim=True)
        eS = P * (eP * gap.abs() + eG * (1 + eP))
        n, w = self.seen.sum(3, keepdim=True).double(), float(T * self.group)
        r = U16 if self.bf16 else 0.0
        turn = lambda x: x.transpose(2, 3).contiguous()
        dq = self.scale * torch.matmul(S, self.K)
        bq = abs(self.scale) * (torch.matmul(eS * (1 + r) + r * S.abs(), self.K.abs()) + (n + 8) * U32 * torch.matmul(S.abs(), self.K.abs()))
        c = self.cached
        cut = lambda x: x[..., c:]
        dk = self.scale * torch.matmul(turn(cut(S)), self.Q)
        bk = abs(self.scale) * (torch.matmul(turn(cut(eS * (1 + r) + r * S.abs())), self.Q.abs()) + (w + 8) * U32 * torch.matmul(turn(cut(S.abs())), self.Q.abs()))
        dv = torch.matmul(turn(cut(P)), D)
        bv = torch.matmul(turn(cut(P * (eP * (1 + r) + r + (w + 8) * U32))), D.abs())
        res = []
        for g, b, shared in ((dq, bq, False), (dk, bk, True), (dv, bv, True)):
            if shared:
                g, b = (x.unflatten(1, (H // self.group, self.group)).sum(2) for x in (g, b))
            if self.bf16:
                b = b * (1 + U16) + U16 * g.abs()
            res.append((g.permute(2, 0, 1, 3), b.permute(2, 0, 1, 3)))
        return res


def next_cache(k, cache, into, positions, first, window, sinks):
    """The cache behind the call, by running its steps one after another over `into` (the cache before it, or what lies there)."""
    T, B = k.shape[:2]
    at = positions_of(positions, first, T, B, k.device)
    new = into.clone()
    for b in range(B):
        rows = [t for t in range(T) if at[t, b] >= 0]
        if not rows:
            if cache is not None:
                new[b] = cache[b]
            continue
        last = rows[-1]
        n = int(at[last, b]) + 1
        for slot in range(window + sinks):
            e = slot_step(slot, n, window, sinks)
            if e < 0:
                continue
            t = last - (n - 1 - e)
            if t >= 0:
                new[b, :, slot] = k[t, b]
            elif cache is not None:
                new[b, :, slot] = cache[b, :, slot]
    return new


def within(got, ref, bound, what=""):
    """Values within their bounds; infinities and NaNs where the reference has them."""
    got, tiny = got.double(), 1e-37
    if ref.numel() == 0:
        return 0.0
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what
    inf = torch.isinf(ref)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], ref[inf]), what
    ok = torch.isfinite(ref)
    worst = float(((got - ref).abs() / (bound + tiny))[ok].max()) if ok.any() else 0.0
    assert worst <= 1.0, (what, worst)
    return worst


# ---- norm and rotation -------------------------------------------------------------------------------------------------------------------
def _turn(x, table, at, R, interleaved, back):
    rows = table.double()[at.clamp(0, table.shape[0] - 1)][:, :, None]
    rows = torch.where((at >= table.shape[0])[:, :, None, None], math.nan, rows)
    c, s = rows[..., : R // 2], rows[..., R // 2:] * (-1.0 if back else 1.0)
    y = x.clone()
    one, two = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    a, b = x[..., one], x[..., two]
    y[..., one], y[..., two] = a * c - b * s, a * s + b * c
    return y


def norm_rotary(x, weight, table, at, eps, interleaved):
    """y and a bound of its error before it is rounded.  at [T][B]"""
    R, D = table.shape[1], x.shape[3]
    x, w = x.double(), torch.ones(D, dtype=torch.float64, device=x.device) if weight is None else weight.double()
    rstd = (x.square().mean(3, keepdim=True) + eps) ** -0.5
    u = x * rstd * w
    y = _turn(u, table, at, R, interleaved, False)
    size = u.abs()
    one, two = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    size[..., one] = size[..., two] = u[..., one].abs() + u[..., two].abs()
    # rstd: half the error of a sum of D squares, its root and reciprocal; then three products and an addition; a table's amplitude is at most 1 here
    bound = (D / 2 + 20) * U32 * size
    on = (at >= 0)[:, :, None, None]
    return torch.where(on, y, 0.0), torch.where(on, bound, 0.0)


def norm_rotary_backward(dy, x, weight, table, at, eps, interleaved):
    """dx, dweight and bounds of their errors (dx: before it is rounded)"""
    R, D = table.shape[1], x.shape[3]
    x, w = x.double(), torch.ones(D, dtype=torch.float64, device=x.device) if weight is None else weight.double()
    rstd = (x.square().mean(3, keepdim=True) + eps) ** -0.5
    on = (at >= 0)[:, :, None, None]
    du = torch.where(on, _turn(dy.double(), table, at, R, interleaved, True), 0.0)
    size = du.abs()
    one, two = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    size[..., one] = size[..., two] = torch.where(on, dy.double().abs()[..., one] + dy.double().abs()[..., two], 0.0)
    g, hat = du * w, x * rstd
    dx = rstd * (g - hat * (g * hat).mean(3, keepdim=True))
    gs = size * w.abs()
    bound = (D + 40) * U32 * rstd * (gs + hat.abs() * (gs * hat.abs()).mean(3, keepdim=True) * 3)
    n = x.shape[0] * x.shape[1] * x.shape[2]
    return (torch.where(on, dx, 0.0), torch.where(on, bound, 0.0)), ((du * hat).sum((0, 1, 2)), (n + D / 2 + 40) * U32 * (size * hat.abs()).sum((0, 1, 2)))
