"""The operators of sequence memories whose speed is tracked: linear attention with a decay per head (whole rollouts, their
gradient, single steps), layer norm (forward, gradient) and rotary positions.

Arrays are time-major like a trajectory: ``[T][B][H][D]`` with B = environments * agents sequences, ``done`` [T][environments]
marks the steps that ended an episode.  ``own`` chooses between the plain form (elementary torch operations in 32 bits) and the
framework's operators.

Definition of linear attention, per sequence and query head h with g = decay[h], state S (Dk x Dv), kv head h * Hk / Hq:
    S_t = [t = 0 or not done_{t-1}] g S_{t-1} + k_t v_t^T        out_t = scale S_t^T q_t        next_state = [not done_{T-1}] S_{T-1}
(S_{-1}: the state given.)
"""
import math

import torch

own = False

_F32, _BF16 = "f32", "bf16"
_DTYPE = {_F32: torch.float32, _BF16: torch.bfloat16}
_EPS = 1e-5
_CHUNK = 64          # steps that the plain form takes at once
_MAX_ELEMENTS = 1 << 27   # of one array of a drawn case


def _attend(name, kind, T, envs, agents, heads, kv_heads, dk, dv, dtype, episode, state):
    return dict(name=name, kind=kind, T=T, envs=envs, agents=agents, heads=heads, kv_heads=kv_heads, dk=dk, dv=dv, dtype=dtype,
                episode=episode, state=state)


def listed():
    return [
        # the smallest benchmarked configuration: one rollout of 16 steps of 64 two-agent environments, 64 hidden units as two heads
        _attend("attend_small", "attend", 16, 64, 2, 2, 2, 32, 32, _F32, 25, True),
        # rollouts of the large bf16 configuration (128 steps, eight agents, 512 hidden units), an eighth of its environments
        _attend("attend_rollout_bf16", "attend", 128, 512, 8, 8, 8, 64, 64, _BF16, 100, True),
        # one long recorded sequence, query heads sharing keys and values: work has to be split over time
        _attend("attend_long_bf16", "attend", 32768, 1, 1, 8, 2, 128, 128, _BF16, 0, False),
        # gradient over a minibatch of sequences of the centralised-critic configuration (128 steps, 128 hidden units)
        _attend("attend_grad_f32", "attend_grad", 128, 1024, 4, 4, 4, 32, 32, _F32, 70, True),
        # gradient at a user's own shape: odd lengths and widths, shared heads, short episodes
        _attend("attend_grad_odd_bf16", "attend_grad", 777, 37, 3, 6, 2, 40, 72, _BF16, 60, True),
        # one step of the smallest configuration: the latency of acting
        _attend("step_small", "step", 1, 64, 2, 2, 2, 32, 32, _F32, 25, True),
        # one step of 4096 four-agent environments: reading and writing the states
        _attend("step_rollout", "step", 1, 4096, 4, 4, 4, 32, 32, _F32, 70, True),
        # norm in front of a block, the large bf16 configuration
        dict(name="norm_rollout_bf16", kind="norm", rows=128 * 4096, width=512, dtype=_BF16, affine=True),
        # its gradient, fp32 networks of 128 units
        dict(name="norm_grad_f32", kind="norm_grad", rows=128 * 4096, width=128, dtype=_F32, affine=True),
        # gradient over rows as wide as an observation of a 7 x 7 window: nothing is a power of two
        dict(name="norm_grad_odd_bf16", kind="norm_grad", rows=10007, width=147, dtype=_BF16, affine=True),
        # positions of one acting step
        dict(name="rotate_small", kind="rotate", T=1, envs=64, agents=2, heads=2, kv_heads=2, dim=32, rotary=32, interleaved=False,
             inverse=False, dtype=_F32, positions=25),
        # positions of a whole rollout, queries and keys, half of each head rotated
        dict(name="rotate_rollout_bf16", kind="rotate", T=128, envs=512, agents=8, heads=8, kv_heads=8, dim=64, rotary=32,
             interleaved=True, inverse=False, dtype=_BF16, positions=4096),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend_grad", "step", "norm", "norm_grad", "rotate"])
    dtype = rng.choice([_F32, _BF16])
    while True:
        if kind in ("norm", "norm_grad"):
            case = dict(kind=kind, rows=_log(rng, 1, 1 << 20), width=_log(rng, 8, 2048), dtype=dtype, affine=rng.random() < 0.8)
            elements = case["rows"] * case["width"]
        else:
            envs, agents = _log(rng, 1, 16384), rng.randint(1, 8)
            kv_heads = _log(rng, 1, 8)
            heads = kv_heads * rng.choice([1, 1, 1, 2, 3])
            T = 1 if kind == "step" else _log(rng, 1, 128) if envs * agents > 64 else _log(rng, 1, 16384)
            if kind == "rotate":
                dim = _log(rng, 4, 128)
                rotary = 2 * max(1, int(rng.choice([0.25, 0.5, 1.0, 1.0]) * dim) // 2)
                case = dict(kind=kind, T=T, envs=envs, agents=agents, heads=heads, kv_heads=kv_heads, dim=dim, rotary=rotary,
                            interleaved=rng.random() < 0.5, inverse=rng.random() < 0.3, dtype=dtype, positions=_log(rng, 1, 8192))
                elements = T * envs * agents * heads * dim
            else:
                dk, dv = (_log(rng, 8, 128) for _ in range(2)) if rng.random() < 0.5 else [rng.choice([16, 32, 64, 128])] * 2
                case = dict(kind=kind, T=T, envs=envs, agents=agents, heads=heads, kv_heads=kv_heads, dk=dk, dv=dv, dtype=dtype,
                            episode=rng.choice([0, 25, 70, 400]), state=rng.random() < 0.7 or kind == "step")
                per_step = envs * agents * heads * max(dk, dv)
                elements = max(T * per_step, 4 * envs * agents * heads * dk * dv)
                if kind == "attend_grad":
                    elements *= 2
        if elements <= _MAX_ELEMENTS:
            return case


# ---- what a program holds before the call ------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = _DTYPE[case["dtype"]]

    def randn(*shape, dtype=dtype):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    kind = case["kind"]
    s = dict(case=case)
    if kind in ("norm", "norm_grad"):
        rows, width = case["rows"], case["width"]
        x = (torch.randn((rows, width), generator=g, device="cuda") * 1.5 + torch.randn((rows, 1), generator=g, device="cuda")).to(dtype)
        s.update(x=x, weight=None, bias=None, out=torch.empty_like(x))
        if case["affine"]:
            s.update(weight=1 + 0.2 * randn(width, dtype=torch.float32), bias=0.2 * randn(width, dtype=torch.float32))
        s.update(mean=torch.empty(rows, device="cuda"), rstd=torch.empty(rows, device="cuda"))
        if kind == "norm_grad":   # what the forward pass left
            x32 = x.float()
            s["mean"] = x32.mean(1)
            s["rstd"] = 1 / torch.sqrt((x32 - s["mean"][:, None]).square().mean(1) + _EPS)
            s["dout"] = randn(rows, width)
            s["dweight"] = torch.empty(width, device="cuda") if case["affine"] else None
            s["dbias"] = torch.empty(width, device="cuda") if case["affine"] else None
        if own:
            import paper_2107_01460_amd as M
            s["workspace"] = M.alloc_workspace(M.layer_norm_workspace(rows, width))
        return s
    T, envs, agents, hq, hk = case["T"], case["envs"], case["agents"], case["heads"], case["kv_heads"]
    B = envs * agents
    if kind == "rotate":
        P, R = case["positions"], case["rotary"]
        angle = torch.arange(P, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * torch.arange(R // 2, dtype=torch.float64) / R)
        table = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
        # each environment is somewhere in its episode and starts anew at its end
        start = torch.randint(0, P, (envs,), generator=g, device="cuda")
        positions = ((start + torch.arange(T, device="cuda")[:, None]) % P).int()
        s.update(q=randn(T, B, hq, case["dim"]), k=randn(T, B, hk, case["dim"]), table=table, positions=positions)
        s.update(q_out=torch.empty_like(s["q"]), k_out=torch.empty_like(s["k"]))
        return s
    dk, dv = case["dk"], case["dv"]
    s.update(q=randn(T, B, hq, dk), k=randn(T, B, hk, dk), v=randn(T, B, hk, dv), scale=dk ** -0.5)
    # one decay per head, horizons from 32 steps on, doubling
    s["decay"] = 1 - 2.0 ** -(5 + torch.arange(hq, device="cuda", dtype=torch.float32) % 6)
    s["done"] = None
    if case["episode"]:
        s["done"] = (torch.rand((T, envs), generator=g, device="cuda") < 1 / case["episode"]).to(torch.uint8)
    state = lambda: randn(B, hq, dk, dv, dtype=torch.float32)
    s["state"] = state() if case["state"] else None
    s["out"] = torch.empty((T, B, hq, dv), dtype=dtype, device="cuda")
    s["next_state"] = torch.empty((B, hq, dk, dv), device="cuda")
    if kind == "attend_grad":
        s.update(dout=randn(T, B, hq, dv), dnext_state=state() if case["state"] else None, dq=torch.empty_like(s["q"]),
                 dk=torch.empty_like(s["k"]), dv=torch.empty_like(s["v"]), dstate=torch.empty((B, hq, dk, dv), device="cuda"))
    if own and kind != "step":
        import paper_2107_01460_amd as M
        s["workspace"] = M.alloc_workspace(M.linear_attention_workspace(s["q"], s["k"], s["v"], backward=kind == "attend_grad"))
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2107_01460_amd as M
    kind = s["case"]["kind"]
    if kind == "attend":
        M.linear_attention(s["q"], s["k"], s["v"], s["decay"], s["out"], s["workspace"], state=s["state"], next_state=s["next_state"],
                           done=s["done"], scale=s["scale"])
        return s["out"], s["next_state"]
    if kind == "attend_grad":
        M.linear_attention_backward(s["q"], s["k"], s["v"], s["decay"], s["dout"], s["dq"], s["dk"], s["dv"], s["workspace"],
                                    state=s["state"], dnext_state=s["dnext_state"], dstate=s["dstate"], done=s["done"], scale=s["scale"])
        return s["dq"], s["dk"], s["dv"], s["dstate"]
    if kind == "step":   # done: of the step before
        M.linear_attention_step(s["q"][0], s["k"][0], s["v"][0], s["decay"], s["state"], s["out"][0], next_state=s["next_state"],
                                done=None if s["done"] is None else s["done"][0], scale=s["scale"])
        return s["out"], s["next_state"]
    if kind == "norm":
        M.layer_norm(s["x"], s["weight"], s["bias"], s["out"], mean=s["mean"], rstd=s["rstd"], eps=_EPS)
        return s["out"], s["mean"], s["rstd"]
    if kind == "norm_grad":
        M.layer_norm_backward(s["dout"], s["x"], s["weight"], s["mean"], s["rstd"], s["out"], s["dweight"], s["dbias"], s["workspace"])
        return (s["out"], s["dweight"], s["dbias"]) if s["case"]["affine"] else (s["out"],)
    M.rotary(s["q"], s["k"], s["table"], s["q_out"], s["k_out"], positions=s["positions"], interleaved=s["case"]["interleaved"],
             inverse=s["case"]["inverse"])
    return s["q_out"], s["k_out"]


def _heads_first(x, heads):
    """[T][B][Hk][D] in 32 bits as [B][heads][T][D], each kv head repeated for the query heads that share it."""
    x = x.float().permute(1, 2, 0, 3)
    return x.repeat_interleave(heads // x.shape[1], 1) if x.shape[1] != heads else x.contiguous()


def _scan(x, y, z, decay, done, state, reverse, inner, inter, update):
    """out_i = inner sum_j g^|i-j| (x_i . y_j) z_j + inter g^(..) x_i S over the j up to i (reverse: from i on) in i's episode,
    S <- g^n S + update sum_j g^(..) y_j z_j^T, chunk by chunk; returns out and S."""
    B, H, T, _ = x.shape
    out = torch.empty((B, H, T, z.shape[3]), device=x.device)
    S = torch.zeros((B, H, x.shape[3], z.shape[3]), device=x.device) if state is None else state
    starts = list(range(0, T, _CHUNK))
    for t0 in reversed(starts) if reverse else starts:
        n = min(_CHUNK, T - t0)
        i = torch.arange(n, device=x.device)
        power = decay[:, None, None] ** (i[:, None] - i[None, :]).abs().float()
        reach = i[:, None] <= i[None, :] if reverse else i[:, None] >= i[None, :]
        first = decay[:, None] ** (i + 1.0)          # from the chunk's start to step i
        last = decay[:, None] ** (n - 1.0 - i)       # from step i to the chunk's end
        carry = (decay ** float(n))[None, :, None, None]
        if done is not None:
            d = done[t0:t0 + n].long().t()           # [B][n]
            before = d.cumsum(1) - d                 # episodes that ended in the chunk before step i
            total = d.sum(1, keepdim=True)
            reach = (reach[None] & (before[:, :, None] == before[:, None, :]))[:, None]
            first = torch.where((before == 0)[:, None], first[None], 0.0)
            last = torch.where((before == total)[:, None], last[None], 0.0)
            carry = torch.where((total == 0)[:, :, None, None], carry, 0.0)
        if reverse:
            first, last = last, first
        xc, yc, zc = x[:, :, t0:t0 + n], y[:, :, t0:t0 + n], z[:, :, t0:t0 + n]
        score = torch.where(reach, torch.matmul(xc, yc.transpose(2, 3).contiguous()) * (power * inner), 0.0)
        out[:, :, t0:t0 + n] = torch.matmul(score, zc) + (first * inter)[..., None] * torch.matmul(xc, S)
        S = carry * S + torch.matmul((yc * (last * update)[..., None]).transpose(2, 3).contiguous(), zc)
    return out, S


def _run_plain(s):
    case = s["case"]
    kind, dtype = case["kind"], _DTYPE[case["dtype"]]
    if kind in ("norm", "norm_grad"):
        x = s["x"].float()
        if kind == "norm":
            mean = x.mean(1)
            centred = x - mean[:, None]
            rstd = 1 / torch.sqrt(centred.square().mean(1) + _EPS)
            y = centred * rstd[:, None]
            if case["affine"]:
                y = y * s["weight"] + s["bias"]
            return y.to(dtype), mean, rstd
        dy = s["dout"].float()
        hat = (x - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["weight"] if case["affine"] else dy
        dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
        return (dx.to(dtype), (dy * hat).sum(0), dy.sum(0)) if case["affine"] else (dx.to(dtype),)
    if kind == "rotate":
        R = case["rotary"]
        rows = s["table"][s["positions"].long().repeat_interleave(case["agents"], 1)][:, :, None]   # [T][B][1][R]
        cos, sin = rows[..., :R // 2], rows[..., R // 2:]
        if case["inverse"]:
            sin = -sin

        def turn(x):
            x = x.float()
            y = x.clone()
            one, two = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
            y[..., one] = x[..., one] * cos - x[..., two] * sin
            y[..., two] = x[..., one] * sin + x[..., two] * cos
            return y.to(dtype)

        return turn(s["q"]), turn(s["k"])
    hq, hk, agents = case["heads"], case["kv_heads"], case["agents"]
    done = None if s["done"] is None else s["done"].repeat_interleave(agents, 1)
    decay, scale = s["decay"], s["scale"]
    q, k, v = _heads_first(s["q"], hq), _heads_first(s["k"], hq), _heads_first(s["v"], hq)
    back = lambda x: x.permute(2, 0, 1, 3).to(dtype).contiguous()
    if kind == "step":
        keep = decay[None, :, None, None]
        if done is not None:
            keep = torch.where(done[0].bool()[:, None, None, None], 0.0, keep)
        S = keep * s["state"] + k[:, :, 0, :, None] * v[:, :, 0, None, :]
        return (scale * (q[:, :, 0, :, None] * S).sum(2)).to(dtype)[None], S
    if kind == "attend":
        out, S = _scan(q, k, v, decay, done, s["state"], False, scale, scale, 1.0)
        return back(out), S
    do = _heads_first(s["dout"], hq)
    turned = lambda S: None if S is None else S.transpose(2, 3).contiguous()
    dq, _ = _scan(do, v, k, decay, done, turned(s["state"]), False, scale, scale, 1.0)
    dv, dS = _scan(k, q, do, decay, done, s["dnext_state"], True, scale, 1.0, scale)
    dk, _ = _scan(v, do, q, decay, done, turned(s["dnext_state"]), True, scale, 1.0, scale)
    if hk != hq:   # the gradient of a shared head: the sum over the query heads that share it
        dk, dv = (g.unflatten(1, (hk, hq // hk)).sum(2) for g in (dk, dv))
    return back(dq), back(dk), back(dv), dS


# ---- in 64 bits, from the definition -----------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    wide = lambda name: None if s.get(name) is None else s[name].double()
    if kind == "norm":
        x = wide("x")
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + _EPS) ** -0.5
        y = (x - mean[:, None]) * rstd[:, None]
        return (y * wide("weight") + wide("bias") if case["affine"] else y), mean, rstd
    if kind == "norm_grad":
        dy, n = wide("dout"), case["width"]
        hat = (wide("x") - wide("mean")[:, None]).mul_(wide("rstd")[:, None])
        dw, db = (dy * hat).sum(0), dy.sum(0)
        g = dy * wide("weight") if case["affine"] else dy
        dx = (g - g.sum(1, keepdim=True) / n - hat * ((g * hat).sum(1, keepdim=True) / n)) * wide("rstd")[:, None]
        return (dx, dw, db) if case["affine"] else (dx,)
    if kind == "rotate":
        R = case["rotary"]
        at = wide("table")[s["positions"].long()].repeat_interleave(case["agents"], 1)[:, :, None]
        turn = torch.complex(at[..., :R // 2].contiguous(), (-1.0 if case["inverse"] else 1.0) * at[..., R // 2:])

        def rotated(x):
            x = x.double()
            if case["interleaved"]:
                y = torch.view_as_real(torch.view_as_complex(x[..., :R].unflatten(-1, (R // 2, 2)).contiguous()) * turn).flatten(-2)
            else:
                z = torch.complex(x[..., :R // 2].contiguous(), x[..., R // 2:R].contiguous()) * turn
                y = torch.cat([z.real, z.imag], -1)
            return torch.cat([y, x[..., R:]], -1)

        return rotated(s["q"]), rotated(s["k"])
    T, hq, hk = case["T"], case["heads"], case["kv_heads"]
    share = torch.arange(hq, device="cuda") // (hq // hk)     # kv head of each query head
    g, scale = wide("decay")[None, :, None, None], s["scale"]
    q, k, v, do = wide("q"), wide("k"), wide("v"), wide("dout")
    alive = None
    if s["done"] is not None:
        alive = 1.0 - s["done"].double().repeat_interleave(case["agents"], 1)
    zero = torch.zeros((case["envs"] * case["agents"], hq, case["dk"], case["dv"]), dtype=torch.float64, device="cuda")
    S = zero.clone() if s["state"] is None else wide("state")
    if kind == "step" and alive is not None:
        S *= alive[0][:, None, None, None]
    result = []
    for t in range(T):
        S = (S * g).addcmul_(k[t][:, share, :, None], v[t][:, share, None, :])
        if kind == "attend_grad":
            result.append(scale * (S * do[t][:, :, None, :]).sum(3))
        else:
            result.append(scale * (S * q[t][:, :, :, None]).sum(2))
        if alive is not None and kind != "step":
            S = S * alive[t][:, None, None, None]
    result = torch.stack(result)
    if kind != "attend_grad":
        return result, S
    R = zero if s["dnext_state"] is None else wide("dnext_state")
    dk, dv = torch.empty_like(k), torch.empty_like(v)
    for t in reversed(range(T)):
        if alive is not None:
            R = R * alive[t][:, None, None, None]
        R = R + scale * q[t][:, :, :, None] * do[t][:, :, None, :]
        dk[t] = (R * v[t][:, share, None, :]).sum(3).unflatten(1, (hk, hq // hk)).sum(2)
        dv[t] = (R * k[t][:, share, :, None]).sum(2).unflatten(1, (hk, hq // hk)).sum(2)
        R = R * g
    return result, dk, dv, R


def work(case):
    kind, size = case["kind"], 4 if case["dtype"] == _F32 else 2
    if kind in ("norm", "norm_grad"):
        n = case["rows"] * case["width"]
        grad = kind == "norm_grad"
        weights = (4 if grad and case["affine"] else 2) * 4 * case["width"] if case["affine"] else 0
        return {"bytes": n * size * (3 if grad else 2) + 8 * case["rows"] + weights, "flops": n * (16 if grad else 8)}
    steps = case["T"] * case["envs"] * case["agents"]
    hq, hk = case["heads"], case["kv_heads"]
    if kind == "rotate":
        return {"bytes": 2 * steps * (hq + hk) * case["dim"] * size + 4 * case["T"] * case["envs"] + 4 * case["positions"] * case["rotary"],
                "flops": 3 * steps * (hq + hk) * case["rotary"]}
    dk, dv = case["dk"], case["dv"]
    states = case["envs"] * case["agents"] * hq * dk * dv * 4
    flags = case["T"] * case["envs"] if case["episode"] else 0
    if kind == "attend_grad":
        return {"bytes": steps * size * (hq * (2 * dk + dv) + hk * 2 * (dk + dv)) + (3 if case["state"] else 1) * states + flags,
                "flops": 10 * steps * hq * dk * dv}
    return {"bytes": steps * size * (hq + hk) * (dk + dv) + (2 if case["state"] else 1) * states + flags, "flops": 4 * steps * hq * dk * dv}
