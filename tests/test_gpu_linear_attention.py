"""Linear attention with a decay per head against the recurrence in 64 bits: whole sequences, gradients, single steps."""
import pytest
import torch

import memory_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
# values as two bf16 parts lose 2^-16 (each part's rounding: 2^-8): a term goes through the scores or through the state
PARTS = {F32: 0.0, BF16: 2.0 ** -16}


@pytest.fixture(scope="module")
def M():
    import paper_2107_01460_amd as m
    assert torch.cuda.is_available()
    return m


def make(T, B, H, Hk, Dk, Dv, dtype, seed=0, episode=0, agents=1, state=True, layout="tbhd"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")

    def arr(H, D):
        if layout == "bhtd":      # sequence-major storage
            return rnd(B, H, T, D).to(dtype).permute(2, 0, 1, 3)
        if layout == "odd":       # a part of wider rows that starts at an odd element
            return rnd(T, B, H, D + 3).to(dtype)[..., 1: D + 1]
        return rnd(T, B, H, D).to(dtype)
    done = None
    if episode:
        done = (torch.rand((T, B // agents), generator=g, device="cuda") < 1 / episode).to(torch.uint8)
    decay = 1 - 2.0 ** -(2 + torch.arange(H, device="cuda", dtype=F32) % 6)
    s = dict(q=arr(H, Dk), k=arr(Hk, Dk), v=arr(Hk, Dv), decay=decay, done=done, scale=Dk ** -0.5, dout=arr(H, Dv))
    s["state"] = rnd(B, H, Dk, Dv) if state else None
    s["dnext"] = rnd(B, H, Dk, Dv) if state else None
    return s


def empty(shape, dtype, layout="tbhd"):
    if layout == "bhtd":
        T, B, H, D = shape
        return torch.full((B, H, T, D), float("nan"), dtype=dtype, device="cuda").permute(2, 0, 1, 3)
    if layout == "odd":
        return torch.full((*shape[:3], shape[3] + 3), float("nan"), dtype=dtype, device="cuda")[..., 1: shape[3] + 1]
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def forward(M, s, layout="tbhd", stream=None):
    q, k, v = s["q"], s["k"], s["v"]
    T, B, H, Dk = q.shape
    out, nxt = empty((T, B, H, v.shape[3]), q.dtype, layout), empty((B, H, Dk, v.shape[3]), F32)
    ws = M.alloc_workspace(M.linear_attention_workspace(q, k, v))
    M.linear_attention(q, k, v, s["decay"], out, ws, state=s["state"], next_state=nxt, done=s["done"], scale=s["scale"], stream=stream)
    return out, nxt


def backward(M, s, layout="tbhd"):
    q, k, v = s["q"], s["k"], s["v"]
    T, B, H, Dk = q.shape
    dq, dk, dv = (empty(x.shape, q.dtype, layout) for x in (q, k, v))
    dstate = empty((B, H, Dk, v.shape[3]), F32)
    ws = M.alloc_workspace(M.linear_attention_workspace(q, k, v, backward=True))
    M.linear_attention_backward(q, k, v, s["decay"], s["dout"], dq, dk, dv, ws, state=s["state"], dnext_state=s["dnext"], dstate=dstate, done=s["done"],
                                scale=s["scale"])
    return dq, dk, dv, dstate


def absolute(s):
    return {n: (x.abs() if n in ("q", "k", "v", "dout", "state", "dnext") and x is not None else x) for n, x in s.items()}


def check(M, s, layout="tbhd", grad=True):
    q, k, v = s["q"], s["k"], s["v"]
    T, (Dk, Dv) = q.shape[0], (q.shape[3], v.shape[3])
    bf16, parts, group = q.dtype == BF16, PARTS[q.dtype], q.shape[2] // k.shape[2]
    n = 1.25 * T + max(Dk, Dv)
    out, nxt = forward(M, s, layout)
    a = absolute(s)
    args = lambda d: (d["q"], d["k"], d["v"], d["decay"], d["state"], d["done"], d["scale"])
    (ro, rs), (ao, as_) = O.attend(*args(s)), O.attend(*args(a))
    O.within(out, ro, ao, n, bf16, parts)
    O.within(nxt, rs, as_, n)
    if not grad:
        return
    got = backward(M, s, layout)
    args = lambda d: (d["q"], d["k"], d["v"], d["decay"], d["dout"], d["state"], d["dnext"], d["done"], d["scale"])
    ref, size = O.attend_backward(*args(s)), O.attend_backward(*args(a))
    for x, r, z in zip(got[:3], ref, size):
        O.within(x, r, z, n + group, bf16, parts)
    O.within(got[3], ref[3], size[3], n)


# widths on both sides of each padded width, lengths on both sides of the sixteen-step tiles
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,B,H,Hk,Dk,Dv", [
    (1, 1, 1, 1, 1, 1), (1, 5, 2, 1, 16, 16), (15, 3, 2, 2, 8, 24), (16, 6, 2, 2, 32, 32), (17, 4, 3, 1, 33, 31), (33, 2, 4, 2, 64, 64),
    (40, 3, 2, 2, 65, 17), (50, 2, 1, 1, 128, 128), (31, 2, 2, 1, 100, 127), (64, 70, 2, 2, 16, 48), (128, 9, 4, 4, 32, 64), (20, 2, 2, 2, 17, 128),
    (40, 3, 2, 2, 48, 80), (18, 2, 2, 1, 70, 44), (35, 2, 1, 1, 90, 112)])
def test_sequences(M, T, B, H, Hk, Dk, Dv, dtype):
    print("case", T, B, H, Hk, Dk, Dv, dtype, flush=True)
    check(M, make(T, B, H, Hk, Dk, Dv, dtype, seed=T + Dk))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("episode", [1, 2, 7, 40])
def test_episodes(M, episode, dtype):
    """Flags from every step to one in forty, shared by three agents, among them the first and the last step's."""
    s = make(53, 12, 2, 2, 32, 20, dtype, seed=episode, episode=episode, agents=3)
    s["done"][0, 1] = s["done"][-1, 2] = s["done"][15, 0] = s["done"][16, 0] = 1
    check(M, s)


# few sequences, cut over time: whole and ragged stretches, episodes that end inside and at their borders, shared heads
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,H,Hk,Dk,Dv,episode", [(512, 1, 1, 32, 32, 0), (1000, 4, 2, 40, 72, 90), (2049, 2, 1, 64, 128, 300), (700, 3, 3, 128, 128, 3)])
def test_long_sequences(M, T, H, Hk, Dk, Dv, episode, dtype):
    s = make(T, 2, H, Hk, Dk, Dv, dtype, seed=T, episode=episode, agents=2)
    if s["done"] is not None:
        for t in (63, 64, 127, 128, T - 1):
            s["done"][t] = 1
    assert M.linear_attention_workspace(s["q"], s["k"], s["v"]) > 0
    check(M, s)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", ["bhtd", "odd"])
def test_strides(M, layout, dtype):
    check(M, make(37, 6, 4, 2, 24, 40, dtype, episode=9, layout=layout), layout)


def test_broadcast_input(M):
    """One query for all steps (stride 0)."""
    s = make(30, 4, 2, 2, 32, 32, F32)
    s["q"] = s["q"][:1].expand(30, -1, -1, -1)
    check(M, s)


@pytest.mark.parametrize("value", [0.0, 1.0, 1e-30])
def test_decay_limits(M, value):
    s = make(40, 3, 2, 2, 16, 16, F32)
    s["decay"] = torch.full((2,), value, device="cuda")
    check(M, s)


def test_without_states(M):
    check(M, make(20, 3, 2, 2, 32, 32, BF16, state=False))
    s = make(20, 3, 2, 2, 32, 32, F32, state=False)
    out = empty(s["dout"].shape, F32)
    M.linear_attention(s["q"], s["k"], s["v"], s["decay"], out, None, scale=s["scale"])
    assert torch.equal(out, forward(M, s)[0])


def test_no_steps_and_no_sequences(M):
    s = make(0, 3, 2, 2, 8, 8, F32)
    out, nxt = forward(M, s)
    assert out.numel() == 0 and torch.equal(nxt, s["state"])
    assert torch.equal(backward(M, s)[3], s["dnext"])
    s["state"] = None
    assert not forward(M, s)[1].any()
    s = make(5, 0, 2, 2, 8, 8, F32)
    forward(M, s)
    backward(M, s)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_not_finite_stays_where_it_belongs(M, bad, dtype):
    """An infinity or a NaN in one step reaches that episode's later steps (its gradient: earlier ones) and nothing else."""
    done = torch.zeros((48, 2), dtype=torch.uint8, device="cuda")
    done[20] = done[37] = 1
    for name in ("q", "k", "v", "dout"):
        s = make(48, 2, 2, 2, 32, 32, dtype, seed=3)
        s["done"] = done
        clean = forward(M, s) + backward(M, s)
        s[name][25, 0, 1, 5] = bad
        out, nxt, dq, dk, dv, dstate = forward(M, s) + backward(M, s)
        args = (s["q"], s["k"], s["v"], s["decay"])
        ref = O.attend(*args, s["state"], done, s["scale"]) + O.attend_backward(*args, s["dout"], s["state"], s["dnext"], done, s["scale"])
        for x, r, c, what in zip((out, nxt, dq, dk, dv, dstate), ref, clean, ("out", "next_state", "dq", "dk", "dv", "dstate")):
            assert torch.equal(x.isfinite(), r.isfinite()), (name, what)
            assert torch.equal(x.isnan(), r.isnan()), (name, what)
            inside = torch.zeros_like(x, dtype=torch.bool)
            if x.shape[0] == 48:
                inside[21:38, 0, 1] = True
            ok = ~inside & x.isfinite()
            O.within(torch.where(ok, x.double(), 0.0), torch.where(ok, c.double(), 0.0), torch.ones_like(x, dtype=torch.float64) * 64, 200, dtype == BF16, 2.0 ** -15)


def test_infinite_state_is_dropped_with_its_episode(M):
    s = make(20, 2, 1, 1, 16, 16, F32)
    s["done"] = torch.zeros((20, 2), dtype=torch.uint8, device="cuda")
    s["done"][3] = 1
    s["state"][0, 0, 2, 3] = float("inf")
    out, nxt = forward(M, s)
    assert not out[:4, 0, 0, 3].isfinite().any() and out[4:].isfinite().all() and out[:, 1].isfinite().all() and nxt.isfinite().all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,H,Hk,Dk,Dv", [(1, 1, 1, 1, 1), (3, 2, 1, 16, 16), (6, 4, 4, 32, 32), (5, 6, 2, 40, 72), (2, 2, 2, 128, 128), (4, 3, 3, 63, 65), (2, 1, 1, 5, 127), (2, 2, 1, 100, 7)])
def test_steps(M, B, H, Hk, Dk, Dv, dtype):
    """One step at a time gives what the whole sequence gives."""
    T = 6
    s = make(T, B, H, Hk, Dk, Dv, dtype, seed=Dk, episode=3)
    (ref, rs), (size, ss) = (O.attend(d["q"], d["k"], d["v"], d["decay"], d["state"], d["done"], d["scale"]) for d in (s, absolute(s)))
    S = s["state"].clone()
    for t in range(T):
        out = empty(ref.shape[1:], dtype)
        M.linear_attention_step(s["q"][t], s["k"][t], s["v"][t], s["decay"], S, out, done=s["done"][t - 1] if t else None, scale=s["scale"])
        O.within(out, ref[t], size[t], 2 * T + Dk, dtype == BF16)
    S = torch.where(s["done"][-1].bool()[:, None, None, None], 0.0, S)
    O.within(S, rs, ss, 2 * T)


def test_step_keeps_the_state_it_is_not_asked_to_change(M):
    s = make(1, 4, 2, 2, 32, 32, F32)
    before, nxt, out = s["state"].clone(), torch.empty_like(s["state"]), empty((4, 2, 32), F32)
    s["state"][1, 0, 3, 3] = float("inf")
    first = torch.tensor([0, 1, 0, 0], dtype=torch.uint8, device="cuda")
    M.linear_attention_step(s["q"][0], s["k"][0], s["v"][0], s["decay"], s["state"], out, next_state=nxt, done=first, scale=1.0)
    s["state"][1, 0, 3, 3] = before[1, 0, 3, 3]
    assert torch.equal(s["state"], before) and nxt.isfinite().all() and out.isfinite().all()


def test_gradient_against_differences(M):
    """out and next_state are linear in each of q, k, v and the state by itself: a difference of any size is the derivative."""
    s = make(45, 4, 4, 2, 24, 20, F32, seed=5, episode=15, agents=2)
    got = dict(zip(("q", "k", "v", "state"), backward(M, s)))
    loss = lambda d: sum(float((x * w.double()).sum()) for x, w in zip(O.attend(d["q"], d["k"], d["v"], d["decay"], d["state"], d["done"], d["scale"]), (s["dout"], s["dnext"])))
    g = torch.Generator(device="cuda").manual_seed(9)
    for name, grad in got.items():
        d = torch.randn(s[name].shape, generator=g, device="cuda").double()
        up, down = ({**s, name: s[name].double() + e * d} for e in (0.5, -0.5))
        diff, dot = loss(up) - loss(down), float((grad.double() * d).sum())
        # each gradient element carries at most 2^-24 (additions + 40) of its terms: 1e-5 of its own scale here
        assert abs(diff - dot) <= 1e-5 * float((grad.double() * d).abs().sum()), name


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_same_bits_twice_and_on_another_stream(M, dtype):
    s = make(600, 3, 4, 2, 48, 64, dtype, episode=50)
    a = forward(M, s) + backward(M, s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b = forward(M, s) + backward(M, s)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_graph_replays(M):
    s = make(200, 2, 2, 1, 32, 32, BF16, episode=30)
    q, k, v = s["q"], s["k"], s["v"]
    ws = M.alloc_workspace(M.linear_attention_workspace(q, k, v, backward=True))
    out, dq, dk, dv = (torch.empty_like(x) for x in (s["dout"], q, k, v))

    def call():
        M.linear_attention(q, k, v, s["decay"], out, ws, state=s["state"], done=s["done"], scale=s["scale"])
        M.linear_attention_backward(q, k, v, s["decay"], s["dout"], dq, dk, dv, ws, state=s["state"], done=s["done"], scale=s["scale"])
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (1, 2, 3):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        call()
        want = [x.clone() for x in (out, dq, dk, dv)]
        for x in (out, dq, dk, dv):
            x.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, (out, dq, dk, dv)))


def test_offsets_past_32_bits(M):
    """Steps 1.2 G elements apart in one 7 GB buffer."""
    far = 1_200_000_000
    whole = torch.empty(2 * far + 4096, dtype=BF16, device="cuda")
    big = torch.as_strided(whole, (3, 2, 2, 32), (far, 64, 32, 1))
    s = make(3, 2, 2, 2, 32, 32, BF16)
    out, nxt = forward(M, s)
    big.copy_(s["k"])
    s["k"] = big
    o2, n2 = forward(M, s)
    assert torch.equal(out, o2) and torch.equal(nxt, n2)
    M.linear_attention(s["q"], s["k"].clone(), s["v"], s["decay"], big, None, state=s["state"], scale=s["scale"])
    assert torch.equal(out, big)
