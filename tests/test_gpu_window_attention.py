"""Attention over a window with first steps: whole rollouts, gradients, single steps and caches against 64 bits."""
import math

import pytest
import torch

import window_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
NAMES = {F32: "f32", BF16: "bf16"}


@pytest.fixture(scope="module")
def M():
    import paper_2107_01460_amd as m
    assert torch.cuda.is_available()
    return m


def positions_for(kind, T, envs, span, g):
    """[T][envs] int32, or None"""
    rand = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device="cuda")
    t = torch.arange(T, device="cuda")[:, None]
    if kind == "none":
        return None
    if kind == "any":      # positions that do not count up
        return rand(-2, 60, T, envs).int()
    begun = -rand(0, 2 * span + 3, envs)[None].expand(T, envs)
    if kind == "whole":
        begun = torch.zeros_like(begun)
    if kind in ("episodes", "ragged", "rare"):
        ended = torch.rand((T, envs), generator=g, device="cuda") < (0.004 if kind == "rare" else 0.06)
        begun = torch.where(ended, t, begun).cummax(0).values
    p = t - begun
    if kind == "ragged":
        length = rand(0, T + 1, envs)
        length[0] = 0
        p = torch.where(t < length, p, -1)
    return p.int()


class Case:
    def __init__(self, T, envs, agents, H, Hk, Dk, Dv, dtype, window, sinks, kind, cached, seed=0):
        self.__dict__.update(locals())
        g = self.g = torch.Generator(device="cuda").manual_seed(seed)
        B = self.B = envs * agents
        randn = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)
        self.q, self.k, self.v, self.dout = randn(T, B, H, Dk), randn(T, B, Hk, Dk), randn(T, B, Hk, Dv), randn(T, B, H, Dv)
        self.positions = positions_for(kind, T, envs, window + sinks, g)
        slots = window + sinks
        self.cache = (randn(B, Hk, slots, Dk), randn(B, Hk, slots, Dv)) if cached else None
        self.scale = Dk ** -0.5

    def forward(self, M, next_cache=None, lse=True, first=0):
        out = torch.full((self.T, self.B, self.H, self.Dv), 7.0, dtype=self.dtype, device="cuda")
        lse = torch.full((self.B, self.H, self.T), 7.0, device="cuda") if lse else None
        M.window_attention(self.q, self.k, self.v, out, self.window, self.sinks, lse=lse, positions=self.positions, cache=self.cache, next_cache=next_cache,
                           scale=self.scale, first_position=first)
        return out, lse

    def backward(self, M, out, lse, dout=None, first=0):
        dq, dk, dv = (torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda") for x in (self.q, self.k, self.v))
        ws = M.alloc_workspace(M.window_attention_workspace(self.q, self.k, self.v, self.window, self.sinks, kind="backward"))
        ws.fill_(255)
        M.window_attention_backward(self.q, self.k, self.v, out, lse, self.dout if dout is None else dout, dq, dk, dv, self.window, self.sinks,
                                    positions=self.positions, cache=self.cache, scale=self.scale, workspace=ws, first_position=first)
        return dq, dk, dv

    def oracle(self, first=0):
        return O.Attention(self.q, self.k, self.v, self.window, self.sinks, self.positions, first, self.cache, self.scale)


def check(M, c, first=0):
    ref = c.oracle(first)
    out, lse = c.forward(M, first=first)
    want, bound, want_lse, lse_bound = ref.forward(c.Dv)
    empty = ~ref.seen.any(3).expand(-1, c.H, -1)
    want = torch.where(empty.permute(2, 0, 1)[..., None], 0.0, want)
    O.within(out, want, bound, "out")
    O.within(lse, want_lse, lse_bound, "lse")
    assert torch.equal(out[empty.permute(2, 0, 1)], torch.zeros_like(out[empty.permute(2, 0, 1)]))
    for name, got, (g, b) in zip(("dq", "dk", "dv"), c.backward(M, out, lse, first=first), ref.backward(out, lse, c.dout)):
        O.within(got, g, b, name)


# (steps, environments, agents, heads, kv heads, dk, dv, window, sinks, positions, cache): each wavefront count, tiles on both sides of 32 and 64, widths on
# both sides of every instance, windows inside, at and across tiles, first steps that fill more than a tile
CASES = [
    (1, 3, 2, 2, 2, 32, 32, 8, 1, "episodes", True), (1, 1, 1, 1, 1, 1, 1, 1, 0, "none", False), (2, 2, 1, 4, 2, 16, 8, 1, 0, "whole", False),
    (16, 4, 2, 2, 2, 32, 32, 8, 1, "episodes", True), (31, 3, 1, 3, 1, 33, 20, 5, 2, "episodes", True), (32, 2, 2, 4, 4, 64, 64, 32, 4, "whole", False),
    (33, 2, 2, 4, 1, 64, 64, 31, 0, "episodes", False), (64, 2, 1, 2, 1, 40, 72, 33, 3, "ragged", True), (65, 3, 1, 6, 2, 128, 128, 64, 4, "episodes", True),
    (100, 2, 2, 8, 2, 96, 96, 7, 1, "episodes", True), (128, 2, 2, 4, 4, 32, 32, 32, 2, "ragged", True), (200, 1, 2, 4, 2, 64, 64, 1000, 0, "none", False),
    (200, 2, 1, 8, 2, 128, 128, 50, 40, "going", True), (150, 2, 1, 6, 2, 40, 72, 20, 70, "episodes", True), (97, 2, 1, 5, 5, 127, 65, 11, 3, "any", True),
    (130, 2, 2, 3, 3, 5, 3, 100, 4, "any", False), (70, 1, 3, 2, 2, 100, 7, 66, 1, "ragged", False), (300, 1, 1, 4, 1, 128, 64, 64, 4, "going", False),
    (260, 1, 1, 1, 1, 64, 128, 3, 33, "whole", False), (48, 2, 1, 7, 1, 24, 24, 16, 4, "going", True),
    # first steps that many tiles of rows see from beyond the window: of one episode, of several, more tiles of them than there are places, positions that do not count up
    (900, 1, 1, 4, 1, 32, 32, 20, 4, "whole", False), (700, 2, 1, 2, 1, 64, 64, 33, 40, "rare", False), (1000, 1, 2, 6, 2, 128, 96, 50, 4, "rare", True),
    (1500, 1, 1, 1, 1, 16, 16, 10, 400, "whole", False), (600, 1, 1, 2, 2, 32, 32, 7, 3, "any", True), (2500, 1, 1, 4, 2, 40, 40, 64, 2, "rare", False)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_against_64_bits(M, case, dtype):
    T, envs, agents, H, Hk, Dk, Dv, window, sinks, kind, cached = case
    check(M, Case(T, envs, agents, H, Hk, Dk, Dv, dtype, window, sinks, kind, cached, seed=T))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("waves", [20, 50, 90])
@pytest.mark.parametrize("D", [32, 64, 96, 128])
def test_every_instance(M, D, waves, dtype):
    check(M, Case(waves, 2, 1, 2, 2, D, D, dtype, 40, 2, "episodes", True, seed=D + waves))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("first", [0, 5, 40, -3, -50])
def test_positions_by_number(M, first, dtype):
    check(M, Case(40, 2, 1, 2, 1, 32, 48, dtype, 12, 2, "none", True, seed=3), first=first)


@pytest.mark.parametrize("scale", [-0.3, 0.0, 3.0])
def test_scales(M, scale):
    for dtype in (F32, BF16):
        c = Case(70, 2, 1, 2, 1, 32, 32, dtype, 40, 2, "episodes", True, seed=4)
        c.scale = scale
        check(M, c)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_strides(M, dtype):
    """Queries, keys and values as columns of one product; sequence-major storage; keys and values that all sequences share; rows that begin at odd addresses."""
    c = Case(50, 3, 2, 4, 2, 24, 24, dtype, 20, 2, "episodes", False, seed=5)
    want, lse = c.forward(M)
    grads = c.backward(M, want, lse)
    fused = torch.cat([c.q, c.k, c.v], 2)
    views = fused.split([4, 2, 2], 2)
    major = [x.permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3) for x in (c.q, c.k, c.v)]
    odd = []
    for x in (c.q, c.k, c.v):
        y = torch.zeros((*x.shape[:3], x.shape[3] + 3), dtype=dtype, device="cuda")
        y[..., 1:-2] = x
        odd.append(y[..., 1:-2])
    for q, k, v in (views, major, odd):
        d = Case(50, 3, 2, 4, 2, 24, 24, dtype, 20, 2, "episodes", False, seed=5)
        d.q, d.k, d.v = q, k, v
        got, got_lse = d.forward(M)
        assert torch.equal(got, want) and torch.equal(got_lse, lse)
        assert all(torch.equal(a, b) for a, b in zip(d.backward(M, got, got_lse), grads))
        wide = [torch.zeros((*x.shape[:3], x.shape[3] + 5), dtype=dtype, device="cuda")[..., 3:-2] for x in (c.q, c.k, c.v)]
        ws = M.alloc_workspace(M.window_attention_workspace(q, k, v, 20, 2, kind="backward"))
        M.window_attention_backward(q, k, v, got, got_lse, c.dout, *wide, 20, 2, positions=c.positions, scale=c.scale, workspace=ws)
        assert all(torch.equal(a, b) for a, b in zip(wide, grads))
        out = torch.zeros((*got.shape[:3], 29), dtype=dtype, device="cuda")
        M.window_attention(q, k, v, out[..., 1:25], 20, 2, positions=c.positions, scale=c.scale)
        assert torch.equal(out[..., 1:25], want) and not out[..., 0].any() and not out[..., 25:].any()
    c.k, c.v = (x[:, :1].expand(-1, c.B, -1, -1) for x in (c.k, c.v))
    check(M, c)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_broadcast_gradient(M, dtype):
    """The gradient of a sum: one number for all elements."""
    c = Case(40, 2, 1, 2, 2, 32, 32, dtype, 16, 1, "episodes", False, seed=6)
    c.dout = torch.ones((1, 1, 1, 32), dtype=dtype, device="cuda").expand(40, 2, 2, 32)
    check(M, c)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("case", [(16, 4, 2, 2, 2, 32, 32, 8, 1, "episodes"), (90, 3, 1, 4, 2, 40, 72, 20, 3, "ragged"), (5, 2, 1, 1, 1, 7, 9, 30, 0, "going"),
                                  (1, 2, 2, 2, 1, 64, 64, 6, 2, "episodes"), (200, 2, 1, 2, 2, 16, 16, 150, 2, "whole"), (40, 3, 1, 2, 1, 16, 24, 11, 4, "any")])
def test_cache_behind_the_call(M, case, dtype):
    """Copies, so bit for bit; slots that hold nothing as they were; in place; without a cache before the call."""
    T, envs, agents, H, Hk, Dk, Dv, window, sinks, kind = case
    c = Case(T, envs, agents, H, Hk, Dk, Dv, dtype, window, sinks, kind, True, seed=T)
    new = tuple(torch.full_like(x, 5.0) for x in c.cache)
    want = [O.next_cache(x, old, n, c.positions, 0, window, sinks) for x, old, n in zip((c.k, c.v), c.cache, new)]
    out, _ = c.forward(M, next_cache=new)
    assert all(torch.equal(a, b) for a, b in zip(new, want))
    in_place = [O.next_cache(x, old, old, c.positions, 0, window, sinks) for x, old in zip((c.k, c.v), c.cache)]
    again, _ = c.forward(M, next_cache=c.cache, lse=False)
    assert torch.equal(out, again) and all(torch.equal(a, b) for a, b in zip(c.cache, in_place))
    c.cache = None
    new = tuple(torch.full_like(x, 5.0) for x in new)
    want = [O.next_cache(x, None, n, c.positions, 0, window, sinks) for x, n in zip((c.k, c.v), new)]
    c.forward(M, next_cache=new)
    assert all(torch.equal(a, b) for a, b in zip(new, want))


def steps(M, c, cache, t0=0):
    """The case's steps one at a time"""
    ws = M.alloc_workspace(M.window_attention_workspace(c.q, c.k, c.v, c.window, c.sinks, kind="step"))
    out = torch.full((c.T, c.B, c.H, c.Dv), 7.0, dtype=c.dtype, device="cuda")
    for t in range(t0, c.T):
        M.window_attention_step(c.q[t], c.k[t], c.v[t], cache, c.positions[t].contiguous(), out[t], c.window, c.sinks, scale=c.scale, workspace=ws)
    return out


STEP_CASES = [(30, 4, 2, 2, 2, 32, 32, 8, 1, "episodes"), (40, 3, 1, 4, 2, 40, 72, 20, 3, "ragged"), (25, 2, 1, 8, 1, 128, 128, 9, 0, "episodes"),
              (12, 2, 1, 3, 1, 5, 3, 4, 2, "going"), (20, 2, 2, 6, 2, 64, 64, 1, 0, "episodes"), (20, 1, 1, 10, 2, 100, 16, 6, 7, "whole"), (9, 1, 2, 2, 1, 16, 4, 300, 4, "going"),
              (6, 1, 1, 8, 2, 128, 128, 3001, 4, "going"), (5, 2, 1, 1, 1, 63, 65, 1111, 1, "going"), (4, 1, 1, 5, 1, 1, 1, 5000, 0, "going"), (4, 1, 2, 4, 4, 8, 128, 2000, 2, "ragged")]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("case", STEP_CASES, ids=lambda c: "-".join(map(str, c)))
def test_single_steps(M, case, dtype):
    """A whole rollout and its steps one at a time, and the caches that both leave."""
    T, envs, agents, H, Hk, Dk, Dv, window, sinks, kind = case
    c = Case(T, envs, agents, H, Hk, Dk, Dv, dtype, window, sinks, kind, True, seed=T)
    whole = tuple(x.clone() for x in c.cache)
    acting = tuple(x.clone() for x in c.cache)
    ref = c.oracle()
    want, bound, *_ = ref.forward(Dv)
    empty = ~ref.seen.any(3).expand(-1, H, -1).permute(2, 0, 1)
    want = torch.where(empty[..., None], 0.0, want)
    O.within(steps(M, c, acting), want, bound, "steps")
    before = c.cache
    c.cache = whole
    c.forward(M, next_cache=whole)
    # a slot that an episode which ended had reached, and the one after it has not, differs: nothing reads it
    at = O.positions_of(c.positions, 0, T, c.B, "cuda")
    for b in range(c.B):
        rows = [t for t in range(T) if at[t, b] >= 0]
        n = int(at[rows[-1], b]) + 1 if rows else window + sinks
        held = [s for s in range(window + sinks) if O.slot_step(s, n, window, sinks) >= 0]
        for x, y in zip(whole, acting):
            assert torch.equal(x[b][:, held], y[b][:, held])
    assert before is not c.cache


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_rollouts_one_after_another(M, dtype):
    """A recording in one call, and in pieces that hand the cache on."""
    c = Case(120, 3, 1, 4, 2, 32, 40, dtype, 24, 3, "episodes", True, seed=8)
    want, bound, *_ = c.oracle().forward(c.Dv)
    cache, got = tuple(x.clone() for x in c.cache), []
    for a, b in ((0, 1), (1, 30), (30, 94), (94, 120)):
        out = torch.empty((b - a, c.B, c.H, c.Dv), dtype=dtype, device="cuda")
        M.window_attention(c.q[a:b], c.k[a:b], c.v[a:b], out, c.window, c.sinks, positions=c.positions[a:b].contiguous(), cache=cache, next_cache=cache, scale=c.scale)
        got.append(out)
    O.within(torch.cat(got), want, bound)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("D,H,Hk", [(32, 2, 2), (64, 4, 1), (128, 2, 1)])
def test_infinities_and_nans_that_a_row_does_not_see(M, D, H, Hk, dtype):
    """In keys, values, queries, gradients and in the cache: a row's results are those without them, unless it sees them."""
    c = Case(110, 2, 1, H, Hk, D, D, dtype, 20, 2, "whole", True, seed=9)
    c.positions[:, 1] += 30   # sequence 1 goes on from the cache
    bad = {"k": (0, 40), "v": (0, 70), "q": (0, 50)}
    for value in (math.inf, -math.inf, math.nan):
        d = Case(110, 2, 1, H, Hk, D, D, dtype, 20, 2, "whole", True, seed=9)
        d.positions = c.positions
        for name, (b, t) in bad.items():
            getattr(d, name)[t, b, 0, 3] = value
        d.cache[1][1, 0, 2 + 9] = value        # step 11 of sequence 1: out of the window, which reaches back to steps 11..29 from row 0 on
        d.cache[0][0] = value                   # sequence 0 begins with the call: its cache holds nothing
        d.cache[1][0] = value
        out, lse = d.forward(M)
        clean = Case(110, 2, 1, H, Hk, D, D, dtype, 20, 2, "whole", True, seed=9)
        clean.positions = c.positions
        ref = clean.oracle()
        want, bound, want_lse, lse_bound = ref.forward(D)
        hit = torch.zeros((110, 2, H), dtype=torch.bool, device="cuda")
        group = H // Hk
        hit[40:60, 0, :group] = True
        hit[70:90, 0, :group] = True
        hit[50, 0, 0] = True
        hit[0, 1, :group] = True                # row 0 is at step 30 and sees steps 11..30
        O.within(torch.where(hit[..., None], 0.0, out.double()), torch.where(hit[..., None], 0.0, want), bound, "out")
        nan_rows = out[70:90, 0, :group, 3]     # a value seen shows (an infinity with a weight; a NaN)
        assert not torch.isfinite(nan_rows).any()
        assert torch.isfinite(out[:, :, :, :3][~hit]).all()
        # gradient: from the clean outputs, so that only the operands carry infinities
        out, lse = clean.forward(M)
        grads = ref.backward(out, lse, clean.dout)
        dout = clean.dout.clone()
        dout[100, 0, 0, 5] = value
        dq, dk, dv = d.backward(M, out, lse, dout=dout)
        rows = torch.zeros((110, 2, H), dtype=torch.bool, device="cuda")      # rows of dq that see or hold something
        rows[40:60, 0, :group] = rows[70:90, 0, :group] = True
        rows[50, 0, 0] = rows[100, 0, 0] = rows[0, 1, :group] = True
        O.within(torch.where(rows[..., None], 0.0, dq.double()), torch.where(rows[..., None], 0.0, grads[0][0]), grads[0][1], "dq")
        cols = torch.zeros((110, 2, Hk), dtype=torch.bool, device="cuda")     # columns that such a row sees
        cols[20:90, 0, 0] = cols[81:101, 0, 0] = cols[:2, 0, 0] = True
        cols[0, 1, 0] = True
        for name, got, (g, b) in (("dk", dk, grads[1]), ("dv", dv, grads[2])):
            O.within(torch.where(cols[..., None], 0.0, got.double()), torch.where(cols[..., None], 0.0, g), b, name)


def test_a_row_that_sees_infinite_scores(M):
    """As the formula has it: a score of +infinity makes its row NaN, one of -infinity takes no part."""
    c = Case(10, 1, 1, 1, 1, 8, 8, F32, 4, 0, "whole", False, seed=10)
    c.q[:, 0, 0, 0], c.q[:, 0, 0, 1:], c.k[3, 0, 0, 0] = 1.0, 0.0, -math.inf
    out, lse = c.forward(M)
    d = c.oracle()
    P = torch.softmax(torch.where(d.seen, d.s, -math.inf), -1)
    want = torch.matmul(P, d.V).permute(2, 0, 1, 3)
    assert float((out.double() - want).abs().max()) < 1e-5 and torch.isfinite(lse).all()
    c.k[3, 0, 0, 0] = math.inf
    out, lse = c.forward(M)
    assert out[3:7].isnan().all() and torch.isfinite(out[:3]).all() and torch.isfinite(out[7:]).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_gradient_against_differences(M, dtype):
    """Along a direction, through the formula in 64 bits."""
    c = Case(40, 2, 1, 4, 2, 16, 24, dtype, 12, 2, "episodes", True, seed=11)
    out, lse = c.forward(M)
    grads = c.backward(M, out, lse)
    e, bound = 1e-5, [b for _, b in c.oracle().backward(out, lse, c.dout)]
    base = {"q": c.q, "k": c.k, "v": c.v}
    for (name, x), g, b in zip(base.items(), grads, bound):
        d = torch.randn(x.shape, generator=c.g, device="cuda", dtype=torch.float64)
        loss = []
        for sign in (1, -1):
            a = {**base, name: x.double() + sign * e * d}
            o, *_ = O.Attention(a["q"], a["k"], a["v"], c.window, c.sinks, c.positions, 0, c.cache, c.scale).forward(24)
            loss.append(float((o * c.dout.double()).sum()))
        # delta comes from the output as it was rounded: what that adds to the gradient is below the output's rounding times the gradient's terms
        rounding = (2.0 ** -8 if dtype == BF16 else 2.0 ** -22) * float((g.double().abs() * d.abs()).sum()) * 4
        assert abs((loss[0] - loss[1]) / (2 * e) - float((g.double() * d).sum())) <= float((b * d.abs()).sum()) + rounding + 1e-6


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_twice_the_same(M, dtype):
    c = Case(300, 4, 2, 4, 2, 64, 64, dtype, 70, 3, "episodes", True, seed=12)
    out, lse = c.forward(M)
    grads = c.backward(M, out, lse)
    for _ in range(3):
        again, lse2 = c.forward(M)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
        assert all(torch.equal(a, b) for a, b in zip(grads, c.backward(M, out, lse)))


def test_no_steps_no_sequences(M):
    for T, envs in ((0, 3), (4, 0), (0, 0)):
        c = Case(T, envs, 1, 2, 1, 16, 16, F32, 4, 1, "none", True, seed=1)
        new = tuple(torch.zeros_like(x) for x in c.cache)
        out, lse = c.forward(M, next_cache=new)
        c.backward(M, out, lse)
        if T == 0:
            assert all(torch.equal(a, b) for a, b in zip(new, c.cache))


def test_another_stream(M):
    c = Case(64, 3, 1, 4, 2, 64, 64, BF16, 20, 2, "episodes", True, seed=13)
    want, want_lse = c.forward(M)
    grads = c.backward(M, want, want_lse)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        out, lse = c.forward(M)
        got = c.backward(M, out, lse)
    s.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and all(torch.equal(a, b) for a, b in zip(got, grads))


def test_replayed(M):
    """A rollout, its gradient and a step in one graph; the caller's data change between replays, and eager calls with their own workspaces run there too."""
    c = Case(50, 3, 2, 4, 2, 32, 32, BF16, 20, 2, "episodes", True, seed=14)
    e = Case(6, 1, 1, 8, 2, 128, 128, BF16, 3000, 4, "going", True, seed=15)
    out, lse = torch.empty_like(c.dout), torch.empty((c.B, c.H, c.T), device="cuda")
    dq, dk, dv, new = torch.empty_like(c.q), torch.empty_like(c.k), torch.empty_like(c.v), tuple(torch.zeros_like(x) for x in c.cache)
    ws = M.alloc_workspace(M.window_attention_workspace(c.q, c.k, c.v, 20, 2, kind="backward"))
    ws2 = M.alloc_workspace(M.window_attention_workspace(e.q, e.k, e.v, 3000, 4, kind="step"))
    row, at = torch.empty((1, 8, 128), dtype=BF16, device="cuda"), e.positions[0].contiguous()

    def work():
        M.window_attention(c.q, c.k, c.v, out, 20, 2, lse=lse, positions=c.positions, cache=c.cache, next_cache=new, scale=c.scale)
        M.window_attention_backward(c.q, c.k, c.v, out, lse, c.dout, dq, dk, dv, 20, 2, positions=c.positions, cache=c.cache, scale=c.scale, workspace=ws)
        M.window_attention_step(e.q[0], e.k[0], e.v[0], e.cache, at, row, 3000, 4, scale=e.scale, workspace=ws2)

    work()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for n in range(4):
        c.q.copy_(torch.randn(c.q.shape, generator=c.g, device="cuda"))
        e.q.copy_(torch.randn(e.q.shape, generator=c.g, device="cuda"))
        for x in (out, lse, dq, dk, dv, row, *new):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, lse, dq, dk, dv, row, *new)]
        for x in (out, lse, dq, dk, dv, row, *new):
            x.zero_()
        work()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, dq, dk, dv, row, *new))), n


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_a_cache_past_32_bits(M, dtype):
    """Offsets in elements past 2^31: a cache of 2^31 and some elements, its last sequence's results those of the sequence alone."""
    window, Hk, D = 65536, 2, 128
    B = 2 ** 31 // (window * Hk * D) + 1
    g = torch.Generator(device="cuda").manual_seed(1)
    cache = tuple(torch.zeros((B, Hk, window, D), dtype=dtype, device="cuda") for _ in range(2))
    for x in cache:
        x[-1] = torch.randn((Hk, window, D), generator=g, device="cuda").to(dtype)
    q, k, v = (torch.randn((1, B, h, D), generator=g, device="cuda").to(dtype) for h in (4, Hk, Hk))
    p = torch.full((B,), 200000, dtype=torch.int32, device="cuda")
    alone = tuple(x[-1:].clone() for x in cache)
    ws = M.alloc_workspace(max(M.window_attention_workspace(x, y, y, window, 0, kind="step") for x, y in ((q, k), (q[:, -1:], k[:, -1:]))))
    out, one = torch.empty_like(q), torch.empty_like(q[:, -1:])
    M.window_attention(q, k, v, out, window, 0, positions=p[None], cache=cache, scale=D ** -0.5)
    M.window_attention(q[:, -1:], k[:, -1:], v[:, -1:], one, window, 0, positions=p[None, -1:], cache=alone, scale=D ** -0.5)
    assert torch.equal(out[:, -1:], one)
    whole = out.clone()
    M.window_attention_step(q[0], k[0], v[0], cache, p, out[0], window, 0, scale=D ** -0.5, workspace=ws)
    assert float((out[0, -1].float() - whole[0, -1].float()).abs().max()) <= (2e-6 if dtype == F32 else 2.0 ** -7 * float(whole[0, -1].float().abs().max()))
    slot = 200000 % window
    assert torch.equal(cache[0][-1, :, slot], k[0, -1]) and torch.equal(cache[1][-1, :, slot], v[0, -1])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_far_positions(M, dtype):
    """Positions up to the largest number, windows and first steps up to the largest there are."""
    c = Case(40, 2, 1, 2, 1, 32, 32, dtype, 12, 3, "whole", True, seed=16)
    c.positions += 2 ** 31 - 1 - 39
    check(M, c)
    step = Case(1, 2, 1, 2, 1, 32, 32, dtype, 12, 3, "whole", True, seed=17)
    step.positions += 2 ** 31 - 1
    want, bound, *_ = step.oracle().forward(32)
    O.within(steps(M, step, step.cache), want, bound)
    c = Case(40, 2, 1, 2, 1, 32, 32, dtype, 2 ** 29, 2 ** 29, "going", False, seed=18)
    check(M, c)
