"""The norm of heads with their rotation in one pass, and its gradient, against 64 bits."""
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


def table_of(P, R):
    angle = torch.arange(P, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * torch.arange(R // 2, dtype=torch.float64) / R)
    return torch.cat([angle.cos(), angle.sin()], 1).float().cuda()


class Case:
    def __init__(self, T, envs, agents, H, Hk, D, R, dtype, P=300, seed=0):
        self.__dict__.update(locals())
        g = torch.Generator(device="cuda").manual_seed(seed)
        B = self.B = envs * agents
        randn = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.q, self.k, self.dq, self.dk = (randn(T, B, h, D).mul(1.5).to(dtype) for h in (H, Hk, H, Hk))
        self.wq, self.wk = 1 + 0.3 * randn(D), 1 + 0.3 * randn(D)
        self.table = table_of(P, R)
        self.positions = torch.randint(0, P, (T, envs), generator=g, device="cuda").int()

    def at(self):
        return self.positions.long().repeat_interleave(self.agents, 1)


def rounded(bound, ref, dtype):
    return bound * (1 + O.U16) + O.U16 * ref.abs() if dtype == BF16 else bound + O.U32 * ref.abs()


def check(M, c, interleaved, eps=1e-6):
    at = c.at()
    qo, ko = torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0)
    M.norm_rotary(c.q, c.k, c.wq, c.wk, c.table, qo, ko, eps=eps, positions=c.positions, interleaved=interleaved)
    for x, w, y in ((c.q, c.wq, qo), (c.k, c.wk, ko)):
        ref, bound = O.norm_rotary(x, w, c.table, at, eps, interleaved)
        O.within(y, ref, rounded(bound, ref, c.dtype), "y")
    gq, gk, gwq, gwk = torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0), torch.full((c.D,), 7.0, device="cuda"), torch.full((c.D,), 7.0, device="cuda")
    ws = M.alloc_workspace(M.norm_rotary_workspace(c.q, c.k))
    ws.fill_(255)
    M.norm_rotary_backward(c.dq, c.dk, c.q, c.k, c.wq, c.wk, c.table, gq, gk, gwq, gwk, ws, eps=eps, positions=c.positions, interleaved=interleaved)
    for x, w, dy, dx, dw in ((c.q, c.wq, c.dq, gq, gwq), (c.k, c.wk, c.dk, gk, gwk)):
        (ref, bound), (ref_w, bound_w) = O.norm_rotary_backward(dy, x, w, c.table, at, eps, interleaved)
        O.within(dx, ref, rounded(bound, ref, c.dtype), "dx")
        O.within(dw, ref_w, bound_w, "dw")
    return qo, ko, gq, gk, gwq, gwk


# widths on both sides of every team of lanes; rotated parts that end and turn inside a vector
WIDTHS = [(2, 2), (3, 2), (4, 4), (7, 6), (8, 8), (9, 4), (16, 8), (24, 12), (31, 30), (32, 32), (33, 32), (40, 20), (64, 32), (64, 6), (80, 48), (127, 126),
          (128, 128), (130, 66), (255, 254), (256, 256)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R", WIDTHS)
def test_against_64_bits(M, D, R, interleaved, dtype):
    check(M, Case(5, 3, 2, 3, 2, D, R, dtype, seed=D), interleaved)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_many_rows(M, dtype):
    """More rows than the gradient's workgroups take at once, the weights' sums the same twice."""
    c = Case(70, 60, 3, 5, 1, 48, 24, dtype, seed=1)
    first, again = check(M, c, False), check(M, c, False)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("D,R", [(32, 16), (36, 20), (50, 26)])
def test_strides_in_place_and_alone(M, D, R, dtype):
    c = Case(6, 2, 2, 4, 2, D, R, dtype, seed=2)
    want_q, want_k, gq, gk, gwq, gwk = check(M, c, False)
    fused = torch.cat([c.q, c.k, c.k], 2)
    before = fused.clone()
    q, k = fused[:, :, :4], fused[:, :, 4:6]
    M.norm_rotary(q, k, c.wq, c.wk, c.table, q, k, positions=c.positions)          # in place, inside one array
    assert torch.equal(q, want_q) and torch.equal(k, want_k) and torch.equal(fused[:, :, 6:], before[:, :, 6:])
    major = c.q.permute(1, 2, 0, 3).contiguous().permute(2, 0, 1, 3)
    odd = torch.zeros((6, 4, 4, D + 3), dtype=dtype, device="cuda")
    M.norm_rotary(major, None, c.wq, None, c.table, odd[..., 1:-2], None, positions=c.positions)
    assert torch.equal(odd[..., 1:-2], want_q) and not odd[..., 0].any() and not odd[..., -2:].any()
    grad = c.dq.clone()
    only = torch.empty(D, device="cuda")
    M.norm_rotary_backward(grad, None, c.q, None, c.wq, None, c.table, grad, None, only, None, M.alloc_workspace(M.norm_rotary_workspace(c.q, None)), positions=c.positions)
    assert torch.equal(grad, gq) and torch.equal(only, gwq)
    plain, ones = torch.empty_like(c.q), torch.ones(D, device="cuda")
    other = torch.empty_like(c.q)
    M.norm_rotary(c.q, None, None, None, c.table, plain, None, first_position=3)
    at = (torch.arange(6, device="cuda") + 3)[:, None].expand(6, 2).int().contiguous()
    M.norm_rotary(c.q, None, ones, None, c.table, other, None, positions=at)
    assert torch.equal(plain, other)
    dx = torch.empty_like(c.q)
    M.norm_rotary_backward(c.dq, None, c.q, None, c.wq, None, c.table, dx, None, positions=c.positions)   # no sums: no workspace
    assert torch.equal(dx, gq)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_rows_without_a_step_and_unknown_positions(M, dtype):
    c = Case(4, 3, 1, 2, 1, 16, 8, dtype, P=10, seed=3)
    c.positions = torch.tensor([[0, 9, -1], [3, -7, 5], [1, 2, 3], [-2 ** 31, 4, 0]], dtype=torch.int32, device="cuda")
    bad = c.positions < 0
    for x in (c.q, c.k, c.dq, c.dk):
        x[bad] = math.nan            # nothing of such a row enters a result
    q, k, gq, gk, gwq, gwk = Case(4, 3, 1, 2, 1, 16, 8, dtype, P=10, seed=3), None, None, None, None, None
    clean = q
    clean.positions = c.positions
    want = check(M, clean, False)
    got = [torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0)]
    M.norm_rotary(c.q, c.k, c.wq, c.wk, c.table, *got, positions=c.positions)
    back = [torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0), torch.empty(16, device="cuda"), torch.empty(16, device="cuda")]
    M.norm_rotary_backward(c.dq, c.dk, c.q, c.k, c.wq, c.wk, c.table, *back, M.alloc_workspace(M.norm_rotary_workspace(c.q, c.k)), positions=c.positions)
    assert all(torch.equal(a, b) for a, b in zip((*got, *back), want))
    assert not got[0][bad].any() and not back[0][bad].any()
    c = Case(4, 3, 1, 2, 1, 16, 8, dtype, P=10, seed=3)
    c.positions[1, 1], c.positions[2, 0] = 10, 2 ** 31 - 1
    out = torch.empty_like(c.q)
    M.norm_rotary(c.q, None, c.wq, None, c.table, out, None, positions=c.positions)
    unknown = (c.positions >= 10)[:, :, None, None]
    assert torch.equal(out[..., :8].isnan(), unknown.expand(4, 3, 2, 8)) and not out[..., 8:].isnan().any()


def test_gradient_against_differences(M):
    c = Case(4, 2, 1, 3, 1, 20, 12, F32, seed=4)
    _, _, gq, _, gwq, _ = check(M, c, True)
    e, at = 1e-5, c.at()
    loss = lambda x, w: float((O.norm_rotary(x, w, c.table, at, 1e-6, True)[0] * c.dq.double()).sum())
    for which, g in ((0, gq), (1, gwq)):
        base = [c.q.double(), c.wq.double()]
        d = torch.randn(g.shape, device="cuda", dtype=torch.float64)
        up, down = list(base), list(base)
        up[which], down[which] = base[which] + e * d, base[which] - e * d
        diff = (loss(*up) - loss(*down)) / (2 * e)
        assert abs(diff - float((g.double() * d).sum())) <= 2e-5 * float((g.double() * d).abs().sum()) + 1e-6


def test_nothing_and_small_and_large_values(M):
    x = torch.empty((0, 4, 2, 16), device="cuda")
    dw = torch.full((16,), 7.0, device="cuda")
    M.norm_rotary(x, None, None, None, table_of(8, 8), x.clone(), None)
    M.norm_rotary_backward(x, None, x, None, None, None, table_of(8, 8), x.clone(), None, dw, None, M.alloc_workspace(M.norm_rotary_workspace(x, None)))
    assert not dw.any()
    for scale in (0.0, 1e-12, 1e15):
        c = Case(3, 2, 1, 2, 1, 32, 16, F32, seed=5)
        c.q.mul_(scale)
        c.k.mul_(scale)
        check(M, c, False)


def test_replayed_and_on_another_stream(M):
    c = Case(20, 4, 2, 4, 2, 64, 32, BF16, seed=6)
    outs = [torch.empty_like(c.q), torch.empty_like(c.k), torch.empty_like(c.q), torch.empty_like(c.k), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")]
    ws = M.alloc_workspace(M.norm_rotary_workspace(c.q, c.k))

    def work():
        M.norm_rotary(c.q, c.k, c.wq, c.wk, c.table, *outs[:2], positions=c.positions)
        M.norm_rotary_backward(c.dq, c.dk, c.q, c.k, c.wq, c.wk, c.table, *outs[2:], ws, positions=c.positions)

    work()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    want = [x.clone() for x in outs]
    with torch.cuda.stream(s):
        work()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for n in range(4):
        c.q.mul_(1.25)
        for x in outs:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in outs]
        work()
        assert all(torch.equal(a, b) for a, b in zip(got, outs)), n
