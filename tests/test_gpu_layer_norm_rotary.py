"""Layer norm and its gradient, rotary positions and their table, against 64 bits."""
import math

import pytest
import torch

import memory_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def M():
    import paper_2107_01460_amd as m
    assert torch.cuda.is_available()
    return m


def rows(n, w, dtype, seed, offset=0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn((n, w + pad), generator=g, device="cuda") * 1.5 + 0.5).to(dtype)
    return x[:, offset: offset + w]


# widths on both sides of every team of lanes, of vector and element accesses
WIDTHS = [1, 3, 8, 27, 64, 128, 129, 147, 255, 256, 512, 520, 1000, 1024, 1032, 2047, 4096, 4104, 16384]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_layer_norm(M, width, dtype):
    n = 67
    x, dy = rows(n, width, dtype, width), rows(n, width, dtype, width + 1)
    w, b = torch.randn(width, device="cuda"), torch.randn(width, device="cuda")
    y, mean, rstd = torch.full_like(x, float("nan")), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    M.layer_norm(x, w, b, y, mean, rstd)
    ref, m, r = O.layer_norm(x, w, b, 1e-5)
    # a value in units of its row's deviation: the mean's error (a sum of `width` terms in teams of lanes, at most 20 additions deep in each) and
    # that of the deviation, each below 40 2^-24 of |x| + |mean|
    hat = (x.double().abs() + m.abs()[:, None]) * r[:, None]
    O.within(y, ref, (hat + 1) * w.double().abs() + b.double().abs(), 40, dtype == BF16)
    O.within(mean, m, x.double().abs().mean(1), 10)
    O.within(rstd, r, r * (1 + (x.double().abs().mean(1) * r) ** 2), 40)
    dx, dw, db = torch.full_like(x, float("nan")), torch.empty(width, device="cuda"), torch.empty(width, device="cuda")
    M.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, M.alloc_workspace(M.layer_norm_workspace(n, width)))
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    u = dy.double() * w.double()
    rs = rstd.double()[:, None]
    want = rs * (u - u.mean(1, keepdim=True) - h * (u * h).mean(1, keepdim=True))
    size = rs * (u.abs() + u.abs().mean(1, keepdim=True) + (h.abs() + hat) * (u * h).abs().mean(1, keepdim=True) + h.abs() * (u.abs() * hat).mean(1, keepdim=True))
    O.within(dx, want, size, 40, dtype == BF16)
    O.within(dw, (dy.double() * h).sum(0), (dy.double().abs() * hat).sum(0), n)
    O.within(db, dy.double().sum(0), dy.double().abs().sum(0), n)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_layer_norm_strided_rows_and_in_place(M, dtype):
    for offset, pad in ((8, 16), (1, 5)):
        x = rows(50, 96, dtype, 3, offset, pad)
        y, flat = torch.empty((50, 96), dtype=dtype, device="cuda"), torch.empty((50, 96), dtype=dtype, device="cuda")
        M.layer_norm(x, None, None, y)
        M.layer_norm(x.contiguous(), None, None, flat)
        ref, m, r = O.layer_norm(x, None, None, 1e-5)
        O.within(y, ref, (x.double().abs() + m.abs()[:, None]) * r[:, None] + 1, 40, dtype == BF16)
        keep = x.clone()
        M.layer_norm(x, None, None, x)
        assert torch.equal(x, y)
        mean, rstd = keep.float().mean(1), torch.ones(50, device="cuda")
        dy = rows(50, 96, dtype, 4, offset, pad)
        dx = torch.empty_like(y)
        M.layer_norm_backward(dy, keep, None, mean, rstd, dx)
        M.layer_norm_backward(dy, keep, None, mean, rstd, dy)
        O.within(dy, dx, dx.abs() + 1, 1000, dtype == BF16)


def test_layer_norm_many_rows(M):
    """More rows than the gradient's workgroups take at once; two runs agree bit for bit; only one of the two sums asked for."""
    n, w = 100003, 40
    x, dy, weight = rows(n, w, F32, 1), rows(n, w, F32, 2), torch.randn(w, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    M.layer_norm(x, weight, None, y, mean, rstd)
    ws = M.alloc_workspace(M.layer_norm_workspace(n, w))
    out = []
    for _ in range(2):
        dx, dw, db = torch.empty_like(x), torch.empty(w, device="cuda"), torch.empty(w, device="cuda")
        M.layer_norm_backward(dy, x, weight, mean, rstd, dx, dw, db, ws)
        out.append((dx, dw, db))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    O.within(out[0][1], (dy.double() * h).sum(0), (dy.double() * h).abs().sum(0), 500)
    O.within(out[0][2], dy.double().sum(0), dy.double().abs().sum(0), 500)
    db = torch.empty(w, device="cuda")
    M.layer_norm_backward(dy, x, weight, mean, rstd, torch.empty_like(x), None, db, ws)
    assert torch.equal(db, out[0][2])


def test_layer_norm_no_rows(M):
    x = torch.empty((0, 32), device="cuda")
    M.layer_norm(x, None, None, torch.empty_like(x))
    dw, db = torch.full((32,), 7.0, device="cuda"), torch.full((32,), 7.0, device="cuda")
    e = torch.empty(0, device="cuda")
    M.layer_norm_backward(x, x, None, e, e, torch.empty_like(x), dw, db, M.alloc_workspace(256))
    assert not dw.any() and not db.any()


def test_layer_norm_rows_that_are_not_finite(M):
    x = rows(20, 100, F32, 1)
    clean = torch.empty((20, 100), device="cuda")
    M.layer_norm(x, None, None, clean)
    x[3, 7], x[9, 99] = float("inf"), float("nan")
    y = torch.empty((20, 100), device="cuda")
    M.layer_norm(x, None, None, y)
    other = [i for i in range(20) if i not in (3, 9)]
    assert torch.equal(y[other], clean[other]) and y[3].isnan().all() and y[9].isnan().all()


def test_layer_norm_large_mean(M):
    """A mean a thousand times the deviation: the variance comes from centred values, not from a difference of squares."""
    x = rows(30, 256, F32, 5) + 1500.0
    y = torch.empty_like(x)
    M.layer_norm(x, None, None, y)
    # the centred value is exact but for the mean's error, 20 2^-24 of 1500, and in units of the deviation 1.5
    assert float((y.double() - O.layer_norm(x, None, None, 1e-5)[0]).abs().max()) <= 20 * 2.0 ** -24 * 1500


def test_layer_norm_gradient_against_differences(M):
    n, w = 9, 50
    x, dy, weight, bias = rows(n, w, F32, 1), rows(n, w, F32, 2), torch.randn(w, device="cuda"), torch.randn(w, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    M.layer_norm(x, weight, bias, y, mean, rstd)
    dx, dw, db = torch.empty_like(x), torch.empty(w, device="cuda"), torch.empty(w, device="cuda")
    M.layer_norm_backward(dy, x, weight, mean, rstd, dx, dw, db, M.alloc_workspace(M.layer_norm_workspace(n, w)))
    loss = lambda x, a, b: float((O.layer_norm(x, a, b, 1e-5)[0] * dy.double()).sum())
    e = 1e-5   # the difference's own error: e^2 of the third derivative, 1e-10 of the scale
    for which, grad in enumerate((dx, dw, db)):
        base = [x.double(), weight.double(), bias.double()]
        d = torch.randn(grad.shape, device="cuda", dtype=torch.float64)
        up, down = list(base), list(base)
        up[which], down[which] = base[which] + e * d, base[which] - e * d
        diff = (loss(*up) - loss(*down)) / (2 * e)
        assert abs(diff - float((grad.double() * d).sum())) <= 2e-5 * float((grad.double() * d).abs().sum()) + 1e-6


# ---- rotary ---------------------------------------------------------------------------------------------------------------
def table_of(P, R, base=10000.0, f=None):
    f = base ** (-2.0 * torch.arange(R // 2, dtype=torch.float64) / R) if f is None else f
    angle = torch.arange(P, dtype=torch.float64)[:, None] * f
    return torch.cat([angle.cos(), angle.sin()], 1)


@pytest.mark.parametrize("scaling", [None, "linear", "base", "by_turns"])
def test_table(M, scaling):
    R, base, factor, L = 64, 10000.0, 8.0, 4096.0
    f = base ** (-2.0 * torch.arange(R // 2, dtype=torch.float64) / R)
    if scaling == "linear":
        f = f / factor
    if scaling == "base":
        f = (base * factor ** (R / (R - 2))) ** (-2.0 * torch.arange(R // 2, dtype=torch.float64) / R)
    if scaling == "by_turns":
        m = ((L * f / (2 * math.pi) - 1.0) / 31.0).clamp(0, 1)
        f = m * f + (1 - m) * f / factor
    got = M.rotary_table(32768, R, base, scaling=scaling, factor=factor, trained_length=L, amplitude=1.25)
    # 64-bit angles of up to 32768: 1e-11; the rounding to fp32: 2^-24 of 1.25
    assert float((got.cpu().double() - 1.25 * table_of(32768, R, f=f)).abs().max()) <= 1.25 * 2.0 ** -24 + 1e-10


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R", [(2, 2), (9, 4), (32, 32), (64, 32), (80, 48), (128, 128), (40, 20), (64, 6), (127, 126)])
def test_rotary(M, D, R, interleaved, dtype):
    T, B, H, Hk, P = 5, 6, 3, 2, 300
    g = torch.Generator(device="cuda").manual_seed(D)
    q, k = (torch.randn((T, B, h, D), generator=g, device="cuda").to(dtype) for h in (H, Hk))
    table = table_of(P, R).float().cuda()
    pos = torch.randint(0, P, (T, B // 2), generator=g, device="cuda").int()
    full = pos.repeat_interleave(2, 1)
    for inverse in (False, True):
        qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
        M.rotary(q, k, table, qo, ko, positions=pos, interleaved=interleaved, inverse=inverse)
        for x, y in ((q, qo), (k, ko)):
            ref, size = O.rotate(x, table, full, interleaved, inverse), O.rotate(x.abs(), table.abs(), full, interleaved, False)
            one, two = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
            size = x.double().abs()   # |x1| + |x2| bounds both terms
            s = size[..., one] + size[..., two]
            size[..., one] = size[..., two] = s
            O.within(y, ref, size, 3, dtype == BF16)
            assert torch.equal(y[..., R:], x[..., R:])
    # in place, alone, by the step's number
    ref = O.rotate(q, table, (torch.arange(T, device="cuda")[:, None] + 7).expand(T, B), interleaved, False)
    alone = q.clone()
    M.rotary(alone, None, table, alone, None, first_position=7, interleaved=interleaved)
    O.within(alone, ref, q.double().abs().sum(-1, keepdim=True).expand_as(ref), 3, dtype == BF16)


def test_rotary_strides_and_turning_back(M):
    g = torch.Generator(device="cuda").manual_seed(1)
    fused = torch.randn((4, 3, 10, 64), generator=g, device="cuda")            # queries, keys and values side by side
    q, k = fused[:, :, :4], fused[:, :, 4:7]
    table = table_of(50, 64).float().cuda()
    want = fused.clone()
    want[:, :, :7] = O.rotate(fused[:, :, :7], table, torch.arange(4, device="cuda")[:, None].expand(4, 3), False, False).float()
    before = fused.clone()
    M.rotary(q, k, table, q, k)
    assert float((fused - want).abs().max()) < 1e-6 and torch.equal(fused[:, :, 7:], before[:, :, 7:])
    M.rotary(q, k, table, q, k, inverse=True)
    assert float((fused - before).abs().max()) < 2e-6
    turned = torch.randn((3, 2, 5, 32), generator=g, device="cuda").permute(2, 0, 1, 3)   # [T][B][H][D] of sequence-major storage
    out = torch.empty((5, 3, 2, 32), device="cuda")
    M.rotary(turned, None, table[:, :32].contiguous(), out, None)
    O.within(out, O.rotate(turned, table[:, :32], torch.arange(5, device="cuda")[:, None].expand(5, 3), False, False), turned.double().abs() + 4, 3)


def test_rotary_unknown_positions_and_empty(M):
    q = torch.ones((2, 3, 1, 8), device="cuda")
    table = table_of(10, 4).float().cuda()
    pos = torch.tensor([[0, 9, 10], [-1, 5, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    M.rotary(q, None, table, out, None, positions=pos)
    bad = ((pos < 0) | (pos >= 10))[:, :, None, None]
    assert torch.equal(out[..., :4].isnan(), bad.expand(2, 3, 1, 4)) and torch.equal(out[..., 4:], q[..., 4:])
    M.rotary(q[:0], None, table, out[:0], None)
    torch.cuda.synchronize()
