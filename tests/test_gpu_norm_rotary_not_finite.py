"""Infinities and NaNs behind the rotated part of a head: elements there are copied, so that none of them enters another one, in both orders of pairs."""
import math

import pytest
import torch

import window_oracle as O
from test_gpu_norm_rotary import BF16, F32, M, NAMES, Case, rounded  # noqa: F401  (M: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R", [(4, 2), (8, 4), (9, 4), (16, 8), (40, 20), (64, 6), (64, 32), (130, 66), (256, 128)])
def test_behind_the_rotated_part(M, D, R, interleaved, dtype, value):  # noqa: F811
    for i in (R, R + 1, D - 1):
        c = Case(3, 2, 1, 2, 1, D, R, dtype, seed=D)
        at = c.at()
        c.q[1, 0, 1, i] = c.k[0, 1, 0, i] = value
        out = [torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0)]
        M.norm_rotary(c.q, c.k, c.wq, c.wk, c.table, *out, positions=c.positions, interleaved=interleaved)
        for x, w, y in ((c.q, c.wq, out[0]), (c.k, c.wk, out[1])):
            ref, bound = O.norm_rotary(x, w, c.table, at, 1e-6, interleaved)
            O.within(y, ref, rounded(bound, ref, dtype), "y")
        # the gradient, of clean inputs
        c = Case(3, 2, 1, 2, 1, D, R, dtype, seed=D)
        c.dq[1, 0, 1, i] = c.dk[0, 1, 0, i] = value
        back = [torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0), torch.full((D,), 7.0, device="cuda"), torch.full((D,), 7.0, device="cuda")]
        M.norm_rotary_backward(c.dq, c.dk, c.q, c.k, c.wq, c.wk, c.table, *back, M.alloc_workspace(M.norm_rotary_workspace(c.q, c.k)), positions=c.positions,
                               interleaved=interleaved)
        for x, w, dy, dx, dw in ((c.q, c.wq, c.dq, back[0], back[2]), (c.k, c.wk, c.dk, back[1], back[3])):
            (ref, bound), (ref_w, bound_w) = O.norm_rotary_backward(dy, x, w, c.table, at, 1e-6, interleaved)
            O.within(dx, ref, rounded(bound, ref, dtype), "dx")
            O.within(dw, ref_w, bound_w, "dw")
            others = torch.arange(D, device="cuda") != i
            assert torch.isfinite(dw[others]).all() and not torch.isfinite(dw[i])
