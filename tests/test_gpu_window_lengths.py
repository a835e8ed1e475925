"""Windows of many tiles, of which most are seen whole, and sequences in numbers that fill no round of the columns' order: against the definition in 64 bits."""
import pytest
import torch

import window_oracle as O
from test_gpu_window_attention import BF16, F32, M, NAMES, Case, check  # noqa: F401  (M: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("D,H,Hk", [(32, 2, 2), (64, 4, 1), (96, 3, 1), (128, 4, 2), (50, 2, 1)])
@pytest.mark.parametrize("window,kind", [(250, "whole"), (257, "rare"), (333, "going"), (300, "ragged"), (600, "rare")])
def test_many_tiles(M, window, kind, D, H, Hk, dtype):  # noqa: F811
    check(M, Case(700, 1 if kind != "ragged" else 3, 1, H, Hk, D, D, dtype, window, 3, kind, kind == "going", seed=window + D))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("D,H,Hk,envs,agents", [(32, 1, 1, 65, 1), (64, 3, 3, 35, 2), (128, 2, 1, 64, 1), (32, 4, 1, 43, 3), (7, 2, 2, 33, 2)])
def test_many_sequences(M, D, H, Hk, envs, agents, dtype):  # noqa: F811
    check(M, Case(70, envs, agents, H, Hk, D, D, dtype, 20, 2, "episodes", True, seed=D + envs))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_infinities_inside_a_long_window(M, dtype):  # noqa: F811
    """A value that is infinite shows in the rows that see it, inside tiles that are seen whole too, and in no others."""
    c = Case(600, 1, 1, 2, 1, 64, 64, dtype, 200, 2, "whole", False, seed=5)
    c.v[150, 0, 0, 7] = float("inf")
    out, _ = c.forward(M)
    sees = torch.zeros(600, dtype=torch.bool, device="cuda")
    sees[150:350] = True
    assert torch.equal(torch.isinf(out[:, 0, 0, 7]), sees) and torch.equal(torch.isinf(out[:, 0, 1, 7]), sees)
    c.v[150, 0, 0, 7] = 0.0
    ref = c.oracle()
    want, bound, _, _ = ref.forward(c.Dv)
    out[..., 7], want[..., 7] = 0.0, 0.0
    O.within(out, want, bound, "out")
