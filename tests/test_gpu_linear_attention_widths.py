"""Linear attention at every pair of padded widths, whole pieces and others: each instance of the scan, output and gradient, against the recurrence in 64 bits."""
import pytest
import torch

from test_gpu_linear_attention import BF16, F32, check, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import paper_2107_01460_amd as m
    assert torch.cuda.is_available()
    return m


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("Dk", [16, 32, 48, 64, 80, 96, 128, 13, 27, 37, 61, 75, 91, 117])
def test_every_width(M, Dk, dtype):
    """70 steps: two whole tiles and a part of one; shared heads, so that the gradients go out in fp32 shares as well."""
    for Dv in (16, 32, 64, 96, 128) if Dk % 16 == 0 else (11, 29, 43, 83, 125):
        for Hk in (3, 1):
            print("case", Dk, Dv, Hk, dtype, flush=True)
            check(M, make(70, 3, 3, Hk, Dk, Dv, dtype, seed=Dk + Dv, episode=25))
