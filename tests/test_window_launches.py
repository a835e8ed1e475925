"""Where a window's calls stop fitting a launch, to the sequence: a grid has fewer than 2^32 work-items, workgroups of rollouts and gradients up to 256 of them."""
import pytest

from test_memory_boundary import OK, SIZE, M, dims  # noqa: F401  (M: the fixture)
from test_window_boundary import LIMIT, attend, back, need, norm, step


def sized(n, **kw):
    return dict(dict(n_steps=1, n_seqs=n, n_heads=1, n_kv_heads=1, dim_k=16, dim_v=16, seqs_per_flag=1), **kw)


@pytest.mark.parametrize("kind", [0, 1])
def test_one_step(M, kind):  # noqa: F811
    """A workgroup for each sequence; of the two plans, by alignment, the one with four wavefronts a workgroup decides."""
    most = LIMIT // 256
    sizes = list(range(most - 3, most + 3))
    assert [need(M, kind, 1, 0, **sized(n))[0] for n in sizes] == [OK] * 3 + [SIZE] * 3
    call = attend if kind == 0 else back
    assert call(M, dims(M, **sized(most)), 1, 0) == SIZE


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("heads,steps,each", [(2, 1, 2), (3, 33, 3), (6, 129, 12), (1, 4096, 32)])
def test_workgroups_of_a_sequence(M, kind, heads, steps, each):  # noqa: F811
    """Heads that share nothing, 128 steps of one a workgroup."""
    most = (LIMIT // 256 - 1) // each
    sizes = [most - 1, most, most + 1, most + 2]
    assert [need(M, kind, 1 << 12, 0, **sized(n, n_heads=heads, n_kv_heads=heads, n_steps=steps))[0] for n in sizes] == [OK, OK, SIZE, SIZE]


def test_steps(M):  # noqa: F811
    """A wavefront for each sequence and key head, four a workgroup of 256."""
    assert need(M, 2, 1, 0, **sized((LIMIT - 256) // 64))[0] == OK and need(M, 2, 1, 0, **sized(LIMIT // 64 - 3))[0] == SIZE
    assert step(M, dims(M, **sized(1 << 26)), 1, 0) == SIZE
