"""Checks of the sequence operators' arguments that need no GPU, in Python and in the library."""
import ctypes as C

import pytest
import torch

from test_memory_boundary import CONFIG, GOOD, OK, M, dims, view  # noqa: F401  (M: the fixture)


def test_workspace_in_host_memory(M):  # noqa: F811
    """The one pointer of a call that a kernel writes without any other tensor's shape: it has to lie on the GPU too, needed or not."""
    for need in (0, 64):
        with pytest.raises(M.MarlError, match="on the GPU"):
            M.binding._workspace(torch.empty(256, dtype=torch.uint8), need)
    assert M.binding._workspace(None, 0) is None


def test_gradient_of_the_state_over_states(M):  # noqa: F811
    """dstate is written while other workgroups still read state and dnext_state: it overlaps neither, wholly or in part."""
    d, v = dims(M), view(M)
    size = d.n_seqs * d.n_heads * d.dim_k * d.dim_v * 4
    grad = lambda state, dnext, dstate, d=d: M.lib().marl_linear_attention_backward(C.byref(d), v, v, v, GOOD, state, None, v, dnext, v, v, v, dstate, GOOD, None)
    for at in (GOOD, GOOD + 16, GOOD + size - 16, GOOD - 16, GOOD - size + 16):
        assert grad(GOOD, None, at) == CONFIG and grad(None, GOOD, at) == CONFIG
    nothing = dims(M, n_seqs=0)
    assert grad(GOOD, GOOD, GOOD, nothing) == OK


def test_next_state_over_a_part_of_the_state(M):  # noqa: F811
    """next_state may be the state, but not a part of it and something else."""
    d, one, v = dims(M), dims(M, n_steps=1), view(M)
    for at in (GOOD + 16, GOOD - 16):
        assert M.lib().marl_linear_attention(C.byref(d), v, v, v, GOOD, GOOD, None, view(M, GOOD + (1 << 20)), at, GOOD, None) == CONFIG
        assert M.lib().marl_linear_attention_step(C.byref(one), v, v, v, GOOD, GOOD, None, view(M, GOOD + (1 << 20)), at, None) == CONFIG


OUT = GOOD + (1 << 24)


def test_outputs_that_begin_where_another_array_does(M):  # noqa: F811
    """Wrong answers in silence otherwise: a wavefront reads an input that another has written its output over."""
    L, d, one = M.lib(), dims(M), dims(M, n_steps=1)
    at = lambda p: view(M, p)
    for bad in range(3):
        q, k, v = (at(GOOD + 4096 * n) for n in range(3))
        assert L.marl_linear_attention(C.byref(d), q, k, v, GOOD, None, None, at(GOOD + 4096 * bad), None, GOOD, None) == CONFIG
        assert L.marl_linear_attention_step(C.byref(one), q, k, v, GOOD, GOOD, None, at(GOOD + 4096 * bad), GOOD, None) == CONFIG
    places = [GOOD + 4096 * n for n in range(4)] + [OUT + 4096 * n for n in range(3)]   # q, k, v, dout, dq, dk, dv
    for i in range(4, 7):
        for j in range(i):
            p = list(places)
            p[i] = p[j]
            q, k, v, dout, dq, dk, dv = map(at, p)
            assert L.marl_linear_attention_backward(C.byref(d), q, k, v, GOOD, None, None, dout, None, dq, dk, dv, None, GOOD, None) == CONFIG, (i, j)


def test_in_place_with_other_strides(M):  # noqa: F811
    L, d = M.lib(), dims(M)
    assert L.marl_layer_norm(0, 4, 8, GOOD, 8, None, None, 1e-5, GOOD, 9, None, None, None) == CONFIG
    for x, dy in ((GOOD, OUT), (OUT, GOOD)):
        assert L.marl_layer_norm_backward(0, 4, 8, dy, 8, x, 8, None, GOOD, GOOD, GOOD, 9, None, None, None, None) == CONFIG
    V = M.binding.View
    q, k, qo, ko = V(GOOD, 64, 32, 16), V(GOOD + 4096, 64, 32, 16), V(OUT, 64, 32, 16), V(OUT + 4096, 64, 32, 16)
    for outs in ((V(GOOD, 128, 32, 16), ko), (qo, V(GOOD + 4096, 64, 48, 16)), (k, ko), (qo, q), (qo, qo)):
        assert L.marl_rotary(C.byref(d), q, k, GOOD, 8, 8, None, 0, 0, 0, *outs, None) == CONFIG


def test_numbers_in_place_of_arrays(M):  # noqa: F811
    """Flags and positions without a dimension are refused like any other wrong shape."""
    with pytest.raises(M.MarlError, match="done"):
        M.binding._flags(torch.tensor(1, dtype=torch.uint8), (4,), 6, "done")
    with pytest.raises(M.MarlError, match="positions"):
        M.rotary(torch.zeros(4, 6, 2, 8), None, torch.zeros(9, 8), torch.zeros(4, 6, 2, 8), None, positions=torch.tensor(3, dtype=torch.int32))
