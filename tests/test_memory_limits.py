"""Sizes that no launch can have: refused with MARL_E_SIZE in front of the first launch, on both sides of the limit, without a GPU."""
import ctypes as C
import os

import pytest

from paper_2107_01460_amd import build
from test_memory_boundary import GOOD, OK, SIZE, dims, view

LIMIT = 1 << 32   # work-items along a dimension of a grid


@pytest.fixture(scope="module")
def M():
    import paper_2107_01460_amd as m
    if not os.path.exists(m.binding._LIB_PATH):
        build.build(verbose=False)
    m.lib()
    return m


def need(M, backward, **kw):
    return M.lib().marl_linear_attention_workspace(C.byref(dims(M, **kw)), backward, C.byref(C.c_int64()))


# work-items of a (sequence, head) pair: a wavefront for each slice of up to 32 columns; in the gradient three times, or twice the one and once the other
@pytest.mark.parametrize("dk,dv,forward,gradient", [(16, 16, 64, 192), (32, 64, 128, 128), (64, 64, 128, 384), (64, 32, 64, 256), (16, 96, 192, 192),
                                                   (128, 96, 192, 512), (128, 128, 256, 768)])
def test_scans(M, dk, dv, forward, gradient):
    for backward, each in ((0, forward), (1, gradient)):
        most = min((LIMIT - 1) // each // 4 * 4, 1 << 26)
        one = dict(n_steps=1, n_heads=1, n_kv_heads=1, dim_k=dk, dim_v=dv, seqs_per_flag=1)
        assert need(M, backward, n_seqs=most, **one) == OK
        assert need(M, backward, n_seqs=most + 4, **one) == SIZE
        d, v = dims(M, n_seqs=most + 4, **one), view(M)
        if backward:
            assert M.lib().marl_linear_attention_backward(C.byref(d), v, v, v, GOOD, None, None, v, None, v, v, v, None, GOOD, None) == SIZE
        else:
            assert M.lib().marl_linear_attention(C.byref(d), v, v, v, GOOD, None, None, v, None, GOOD, None) == SIZE


def test_states_alone(M):
    """No steps: a copy of the states, a work-item an element."""
    one = dict(n_steps=0, n_heads=1, n_kv_heads=1, dim_k=128, dim_v=128, seqs_per_flag=1)
    assert need(M, 0, n_seqs=(1 << 18) - 1, **one) == OK and need(M, 0, n_seqs=1 << 18, **one) == SIZE
    d, v = dims(M, n_seqs=1 << 18, **one), view(M)
    assert M.lib().marl_linear_attention(C.byref(d), v, v, v, GOOD, GOOD, None, v, GOOD, None, None) == SIZE


def test_long_and_many(M):
    """The shares of shared heads: a size in bytes that 64 bits hold."""
    assert need(M, 1, n_steps=1 << 30, n_seqs=1 << 22, n_heads=2, n_kv_heads=1, seqs_per_flag=1) == SIZE


@pytest.mark.parametrize("dk,dv,each", [(64, 64, 256), (16, 16, 64), (8, 65, 256), (31, 33, 64)])
def test_steps(M, dk, dv, each):
    n = LIMIT // each
    d, v = dims(M, n_steps=1, n_seqs=n, n_heads=1, n_kv_heads=1, dim_k=dk, dim_v=dv, seqs_per_flag=1), view(M)
    assert M.lib().marl_linear_attention_step(C.byref(d), v, v, v, GOOD, GOOD, None, v, GOOD, None) == SIZE


def test_rotary(M):
    L, v = M.lib(), view(M)
    turn = lambda **kw: L.marl_rotary(C.byref(dims(M, **kw)), v, v, GOOD, 8, 8, None, 0, 0, 0, v, v, None)
    # four items of sixteen bytes a head of 16, four heads of q and two of k: 24 items a token, four to a work-item
    assert turn(n_steps=1 << 20, n_seqs=1 << 14) == SIZE
    assert turn(n_steps=(1 << 31) - 1, n_seqs=1 << 30, n_heads=1 << 14, n_kv_heads=1 << 14, dim_k=1024, seqs_per_flag=1) == SIZE   # (a product past 64 bits)
    none = M.binding.RotaryDims(n_positions=(1 << 31) - 1, rotary_dim=4, scaling=0, base=1e4, factor=1.0, trained_length=1.0, slow=1.0, fast=2.0, amplitude=1.0)
    assert L.marl_rotary_table(C.byref(none), GOOD, None) == SIZE
