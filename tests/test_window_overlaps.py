"""What a call writes and another array of its own: refused where they share memory, however the one begins, and taken where one lies between the other's rows."""
import ctypes as C
import os
import random
import shutil
import subprocess

import pytest
import torch

from paper_2107_01460_amd import build
from test_memory_boundary import CONFIG, GOOD, M, dims  # noqa: F401  (M: the fixture)
from test_window_boundary import DK, DOUT, DQ, DV, FAR, K, KEYS, LSE, OUT, POS, Q, V, VALUES, WS, attend, back, norm, norm_back, step

# of the calls below: 4 steps of 6 sequences in fp32, 4 heads on 2, 16 and 32 wide, in views of 64, 32 and 16 elements
OLD = (FAR, FAR + KEYS)
STEP = 4 * (32 * 5 + 16 + 16)                    # bytes of the shortest view, a step of k, whose rows lie side by side
LONG = 4 * (64 * 3 + 32 * 5 + 16 * 3 + 32)       # of out's


def around(begin, size):
    """Places in front of memory from which a view runs into it, by most of the view and by its end, and one at the memory's own end"""
    return [begin - 64, begin - STEP + 64, begin + size - 4]


def test_views_that_run_into_caches(M):  # noqa: F811
    for x in around(FAR, KEYS) + around(FAR + KEYS, VALUES):
        assert attend(M, old=OLD, out=x) == CONFIG and attend(M, new=OLD, out=x) == CONFIG and step(M, old=OLD, out=x) == CONFIG
        for y in ("q", "k", "v"):
            assert attend(M, new=OLD, **{y: x}) == CONFIG and step(M, old=OLD, **{y: x}) == CONFIG
        for y in ("dq", "dk", "dv"):
            assert back(M, old=OLD, **{y: x}) == CONFIG, y


def test_vectors_that_run_into_others(M):  # noqa: F811
    lse, pos = 6 * 4 * 4 * 4, 4 * 3 * 4              # bytes
    for x in (FAR - lse + 4, FAR + KEYS + VALUES - 4):
        assert attend(M, old=OLD, lse=x) == CONFIG and attend(M, new=OLD, lse=x) == CONFIG
    assert attend(M, lse=POS + pos - 4, pos=POS) == CONFIG and attend(M, lse=POS - lse + 4, pos=POS) == CONFIG
    assert attend(M, new=OLD, pos=FAR - pos + 4) == CONFIG and step(M, old=OLD, pos=FAR - 8) == CONFIG
    for x in (OUT - 4, OUT + LONG - 64, Q + 8, V + 128):       # inside a view, or into its beginning
        assert attend(M, lse=x) == CONFIG
    for p in (DQ, DK, DV):
        assert back(M, lse=p + 16) == CONFIG and back(M, lse=p - lse + 4) == CONFIG and back(M, pos=p + 4) == CONFIG
    assert attend(M, pos=OUT + 4) == CONFIG and step(M, pos=OUT - 8) == CONFIG


def test_workspaces_that_others_lie_in(M):  # noqa: F811
    for p in (Q, K, V, OUT, DOUT, DQ, DK, DV):
        assert back(M, ws=p) == CONFIG and back(M, ws=p - 64) == CONFIG and back(M, ws=p + 64) == CONFIG
    assert back(M, ws=LSE) == CONFIG and back(M, ws=LSE + 16) == CONFIG and back(M, ws=POS, pos=POS) == CONFIG and back(M, ws=FAR + 64, old=OLD) == CONFIG
    many = dims(M, n_steps=1, n_seqs=2, seqs_per_flag=1)
    caches = (FAR, FAR << 1)
    for p in (Q, K, V, OUT, POS, FAR + 128):
        assert step(M, many, 4096, 0, old=caches, ws=p) == CONFIG, hex(p)


def test_norm(M):  # noqa: F811
    for x in (OUT, OUT + 64, OUT - 240, DOUT - 240):       # a table of 256 bytes
        assert norm(M, table=x) == CONFIG and norm_back(M, table=x) == CONFIG
    for x in (dict(qw=OUT + 4), dict(kw=DOUT - 60), dict(pos=OUT + 8), dict(pos=DOUT - 44)):
        assert norm(M, **x) == CONFIG and norm_back(M, **x) == CONFIG, x
    for p in (OUT, DOUT, Q, K, DQ, DK):
        assert norm_back(M, dqw=p + 4) == CONFIG and norm_back(M, dkw=p - 60) == CONFIG and norm_back(M, ws=p - 64) == CONFIG
    assert norm_back(M, dkw=FAR + 60) == CONFIG and norm_back(M, dqw=WS + 64) == CONFIG and norm_back(M, ws=POS, pos=POS + 64) == CONFIG
    assert norm_back(M, qw=WS + 4) == CONFIG and norm_back(M, table=WS + 256) == CONFIG


SOURCE = """
#include "attention_checks.h"
extern "C" int32_t touch(uint64_t data, const int64_t* strides, const int32_t* counts, int32_t dim, int32_t elem, uint64_t from, uint64_t bytes) {
  const marl_view v = {reinterpret_cast<void*>(data), strides[0], strides[1], strides[2]};
  marl_attention_dims d{};
  d.precision = elem == 4 ? 0 : 1;
  d.n_steps = counts[0];
  d.n_seqs = counts[1];
  return marl::touches(v, d, counts[2], dim, {from, bytes});
}
"""


@pytest.fixture(scope="module")
def touch(tmp_path_factory):
    if shutil.which("hipcc") is None:
        pytest.skip("needs hipcc")
    folder = tmp_path_factory.mktemp("touch")
    src, so = str(folder / "touch.hip"), str(folder / "touch.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.check_call(["hipcc", *build.FLAGS, "-shared", src, "-o", so])
    f = C.CDLL(so).touch
    f.argtypes = [C.c_uint64, C.POINTER(C.c_int64), C.POINTER(C.c_int32), C.c_int32, C.c_int32, C.c_uint64, C.c_uint64]
    return lambda data, strides, counts, dim, elem, begin, size: bool(f(data, (C.c_int64 * 3)(*strides), (C.c_int32 * 3)(*counts), dim, elem, begin, size))


def test_which_memory_a_view_touches(touch):
    """Against every byte of every row; strides in any order, negative ones among them, rows of one head beside each other or with gaps."""
    rng = random.Random(1)
    seen = {True: 0, False: 0}
    for _ in range(4000):
        dim, elem = rng.randint(1, 5), rng.choice((2, 4))
        counts = [rng.randint(1, 4) for _ in range(3)]
        strides, size = [0, 0, 0], dim + rng.randint(0, 3)
        for n in rng.sample(range(3), 3):                        # each dimension's places behind the ones inside it
            strides[n] = size * rng.choice((1, 1, -1))
            size = size * counts[n] + rng.randint(0, 9)
        data = 1 << 20
        rows = {data + elem * (t * strides[0] + b * strides[1] + h * strides[2]) for t in range(counts[0]) for b in range(counts[1]) for h in range(counts[2])}
        taken = {x + e for x in rows for e in range(dim * elem)}
        begin, length = rng.randint(min(taken) - 24, max(taken) + 24), rng.randint(1, 40)
        want = any(x in taken for x in range(begin, begin + length))
        assert touch(data, strides, counts, dim, elem, begin, length) == want, (strides, counts, dim, elem, begin - data, length)
        seen[want] += 1
    assert min(seen.values()) > 400


def test_the_largest_strides(touch):
    big = (1 << 62) // 4
    assert touch(1 << 40, (big, -big, 7), (3, 2, 2), 4, 4, 1 << 40, 1)
    assert not touch(1 << 40, (big, -big, 7), (3, 2, 2), 4, 4, (1 << 40) + 64, 64) and not touch(1 << 40, (0, 0, 0), (5, 5, 5), 4, 4, (1 << 40) + 16, 64)
    assert not touch(1 << 40, (1, 2, 3), (5, 5, 5), 4, 4, 1 << 40, 0)


@pytest.mark.gpu
def test_arrays_between_the_rows_of_others(M):  # noqa: F811
    """All of a call's arrays in one piece of memory, the caches and statistics between the steps of the views: taken, with the results of arrays of their own."""
    T, B, H, D, window, sinks = 6, 3, 2, 32, 5, 1
    g = torch.Generator(device="cuda").manual_seed(2)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    one = B * H * D                                  # elements of a step of an array
    step_ = 8 * one                                  # from one step to the next: room for eight arrays' rows
    memory = torch.zeros(T * step_, device="cuda")
    at = lambda n, T=T: memory[n * one:].as_strided((T, B, H, D), (step_, H * D, D, 1))
    q, k, v, out, dq, dk, dv = (at(n) for n in range(7))
    for x in (q, k, v):
        x.copy_(rand(T, B, H, D))
    # (behind a step's rows of the seven arrays one array's room is left: the statistics, and half of a cache of shape [3][2][1][...] do not fit; small ones do)
    lse = memory[7 * one: 7 * one + B * H * T].view(B, H, T)
    cache = tuple(memory[step_ * (1 + n) + 7 * one: step_ * (1 + n) + 7 * one + B * H * 1 * 16].view(B, H, 1, 16) for n in range(2))
    p = torch.arange(T, dtype=torch.int32, device="cuda")[:, None].repeat(1, B)
    own = [x.clone(memory_format=torch.contiguous_format) for x in (q, k, v)]
    want, want_lse = torch.empty_like(own[0]), torch.empty(B, H, T, device="cuda")
    M.window_attention(*own, want, window, sinks, lse=want_lse, positions=p)
    M.window_attention(q, k, v, out, window, sinks, lse=lse, positions=p)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    grads = [torch.empty_like(x) for x in own]
    ws = M.alloc_workspace(M.window_attention_workspace(*own, window, sinks, kind="backward"))
    M.window_attention_backward(*own, want, want_lse, want, *grads, window, sinks, positions=p, workspace=ws)
    M.window_attention_backward(q, k, v, out, lse, want, dq, dk, dv, window, sinks, positions=p, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(grads, (dq, dk, dv)))
    # a window of one step on heads of 16: its cache between the steps of the views that the call reads and writes
    narrow = [x[..., :16] for x in (q, k, v)]
    want = torch.empty(T, B, H, 16, device="cuda")
    after = tuple(torch.zeros(B, H, 1, 16, device="cuda") for _ in range(2))
    M.window_attention(*[x.contiguous() for x in narrow], want, 1, 0, positions=p, next_cache=after)
    M.window_attention(*narrow, out[..., :16], 1, 0, positions=p, next_cache=cache)
    assert torch.equal(out[..., :16], want) and all(torch.equal(a, b) for a, b in zip(cache, after))
