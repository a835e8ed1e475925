"""Window attention and norm with rotation refuse bad arguments on the host, before anything is launched; and their kernels' listings."""
import ctypes as C
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

from paper_2107_01460_amd import build
from test_matrix_product_chains import mixed_chains
from test_memory_boundary import ALIGN, BAD_DIMS, CONFIG, GOOD, NULL, OK, SIZE, M, dims, view  # noqa: F401  (M: the fixture)
from test_rollout_waits import pending_writes_at_barriers

LIMIT = 1 << 32          # work-items along a dimension of a grid
SLOTS = 8 + 2            # of the calls below
KEYS, VALUES = 6 * 2 * SLOTS * 16 * 4, 6 * 2 * SLOTS * 32 * 4     # bytes of their caches
Q, K, V, OUT, DOUT, DQ, DK, DV = (GOOD + (n << 16) for n in range(8))
LSE, POS, WS, FAR = GOOD + (9 << 16), GOOD + (10 << 16), GOOD + (11 << 16), GOOD + (1 << 24)


def need(M, kind, window=8, sinks=2, d=None, **kw):
    n = C.c_int64()
    d = dims(M, **kw) if d is None else d
    return M.lib().marl_window_attention_workspace(C.byref(d), window, sinks, kind, C.byref(n)), n.value


def cache(M, keys=None, values=None):
    return M.binding.WindowCache(keys, values)


def attend(M, d=None, window=8, sinks=2, q=Q, k=K, v=V, pos=None, first=0, old=(None, None), out=OUT, lse=None, new=(None, None), views={}):
    at = lambda name, p: views.get(name, view(M, p))
    d = dims(M) if d is None else d
    return M.lib().marl_window_attention(C.byref(d), window, sinks, at("q", q), at("k", k), at("v", v), pos, first, cache(M, *old), at("out", out), lse, cache(M, *new),
                                         None, None)


def back(M, d=None, window=8, sinks=2, pos=None, first=0, old=(None, None), lse=LSE, ws=WS, views={}, **kw):
    p = dict(q=Q, k=K, v=V, out=OUT, dout=DOUT, dq=DQ, dk=DK, dv=DV)
    p.update(kw)
    at = [views.get(name, view(M, x)) for name, x in p.items()]
    d = dims(M) if d is None else d
    return M.lib().marl_window_attention_backward(C.byref(d), window, sinks, *at[:3], pos, first, cache(M, *old), at[3], lse, *at[4:], ws, None)


def step(M, d=None, window=8, sinks=2, q=Q, k=K, v=V, pos=POS, old=(FAR, FAR + KEYS), out=OUT, ws=WS, views={}):
    at = lambda name, p: views.get(name, view(M, p))
    d = dims(M, n_steps=1) if d is None else d
    return M.lib().marl_window_attention_step(C.byref(d), window, sinks, at("q", q), at("k", k), at("v", v), pos, cache(M, *old), at("out", out), ws, None)


@pytest.mark.parametrize("change,code", BAD_DIMS)
def test_window_sizes(M, change, code):  # noqa: F811
    d = dims(M, **change)
    assert all(need(M, kind, d=d)[0] == code for kind in range(3))
    assert attend(M, d) == code and back(M, d) == code and step(M, d) == code


@pytest.mark.parametrize("window,sinks", [(0, 2), (-1, 0), (8, -1), ((1 << 30) + 1, 0), (1 << 30, 1), (5, 1 << 30), ((1 << 31) - 1, (1 << 31) - 1)])
def test_windows(M, window, sinks):  # noqa: F811
    assert all(need(M, kind, window, sinks)[0] == CONFIG for kind in range(3))
    assert attend(M, None, window, sinks) == CONFIG and back(M, None, window, sinks) == CONFIG and step(M, None, window, sinks) == CONFIG


def test_the_largest_windows(M):  # noqa: F811
    assert need(M, 0, 1 << 30, 0) == (OK, 0) and need(M, 1, 1, (1 << 30) - 1)[0] == OK and need(M, 2, (1 << 30) - 1, 1)[0] == OK
    assert need(M, 0, 1 << 30, 0, n_seqs=1 << 20, n_heads=2, seqs_per_flag=1)[0] == SIZE    # a cache whose size 64 bits do not hold


def test_attention_pointers(M):  # noqa: F811
    d = dims(M)
    n = C.c_int64()
    L = M.lib()
    assert L.marl_window_attention_workspace(None, 8, 2, 0, C.byref(n)) == NULL and L.marl_window_attention_workspace(C.byref(d), 8, 2, 0, None) == NULL
    assert need(M, 3)[0] == CONFIG and need(M, -1)[0] == CONFIG
    for x in ("q", "k", "v", "out"):
        assert attend(M, **{x: None}) == NULL and attend(M, **{x: GOOD + 2}) == ALIGN and attend(M, dims(M, precision=1), **{x: GOOD + 1}) == ALIGN
        assert step(M, **{x: None}) == NULL and step(M, **{x: GOOD + 2}) == ALIGN
    for x in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        assert back(M, **{x: None}) == NULL and back(M, **{x: GOOD + 2}) == ALIGN
    assert back(M, lse=None) == NULL and back(M, ws=None) == NULL and back(M, ws=WS + 8) == ALIGN and back(M, lse=LSE + 2) == ALIGN
    assert attend(M, lse=LSE + 2) == ALIGN and attend(M, pos=POS + 2) == ALIGN and back(M, pos=POS + 1) == ALIGN and step(M, pos=POS + 2) == ALIGN
    assert step(M, pos=None) == NULL and step(M, old=(None, None)) == NULL and step(M, dims(M, n_steps=4)) == SIZE and step(M, dims(M, n_steps=0)) == SIZE
    for bad in ((FAR, None), (None, FAR)):
        assert attend(M, old=bad) == NULL and attend(M, new=bad) == NULL and back(M, old=bad) == NULL and step(M, old=bad) == NULL
    for bad in ((FAR + 4, FAR + KEYS), (FAR, FAR + KEYS + 8)):
        assert attend(M, old=bad) == ALIGN and attend(M, new=bad) == ALIGN and back(M, old=bad) == ALIGN and step(M, old=bad) == ALIGN
    many = dims(M, n_steps=1, n_seqs=2, seqs_per_flag=1)
    assert need(M, 2, 4096, 0, d=many)[1] > 0 and step(M, many, 4096, 0, old=(FAR, FAR << 1), ws=None) == NULL
    nothing = dims(M, n_seqs=0)
    assert attend(M, nothing, q=None) == OK and back(M, nothing, q=None, lse=None, ws=None) == OK and step(M, dims(M, n_steps=1, n_seqs=0), q=None) == OK
    assert back(M, dims(M, n_steps=0), q=None, lse=None, ws=None) == OK and attend(M, dims(M, n_steps=0), q=None) == OK


def test_positions_by_number(M):  # noqa: F811
    assert attend(M, first=(1 << 31) - 4) == SIZE and back(M, first=(1 << 31) - 4) == SIZE
    assert attend(M, dims(M, n_seqs=0), first=(1 << 31) - 5) == OK


def test_outputs_that_overlap_themselves(M):  # noqa: F811
    View = M.binding.View
    for strides in ((0, 32, 16), (64, 0, 16), (64, 32, 0)):
        assert attend(M, views=dict(out=View(OUT, *strides))) == CONFIG
        for x, p in (("dq", DQ), ("dk", DK), ("dv", DV)):
            assert back(M, views={x: View(p, *strides)}) == CONFIG
    for strides in ((64, 0, 16), (64, 32, 0)):
        assert step(M, views=dict(out=View(OUT, *strides))) == CONFIG


def test_places(M):  # noqa: F811
    """An output that begins where another array does, or inside a cache that the call reads or writes: wrong answers in silence otherwise."""
    for x in (Q, K, V):
        assert attend(M, out=x) == CONFIG and step(M, out=x) == CONFIG
    for x in (Q, K, V, OUT, POS):
        assert attend(M, lse=x, pos=POS) == CONFIG
    assert attend(M, out=POS, pos=POS) == CONFIG and step(M, out=POS) == CONFIG
    names = dict(q=Q, k=K, v=V, out=OUT, dout=DOUT, dq=DQ, dk=DK, dv=DV)
    for g in ("dq", "dk", "dv"):
        for x in names:
            if x != g:
                assert back(M, **{g: names[x]}) == CONFIG, (g, x)
        assert back(M, **{g: LSE}) == CONFIG and back(M, **{g: POS}, pos=POS) == CONFIG
        assert back(M, **{g: FAR + 64}, old=(FAR, FAR + KEYS)) == CONFIG and back(M, **{g: FAR + KEYS + 64}, old=(FAR, FAR + KEYS)) == CONFIG
    for old in ((FAR, FAR + KEYS), (FAR + VALUES, FAR)):
        for x in (old[0], old[0] + KEYS - 4, old[1], old[1] + VALUES - 4):
            assert attend(M, old=old, out=x) == CONFIG and attend(M, old=old, lse=x) == CONFIG
            assert attend(M, new=old, out=x) == CONFIG and attend(M, new=old, lse=x) == CONFIG and attend(M, new=old, pos=x) == CONFIG
            assert step(M, old=old, out=x) == CONFIG and step(M, old=old, pos=x) == CONFIG
            for y in ("q", "k", "v"):
                assert attend(M, new=old, **{y: x}) == CONFIG and step(M, old=old, **{y: x}) == CONFIG
    # caches: the next one may be the one before, but no part of it and no other's
    old = (FAR, FAR + KEYS)
    other = FAR + (1 << 22)
    for new in ((FAR + 16, other), (other, FAR + KEYS - 16), (other, FAR + KEYS + 16), (FAR - 16, other), (FAR, other), (other, FAR + KEYS), (other, other + 16)):
        assert attend(M, old=old, new=new) == CONFIG, new
    assert step(M, old=(FAR, FAR + 16)) == CONFIG
    # (nothing of it is launched without sequences, so the check alone is seen)
    assert attend(M, dims(M, n_seqs=0), old=old, new=old) == OK


@pytest.mark.parametrize("kind,each", [(0, 64), (1, 64), (2, 64)])
def test_launches(M, kind, each):  # noqa: F811
    """More workgroups than a grid has: refused by the workspace's size and by the call, in front of the first launch."""
    one = dict(n_steps=1, n_heads=1, n_kv_heads=1, dim_k=16, dim_v=16, seqs_per_flag=1)
    most = LIMIT // each
    sizes = [n for n in range(most - 64, most + 64, 16) if n <= 1 << 26]
    codes = [need(M, kind, 1, 0, n_seqs=n, **one)[0] for n in sizes]
    assert set(codes) <= {OK, SIZE} and codes == sorted(codes, reverse=True)
    big = dims(M, n_seqs=1 << 26, **{**one, "n_steps": 4096 if kind < 2 else 1})
    d = need(M, kind, 1, 0, d=big)[0]
    assert d == SIZE or kind == 2
    if kind == 0:
        assert attend(M, big, 1, 0) == SIZE
    elif kind == 1:
        assert back(M, big, 1, 0) == SIZE
    assert attend(M, dims(M, n_seqs=1 << 20, **one), 1 << 20, 0, new=(1 << 40, 1 << 50)) == SIZE      # the cache's own launch


# ---- norm and rotation -------------------------------------------------------------------------------------------------------------------
def norm(M, d=None, q=Q, k=K, qw=None, kw=None, eps=1e-6, table=GOOD, P=8, R=8, pos=None, first=0, inter=0, qo=OUT, ko=DOUT, views={}):
    at = lambda name, p: views.get(name, view(M, p))
    d = dims(M) if d is None else d
    return M.lib().marl_norm_rotary(C.byref(d), at("q", q), at("k", k), qw, kw, eps, table, P, R, pos, first, inter, at("qo", qo), at("ko", ko), None)


def norm_back(M, d=None, eps=1e-6, table=GOOD, P=8, R=8, pos=None, first=0, inter=0, qw=None, kw=None, dqw=FAR, dkw=FAR + 4096, ws=WS, views={}, **kw_):
    p = dict(dqo=DQ, dko=DK, q=Q, k=K, dq=OUT, dk=DOUT)
    p.update(kw_)
    at = {name: views.get(name, view(M, x)) for name, x in p.items()}
    d = dims(M) if d is None else d
    return M.lib().marl_norm_rotary_backward(C.byref(d), at["dqo"], at["dko"], at["q"], at["k"], qw, kw, eps, table, P, R, pos, first, inter, at["dq"], at["dk"], dqw, dkw,
                                             ws, None)


def both(M, d=None, **kw):
    codes = {norm(M, d, **kw), norm_back(M, d, **kw)}
    assert len(codes) == 1, codes
    return codes.pop()


def test_norm_arguments(M):  # noqa: F811
    for x in (dict(P=0), dict(R=0), dict(R=18), dict(first=(1 << 31) - 4)):
        assert both(M, **x) == SIZE, x
    for x in (dict(R=7), dict(inter=2), dict(inter=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert both(M, **x) == CONFIG, x
    for change, code in ((dict(precision=2), CONFIG), (dict(n_steps=-1), SIZE), (dict(n_seqs=-2), SIZE), (dict(n_heads=0), CONFIG), (dict(n_kv_heads=0), CONFIG),
                         (dict(dim_k=0), SIZE), (dict(dim_k=257), SIZE), (dict(seqs_per_flag=0), CONFIG), (dict(seqs_per_flag=4), CONFIG),
                         (dict(n_steps=1 << 30, n_seqs=1 << 30, seqs_per_flag=1), SIZE), (dict(n_heads=(1 << 14) + 1), CONFIG)):
        assert both(M, dims(M, **change)) == code, change
        assert M.lib().marl_norm_rotary_workspace(C.byref(dims(M, **change)), C.byref(C.c_int64())) == code
    assert both(M, q=None) == NULL and both(M, table=None) == NULL and both(M, q=Q + 2) == ALIGN and both(M, pos=POS + 2) == ALIGN and both(M, k=K + 1) == ALIGN
    assert both(M, table=GOOD + 4) == ALIGN and both(M, qw=FAR + 2) == ALIGN and both(M, kw=FAR + 1) == ALIGN
    assert norm(M, qo=None) == NULL and norm(M, ko=None) == NULL and norm(M, qo=OUT + 2) == ALIGN
    assert norm_back(M, ws=None) == NULL and norm_back(M, ws=WS + 4) == ALIGN and norm_back(M, dqw=FAR + 2) == ALIGN and norm_back(M, dkw=FAR) == CONFIG
    for x in ("dqo", "dko", "dq", "dk"):
        assert norm_back(M, **{x: None}) == NULL and norm_back(M, **{x: GOOD + 2}) == ALIGN
    assert M.lib().marl_norm_rotary_workspace(None, C.byref(C.c_int64())) == NULL and M.lib().marl_norm_rotary_workspace(C.byref(dims(M)), None) == NULL


def test_norm_of_nothing(M):  # noqa: F811
    for change in (dict(n_steps=0), dict(n_seqs=0)):
        assert norm(M, dims(M, **change), q=None) == OK
        assert norm_back(M, dims(M, **change), q=None, dqw=None, dkw=None, ws=None) == OK


def test_norm_places(M):  # noqa: F811
    """In place only over its own input, with its strides."""
    View = M.binding.View
    other, narrow = View(Q, 128, 32, 16), View(K, 64, 48, 16)
    assert norm(M, views=dict(qo=other)) == CONFIG and norm(M, views=dict(ko=narrow)) == CONFIG
    for x in (dict(qo=K), dict(ko=Q), dict(qo=DOUT)):
        assert norm(M, **x) == CONFIG
    assert norm_back(M, views=dict(dq=other)) == CONFIG and norm_back(M, views=dict(dk=View(DK, 64, 48, 16))) == CONFIG
    for x in (dict(dq=K), dict(dq=DK), dict(dq=DOUT), dict(dk=Q), dict(dk=DQ), dict(dk=OUT)):
        assert norm_back(M, **x) == CONFIG, x
    for strides in ((0, 32, 16), (64, 0, 16), (64, 32, 0)):
        for x, p in (("qo", OUT), ("ko", DOUT)):
            assert norm(M, views={x: View(p, *strides)}) == CONFIG
        for x, p in (("dq", OUT), ("dk", DOUT)):
            assert norm_back(M, views={x: View(p, *strides)}) == CONFIG


# ---- Python ------------------------------------------------------------------------------------------------------------------------------
def refusals(M, device):  # noqa: F811
    """Calls whose tensors do not fit: shapes, types, strides, workspaces, compared before the library is called."""
    new = lambda *s, **kw: torch.zeros(*s, device=device, **kw)
    i32 = lambda *s: new(*s, dtype=torch.int32)
    q, k, out, lse = new(4, 6, 4, 16), new(4, 6, 2, 16), new(4, 6, 4, 16), new(6, 4, 4)
    old = (new(6, 2, 10, 16), new(6, 2, 10, 16))
    for change in (dict(q=q.half()), dict(q=q[0]), dict(k=k[:3]), dict(v=k.bfloat16()), dict(v=k[0]), dict(out=out[..., :8]), dict(q=q.transpose(2, 3)),
                   dict(lse=lse[:, :3]), dict(lse=lse.double()), dict(lse=new(6, 4, 8)[..., ::2]), dict(positions=i32(4, 4)), dict(positions=i32(3, 6)),
                   dict(positions=new(4, 6)), dict(positions=i32(6, 4).t()), dict(cache=(old[0][:, :, :9], old[1])), dict(cache=(old[0].bfloat16(), old[1])),
                   dict(next_cache=(old[0], old[1][:5])), dict(next_cache=(new(2, 6, 10, 16).transpose(0, 1), old[1])), dict(window=9)):
        yield lambda c=change: M.window_attention(**{**dict(q=q, k=k, v=k, out=out, window=8, sinks=2, cache=old), **c})
    grads = dict(q=q, k=k, v=k, out=out, lse=lse, dout=out, dq=q.clone(), dk=k.clone(), dv=k.clone(), window=8, sinks=2, workspace=new(1 << 16, dtype=torch.uint8))
    for change in (dict(dout=out[:3]), dict(dq=q.bfloat16()), dict(dk=q), dict(dv=k.transpose(2, 3)), dict(lse=lse[0]), dict(workspace=None),
                   dict(workspace=new(64, dtype=torch.uint8)), dict(positions=i32(4, 5)), dict(cache=(old[0][:3], old[1]))):
        yield lambda c=change: M.window_attention_backward(**{**grads, **c})
    for change in (dict(q=q), dict(k=k), dict(v=k[0].half()), dict(positions=i32(4)), dict(positions=i32(1, 6)), dict(positions=new(6)), dict(out=out[0, :, :3]),
                   dict(cache=(old[0], old[1][:, :, 1:])), dict(window=7)):
        yield lambda c=change: M.window_attention_step(**{**dict(q=q[0], k=k[0], v=k[0], cache=old, positions=i32(6), out=out[0], window=8, sinks=2), **c})
    many = (new(1, 1, 4096, 16), new(1, 1, 4096, 16))
    yield lambda: M.window_attention_step(new(1, 1, 16), new(1, 1, 16), new(1, 1, 16), many, i32(1), new(1, 1, 16), 4096)     # shared out: needs a workspace
    table, w = new(9, 8), new(16)
    for change in (dict(table=table[0]), dict(table=table.double()), dict(positions=new(4, 6)), dict(positions=i32(4, 5)), dict(q_out=out.bfloat16()), dict(k=k[0]),
                   dict(q_weight=w[:8]), dict(k_weight=w.double()), dict(k_out=out), dict(q=q.half())):
        yield lambda c=change: M.norm_rotary(**{**dict(q=q, k=k, q_weight=w, k_weight=w, table=table, q_out=out, k_out=k.clone()), **c})
    grads = dict(dq_out=out, dk_out=k, q=q, k=k, q_weight=w, k_weight=w, table=table, dq=q.clone(), dk=k.clone(), dq_weight=w.clone(), dk_weight=w.clone(),
                 workspace=new(1 << 18, dtype=torch.uint8))
    for change in (dict(dq_out=k), dict(dk=k[:3]), dict(dq_weight=w[:4]), dict(dk_weight=w.bfloat16()), dict(workspace=None), dict(workspace=new(4096, dtype=torch.uint8)),
                   dict(q=q[0])):
        yield lambda c=change: M.norm_rotary_backward(**{**grads, **c})


@pytest.mark.gpu
def test_tensors_that_do_not_fit_are_refused(M):  # noqa: F811
    for call in refusals(M, "cuda"):
        with pytest.raises(M.MarlError, match="marl error -3"):
            call()


def test_tensors_in_host_memory_are_refused(M):  # noqa: F811
    q, i = torch.zeros(4, 6, 4, 16), torch.zeros(6, dtype=torch.int32)
    old = (torch.zeros(6, 4, 8, 16), torch.zeros(6, 4, 8, 16))
    table = torch.zeros(9, 8)
    for call in (lambda: M.window_attention(q, q, q, q.clone(), 8), lambda: M.window_attention(q, q, q, q.clone(), 8, cache=old),
                 lambda: M.window_attention_backward(q, q, q, q, torch.zeros(6, 4, 4), q, *[q.clone() for _ in range(3)], 8),
                 lambda: M.window_attention_step(q[0], q[0], q[0], old, i, q[0].clone(), 8), lambda: M.norm_rotary(q, None, None, None, table, q, None),
                 lambda: M.norm_rotary_backward(q, None, q, None, None, None, table, q, None)):
        with pytest.raises(M.MarlError, match="on the GPU"):
            call()


def test_other_arguments_that_are_refused(M):  # noqa: F811
    q = torch.zeros(4, 6, 4, 16)
    with pytest.raises(M.MarlError, match="positions"):       # a number in place of an array
        M.binding._positions(torch.tensor(3, dtype=torch.int32), (4,), 6)
    with pytest.raises(M.MarlError, match="marl error -3"):
        M.window_attention_workspace(q, q, q, 0)
    with pytest.raises(M.MarlError, match="float32 or bfloat16"):
        M.norm_rotary_workspace(q.half(), None)
    with pytest.raises(M.MarlError, match="kind"):
        M.window_attention_workspace(q, q, q, 8, kind="sideways")


def test_tensors_on_another_gpu(M, monkeypatch):  # noqa: F811
    class On:
        def __init__(self, device):
            self.get_device = lambda: device
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    M.binding._here(On(1), None, On(1))
    M.binding._here()
    for bad in ((On(0),), (On(1), On(0)), (On(1), None, On(-1)), (On(-1),), (On(0), On(1))):
        with pytest.raises(M.MarlError, match="current"):
            M.binding._here(*bad)


@pytest.mark.gpu
def test_calls_on_another_gpu(M, monkeypatch):  # noqa: F811
    new = lambda *s, **kw: torch.zeros(*s, device="cuda", **kw)
    q, w, table, at = new(4, 6, 4, 16), new(16), new(9, 8), new(6, dtype=torch.int32)
    old = (new(6, 4, 8, 16), new(6, 4, 8, 16))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: M.window_attention(q, q, q, q.clone(), 8), lambda: M.window_attention_step(q[0], q[0], q[0], old, at, q[0].clone(), 8),
                 lambda: M.window_attention_backward(q, q, q, q, new(6, 4, 4), q, *[q.clone() for _ in range(3)], 8, workspace=new(1 << 16)),
                 lambda: M.norm_rotary(q, None, w, None, table, q.clone(), None),
                 lambda: M.norm_rotary_backward(q, None, q, None, w, None, table, q.clone(), None)):
        with pytest.raises(M.MarlError, match="current"):
            call()


def test_workspaces(M):  # noqa: F811
    assert need(M, 0) == (OK, 0)
    assert need(M, 2, n_steps=1, n_seqs=65536) == (OK, 0)                            # many sequences: a cache is read by one wavefront
    assert 0 < need(M, 2, 4096, 64, n_steps=1, n_seqs=2)[1] < 1 << 24
    assert need(M, 1, n_steps=128, n_seqs=64)[1] < 2 * 128 * 64 * 4 * 4 + (1 << 16)   # a number a row, and little else
    assert need(M, 1, 1 << 12, 1 << 20, n_steps=1 << 16, n_seqs=1, seqs_per_flag=1)[1] < 1 << 28
    q = torch.zeros(4, 6, 4, 16)
    assert M.window_attention_workspace(q, q, q, 8, kind="backward") == need(M, 1, 8, 0, n_kv_heads=4, dim_v=16)[1]
    assert M.norm_rotary_workspace(q, None) > 0


# ---- listings ----------------------------------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def window_listings(tmp_path_factory):
    if shutil.which("hipcc") is None:
        pytest.skip("needs hipcc")
    folder = tmp_path_factory.mktemp("window_listings")

    def listing(src):
        out = str(folder / src.replace(".hip", ".s"))
        subprocess.check_call(["hipcc", *build.flags(src), "--cuda-device-only", "-S", os.path.join(build.CSRC, src), "-o", out])
        with open(out) as f:
            return f.read()

    with ThreadPoolExecutor(max_workers=4) as ex:
        return dict(zip(build.WINDOW_SOURCES, ex.map(listing, build.WINDOW_SOURCES)))


KERNELS = {"window_attention_f32.hip": ["window_rows_kernel", "window_columns_kernel"], "window_attention_bf16.hip": ["window_rows_kernel", "window_columns_kernel"],
           "window_attention.hip": ["window_step_kernel", "window_cache_kernel"], "norm_rotary.hip": ["norm_rotary_kernel", "norm_weight_kernel"]}


@pytest.mark.parametrize("src", build.WINDOW_SOURCES)
def test_no_lds_write_is_pending_at_a_barrier(window_listings, src):
    text = window_listings[src]
    found = pending_writes_at_barriers(text)
    for name in KERNELS[src]:
        assert re.search(rf"^_Z\S*{name}\S*:", text, re.M), name
    assert {k: v for k, v in found.items() if v} == {}
    assert "v_pk_fma_f32" not in text and "v_pk_mul_f32" not in text and "v_pk_add_f32" not in text
    assert mixed_chains(text) == []


def test_matrix_products(window_listings):
    assert set(re.findall(r"v_mfma_\w+?_(\d+x\d+x\d+)", window_listings["window_attention_bf16.hip"])) == {"32x32x16"}
    assert set(re.findall(r"v_mfma_\w+?_(\d+x\d+x\d+)", window_listings["window_attention_f32.hip"])) == {"32x32x2"}
