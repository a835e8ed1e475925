"""The sequence operators refuse bad arguments on the host, before anything is launched; and their kernels' barriers in the listing."""
import ctypes as C
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

from paper_2107_01460_amd import build
from test_rollout_waits import pending_writes_at_barriers

OK, NULL, ALIGN, CONFIG, SIZE = 0, -1, -2, -3, -5
GOOD = 0x10000


@pytest.fixture(scope="module")
def M():
    import paper_2107_01460_amd as m
    if not os.path.exists(m.binding._LIB_PATH):
        build.build(verbose=False)
    m.lib()
    return m


def dims(M, **kw):
    d = dict(precision=0, n_steps=4, n_seqs=6, n_heads=4, n_kv_heads=2, dim_k=16, dim_v=32, seqs_per_flag=2, scale=1.0)
    d.update(kw)
    return M.binding.AttentionDims(*d.values())


def view(M, data=GOOD):
    return M.binding.View(data, 64, 32, 16)


def attend(M, d, q=GOOD, decay=GOOD, state=None, out=GOOD, nxt=None, ws=GOOD):
    v = lambda p=GOOD: view(M, p)
    return M.lib().marl_linear_attention(C.byref(d), v(q), v(), v(), decay, state, None, v(out), nxt, ws, None)


BAD_DIMS = [(dict(precision=2), CONFIG), (dict(n_steps=-1), SIZE), (dict(n_seqs=-2), SIZE), (dict(n_heads=0), CONFIG), (dict(n_kv_heads=3), CONFIG),
            (dict(n_kv_heads=0), CONFIG), (dict(dim_k=0), CONFIG), (dict(dim_k=129), CONFIG), (dict(dim_v=256), CONFIG), (dict(seqs_per_flag=0), CONFIG),
            (dict(seqs_per_flag=4), CONFIG), (dict(n_seqs=1 << 26, n_heads=4), SIZE), (dict(n_steps=(1 << 30) + 1), SIZE)]


@pytest.mark.parametrize("change,code", BAD_DIMS)
def test_attention_sizes(M, change, code):
    d, n = dims(M, **change), C.c_int64()
    v = view(M)
    assert M.lib().marl_linear_attention_workspace(C.byref(d), 0, C.byref(n)) == code
    assert attend(M, d) == code
    assert M.lib().marl_linear_attention_backward(C.byref(d), v, v, v, GOOD, None, None, v, None, v, v, v, None, GOOD, None) == code
    assert M.lib().marl_linear_attention_step(C.byref(d), v, v, v, GOOD, GOOD, None, v, GOOD, None) == code


def test_attention_pointers(M):
    L, d, v = M.lib(), dims(M), view(M)
    assert attend(M, d, q=None) == NULL and attend(M, d, out=None) == NULL and attend(M, d, decay=None) == NULL
    assert attend(M, d, q=GOOD + 2) == ALIGN and attend(M, d, state=GOOD + 4) == ALIGN and attend(M, d, nxt=GOOD + 8) == ALIGN
    assert attend(M, d, decay=GOOD + 2) == ALIGN
    assert attend(M, dims(M, precision=1), out=GOOD + 1) == ALIGN
    long = dims(M, n_steps=4096, n_seqs=2)
    assert attend(M, long, ws=None) == NULL and attend(M, long, ws=GOOD + 8) == ALIGN
    grad = lambda dq, ws=GOOD, d=d: L.marl_linear_attention_backward(C.byref(d), v, v, v, GOOD, None, None, v, None, view(M, dq), v, v, None, ws, None)
    assert grad(None) == NULL and grad(GOOD + 2) == ALIGN and grad(GOOD, None) == NULL   # shared heads: a workspace is needed
    step = lambda d, q=GOOD, s=GOOD, n=GOOD: L.marl_linear_attention_step(C.byref(d), view(M, q), v, v, GOOD, s, None, v, n, None)
    one = dims(M, n_steps=1)
    assert step(d) == SIZE and step(one, q=None) == NULL and step(one, s=None) == NULL and step(one, n=None) == NULL and step(one, s=GOOD + 4) == ALIGN
    assert L.marl_linear_attention(None, v, v, v, GOOD, None, None, v, None, None, None) == NULL
    assert L.marl_linear_attention_workspace(C.byref(d), 0, None) == NULL
    assert attend(M, dims(M, n_seqs=0), q=None, ws=None) == OK     # nothing to do


def test_outputs_that_overlap_themselves(M):
    L, d = M.lib(), dims(M)
    one, V = dims(M, n_steps=1), M.binding.View
    v = view(M)
    for bad in (V(GOOD, 0, 32, 16), V(GOOD, 64, 0, 16), V(GOOD, 64, 32, 0)):
        assert L.marl_linear_attention(C.byref(d), v, v, v, GOOD, None, None, bad, None, GOOD, None) == CONFIG
        for k in range(3):
            out = [bad if i == k else v for i in range(3)]
            assert L.marl_linear_attention_backward(C.byref(d), v, v, v, GOOD, None, None, v, None, *out, None, GOOD, None) == CONFIG
        assert L.marl_rotary(C.byref(d), v, v, GOOD, 8, 8, None, 0, 0, 0, v, bad, None) == CONFIG
    assert L.marl_linear_attention_step(C.byref(one), v, v, v, GOOD, GOOD, None, V(GOOD, 0, 0, 16), GOOD, None) == CONFIG
    assert L.marl_layer_norm(0, 4, 8, GOOD, 8, None, None, 1e-5, GOOD, 7, None, None, None) == CONFIG
    assert L.marl_layer_norm_backward(0, 4, 8, GOOD, 8, GOOD, 8, None, GOOD, GOOD, GOOD, 0, None, None, None, None) == CONFIG


def test_attention_workspace(M):
    n = C.c_int64()
    need = lambda back, **kw: (M.lib().marl_linear_attention_workspace(C.byref(dims(M, **kw)), back, C.byref(n)), n.value)[1]
    assert need(0, n_steps=128, n_seqs=65536) == 0                      # many sequences: nothing is cut
    assert need(1, n_steps=128, n_seqs=65536, n_kv_heads=4) == 0
    assert need(1, n_steps=128, n_seqs=65536) == 128 * 65536 * 4 * (16 + 32) * 4
    assert need(0, n_steps=4096, n_seqs=2) > 0
    assert need(0, n_steps=1 << 20, n_seqs=1, seqs_per_flag=1) < 1 << 27   # as many stretches as fill the chip, not as many as there are steps


def test_layer_norm_arguments(M):
    L, n = M.lib(), C.c_int64()
    norm = lambda p=0, rows=4, w=8, x=GOOD, y=GOOD, weight=None, eps=1e-5, mean=None: L.marl_layer_norm(p, rows, w, x, 8, weight, None, eps, y, 8, mean, None, None)
    assert norm(p=2) == CONFIG and norm(rows=-1) == SIZE and norm(w=0) == SIZE and norm(w=16385) == SIZE and norm(x=None) == NULL and norm(y=None) == NULL
    assert norm(x=GOOD + 2) == ALIGN and norm(p=1, x=GOOD + 1) == ALIGN and norm(weight=GOOD + 1) == ALIGN and norm(mean=GOOD + 2) == ALIGN
    assert norm(eps=-1.0) == CONFIG and norm(eps=float("nan")) == CONFIG and norm(rows=0, x=None, y=None) == OK
    grad = lambda p=0, rows=4, w=8, dy=GOOD, mean=GOOD, dx=GOOD, dw=GOOD, ws=GOOD: L.marl_layer_norm_backward(p, rows, w, dy, 8, GOOD, 8, None, mean, GOOD, dx, 8, dw, None, ws, None)
    assert grad(p=3) == CONFIG and grad(rows=-1) == SIZE and grad(w=0) == SIZE and grad(dy=None) == NULL and grad(mean=None) == NULL and grad(dx=None) == NULL
    assert grad(ws=None) == NULL and grad(ws=GOOD + 4) == ALIGN and grad(dw=GOOD + 1) == ALIGN and grad(dy=GOOD + 2) == ALIGN
    assert L.marl_layer_norm_workspace(4, 8, None) == NULL and L.marl_layer_norm_workspace(4, 0, C.byref(n)) == SIZE
    assert L.marl_layer_norm_workspace(1 << 30, 16384, C.byref(n)) == OK and n.value < 1 << 30


def test_rotary_arguments(M):
    L = M.lib()
    none = M.binding.View(None, 0, 0, 0)

    def turn(d=None, q=GOOD, k=GOOD, table=GOOD, P=8, R=8, pos=None, inter=0, inv=0, out=GOOD):
        d = dims(M) if d is None else d
        return L.marl_rotary(C.byref(d), view(M, q), view(M, k), table, P, R, pos, 0, inter, inv, view(M, out), view(M, out), None)
    assert turn(q=None) == NULL and turn(table=None) == NULL and turn(out=None) == NULL and turn(q=GOOD + 2) == ALIGN and turn(table=GOOD + 4) == ALIGN
    assert turn(pos=GOOD + 2) == ALIGN and turn(R=7) == CONFIG and turn(R=0) == SIZE and turn(R=18) == SIZE and turn(P=0) == SIZE
    assert turn(inter=2) == CONFIG and turn(inv=-1) == CONFIG and turn(dims(M, precision=5)) == CONFIG and turn(dims(M, seqs_per_flag=4)) == CONFIG
    assert turn(dims(M, n_kv_heads=0)) == CONFIG and turn(dims(M, dim_k=2000)) == SIZE and turn(dims(M, n_steps=-1)) == SIZE
    assert turn(dims(M, n_steps=0), q=None) == OK
    assert L.marl_rotary(None, none, none, GOOD, 8, 8, None, 0, 0, 0, none, none, None) == NULL

    def table(**kw):
        d = dict(n_positions=8, rotary_dim=8, scaling=0, base=1e4, factor=2.0, trained_length=64.0, slow=1.0, fast=32.0, amplitude=1.0)
        at = kw.pop("at", GOOD)
        d.update(kw)
        return L.marl_rotary_table(C.byref(M.binding.RotaryDims(*d.values())), at, None)
    assert table(n_positions=0) == SIZE and table(rotary_dim=0) == SIZE and table(rotary_dim=5) == CONFIG and table(scaling=4) == CONFIG
    assert table(base=0.0) == CONFIG and table(scaling=1, factor=0.0) == CONFIG and table(scaling=2, rotary_dim=2) == CONFIG
    assert table(scaling=3, trained_length=0.0) == CONFIG and table(scaling=3, fast=1.0) == CONFIG and table(at=None) == NULL and table(at=GOOD + 8) == ALIGN
    assert L.marl_rotary_table(None, GOOD, None) == NULL


def refusals(M, device):
    """Calls whose tensors do not fit: shapes, types, strides, workspaces, compared before the library is called."""
    new = lambda *s, **kw: torch.zeros(*s, device=device, **kw)
    q, k = new(4, 6, 4, 16), new(4, 6, 2, 16)
    decay, out = new(4), new(4, 6, 4, 16)
    u8 = lambda *s: new(*s, dtype=torch.uint8)
    for change in (dict(q=q.half()), dict(q=q[0]), dict(k=k[:3]), dict(v=k.bfloat16()), dict(decay=decay[:3]), dict(decay=decay.double()), dict(out=out[..., :8]),
                   dict(q=q.transpose(2, 3)), dict(state=new(6, 4, 16, 15)), dict(done=u8(4, 4)), dict(done=u8(3, 6)), dict(done=new(4, 6)),
                   dict(next_state=new(4, 6, 16, 16).transpose(0, 1))):
        yield lambda c=change: M.linear_attention(**{**dict(q=q, k=k, v=k, decay=decay, out=out), **c})
    yield lambda: M.linear_attention(new(4096, 1, 1, 16), *[new(4096, 1, 1, 16)] * 2, decay[:1], new(4096, 1, 1, 16))   # long: needs a workspace
    yield lambda: M.linear_attention_backward(q, k, k, decay, out, q.clone(), k.clone(), k.clone(), u8(64))                # shared heads: too small a one
    for change in (dict(q=q), dict(state=new(6, 4, 16, 8)), dict(done=u8(4)), dict(done=u8(1, 6)), dict(out=out[0, :, :3]), dict(k=k[0].half())):
        yield lambda c=change: M.linear_attention_step(**{**dict(q=q[0], k=k[0], v=k[0], decay=decay, state=new(6, 4, 16, 16), out=out[0]), **c})
    x = new(5, 8)
    for args in ((x.half(), None, None, x), (x, new(7), None, x), (x, None, None, x[:4]), (x.t(), None, None, x.t()), (x, None, new(8).double(), x)):
        yield lambda a=args: M.layer_norm(*a)
    yield lambda: M.layer_norm_backward(x, x, None, new(5), new(5), x.clone(), new(8), None, u8(4))
    yield lambda: M.layer_norm_backward(x, x, None, new(4), new(5), x.clone())
    table = new(9, 8)
    for change in (dict(table=table[0]), dict(positions=new(4, 6)), dict(positions=new(4, 5, dtype=torch.int32)), dict(q_out=out.bfloat16()), dict(k=k[0])):
        yield lambda c=change: M.rotary(**{**dict(q=q, k=k, table=table, q_out=out, k_out=k.clone()), **c})


@pytest.mark.gpu
def test_tensors_that_do_not_fit_are_refused(M):
    for call in refusals(M, "cuda"):
        with pytest.raises(M.MarlError, match="marl error -3"):
            call()


def test_tensors_in_host_memory_are_refused(M):
    q, x = torch.zeros(4, 6, 4, 16), torch.zeros(5, 8)
    for call in (lambda: M.linear_attention(q, q, q, torch.ones(4), q.clone()), lambda: M.layer_norm(x, None, None, x), lambda: M.rotary(q, None, x, q, None),
                 lambda: M.linear_attention_step(q[0], q[0], q[0], torch.ones(4), torch.zeros(6, 4, 16, 16), q[0].clone())):
        with pytest.raises(M.MarlError, match="on the GPU"):
            call()


@pytest.fixture(scope="module")
def memory_listings(tmp_path_factory):
    if shutil.which("hipcc") is None:
        pytest.skip("needs hipcc")
    folder = tmp_path_factory.mktemp("memory_listings")

    def listing(src):
        out = str(folder / src.replace(".hip", ".s"))
        subprocess.check_call(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, src), "-o", out])
        with open(out) as f:
            return f.read()

    with ThreadPoolExecutor(max_workers=8) as ex:
        return dict(zip(build.MEMORY_SOURCES, ex.map(listing, build.MEMORY_SOURCES)))


KERNELS = {"linear_attention.hip": ["step_kernel", "join_kernel", "sum_heads"], "linear_attention_f32.hip": ["scan_kernel"],
           "linear_attention_bf16.hip": ["scan_kernel"], "layer_norm.hip": ["layer_norm_kernel", "layer_norm_backward", "column_sum"], "rotary.hip": ["rotary_kernel"]}


@pytest.mark.parametrize("src", build.MEMORY_SOURCES)
def test_no_lds_write_is_pending_at_a_barrier(memory_listings, src):
    found = pending_writes_at_barriers(memory_listings[src])
    for name in KERNELS[src]:
        assert any(name in k for k in found), name
    assert {k: v for k, v in found.items() if v} == {}
    assert "v_pk_fma_f32" not in memory_listings[src] and "v_pk_mul_f32" not in memory_listings[src] and "v_pk_add_f32" not in memory_listings[src]
