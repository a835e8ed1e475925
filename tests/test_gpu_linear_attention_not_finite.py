"""Infinities and NaNs in linear attention where they take other ways through the library: sequences cut over time (the states of the stretches, their
join), query heads that share keys and values (shares in fp32), widths and lengths that are no whole tiles, several slices of columns."""
import pytest
import torch

import memory_oracle as O
from test_gpu_linear_attention import BF16, F32, PARTS, absolute, backward, forward, make

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def M():
    import paper_2107_01460_amd as m
    assert torch.cuda.is_available()
    return m


def same_places(M, s):
    """Infinities and NaNs lie where the recurrence in 64 bits has them, and what is finite is as exact as anywhere."""
    q, v = s["q"], s["v"]
    T, n, group = q.shape[0], 1.25 * q.shape[0] + max(q.shape[3], v.shape[3]), q.shape[2] // v.shape[2]
    bf16, parts = q.dtype == BF16, PARTS[q.dtype]

    def reference(d):
        args = (d["q"], d["k"], d["v"], d["decay"])
        return O.attend(*args, d["state"], d["done"], d["scale"]) + O.attend_backward(*args, d["dout"], d["state"], d["dnext"], d["done"], d["scale"])
    for x, r, z, name in zip(forward(M, s) + backward(M, s), reference(s), reference(absolute(s)), ("out", "next_state", "dq", "dk", "dv", "dstate")):
        assert torch.equal(x.isnan(), r.isnan()), (name, "NaNs")
        assert torch.equal(x.isfinite(), r.isfinite()), (name, "infinities")
        assert torch.equal(x[x.isinf()].double(), r[r.isinf()]), (name, "signs")
        ok = r.isfinite()
        state = name in ("next_state", "dstate")
        O.within(x[ok], r[ok], z[ok], n + group, bf16 and not state, 0.0 if state else parts)


# stretches of 64 steps; over one of them a decay of 0.1 leaves a power of 1e-64, which 32 bits do not hold; one of 0 leaves nothing but what is not finite
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("decay", [0.0, 0.1, 0.75, 0.99])
@pytest.mark.parametrize("bad,at", [(NAN, 10), (INF, 10), (-INF, 300), (NAN, 300), (NAN, 511)])
def test_in_a_sequence_that_is_cut(M, bad, at, decay, dtype):
    """In k, q, v and dout in turn, without an end, with one behind it and with several: twelve pairs of sequences, the first of each pair with the bad value and the ends."""
    kinds = [(name, ends) for name in ("k", "q", "v", "dout") for ends in ((), (400,), (5, 64, 383))]
    s = make(512, 2 * len(kinds), 2, 1, 32, 16, dtype, seed=at)
    s["decay"] = torch.tensor([decay, 0.9], device="cuda")
    s["done"] = torch.zeros((512, 2 * len(kinds)), dtype=torch.uint8, device="cuda")
    for i, (name, ends) in enumerate(kinds):
        for t in ends:
            s["done"][t, 2 * i] = 1
        s[name][at, 2 * i, 0, 7] = bad
    assert M.linear_attention_workspace(s["q"], s["k"], s["v"]) > 0
    same_places(M, s)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("decay", [0.0, 0.1, 0.99])
def test_states_given_to_a_sequence_that_is_cut(M, decay, dtype):
    for bad in (NAN, INF):
        for ends in ((), (200,)):
            s = make(512, 2, 2, 2, 16, 32, dtype, seed=4)
            s["decay"] = torch.full((2,), decay, device="cuda")
            s["done"] = torch.zeros((512, 2), dtype=torch.uint8, device="cuda")
            for t in ends:
                s["done"][t, 1] = 1
            s["state"][1, 0, 3, 5] = s["dnext"][1, 1, 2, 6] = bad
            same_places(M, s)


# shared heads, widths on no tile's border, more than one slice, a last tile that is not whole; cut and uncut
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,B,H,Hk,Dk,Dv", [(45, 6, 6, 2, 40, 72), (75, 4, 3, 1, 33, 127), (19, 3, 2, 1, 128, 40), (7, 5, 4, 2, 5, 3), (333, 1, 4, 2, 40, 72)])
@pytest.mark.parametrize("bad", [NAN, INF])
def test_shared_heads_and_odd_sizes(M, bad, T, B, H, Hk, Dk, Dv, dtype):
    for name in ("k", "q", "v", "dout"):
        s = make(T, B, H, Hk, Dk, Dv, dtype, seed=T, episode=20)
        print("case", name, bad, T, B, H, Hk, Dk, Dv, dtype, flush=True)
        d = s[name].shape[3] - 1
        s[name][T // 2, 0, 0, d] = bad
        s[name][T - 1, B - 1, s[name].shape[2] - 1, 0] = bad
        same_places(M, s)
