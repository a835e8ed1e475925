"""What the sequence operators write counts as changed for autograd: a backward pass that needs the old values raises, as behind torch's own in-place operations."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import paper_2107_01460_amd as m
    assert torch.cuda.is_available()
    return m


def test_a_step_on_the_states_of_a_pending_gradient(M):
    torch.manual_seed(0)
    c = M.MemoryCritic(8, width=16, heads=2, layers=1, max_episode=20)
    obs, positions = torch.randn(3, 4, 8, device="cuda"), torch.arange(3, dtype=torch.int32, device="cuda")[:, None].repeat(1, 4)
    state = [torch.randn_like(s) for s in c.initial_state(4)]
    values, _ = c(obs, positions, None, state)
    c.step(obs[0], positions[0], state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        values.sum().backward()
    values, _ = c(obs, positions, None, state)
    c.step(obs[0], positions[0], [s.clone() for s in state])
    values.sum().backward()


def test_every_output(M):
    new = lambda *s: torch.randn(*s, device="cuda")
    q, decay, state = new(2, 3, 2, 8), torch.rand(2, device="cuda"), new(3, 2, 8, 8)
    x, mean, rstd = new(5, 8), new(5), new(5).abs()
    out, nxt, dq, dk, dv, ds, y, dw, db = new(2, 3, 2, 8), new(3, 2, 8, 8), new(2, 3, 2, 8), new(2, 3, 2, 8), new(2, 3, 2, 8), new(3, 2, 8, 8), new(5, 8), new(8), new(8)
    ko, table = new(2, 3, 2, 8), M.rotary_table(4, 8)
    for call, written in (
            (lambda: M.linear_attention(q, q, q, decay, out, state=state, next_state=nxt), (out, nxt)),
            (lambda: M.linear_attention(q, q, q, decay, out), (out,)),
            (lambda: M.linear_attention_backward(q, q, q, decay, out, dq, dk, dv, dstate=ds), (dq, dk, dv, ds)),
            (lambda: M.linear_attention_step(q[0], q[0], q[0], decay, state, out[0]), (state, out)),
            (lambda: M.linear_attention_step(q[0], q[0], q[0], decay, state, out[0], next_state=nxt), (nxt, out)),
            (lambda: M.layer_norm(x, None, None, y, mean, rstd), (y, mean, rstd)),
            (lambda: M.layer_norm_backward(x, x, None, mean, rstd, y, dw, db, M.alloc_workspace(M.layer_norm_workspace(5, 8))), (y, dw, db)),
            (lambda: M.rotary(q, q, table, out, ko), (out, ko)),
            (lambda: M.rotary(out, None, table, out, None), (out,))):
        everything = (q, decay, state, x, mean, rstd, out, nxt, dq, dk, dv, ds, y, dw, db, ko, table)
        before = [t._version for t in everything]
        call()
        for t, b in zip(everything, before):
            assert (t._version > b) == any(t is w for w in written)
    with torch.inference_mode():   # tensors without a version
        z = new(5, 8)
        M.layer_norm(z, None, None, z)
