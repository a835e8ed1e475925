"""Integers past 32 bits are refused where they would otherwise arrive as others: windows, first steps, positions by number, sizes of tables."""
import pytest
import torch

from test_memory_boundary import M  # noqa: F401  (the fixture)

PAST = [2 ** 31, 2 ** 32, 2 ** 32 + 8, -2 ** 31 - 1, -2 ** 32 + 8, 2 ** 63, 2 ** 64 + 8]


@pytest.mark.parametrize("n", PAST)
@pytest.mark.parametrize("kind", ["forward", "backward", "step"])
def test_workspaces(M, kind, n):  # noqa: F811
    q = torch.zeros(1, 6, 4, 16)
    for window, sinks in ((n, 0), (8, n)):
        with pytest.raises(M.MarlError, match="marl error -3"):
            M.window_attention_workspace(q, q, q, window, sinks, kind=kind)


@pytest.mark.parametrize("n", PAST)
def test_sizes(M, n):  # noqa: F811
    for call in (lambda: M.layer_norm_workspace(4, n), lambda: M.rotary_table(n, 8), lambda: M.rotary_table(8, n)):
        with pytest.raises(M.MarlError, match="marl error -3"):
            call()


def calls(M, device, n):  # noqa: F811
    new = lambda *s, **kw: torch.zeros(*s, device=device, **kw)
    q, lse, table, at = new(1, 6, 4, 16), new(6, 4, 1), new(9, 8), new(6, dtype=torch.int32)
    ws = new(1 << 16, dtype=torch.uint8)
    old = (new(6, 4, 8, 16), new(6, 4, 8, 16))
    for looks in (dict(window=n), dict(window=8, sinks=n), dict(window=8, first_position=n)):
        yield lambda a=looks: M.window_attention(q, q, q, q.clone(), **a)
        yield lambda a=looks: M.window_attention_backward(q, q, q, q, lse, q, q.clone(), q.clone(), q.clone(), workspace=ws, **a)
    for looks in (dict(window=n), dict(window=8, sinks=n)):
        yield lambda a=looks: M.window_attention_step(q[0], q[0], q[0], old, at, q[0].clone(), **a)
    yield lambda: M.norm_rotary(q, None, None, None, table, q.clone(), None, first_position=n)
    yield lambda: M.norm_rotary_backward(q, None, q, None, None, None, table, q.clone(), None, first_position=n)
    yield lambda: M.rotary(q, None, table, q.clone(), None, first_position=n)


@pytest.mark.gpu
@pytest.mark.parametrize("n", PAST)
def test_calls(M, n):  # noqa: F811
    for call in calls(M, "cuda", n):
        with pytest.raises(M.MarlError, match="marl error -3"):
            call()


@pytest.mark.parametrize("n", PAST)
def test_calls_reach_no_library(M, monkeypatch, n):  # noqa: F811
    """The same calls without a GPU: refused in front of the library, which is not called."""
    class None_:
        def __getattr__(self, name):
            raise AssertionError(name)
    monkeypatch.setattr(M.binding, "lib", lambda: None_())
    monkeypatch.setattr(M.binding, "_here", lambda *t: None)
    monkeypatch.setattr(M.binding, "_stream", lambda s: None)
    for name in ("_view", "_step_view", "_floats", "_cache", "_workspace"):
        monkeypatch.setattr(M.binding, name, lambda *a: None)
    monkeypatch.setattr(M.binding, "_positions", lambda *a: (None, 1))
    for call in calls(M, "cpu", n):
        with pytest.raises(M.MarlError, match="marl error -3"):
            call()


@pytest.mark.gpu
def test_the_largest_that_there_are(M):  # noqa: F811
    q, k = torch.ones(2, 1, 1, 8, device="cuda"), torch.full((2, 1, 1, 8), 2.0, device="cuda")
    out = torch.empty_like(q)
    M.window_attention(q, q, k, out, 2 ** 30, 0, first_position=2 ** 31 - 3)
    assert torch.equal(out, k)
    M.window_attention(q, q, k, out, 2 ** 30 - 1, 1, first_position=-2 ** 31)      # no row holds a step
    assert not out.any()
