"""Which stream's memory the buffers of paper_2507_03220_amd/block.py are: torch gives a freed tensor's memory to later work of the stream that it was allocated on, so a buffer that
another stream's kernels use may be somebody else's by then.  The calls and torch's allocator are stood in for; no GPU is touched."""
import contextlib

import pytest
import torch

from paper_2507_03220_amd import binding as sb
from paper_2507_03220_amd import block as blk

HERE = 5                                                   # the stream that is torch's current one


@pytest.fixture
def world(monkeypatch):
    """Tensors remember the stream they were allocated in the order of (and which others were made to wait for them), calls the tensors that they were given."""
    class World:
        order, home, shared, calls = [HERE], {}, set(), []
    w = World()
    w.order, w.home, w.shared, w.calls = [HERE], {}, set(), []

    @contextlib.contextmanager
    def on(stream):
        w.order.append(stream)
        yield
        w.order.pop()
    empty = torch.empty

    def fake_empty(*a, device=None, **kw):
        t = empty(*a, **kw)
        w.home[t.data_ptr()] = (w.order[-1], t)            # (held: no address comes twice)
        return t

    def call(name, stream_at):
        def f(*a, stream=None):
            w.calls.append((name, stream if stream is not None else a[stream_at], [x.data_ptr() for x in a if isinstance(x, torch.Tensor)]))
        return f
    monkeypatch.setattr(blk, "_on", on)
    monkeypatch.setattr(blk, "_also_on", lambda t, stream: w.shared.add((t.data_ptr(), stream)), raising=False)
    monkeypatch.setattr(torch, "empty", fake_empty)
    for name, at in (("symb_norm_fwd", 4), ("symb_base_linear_fwd", 8), ("symb_adapter_grad", 7), ("symb_base_linear_bwd_input", 7), ("symb_norm_bwd", 7)):
        monkeypatch.setattr(sb, name, call(name, at))
    return w


def _check(w):
    assert w.calls
    for name, stream, tensors in w.calls:
        for at in tensors:
            if at in w.home:
                assert w.home[at][0] == stream or (at, stream) in w.shared, (name, stream, w.home[at][0])


def _projection():
    W = torch.zeros(24, 16, dtype=torch.bfloat16)
    return blk.NormedProjection(None, W, [3, 2], [sb.Norm(), sb.Norm()], [sb.Adapter(), sb.Adapter()]), torch.zeros(5, 16, dtype=torch.bfloat16), torch.zeros(5, 24, dtype=torch.bfloat16)


@pytest.mark.parametrize("forward,backward", [((HERE,), HERE), ((9,), 9), ((0,), 0), ((9, HERE), HERE), ((HERE, 9), 9), ((9,), 11), ((9, 9, 11), 9)])
def test_a_normed_projection_on_any_stream(world, forward, backward):
    run, X, dY = _projection()
    for s in forward:
        y = run.forward(X, None, s)
        assert y is run.Y and y.shape == (5, 24)
    n = run.N
    d = run.backward(X, dY, stream=backward)
    assert d is run.dX and d.shape == X.shape and run.N is n                 # (the rows of the last forward pass)
    _check(world)


def test_buffers_stay_while_the_stream_does(world):
    run, X, dY = _projection()
    a = run.forward(X, None, 9), run.N, run.ws, run.backward(X, dY, stream=9), run.dN
    b = run.forward(X, None, 9), run.N, run.ws, run.backward(X, dY, stream=9), run.dN
    assert all(x is y for x, y in zip(a, b))


def test_a_backward_pass_needs_a_forward_pass(world):
    run, X, dY = _projection()
    with pytest.raises(RuntimeError):
        run.backward(X, dY)
    assert not world.calls
