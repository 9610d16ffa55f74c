"""The guard of captures (a backward pass that is captured beside a living eager graph of the same leaf ends the process), on the CPU: what it sees of
graphs, with torch's answers about streams replaced."""
import sys
import threading

import pytest
import torch

from paper_2602_08007_b200 import layers


class Through(torch.autograd.Function):
    """A differentiable call with the guard in front, as the layers have it."""

    @staticmethod
    def forward(ctx, graph, x, w):
        layers._guard_capture(ctx, graph, x, w)
        return x * w

    @staticmethod
    def backward(ctx, dy):
        return None, dy, dy


def through(x, w):
    return Through.apply(torch.is_grad_enabled(), x, w)


@pytest.fixture
def capturing(monkeypatch):
    """A switch per thread: whether the current stream is being captured."""
    state = threading.local()
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: getattr(state, "on", False))
    return state


def leaf():
    return torch.ones(3, requires_grad=True)


def test_a_living_graph_of_the_leaf_is_refused(capturing):
    w, other = leaf(), leaf()
    y = through(torch.ones(3), w)
    capturing.on = True
    through(torch.ones(3), other)
    with torch.no_grad():
        through(torch.ones(3), w)
    with pytest.raises(RuntimeError, match="still alive"):
        through(torch.ones(3), w)
    del y
    through(torch.ones(3), w)


def test_threads_that_make_graphs_do_not_disturb_a_capture(capturing):
    """Graphs come and go in other threads while a capture looks through those that live."""
    stop, failed, interval = threading.Event(), [], sys.getswitchinterval()
    sys.setswitchinterval(1e-6)

    def make():
        try:
            held = []
            while not stop.is_set():
                held.append(through(torch.ones(3), leaf()))
                if len(held) > 200:
                    del held[:100]
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=make) for _ in range(3)]
    for t in threads:
        t.start()
    try:
        capturing.on = True
        for _ in range(300):
            through(torch.ones(3), leaf())
    except Exception as e:
        failed.append(e)
    finally:
        sys.setswitchinterval(interval)
        stop.set()
        for t in threads:
            t.join()
    assert not failed


def test_leaves_that_reach_a_call_through_others_are_seen(capturing):
    """A weight that is cast, viewed or computed on the way; a leaf that the input of a call came from; and leaves that have nothing to do with each other."""
    w, x, other = leaf(), leaf(), leaf()
    y = through((2 * x).exp(), w.double().float().view(3))
    capturing.on = True
    for a, b in ((torch.ones(3), w), (torch.ones(3), w * 3), (x, other), (x.sin(), other.neg())):
        with pytest.raises(RuntimeError, match="still alive"):
            through(a, b)
            pytest.fail("was taken")
    z = through(other.exp(), other * 2).sum()
    del y
    through(x * 2, w.double().float())
    assert z.requires_grad


def test_leaves_are_not_held_beyond_their_graph(capturing):
    """The guard itself keeps nothing alive."""
    import weakref
    w = leaf()
    y = through(torch.ones(3), w)
    gone, node = weakref.ref(y.grad_fn), y.grad_fn
    assert node in layers._EAGER and not any(isinstance(v, (torch.Tensor, list, tuple)) for v in vars(node).values())
    del y, node
    assert gone() is None


def test_graphs_of_other_streams_are_not_refused(capturing, monkeypatch):
    """Only the default stream cannot be reached from a capture.  A graph of another stream that may share accumulators with one of the default stream counts as
    one of its own, even when that one is gone."""
    where = threading.local()
    monkeypatch.setattr(layers, "_on_default_stream", lambda t: getattr(where, "default", True))
    w = leaf()
    where.default = False
    y = through(torch.ones(3), w)
    capturing.on = True
    through(torch.ones(3), w)
    capturing.on = False
    where.default = True
    z = through(torch.ones(3), w)
    where.default = False
    y = through(torch.ones(3), w)
    del z
    capturing.on = True
    with pytest.raises(RuntimeError, match="still alive"):
        through(torch.ones(3), w)
    assert y.requires_grad
