"""Dense plans on streams other than the one their memory belongs to (GPU)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
BUSY = 200_000_000      # clock cycles for which a stream is held up: a tenth of a second


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def rand(n, seed):
    return torch.randn(n, generator=torch.Generator().manual_seed(seed)).cuda()


def spans(tensors):
    return [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors if t.numel()]


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("call", ["step", "grad_norm", "copy_state"])
def test_a_dropped_plan_keeps_its_memory_until_its_calls_are_done(tsr, call, given):
    """A plan is called on a stream that is held up, and dropped: nothing that it allocated is given to anyone else before the
    stream gets there.  The stream is an argument or torch's current one."""
    p, g = rand(300_000, 1), rand(300_000, 2)
    q = p.clone()
    want = tsr.DensePlan([q], [g], state_dtype=F8)
    want.step(tsr.make_hyper(1))
    dst = [torch.zeros(300_000, device="cuda") for _ in (0, 1)]
    out = torch.zeros(2, device="cuda")
    plan = tsr.DensePlan([p], [g], state_dtype=F8)
    into = tsr.DensePlan(None, None, states=[tuple(dst)])
    plan.step(tsr.make_hyper(1))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    mine = spans([plan.workspace, plan._result, into.workspace] + [t for s in plan.states for t in s])
    sizes = [b - a for a, b in mine]
    kw = dict(stream=side) if given else {}
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    with torch.cuda.stream(side if not given else torch.cuda.current_stream()):
        if call == "step":
            plan.step(tsr.make_hyper(2), **kw)
        elif call == "grad_norm":
            plan.grad_norm(1.0, out=out, **kw)
        else:
            into.copy_state(plan, **kw)
    del plan, into
    others = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
    late = side.query()
    if call == "step":
        used = mine[0:1] + mine[3:]
    elif call == "grad_norm":
        used = mine[0:1]
    else:
        used = mine[0:1] + mine[2:]
    clash = [(a, b) for a, b in spans(others) for c, d in used if a < d and c < b]
    side.synchronize()
    assert not late          # the stream was still held up when memory was asked for
    assert not clash
    if call == "step":
        want.step(tsr.make_hyper(2))
        assert torch.equal(p, q)
    elif call == "grad_norm":
        assert torch.equal(out, want.grad_norm(1.0))
    else:
        ref = [torch.zeros(300_000, device="cuda") for _ in (0, 1)]
        tsr.DensePlan(None, None, states=[tuple(ref)]).copy_state(want)
        assert torch.equal(dst[0], ref[0]) and torch.equal(dst[1], ref[1])


def test_a_plan_bound_again_keeps_its_old_tables_until_its_calls_are_done(tsr):
    """bind() waits for the device, so a step that is still to run sees the tables that it was called with."""
    p, g = rand(100_000, 1), rand(100_000, 2)
    q, h = p.clone(), rand(100_000, 3)
    plan = tsr.DensePlan([p], [g])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    plan.step(tsr.make_hyper(1), stream=side)
    plan.grads[0] = h
    plan.bind()
    plan.step(tsr.make_hyper(2))
    want = tsr.DensePlan([q], [g])
    want.step(tsr.make_hyper(1))
    want.grads[0] = h
    want.bind()
    want.step(tsr.make_hyper(2))
    assert torch.equal(p, q)


def test_norms_of_a_plan_on_two_streams_run_one_after_the_other(tsr):
    """They share partial sums.  While the first is held up, the second has not run either; both results are right."""
    g = rand(3_000_000, 1)
    plan = tsr.DensePlan(None, [g])
    want = plan.grad_norm(1.0).clone()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    a, b = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
        plan.grad_norm(1.0, out=a)
        first = torch.cuda.Event()
        first.record()
    plan.grad_norm(1.0, out=b, stream=other)
    held_up = not first.query()
    other.synchronize()
    assert held_up and first.query()      # the second was through only after the first
    assert torch.equal(a, want) and torch.equal(b, want)
    c = plan.grad_norm(1.0)               # back on the default stream, many times on either
    for k in range(20):
        with torch.cuda.stream((side, other)[k % 2]):
            plan.grad_norm(1.0, out=(a, b)[k % 2])
    torch.cuda.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want) and torch.equal(c, want)


def test_a_norm_is_captured_after_norms_on_other_streams(tsr):
    g = rand(100_000, 1)
    plan = tsr.DensePlan(None, [g])
    want = plan.grad_norm(1.0).clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        plan.grad_norm(1.0)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = plan.grad_norm(1.0)
    out.zero_()
    graph.replay()
    assert torch.equal(out, want)
    with torch.cuda.stream(side):
        plan.grad_norm(1.0, out=out)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_a_plan_made_on_a_side_stream_keeps_its_memory_too(tsr):
    """Its memory belongs to the side stream; its calls are on the default one, which is held up when the plan is dropped."""
    side = torch.cuda.Stream()
    p, g = rand(300_000, 1), rand(300_000, 2)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        plan = tsr.DensePlan([p], [g], state_dtype=F8)
        mine = spans([plan.workspace] + [t for s in plan.states for t in s])
    q = p.clone()
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    plan.step(tsr.make_hyper(1))
    done = torch.cuda.Event()
    done.record()
    del plan
    with torch.cuda.stream(side):
        others = [torch.empty(b - a, dtype=torch.uint8, device="cuda") for a, b in mine for _ in range(4)]
    late = done.query()
    clash = [(a, b) for a, b in spans(others) for c, d in mine if a < d and c < b]
    torch.cuda.synchronize()
    assert not late and not clash
    tsr.DensePlan([q], [g], state_dtype=F8).step(tsr.make_hyper(1))
    assert torch.equal(p, q)
