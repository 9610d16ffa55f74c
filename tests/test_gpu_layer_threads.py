"""Layer calls of several host threads at once."""
import ctypes
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def norm_call(tsr, cols, dtype):
    x = torch.randn(8, cols, device="cuda").to(dtype)
    y = torch.empty_like(x)
    kind = tsr.TSR_BF16 if dtype == torch.bfloat16 else tsr.TSR_F32
    desc = tsr.NormDesc(8, cols, kind, tsr.TSR_F32, tsr.TSR_F32, 1, 0, 1e-5)
    m, n = tsr.Matrix(x.data_ptr(), cols), tsr.Matrix(y.data_ptr(), cols)
    return (x, y), lambda stream: tsr.lib().tsr_norm_forward(ctypes.byref(desc), m, None, None, n, None, stream)


def norm_backward_call(tsr, cols):
    x, dy, dx = (torch.randn(8, cols, device="cuda") for _ in range(3))
    stats = torch.ones(8, 2, device="cuda")
    desc = tsr.NormDesc(8, cols, tsr.TSR_F32, tsr.TSR_F32, tsr.TSR_F32, 1, 0, 0.0)
    m = [tsr.Matrix(t.data_ptr(), cols) for t in (dy, x, dx)]
    return (x, dy, dx, stats), lambda stream: tsr.lib().tsr_norm_backward(ctypes.byref(desc), m[0], m[1], None, stats.data_ptr(), m[2], None, None, None, 0, stream)


def few_call(tsr, ins):
    x, w, y = torch.randn(8, ins, device="cuda"), torch.randn(16, ins, device="cuda"), torch.empty(8, 16, device="cuda")
    desc = tsr.LinearDesc(8, ins, 16, tsr.TSR_F32, tsr.TSR_F32, tsr.TSR_F32, tsr.TSR_F32, 0, 0, tsr.DropoutDesc(0.0, 0, 0, 0, None))
    none = tsr.Matrix(None, 0)
    io = tsr.LinearIO(tsr.Matrix(x.data_ptr(), ins), tsr.Matrix(w.data_ptr(), ins), none, none, tsr.Matrix(y.data_ptr(), 16), None)
    return (x, w, y), lambda stream: tsr.lib().tsr_linear_forward(ctypes.byref(desc), ctypes.byref(io), None, 0, stream)


@pytest.mark.parametrize("which", ["few rows", "norm forward", "norm backward"])
def test_sizes_of_other_threads_do_not_matter(tsr, which):
    """Two sizes of one kernel, whose shared memory differs, by two threads each on streams of their own: no call is refused, and each has its own result."""
    make = {"few rows": lambda n: few_call(tsr, 1600 if n else 3000), "norm forward": lambda n: norm_call(tsr, 1100 if n else 2048, torch.bfloat16),
            "norm backward": lambda n: norm_backward_call(tsr, 600 if n else 1024)}[which]
    calls = [make(i % 2) for i in range(4)]
    streams = [torch.cuda.Stream() for _ in calls]
    wants = []
    for held, call in calls:
        assert call(None) == 0
        torch.cuda.synchronize()
        wants.append([t.clone() for t in held])
    refused = [0] * len(calls)
    ready = threading.Barrier(len(calls))

    def work(i):
        torch.cuda.set_device(0)
        stream = streams[i].cuda_stream
        ready.wait()
        for rep in range(4000):
            refused[i] += calls[i][1](stream) != 0
            if rep % 256 == 255:
                streams[i].synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert refused == [0] * len(calls)
    for (held, _), want in zip(calls, wants):
        for a, b in zip(held, want):
            assert torch.equal(a, b)
