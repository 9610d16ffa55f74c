"""What the dense-plan calls refuse and compute on the host (no GPU needed)."""
import ctypes

import numpy as np
import pytest

import dense_model as dm


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    from paper_2602_08007_b200 import build as b
    b.build()
    return t


def create(tsr, descs, count=None):
    arr = (tsr.DenseDesc * max(len(descs), 1))(*descs)
    plan = ctypes.c_void_p(1)
    rc = tsr.lib().tsr_dense_plan_create(ctypes.byref(plan), arr, len(descs) if count is None else count)
    return rc, plan


def desc(tsr, **kw):
    d = dict(rows=4, cols=8, ldp=8, ldg=8, ldi=8, p_dtype=0, g_dtype=0, state=0, flags=0, lr_mult=1.0, wd_mult=1.0)
    d.update(kw)
    return tsr.DenseDesc(*d.values())


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 2), (dict(cols=-1), 2), (dict(ldp=7), 2), (dict(ldg=7), 2), (dict(p_dtype=2), 6), (dict(g_dtype=-1), 6),
    (dict(state=2), 6), (dict(flags=3), 1), (dict(flags=4), 1), (dict(lr_mult=float("nan")), 1), (dict(wd_mult=float("inf")), 1),
    (dict(rows=1 << 40, cols=1 << 40, ldp=1 << 40, ldg=1 << 40), 2), (dict(rows=1 << 20, ldp=1 << 60), 2), (dict(rows=1 << 20, ldg=1 << 60), 2),
])
def test_create_refuses(tsr, change, status):
    rc, plan = create(tsr, [desc(tsr), desc(tsr, **change)])
    assert rc == status and not plan.value


def test_what_a_flag_leaves_out_is_not_looked_at(tsr):
    for d in (desc(tsr, flags=1, state=9, p_dtype=9, ldp=0), desc(tsr, flags=2, ldp=0, ldg=0, p_dtype=9, g_dtype=9), desc(tsr, rows=0), desc(tsr, cols=0),
              desc(tsr, ldi=-5)):
        rc, plan = create(tsr, [d])
        assert rc == 0
        assert tsr.lib().tsr_dense_plan_destroy(plan) == 0


def test_calls_before_bind_and_bad_binds(tsr):
    L = tsr.lib()
    assert L.tsr_dense_plan_create(None, None, 0) == 1
    assert create(tsr, [], -1)[0] == 1
    rc, plan = create(tsr, [desc(tsr), desc(tsr, state=1)])
    assert rc == 0
    h = tsr.make_hyper(1)
    assert L.tsr_dense_plan_step(plan, ctypes.byref(h), None, 0, 0, None) == 11
    assert b"bind" in L.tsr_dense_plan_last_error(plan)
    out = ctypes.c_float()
    assert L.tsr_dense_plan_grad_norm(plan, 1.0, ctypes.addressof(out), None) == 11
    assert L.tsr_dense_plan_copy_state(plan, plan, None) == 11
    assert L.tsr_dense_plan_step(plan, None, None, 0, 0, None) == 1
    assert L.tsr_dense_plan_grad_norm(plan, 1.0, None, None) == 1
    size = ctypes.c_size_t()
    assert L.tsr_dense_plan_workspace_bytes(plan, ctypes.byref(size)) == 0 and size.value > 0
    buf = ctypes.create_string_buffer(size.value + 256)       # only checked, never passed on
    ws = (ctypes.addressof(buf) + 255) // 256 * 256
    P = tsr.DensePtrs
    good = [P(64, 64, 64, 64, None, None), P(64, 64, 64, 64, 64, None)]
    bad = [
        (None, 2, ws, size.value, 1), (good, 1, ws, size.value, 1), (good, 2, None, size.value, 4), (good, 2, ws, size.value - 1, 4), (good, 2, ws + 8, size.value, 3),
        ([P(None, 64, 64, 64, None, None), good[1]], 2, ws, size.value, 1), ([P(64, None, 64, 64, None, None), good[1]], 2, ws, size.value, 1),
        ([good[0], P(64, 64, 64, 64, None, None)], 2, ws, size.value, 1), ([good[0], P(64, 64, None, 64, 64, None)], 2, ws, size.value, 1),
        ([P(66, 64, 64, 64, None, None), good[1]], 2, ws, size.value, 3), ([good[0], P(64, 64, 65, 65, 68, None)], 2, ws, size.value, 3),
        ([P(64, 64, 64, 64, None, 65), good[1]], 2, ws, size.value, 3),
    ]
    for ptrs, count, w, n, status in bad:
        arr = None if ptrs is None else (P * len(ptrs))(*ptrs)
        assert L.tsr_dense_plan_bind(plan, arr, count, w, n) == status, (ptrs and ptrs[0].param, count, n, status)
    L.tsr_dense_plan_destroy(plan)
    for call in (lambda: L.tsr_dense_plan_destroy(None), lambda: L.tsr_dense_plan_step(None, ctypes.byref(h), None, 0, 0, None),
                 lambda: L.tsr_dense_plan_bind(None, None, 0, None, 0), lambda: L.tsr_dense_plan_grad_norm(None, 1.0, None, None),
                 lambda: L.tsr_dense_plan_copy_state(None, None, None), lambda: L.tsr_dense_plan_workspace_bytes(None, None)):
        assert call() == 1
    assert L.tsr_dense_plan_last_error(None) == b""


def test_the_models_of_the_8_bit_form_agree_with_each_other():
    """Rounding to nearest picks the closest value; stochastic rounding picks a neighbour, the upper one as often as the
    remainder says, over all 16-bit words."""
    rng = np.random.default_rng(1)
    y = np.concatenate([rng.uniform(0, 448, 500), 2.0 ** rng.uniform(-12, 8.8, 500), dm.POSITIVE]).astype(np.float32)
    near = dm.E4M3[dm.quantise(y, 1.0)]
    assert np.all(np.abs(near - y) <= np.abs(dm.POSITIVE[None, :] - y[:, None]).min(axis=1))
    words = np.arange(1 << 16)
    for x in y[:40].tolist() + [0.001, 0.0156, 0.01562, 2.0 ** -9, 0.0, 448.0]:
        x = np.float32(x)
        c = dm.E4M3[dm.quantise(np.full(1 << 16, x, np.float32), 1.0, words)]
        assert np.all(np.abs(c - x) < dm.spacing(max(x, 1e-30)) + (x == 0))
        assert abs(c.mean() - x) <= dm.spacing(max(x, 1e-30)) * 2.0 ** -15


def test_the_table_fits_its_room(tmp_path):
    """Shapes, pitches, types and alignments: the table that a binding fills is never larger than the room planned for it."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "dense_table")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-I", os.path.join(root, "include"), "-I", os.path.join(root, "paper_2602_08007_b200", "csrc"),
                           os.path.join(root, "tests", "dense_table.cpp"), "-o", exe])
    run = subprocess.run([exe], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout


@pytest.mark.parametrize("rows,cols,pitch", [(1, 40_000_000, 0), (32000, 2048, 0), (32000, 2048, 8), (2, 3_000_000, 1 << 30)])
def test_the_workspace_holds_the_chunks_of_any_binding(tsr, rows, cols, pitch):
    """Codes off an 8-byte border, or a pitch beyond 32 bits, make chunks of eight blocks, 16 bytes each in the table."""
    rc, plan = create(tsr, [desc(tsr, rows=rows, cols=cols, ldp=cols + pitch, ldg=cols + pitch, ldi=cols, state=1)])
    assert rc == 0
    size = ctypes.c_size_t()
    assert tsr.lib().tsr_dense_plan_workspace_bytes(plan, ctypes.byref(size)) == 0
    blocks = -(-rows * cols // tsr.DENSE_BLOCK)
    assert size.value >= 16 * -(-blocks // 8)
    tsr.lib().tsr_dense_plan_destroy(plan)
