"""Refusals of the experts' products, the 8-bit products and AdamW: every bad argument is reported on the host, before
any device work (no call here reaches a kernel launch)."""
import ctypes

import pytest

from paper_2606_27866_amd import flexmoe as fm

FAKE = 0x100000  # never dereferenced


def code_of(f, *args, **kw):
    with pytest.raises(fm.FlexMoEError) as ei:
        f(*args, **kw)
    assert fm.flexmoe_last_error()
    return ei.value.code


def grouped(**kw):
    a = dict(groups=4, N=48, K=40, max_rows=100)
    a.update(kw)
    return fm.make_grouped_desc(**a)


BAD_DESC = [
    (dict(dtype=5), -5), (dict(dw_dtype=2), -5), (dict(groups=0), -2), (dict(groups=257), -2), (dict(N=0), -2), (dict(K=0), -2),
    (dict(N=(1 << 21) + 1), -2), (dict(max_rows=-1), -2), (dict(max_rows=(1 << 30) + 1), -2), (dict(K=41), -2),  # packed rows of 41
    (dict(ldx=32), -2), (dict(ldx=44), -2), (dict(ldw=36), -2), (dict(ldy=50), -2), (dict(lddw=42), -2), (dict(ldw=(1 << 21) + 8), -2),
]


@pytest.mark.parametrize("kw,code", BAD_DESC)
def test_grouped_descriptor(kw, code):
    D = grouped(**kw)
    assert code_of(fm.flexmoe_grouped_workspace_bytes, D, 1) == -2
    assert code_of(fm.flexmoe_grouped_forward, D, 1, FAKE, FAKE, FAKE, None, FAKE, FAKE, 1 << 40, 0) == code


def test_grouped_keep_axis_out_of_range():
    D = grouped()
    D.keep_axis = 3
    assert code_of(fm.flexmoe_grouped_forward, D, 1, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, 0) == -1


@pytest.mark.parametrize("f", [fm.flexmoe_grouped_forward, fm.flexmoe_grouped_input_grad, fm.flexmoe_grouped_weight_grad])
def test_grouped_arguments(f):
    more = (0,) if f is fm.flexmoe_grouped_weight_grad else ()

    def call(D=grouped(), R=10, a=FAKE, b=FAKE, offsets=FAKE, keep=None, c=FAKE):
        f(D, R, a, b, offsets, keep, c, *more, FAKE, 1 << 40, 0)

    for kw, code in [(dict(a=None), -1), (dict(b=None), -1), (dict(c=None), -1), (dict(offsets=None), -1), (dict(R=-1), -1),
                     (dict(R=101), -2), (dict(keep=FAKE), -1), (dict(D=grouped(keep_axis="N")), -1),
                     (dict(a=FAKE + 8), -1), (dict(b=FAKE + 4), -1), (dict(c=FAKE + 2), -1), (dict(offsets=FAKE + 2), -1),
                     (dict(D=grouped(keep_axis="K"), keep=FAKE + 1), -1)]:
        assert code_of(call, **kw) == code, kw
    if not more:
        call(R=0)  # nothing to do
    assert code_of(fm.flexmoe_grouped_weight_grad, grouped(), 1, FAKE, FAKE, FAKE, None, FAKE, 2, FAKE, 1 << 40, 0) == -1


def test_grouped_workspace_serves_fewer_rows():
    for shape in (dict(groups=1, N=256, K=1024), dict(groups=8, N=512, K=256), dict(groups=3, N=77, K=88, ldy=80, ldw=88)):
        D = grouped(max_rows=5000, **shape)
        sizes = [fm.flexmoe_grouped_workspace_bytes(D, R) for R in (0, 1, 2, 17, 64, 65, 300, 1000, 4999, 5000)]
        assert sizes == sorted(sizes) and all(n >= 256 for n in sizes)


def test_quantized_refusals():
    ok = dict(groups=1, N=48, K=64, max_rows=10)
    f = fm.flexmoe_quantized_forward
    args = (FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, 1 << 40, 0)
    for kw, code in [(dict(ok, K=131072), -2), (dict(ok, K=40), -2), (dict(ok, ldx=72), -2), (dict(ok, dtype=9), -5), (dict(ok, groups=300), -2)]:
        assert code_of(f, fm.make_grouped_desc(**kw), 1, *args) == code, kw
    D = fm.make_grouped_desc(**ok)
    for i in (0, 1, 2, 3, 4, 6):
        bad = list(args)
        bad[i] = None
        assert code_of(f, D, 1, *bad) == -1, i
    assert code_of(f, D, 11, *args) == -2
    f(D, 0, *args)


def test_quantize_refusals():
    f = fm.flexmoe_quantize_rows
    ok = dict(rows=2, cols=32, dtype=fm.FLEXMOE_BF16, x=FAKE, x_gate=None, ldx=0, q=FAKE, ldq=0, scale=FAKE, stream=0)
    for kw, code in [(dict(dtype=3), -5), (dict(rows=-1), -1), (dict(cols=0), -2), (dict(cols=36), -2), (dict(ldx=36), -2), (dict(ldx=24), -2),
                     (dict(ldq=40), -2), (dict(x=None), -1), (dict(q=None), -1), (dict(scale=None), -1), (dict(x=FAKE + 2), -1),
                     (dict(x_gate=FAKE + 8), -1), (dict(q=FAKE + 8), -1), (dict(scale=FAKE + 2), -1)]:
        assert code_of(f, **dict(ok, **kw)) == code, kw
    f(**dict(ok, rows=0))


def adamw(n=5, **kw):
    a = dict(param_dtype=fm.FLEXMOE_F32, grad_dtype=fm.FLEXMOE_F32, state_bits=32, seed=0, step=1, lr=1e-3, beta1=0.9, beta2=0.99,
             eps=1e-8, weight_decay=0.0, grad_scale=1.0)
    t = dict(param=FAKE, grad=FAKE, m=FAKE, v=FAKE, m_scale=None, v_scale=None, master=None, n=n)
    for k, v in kw.items():
        (a if k in a else t)[k] = v
    tensors = (fm.flexmoe_adamw_tensor * 1)(fm.flexmoe_adamw_tensor(**t))
    fm.flexmoe_adamw_step(fm.flexmoe_adamw_desc(**a), tensors, stream=0)


@pytest.mark.parametrize("kw,code", [
    (dict(param_dtype=4), -5), (dict(grad_dtype=-1), -5), (dict(state_bits=16), -1), (dict(step=0), -1), (dict(beta1=1.0), -1),
    (dict(beta2=-0.1), -1), (dict(beta1=float("nan")), -1), (dict(eps=0.0), -1), (dict(eps=float("inf")), -1), (dict(lr=float("nan")), -1),
    (dict(grad_scale=float("inf")), -1), (dict(n=-1), -1), (dict(n=(1 << 40) + 1), -2), (dict(param=None), -1), (dict(grad=None), -1),
    (dict(m=None), -1), (dict(v=None), -1), (dict(m_scale=FAKE), -1), (dict(state_bits=8), -1), (dict(state_bits=8, m_scale=FAKE), -1),
    (dict(master=FAKE), -1), (dict(param=FAKE + 2), -1), (dict(grad=FAKE + 1), -1), (dict(m=FAKE + 2), -1),
    (dict(param_dtype=fm.FLEXMOE_BF16, master=FAKE + 2), -1), (dict(state_bits=8, m_scale=FAKE + 2, v_scale=FAKE), -1),
])
def test_adamw_refusals(kw, code):
    assert code_of(adamw, **kw) == code


def test_adamw_nothing_to_do():
    adamw(n=0, param=None, grad=None, m=None, v=None)
    D = fm.flexmoe_adamw_desc(1, 1, 8, 0, 1, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1.0)
    assert fm.lib().flexmoe_adamw_step(ctypes.byref(D), None, 0, None) == 0
    assert fm.lib().flexmoe_adamw_step(ctypes.byref(D), None, 1, None) == -1
    assert fm.lib().flexmoe_adamw_step(ctypes.byref(D), None, -1, None) == -1
    assert fm.lib().flexmoe_adamw_step(None, None, 0, None) == -1


def test_adamw_read_state_refusals():
    f = fm.flexmoe_adamw_read_state
    assert code_of(f, 1, FAKE, FAKE, FAKE, FAKE, 7, FAKE, FAKE, 0) == -5
    assert code_of(f, -1, FAKE, FAKE, FAKE, FAKE, 0, FAKE, FAKE, 0) == -1
    assert code_of(f, 1, FAKE, FAKE, None, FAKE, 0, FAKE, FAKE, 0) == -1
    assert code_of(f, 1, FAKE, FAKE, FAKE, FAKE, 0, FAKE + 2, FAKE, 0) == -1
    f(0, None, None, None, None, 0, None, None, 0)


def test_tensor_column_refuses_what_is_no_gpu_tensor():
    import numpy as np
    import torch
    table, sizes = np.zeros(4, np.uint64), np.array([3, 4], np.int64)
    column = fm.tensors().column
    assert column([], 0, 0, 0, 8) == -1
    assert column([torch.zeros(3), torch.zeros(4)], sizes.ctypes.data, 0, table.ctypes.data, 8) == 0  # not on the GPU
    assert column([None, torch.zeros(4)], sizes.ctypes.data, 0, table.ctypes.data, 8) == 0
    assert not table.any()
    with pytest.raises(TypeError):
        column((), 0, 0, 0, 8)


def test_products_run_with_any_workspace():
    """Too little workspace is no error (reductions are split less); a misaligned one is."""
    D = grouped()
    assert code_of(fm.flexmoe_grouped_forward, D, 1, FAKE, FAKE, FAKE, None, FAKE, FAKE + 8, 1 << 20, 0) == -4
