"""The matrix memory's operators without a GPU: the library's own checks of arguments (nothing is launched) and the
64-bit definitions the GPU tests compare with, held against differences."""
import ctypes as C

import numpy as np
import pytest

import memory_ref as ref
from paper_1804_05834_amd import dqn, seq


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(dqn.LIB_PATH):
        dqn.build()
    return dqn.lib()


def said(lib):
    return lib.dqn_last_error(None).decode()


P = 1 << 20      # an address that is aligned; no call below gets as far as using it


def packed(layout, fields, kw):
    """The bytes of a struct of arguments from its fields' values (a tuple: several numbers), some of them replaced."""
    assert set(kw) <= set(fields)
    flat = []
    for k, v in fields.items():
        v = kw.get(k, v)
        flat += list(v) if isinstance(v, tuple) else [v or 0]
    return layout.pack(*flat)


# ------------------------------------------------------------------ gated delta rule
IN = (128, 32, 8)        # strides of [2][4][4][8]
GATE = (16, 4, 1)


def delta_args(**kw):
    return packed(seq.DELTA_ARGS, dict(dtype=0, B=2, H=4, Dk=8, Dv=8, scale=1.0, T=4, q=P, k=P, v=P, f=P, b=P, q_s=IN, k_s=IN, v_s=IN, f_s=GATE, b_s=GATE,
                                       s0=0, reset=0, reset_bs=0, reset_ts=0, o=P, o_s=IN, s_last=0, carry=0, workspace=0), kw)


def delta_grad_args(**kw):
    return packed(seq.DELTA_GRAD_ARGS, dict(dtype=0, B=2, H=4, Dk=8, Dv=8, scale=1.0, T=4, q=P, k=P, v=P, f=P, b=P, q_s=IN, k_s=IN, v_s=IN, f_s=GATE, b_s=GATE,
                                            carry=P, reset=0, reset_bs=0, reset_ts=0, dout=P, dout_s=IN, dlast=0, dq=P, dk=P, dv=P, df=P, db=P,
                                            dq_s=IN, dk_s=IN, dv_s=IN, df_s=GATE, db_s=GATE, ds0=0, workspace=P), kw)


BOTH = [dict(dtype=2), dict(B=-1), dict(B=65536), dict(H=-1), dict(H=65536), dict(B=2000, H=2000), dict(Dk=0), dict(Dk=129), dict(Dv=0), dict(Dv=129), dict(T=-1),
        dict(T=1 << 40), dict(B=65535, H=16, T=2000), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(k=P + 2), dict(v=None), dict(f=P + 1), dict(b=None),
        dict(q_s=(-1, 32, 8)), dict(k_s=(128, 1 << 60, 8)), dict(v_s=(128, 32, -8)), dict(f_s=(16, -4, 1)), dict(b_s=(1 << 60, 4, 1)),
        dict(reset=P, reset_ts=-1), dict(reset=P, reset_bs=1 << 60)]


@pytest.mark.parametrize("kw", BOTH + [dict(o=None), dict(o=P + 2), dict(o_s=(128, 32, 7)), dict(o_s=(128, 31, 8)), dict(o_s=(127, 32, 8)), dict(o_s=(0, 32, 8)), dict(o_s=(8, 32, 16)),
                                       dict(s0=P + 2), dict(s_last=P + 1), dict(carry=P + 2)])
def test_delta_refuses(lib, kw):
    assert lib.dqn_delta_forward(delta_args(**kw), None) == dqn.ERR_INVALID_ARG and "dqn_delta_forward" in said(lib)


@pytest.mark.parametrize("kw", BOTH + [dict(carry=None), dict(dout=None), dict(dout_s=(128, -1, 8)), dict(dq=None), dict(dk=P + 2), dict(dv_s=(128, 32, 4)), dict(df_s=(16, 1, 1)),
                                       dict(db_s=(4, 4, 1)), dict(dq_s=(0, 0, 0)), dict(dlast=P + 2), dict(ds0=P + 1), dict(workspace=None), dict(workspace=P + 8)])
def test_delta_backward_refuses(lib, kw):
    assert lib.dqn_delta_backward(delta_grad_args(**kw), None) == dqn.ERR_INVALID_ARG and "dqn_delta_backward" in said(lib)


def test_delta_sizes_and_nothing(lib):
    a, b, c = C.c_size_t(), C.c_size_t(), C.c_size_t()
    assert lib.dqn_delta_sizes(1, 2, 100, 3, 8, 5, C.byref(a), C.byref(b), C.byref(c)) == dqn.OK and a.value > 0 and a.value % 4 == 0
    for args in ((2, 2, 100, 3, 8, 5), (0, -1, 100, 3, 8, 5), (0, 2, -1, 3, 8, 5), (0, 2, 100, 3, 0, 5), (0, 2, 100, 3, 8, 200), (0, 2, 1 << 62, 3, 8, 5)):
        assert lib.dqn_delta_sizes(*args, C.byref(a), C.byref(b), C.byref(c)) == dqn.ERR_INVALID_ARG and "dqn_delta_sizes" in said(lib)
    assert lib.dqn_delta_sizes(1, 2, 100, 3, 8, 5, None, C.byref(b), C.byref(c)) == dqn.ERR_INVALID_ARG
    for fn in (lib.dqn_delta_forward, lib.dqn_delta_backward):
        assert fn(None, None) == dqn.ERR_INVALID_ARG
    assert lib.dqn_delta_forward(delta_args(B=0), None) == lib.dqn_delta_forward(delta_args(H=0, q=None), None) == dqn.OK
    assert lib.dqn_delta_backward(delta_grad_args(B=0), None) == lib.dqn_delta_backward(delta_grad_args(H=0, q=None), None) == dqn.OK


def delta_case(r, B=2, T=5, H=2, Dk=3, Dv=2):
    def unit():
        x = r.randn(B, T, H, Dk)
        return x / np.sqrt((x * x).sum(3, keepdims=True))
    return unit(), unit(), r.randn(B, T, H, Dv), r.randn(B, T, H) + 1, r.randn(B, T, H), r.randn(B, H, Dk, Dv)


def test_gradients_of_the_delta_rule_are_differences():
    r = np.random.RandomState(1)
    x = delta_case(r)
    do, dl = r.randn(*x[2].shape), r.randn(*x[5].shape)
    reset = r.rand(2, 5) < 0.3

    def loss(*x):
        o, last = ref.delta(*x, reset=reset, scale=0.7)[:2]
        return (o * do).sum() + (last * dl).sum()

    grads, _ = ref.delta_backward(do, *x, reset=reset, dlast=dl, scale=0.7)
    for k in range(6):
        for at in np.ndindex(x[k].shape):
            up, down = [v.copy() for v in x], [v.copy() for v in x]
            up[k][at] += 1e-5
            down[k][at] -= 1e-5
            assert abs((loss(*up) - loss(*down)) / 2e-5 - grads[k][at]) < 1e-7
