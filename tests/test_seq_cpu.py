"""The recurrent network's operators without a GPU: the library's own checks of arguments (nothing is launched), the
64-bit definitions the GPU tests compare with, held against differences and against torch."""
import ctypes as C

import numpy as np
import pytest
import torch

import seq_ref as ref
from paper_1804_05834_amd import dqn, seq


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(dqn.LIB_PATH):
        dqn.build()
    return dqn.lib()


def said(lib):
    return lib.dqn_last_error(None).decode()


def test_sizes_and_null_arguments(lib):
    a, b = C.c_size_t(), C.c_size_t()
    assert lib.dqn_scan_sizes(0, 2, 100, 64, C.byref(a), C.byref(b)) == dqn.OK and a.value > 0 and a.value % 4 == 0
    assert lib.dqn_scan_sizes(0, 0, 100, 64, C.byref(a), C.byref(b)) == dqn.OK and a.value == 0
    for args in ((2, 2, 100, 64), (0, -1, 100, 64), (0, 65536, 100, 64), (0, 2, -1, 64), (0, 2, 1 << 60, 64), (0, 60000, 1 << 32, 1 << 30)):
        assert lib.dqn_scan_sizes(*args, C.byref(a), C.byref(b)) == dqn.ERR_INVALID_ARG and "dqn_scan_sizes" in said(lib)
    assert lib.dqn_scan_sizes(0, 1, 1, 1, None, None) == dqn.ERR_INVALID_ARG
    for fn in (lib.dqn_scan_forward, lib.dqn_scan_backward, lib.dqn_norm_forward, lib.dqn_norm_backward, lib.dqn_rows_product):
        assert fn(None, None) == dqn.ERR_INVALID_ARG
    assert lib.dqn_norm_sizes(-1, 4, C.byref(a)) == lib.dqn_norm_sizes(4, 0, C.byref(a)) == lib.dqn_norm_sizes(4, 16385, C.byref(a)) == dqn.ERR_INVALID_ARG
    assert lib.dqn_rows_quantize(0, 3, 4, None, 4, None, 16, None, None) == dqn.ERR_INVALID_ARG
    assert lib.dqn_adamw_sizes(None, 1, 32, None) == lib.dqn_adamw_step(None, 0.1, 0.9, 0.99, 1e-8, 1, 0, None) == dqn.ERR_INVALID_ARG
    assert lib.dqn_adamw_destroy(None) == dqn.OK


P = 1 << 20      # an address that is aligned; no call below gets as far as using it


def packed(layout, fields, kw):
    """The bytes of a struct of arguments from its fields' values, some of them replaced."""
    assert set(kw) <= set(fields)
    return layout.pack(*(kw.get(k, v) or 0 for k, v in fields.items()))


def scan_args(**kw):
    return packed(seq.SCAN_ARGS, dict(dtype=0, B=2, C=8, T=4, f=P, x=P, f_bs=32, f_ts=8, x_bs=32, x_ts=8, h0=0, reset=0, reset_bs=0, reset_ts=0, h=P, h_bs=32, h_ts=8,
                                      h_last=0, carry=0, workspace=0), kw)


@pytest.mark.parametrize("kw", [dict(dtype=5), dict(B=-1), dict(B=70000), dict(C=-2), dict(T=-1), dict(f=None), dict(x=None), dict(h=None), dict(f=P + 2),
                                dict(h=P + 1), dict(f_bs=-1), dict(x_ts=-8), dict(h_ts=7), dict(h_bs=8), dict(f_ts=1 << 60), dict(h0=P + 2), dict(h_last=P + 1), dict(f_ts=(1 << 24) + 1), dict(B=60000, C=60000),
                                dict(carry=P + 2), dict(reset=P, reset_ts=-1), dict(reset=P, reset_bs=1 << 60)])
def test_scan_refuses(lib, kw):
    assert lib.dqn_scan_forward(scan_args(**kw), None) == dqn.ERR_INVALID_ARG and "dqn_scan_forward" in said(lib)


def test_scan_of_nothing_does_nothing(lib):
    assert lib.dqn_scan_forward(scan_args(B=0), None) == lib.dqn_scan_forward(scan_args(C=0, f=None), None) == dqn.OK


def grad_args(**kw):
    return packed(seq.SCAN_GRAD_ARGS, dict(dtype=0, B=2, C=8, T=4, f=P, x=P, f_bs=32, f_ts=8, x_bs=32, x_ts=8, carry=P, reset=0, reset_bs=0, reset_ts=0, dh=P, dh_bs=32, dh_ts=8,
                                           dlast=0, df=P, dx=P, df_bs=32, df_ts=8, dx_bs=32, dx_ts=8, dh0=0, workspace=0), kw)


@pytest.mark.parametrize("kw", [dict(carry=None), dict(dh=None), dict(df=None), dict(dx=P + 2), dict(df_ts=4), dict(dx_bs=0), dict(dh_ts=-1), dict(dlast=P + 2), dict(dh0=P + 3)])
def test_scan_backward_refuses(lib, kw):
    assert lib.dqn_scan_backward(grad_args(**kw), None) == dqn.ERR_INVALID_ARG and "dqn_scan_backward" in said(lib)


def norm_args(**kw):
    return packed(seq.NORM_ARGS, dict(dtype=0, C=8, M=4, x=P, residual=0, x_rs=8, residual_rs=0, weight=P, eps=1e-6, r=0, r_rs=0, y=P, y_rs=8, q=0, q_rs=0, scale=0, rstd=0), kw)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(C=0), dict(C=16385), dict(M=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(x=P + 2), dict(weight=None), dict(y=None),
                                dict(y=P, q=P, q_rs=16, scale=P), dict(y=None, q=P, q_rs=16), dict(y=None, q=P + 8, q_rs=16, scale=P), dict(y=None, q=P, q_rs=8, scale=P),
                                dict(y_rs=7), dict(x_rs=-1), dict(r=P, r_rs=4), dict(residual=P + 1), dict(x_rs=1 << 60)])
def test_norm_refuses(lib, kw):
    assert lib.dqn_norm_forward(norm_args(**kw), None) == dqn.ERR_INVALID_ARG and "dqn_norm_forward" in said(lib)


def norm_grad_args(**kw):
    return packed(seq.NORM_GRAD_ARGS, dict(dtype=0, C=8, M=4, dy=P, x=P, residual=0, dr=0, dy_rs=8, x_rs=8, residual_rs=0, dr_rs=0, weight=P, rstd=P, dx=P, dx_rs=8, dw=P,
                                           workspace=P), kw)


@pytest.mark.parametrize("kw", [dict(dy=None), dict(x=None), dict(residual=P + 2), dict(rstd=None), dict(weight=None), dict(dx=None), dict(dx_rs=7), dict(dw=None), dict(workspace=None), dict(workspace=P + 4),
                                dict(dr=P + 2), dict(C=0), dict(M=-3)])
def test_norm_backward_refuses(lib, kw):
    assert lib.dqn_norm_backward(norm_grad_args(**kw), None) == dqn.ERR_INVALID_ARG and "dqn_norm_backward" in said(lib)


def product_args(**kw):
    return packed(seq.PRODUCT_ARGS, dict(dtype=1, N=8, K=20, M=4, a=P, w=P, a_rs=32, w_rs=32, a_scale=P, w_scale=P, bias=0, y=P, y_rs=8), kw)


@pytest.mark.parametrize("kw", [dict(dtype=9), dict(M=-1), dict(N=-1), dict(K=-1), dict(N=1 << 21), dict(a=None), dict(a=P + 8), dict(w=P + 1), dict(a_rs=24), dict(w_rs=16), dict(a_scale=None),
                                dict(w_scale=P + 2), dict(bias=P + 1), dict(y=None), dict(y_rs=7), dict(y=P + 1)])
def test_product_refuses(lib, kw):
    assert lib.dqn_rows_product(product_args(**kw), None) == dqn.ERR_INVALID_ARG and "dqn_rows_product" in said(lib)


def test_adamw_refuses(lib):
    t = (seq._AdamWTensor * 2)(seq._AdamWTensor(P, P, None, 300, 0.0), seq._AdamWTensor(P, P, None, 0, 0.5))
    out = seq._AdamWBytes()
    assert lib.dqn_adamw_sizes(t, 2, 8, C.byref(out)) == dqn.OK
    assert (out.elements, out.m, out.v, out.m_scale, out.v_scale) == (512, 512, 512, 8, 8) and out.plan % 256 == 0 and out.plan > 0
    assert lib.dqn_adamw_sizes(t, 2, 32, C.byref(out)) == dqn.OK and (out.m, out.m_scale) == (2048, 0)
    h, bufs = C.c_void_p(), seq._AdamWBuffers(P, P, P, P, P)
    for count, bits in ((0, 8), (70000, 8), (2, 16)):
        assert lib.dqn_adamw_sizes(t, count, bits, C.byref(out)) == dqn.ERR_INVALID_ARG
        assert lib.dqn_adamw_init(C.byref(h), t, count, bits, 0, C.byref(bufs), None) == dqn.ERR_INVALID_ARG and not h.value
    for field, value in (("n", -1), ("n", 1 << 60), ("param", None), ("param", P + 2), ("grad", None), ("grad", P + 1), ("copy", P + 1), ("decay", -1.0), ("decay", float("inf"))):
        bad = (seq._AdamWTensor * 1)(seq._AdamWTensor(P, P, None, 300, 0.0))
        setattr(bad[0], field, value)
        assert lib.dqn_adamw_init(C.byref(h), bad, 1, 8, 0, C.byref(bufs), None) == dqn.ERR_INVALID_ARG and not h.value, field
    for field in ("m", "v", "m_scale", "v_scale", "plan"):
        b = seq._AdamWBuffers(P, P, P, P, P)
        setattr(b, field, P + 64)
        assert lib.dqn_adamw_init(C.byref(h), t, 2, 8, 0, C.byref(b), None) == dqn.ERR_INVALID_ARG and "256-byte" in said(lib)
    assert lib.dqn_adamw_init(C.byref(h), t, 2, 8, 3, C.byref(bufs), None) == dqn.ERR_INVALID_ARG


# ------------------------------------------------------------------ the definitions themselves
def test_gradients_of_the_definitions_are_differences():
    r = np.random.RandomState(0)
    B, T, Ch = 2, 6, 3
    f, x, h0, dh, dl = r.randn(B, T, Ch), r.randn(B, T, Ch), r.randn(B, Ch), r.randn(B, T, Ch), r.randn(B, Ch)
    reset = r.rand(B, T) < 0.2

    def loss(f, x, h0):
        h, last = ref.scan(f, x, h0, reset)[:2]
        return (h * dh).sum() + (last * dl).sum()

    grads, _ = ref.scan_backward(dh, f, x, h0, reset, dl)
    for k in range(3):
        args = [f, x, h0]
        for at in np.ndindex(args[k].shape):
            up, down = [v.copy() for v in args], [v.copy() for v in args]
            up[k][at] += 1e-5
            down[k][at] -= 1e-5
            assert abs((loss(*up) - loss(*down)) / 2e-5 - grads[k][at]) < 1e-7
    xr, w, dy, dr = r.randn(3, 5), r.randn(5), r.randn(3, 5), r.randn(3, 5)

    def nloss(x, w):
        rr, y = ref.norm(x, w, eps=1e-3)[:2]
        return (y * dy).sum() + (rr * dr).sum()

    rr, _, rstd = ref.norm(xr, w, eps=1e-3)[:3]
    grads, _ = ref.norm_backward(dy, rr, rstd, w, dr)
    for k in range(2):
        args = [xr, w]
        for at in np.ndindex(args[k].shape):
            up, down = [v.copy() for v in args], [v.copy() for v in args]
            up[k][at] += 1e-5
            down[k][at] -= 1e-5
            assert abs((nloss(*up) - nloss(*down)) / 2e-5 - grads[k][at]) < 1e-7


def test_eight_bit_numbers_are_torchs():
    codes = np.arange(256, dtype=np.uint8)
    for mine, kind in ((ref.e4m3, torch.float8_e4m3fn), (ref.e5m2, torch.float8_e5m2)):
        assert np.array_equal(mine(codes), torch.from_numpy(codes).view(kind).double().numpy(), equal_nan=True)


def test_random_rounding_keeps_the_mean_and_the_draws_are_the_librarys():
    from paper_1804_05834_amd import synth
    d = ref.draws(12345, 1 << 16)
    assert np.array_equal(d.view(np.int64), synth.mix64(12345, torch.arange(1 << 15)).numpy())
    v = np.full(1 << 16, 0.3, np.float32)
    v[::256] = 1.0      # the block's largest
    qm, sm, qv, sv = ref.moments8(v, v, 99)
    rest = np.arange(v.size) % 256 != 0
    assert abs((qm * np.repeat(sm, 256))[rest].mean() / 0.3 - 1) < 1e-3 and abs((qv * np.repeat(sv, 256))[rest].mean() / 0.3 - 1) < 1e-3
    assert (qm[~rest] == 448).all() and (qv[~rest] == 57344).all()


def test_scan_refuses_more_states_than_a_launch_has_threads_for(lib):
    a, b = C.c_size_t(), C.c_size_t()
    for B, c in ((65535, 4097), (17, 1 << 24), (4097, 65536)):
        for T in (1, 9, 100, 5000):
            assert lib.dqn_scan_sizes(0, B, T, c, C.byref(a), C.byref(b)) == dqn.ERR_INVALID_ARG and "2^28" in said(lib)
    for B, c in ((65535, 4096), (16, 1 << 24), (4096, 65536)):
        assert lib.dqn_scan_sizes(0, B, 100, c, C.byref(a), C.byref(b)) == dqn.OK
