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
                                       s0=0, reset=0, reset_bs=0, reset_ts=0, o=P, o_s=IN, s_last=0, carry=0, workspace=P), kw)


def delta_grad_args(**kw):
    return packed(seq.DELTA_GRAD_ARGS, dict(dtype=0, B=2, H=4, Dk=8, Dv=8, scale=1.0, T=4, q=P, k=P, v=P, f=P, b=P, q_s=IN, k_s=IN, v_s=IN, f_s=GATE, b_s=GATE,
                                            carry=P, reset=0, reset_bs=0, reset_ts=0, dout=P, dout_s=IN, dlast=0, dq=P, dk=P, dv=P, df=P, db=P,
                                            dq_s=IN, dk_s=IN, dv_s=IN, df_s=GATE, db_s=GATE, ds0=0, workspace=P), kw)


BOTH = [dict(dtype=2), dict(B=-1), dict(B=65536), dict(H=-1), dict(H=65536), dict(B=2000, H=2000), dict(Dk=0), dict(Dk=129), dict(Dv=0), dict(Dv=129), dict(T=-1),
        dict(T=1 << 40), dict(B=65535, H=16, T=1000), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(k=P + 2), dict(v=None), dict(f=P + 1), dict(b=None),
        dict(q_s=(-1, 32, 8)), dict(k_s=(128, 1 << 60, 8)), dict(v_s=(128, (1 << 24) + 1, 8)), dict(v_s=(128, 32, -8)), dict(f_s=(16, -4, 1)), dict(b_s=(1 << 60, 4, 1)),
        dict(reset=P, reset_ts=-1), dict(reset=P, reset_bs=1 << 60)]


@pytest.mark.parametrize("kw", BOTH + [dict(o=None), dict(o=P + 2), dict(o_s=(128, 32, 7)), dict(o_s=(128, 31, 8)), dict(o_s=(127, 32, 8)), dict(o_s=(0, 32, 8)), dict(o_s=(8, 32, 16)),
                                       dict(s0=P + 2), dict(s_last=P + 1), dict(carry=P + 4), dict(workspace=None), dict(workspace=P + 8)])
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


# ------------------------------------------------------------------ queries and keys per head
TURNS = (C.c_double * 2)(0.1, 0.01)
SHAPE = dict(dtype=0, Hq=3, Hk=2, D=8, R=4)


def heads_args(**kw):
    return packed(seq.HEADS_ARGS, dict(SHAPE, eps=1e-6, M=4, q=P, k=P, q_rs=24, q_hs=8, k_rs=16, k_hs=8, q_weight=P, k_weight=P, position=P, turns=C.addressof(TURNS),
                                       yq=P, yk=P, yq_rs=24, yq_hs=8, yk_rs=16, yk_hs=8, rstd=P), kw)


def heads_grad_args(**kw):
    return packed(seq.HEADS_GRAD_ARGS, dict(SHAPE, M=4, dyq=P, dyk=P, q=P, k=P, dyq_rs=24, dyq_hs=8, dyk_rs=16, dyk_hs=8, q_rs=24, q_hs=8, k_rs=16, k_hs=8, q_weight=P, k_weight=P,
                                            rstd=P, position=P, turns=C.addressof(TURNS), dq=P, dk=P, dq_rs=24, dq_hs=8, dk_rs=16, dk_hs=8, dq_weight=P, dk_weight=P, workspace=P), kw)


NAN_TURNS = (C.c_double * 2)(0.1, float("nan"))
HEADS_BOTH = [dict(dtype=3), dict(Hq=-1), dict(Hk=65536), dict(D=0), dict(D=257), dict(R=3), dict(R=-2), dict(R=10), dict(M=-1), dict(M=1 << 31), dict(q=None), dict(k=P + 2), dict(q_rs=-1),
              dict(k_hs=1 << 60), dict(q_weight=None), dict(k_weight=P + 1), dict(position=None), dict(position=P + 2), dict(turns=None), dict(turns=C.addressof(NAN_TURNS)), dict(rstd=P + 2)]


@pytest.mark.parametrize("kw", HEADS_BOTH + [dict(eps=-1.0), dict(eps=float("nan")), dict(yq=None), dict(yk=P + 1), dict(yq_hs=7), dict(yk_rs=8), dict(yq_rs=0)])
def test_heads_refuses(lib, kw):
    assert lib.dqn_heads_forward(heads_args(**kw), None) == dqn.ERR_INVALID_ARG and "dqn_heads_forward" in said(lib)


@pytest.mark.parametrize("kw", HEADS_BOTH + [dict(rstd=None), dict(dyq=None), dict(dyk_rs=-1), dict(dq=None), dict(dk=P + 2), dict(dq_hs=4), dict(dk_rs=0), dict(dq_weight=None),
                                             dict(dk_weight=P + 2), dict(workspace=None), dict(workspace=P + 4)])
def test_heads_backward_refuses(lib, kw):
    assert lib.dqn_heads_backward(heads_grad_args(**kw), None) == dqn.ERR_INVALID_ARG and "dqn_heads_backward" in said(lib)


def test_heads_sizes_nothing_and_rotations(lib):
    a = C.c_size_t()
    assert lib.dqn_heads_sizes(0, 1, 1, 8, C.byref(a)) == dqn.OK and a.value > 0 and a.value % 4 == 0
    for args in ((-1, 1, 1, 8), (4, -1, 1, 8), (4, 1, 1, 0), (4, 1, 1, 257)):
        assert lib.dqn_heads_sizes(*args, C.byref(a)) == dqn.ERR_INVALID_ARG
    assert lib.dqn_heads_sizes(4, 1, 1, 8, None) == lib.dqn_heads_forward(None, None) == lib.dqn_heads_backward(None, None) == dqn.ERR_INVALID_ARG
    assert lib.dqn_heads_forward(heads_args(M=0), None) == lib.dqn_heads_forward(heads_args(Hq=0, Hk=0, q=None), None) == dqn.OK
    r = seq.rotation(8, 100.0)
    assert r.R == 8 and seq.rotation(8, 100.0) is r and seq.rotation(0).R == 0
    assert np.allclose(np.array(r._turns) * 2 * np.pi, 100.0 ** (-np.arange(4) / 4))
    for bad in ((7,), (-2,), (8, 0.0)):
        with pytest.raises(ValueError):
            seq.rotation(*bad)


def test_gradients_of_the_heads_are_differences():
    r = np.random.RandomState(2)
    x, w, dy, pos, turns = r.randn(3, 2, 7), r.randn(7), r.randn(3, 2, 7), np.array([0, 5, -1000003]), [0.13, 0.011]

    def loss(x, w):
        return (ref.heads(x, w, pos, turns, 1e-3)[0] * dy).sum()

    grads, _ = ref.heads_backward(dy, x, w, pos, turns, 1e-3)
    for k in range(2):
        args = [x, w]
        for at in np.ndindex(args[k].shape):
            up, down = [v.copy() for v in args], [v.copy() for v in args]
            up[k][at] += 1e-5
            down[k][at] -= 1e-5
            assert abs((loss(*up) - loss(*down)) / 2e-5 - grads[k][at]) < 1e-7


# ------------------------------------------------------------------ steps for matrices
def test_muon_refuses(lib):
    t = (seq._MuonMatrix * 2)(seq._MuonMatrix(P, P, P, None, 30, 70, 0.0), seq._MuonMatrix(None, None, None, None, 0, 5, 0.5))
    plan, work, h = C.c_size_t(), C.c_size_t(), C.c_void_p()
    assert lib.dqn_muon_sizes(t, 2, C.byref(plan), C.byref(work)) == dqn.OK and plan.value % 256 == 0 and work.value % 256 == 0 and work.value > 0
    assert lib.dqn_muon_sizes(t, 2, None, C.byref(work)) == dqn.ERR_INVALID_ARG
    for count in (0, 65537):
        assert lib.dqn_muon_sizes(t, count, C.byref(plan), C.byref(work)) == dqn.ERR_INVALID_ARG
    for field, value in (("rows", -1), ("cols", -1), ("rows", (1 << 20) + 1), ("param", None), ("param", P + 2), ("momentum", None), ("momentum", P + 1), ("grad", None), ("copy", P + 1),
                         ("decay", -1.0), ("decay", float("nan"))):
        bad = (seq._MuonMatrix * 1)(seq._MuonMatrix(P, P, P, None, 30, 70, 0.0))
        setattr(bad[0], field, value)
        assert lib.dqn_muon_init(C.byref(h), bad, 1, 0, P, P, None) == dqn.ERR_INVALID_ARG and not h.value, field
    big = (seq._MuonMatrix * 1)(seq._MuonMatrix(P, P, P, None, 65537, 65537, 0.0))
    assert lib.dqn_muon_sizes(big, 1, C.byref(plan), C.byref(work)) == dqn.ERR_INVALID_ARG
    for plan_at, work_at, kind in ((None, P, 0), (P + 64, P, 0), (P, None, 0), (P, P + 16, 0), (P, P, 2)):
        assert lib.dqn_muon_init(C.byref(h), t, 2, kind, plan_at, work_at, None) == dqn.ERR_INVALID_ARG and not h.value
    odd = (seq._MuonMatrix * 1)(seq._MuonMatrix(P, P, P + 2, None, 30, 70, 0.0))
    assert lib.dqn_muon_init(C.byref(h), odd, 1, 0, P, P, None) == dqn.ERR_INVALID_ARG
    assert lib.dqn_muon_init(None, t, 2, 0, P, P, None) == lib.dqn_muon_step(None, 0.1, 0.9, 1, 1e-7, 5, None) == dqn.ERR_INVALID_ARG
    assert lib.dqn_muon_destroy(None) == dqn.OK


def test_muon_refuses_buffers_that_lie_on_each_other(lib):
    """The same matrix twice would be written by two workgroups at once."""
    h, n = C.c_void_p(), 30 * 70
    apart = [P + 4096 * 1024 * i for i in range(8)]
    for which, what in ((("param", "param"), 0), (("momentum", "momentum"), 0), (("param", "momentum"), 4 * n - 4), (("copy", "copy"), 2 * n - 2), (("grad", "param"), 0), (("momentum", "grad"), 4 * n - 4),
                        (("param", "grad"), 2 * n)):
        t = (seq._MuonMatrix * 2)(*(seq._MuonMatrix(*apart[4 * i:4 * i + 4], 30, 70, 0.0) for i in range(2)))
        setattr(t[1], which[1], getattr(t[0], which[0]) + what)
        assert lib.dqn_muon_init(C.byref(h), t, 2, 0, P, P, None) == dqn.ERR_INVALID_ARG and not h.value, which
        assert b"another buffer" in lib.dqn_last_error(None)


def test_the_rounds_take_singular_values_near_one():
    r = np.random.RandomState(3)
    for n, m in ((5, 40), (40, 5), (8, 8)):
        u, _, v = np.linalg.svd(r.randn(n, m), full_matrices=False)
        g = (u * np.linspace(0.2, 1.0, u.shape[1])) @ v
        p, mom, bound = ref.muon(np.zeros((n, m)), g, np.zeros((n, m)), 1.0, 0.9, eps=0.0)
        x = -p / np.sqrt(max(1, n / m))
        s = np.linalg.svd(x, compute_uv=False)
        assert 0.6 < s.min() and s.max() < 1.25 and np.allclose(np.abs(u.T @ x @ v.T - np.diag(np.diag(u.T @ x @ v.T))).max(), 0, atol=1e-9)
        assert np.allclose(mom, g) and 0 < bound < 0.1 * np.sqrt((p * p).sum())
