"""The gates of the matrix memory: the gradient of one that is nearly shut, against its own size, and what is not finite in front of one that is shut."""
import numpy as np
import pytest
import torch

import memory_ref as ref
from paper_1804_05834_amd import seq
from test_gpu_memory import DEV, Delta, host

pytestmark = pytest.mark.gpu


def gate_bounds(c):
    """The gradient of f in 64 bits and a bound of its error in the size of each gate.

    df_t = a_t (1 - a_t) <D_t, S_{t-1}>, D_t being the gradient of what step t keeps of the state.  Formed within a tile it is a sum of products of
    what steps before t wrote, u_j, or the state that entered, with what steps from t on ask of it, q_i do_i and k_i dv_i, or the gradient that
    leaves; each has a_t as a factor, so with keys and queries no longer than one, the sums of sizes
      B_{t+1} = a_t B_t + |u_t|,  A_t = a_{t+1} A_{t+1} + |scale do_t| + |dv_t|
    (0 where an episode starts) bound the terms by a_t A_t B_t, and their errors follow from those of u and dv: an error of the state or of its
    gradient does not grow with the steps, each adds eps of the sizes that it works with, and so u and dv are off by that error and eps of those sizes.
    eps: fp32 sums of up to Dk + TILE products.  bf16 inputs: numbers are also kept as two bf16 of eight bits, the upper one cut off, so that a
    product of two such, without that of the lower ones, is 2^-14 off, and four of them 2^-16 each at most on the way."""
    q, k, v, f, b, do = (host(x) for x in (*c.inputs(), c.do))
    s0, reset, dlast = (None if x is None else host(x) for x in (c.s0, c.reset, c.dlast))
    B, T, H, Dk = q.shape
    eps = (Dk + ref.TILE + 16) * ref.U + (2.0 ** -14 + 4 * 2.0 ** -16 if c.dt is torch.bfloat16 else 0.0)
    grads, _ = ref.delta_backward(do, q, k, v, f, b, s0, reset, dlast, c.scale)
    states = ref.delta(q, k, v, f, b, s0, reset, c.scale)[4]
    a, beta = 1 / (1 + np.exp(-f)), 1 / (1 + np.exp(-b))
    cut = np.zeros((B, T, 1), bool) if reset is None else (reset != 0)[:, :, None]
    norm = lambda x: np.sqrt((x * x).sum(-1))  # noqa: E731
    nv, no, ndv = norm(v), abs(c.scale) * norm(do), norm(grads[2])
    before, e_before = np.zeros((B, T, H)), np.zeros((B, T, H))      # B_t and its error
    S = np.sqrt((states[0] ** 2).sum((2, 3)))
    dS, e = eps * S, eps * S
    for t in range(T):
        S, dS, e = (np.where(cut[:, t], 0.0, x) for x in (S, dS, e))
        before[:, t], e_before[:, t] = S, dS
        old = np.where(cut[:, t, :, None, None], 0.0, states[t])
        u = beta[:, t] * norm(v[:, t] - a[:, t, :, None] * (old * k[:, t, :, :, None]).sum(2))
        du = a[:, t] * e + eps * (S + nv[:, t] + u)
        e = a[:, t] * e + eps * (S + nv[:, t])
        S, dS = a[:, t] * S + u, a[:, t] * dS + du
    bound = np.zeros((B, T, H))
    A = np.zeros((B, H)) if dlast is None else np.sqrt((dlast ** 2).sum((2, 3)))
    dA, e = eps * A, eps * A
    for t in range(T - 1, -1, -1):
        ddv = e + eps * (A + no[:, t] + ndv[:, t])
        e = e + eps * (A + no[:, t])
        A, dA = A + no[:, t] + ndv[:, t], dA + ddv + eps * no[:, t]
        bound[:, t] = a[:, t] * (1 - a[:, t]) * (A * e_before[:, t] + dA * before[:, t] + eps * A * before[:, t])
        A, dA, e = (np.where(cut[:, t], 0.0, a[:, t] * x) for x in (A, dA, e))
    return grads[3], bound + 8 * ref.U * np.abs(grads[3]) * (1 + np.abs(f))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("f", [-4.0, -8.0, -12.0, -20.0])
@pytest.mark.parametrize("which", ["one", "some", "all"])
@pytest.mark.parametrize("T,Dk,Dv,state", [(70, 64, 64, True), (45, 20, 100, False), (600, 16, 24, True), (40, 128, 128, True)])
def test_the_gradient_of_a_gate_that_is_nearly_shut(dtype, f, which, T, Dk, Dv, state):
    c = Delta(20 + T, dtype, 1, T, 2, Dk, Dv, state=state, resets=0.01)
    at = {"one": slice(21, 22), "some": slice(5, None, 9), "all": slice(None)}[which]
    c.f[:, at] = f
    grads = c.run()[2]
    want, bound = gate_bounds(c)
    ref.within(host(grads[3]), want, bound, (), c.dt is torch.bfloat16, "df")
    c.check(*c.run())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,T,H,Dk,Dv", [(2, 5, 2, 16, 24), (3, 50, 2, 64, 64), (1, 700, 1, 32, 40), (2, 33, 1, 128, 128)])
def test_the_first_gate_has_nothing_to_keep(dtype, B, T, H, Dk, Dv):
    c = Delta(30 + T, dtype, B, T, H, Dk, Dv, state=False, resets=0)
    grads = c.run()[2]
    assert (grads[3][:, 0] == 0).all() and not (grads[3][:, 1] == 0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("shut", [-200.0, -100.0])
@pytest.mark.parametrize("at", [31, 32, 33, 64])
@pytest.mark.parametrize("B,T,Dk,Dv", [(2, 100, 16, 24), (1, 70, 64, 64), (1, 640, 32, 32)])
def test_a_gate_that_is_shut_ends_no_episode(dtype, bad, shut, at, B, T, Dk, Dv):
    """Zero times what is not finite is a NaN, wherever in a tile the gate stands and however the sequence is gone through: a value that is not
    finite reaches the steps behind the gate, a gradient the steps before it."""
    for what in ("v", "do", "s0", "dlast"):
        c = Delta(50 + at, dtype, B, T, 2, Dk, Dv, resets=0)
        c.reset = torch.zeros(B, T, dtype=torch.uint8, device=DEV)
        c.reset[:, [2, 67]] = 1
        c.f[:, at, 0] = shut
        if what in ("v", "do"):
            getattr(c, what)[0, 10 if what == "v" else 66, 0, 1] = bad
        else:
            c.reset.zero_()
            getattr(c, what)[0, 0, 3, 1] = bad
        with np.errstate(all="ignore"):
            (o, last), _, want, _ = c.exact()
        got = c.run()
        for name, x, y in zip(("o", "last", "dq", "dk", "dv", "df", "db", "ds0"), (got[0], got[1], *got[2]), (o, last, *want)):
            assert (np.isfinite(host(x)) == np.isfinite(y)).all(), (what, name)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("at", [3, 7])
def test_a_gate_that_is_shut_ends_no_episode_of_few_steps(dtype, at):
    c = Delta(60, dtype, 2, 8, 2, 16, 16, resets=0)
    c.f[:, at] = -200.0
    c.v[0, 1, 0, 5] = float("nan")
    o, last = seq.delta(*c.inputs(), s0=c.s0, reset=c.reset, scale=c.scale)
    p, other, _ = seq.delta(*c.inputs(), s0=c.s0, reset=c.reset, scale=c.scale, save=True)
    assert torch.equal(o.isnan(), p.isnan()) and torch.equal(last.isnan(), other.isnan())
    assert o[0, 1:, 0, 5].isnan().all() and int(o.isnan().sum()) == 7
