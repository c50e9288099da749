"""The matrix memory's operators where there is much: elements further apart than 32 bits reach, more tiles than compute units, many ranges."""
import pytest
import torch

from paper_1804_05834_amd import seq
from test_gpu_memory import DEV, Delta, Heads

pytestmark = pytest.mark.gpu
FAR = 1 << 24       # elements from step to step, the most that is allowed


class Apart:
    """One buffer, of whose rows, FAR apart, each tensor has a few elements."""

    def __init__(self, rows, dtype):
        self.x, self.at = torch.empty((rows - 1) * FAR + 8192, dtype=dtype, device=DEV), 0

    def empty(self, B, T, *rest):
        strides = [1] if rest else []
        for n in reversed(rest[1:]):
            strides.insert(0, strides[0] * n)
        size = rest[0] * strides[0] if rest else 1
        t = self.x.as_strided((B, T, *rest), ((size + 7) // 8 * 8, FAR, *strides), self.at)
        self.at += B * ((size + 7) // 8 * 8)
        assert self.at <= 8192
        return t

    def copy(self, x):
        return self.empty(*x.shape).copy_(x)


@pytest.mark.parametrize("dtype,T", [("bf16", 5), ("bf16", 300), ("fp32", 300)])
def test_delta_steps_far_apart(dtype, T):
    c = Delta(40, dtype, 2, T, 2, 16, 24)
    want = c.run()
    far = Apart(T, c.dt)
    few = seq.delta(*c.inputs(), s0=c.s0, reset=c.reset, scale=c.scale)
    o = far.empty(*c.v.shape)
    c.q, c.k, c.v, c.f, c.b, c.do = (far.copy(x) for x in (c.q, c.k, c.v, c.f, c.b, c.do))
    outs = tuple(far.empty(*x.shape) for x in c.inputs())
    got = c.run(out=outs)
    again = seq.delta(*c.inputs(), s0=c.s0, reset=c.reset, scale=c.scale, out=o)
    assert again[0] is o and torch.equal(o, few[0]) and torch.equal(again[1], few[1])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for x, y in zip(got[2], want[2]):
        assert torch.equal(x, y)
    assert got[2][0].data_ptr() == outs[0].data_ptr()


def test_delta_takes_five_outputs_or_none():
    c = Delta(41, "fp32", 1, 3, 1, 4, 4)
    carry = seq.delta(*c.inputs(), save=True)[2]
    with pytest.raises(ValueError, match="out"):
        seq.delta_backward(c.do, *c.inputs(), carry, out=(None,) * 4)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_heads_rows_far_apart(dtype):
    c = Heads(42, dtype, 260, 2, 1, 24, 16)
    want = c.run()
    far = Apart(260, c.dt)
    views = [far.copy(x[None])[0] for x in (c.q, c.k, c.dyq, c.dyk)]
    outs = [far.empty(1, *x.shape)[0] for x in (c.q, c.k, c.q, c.k)]
    got = c.run(*views, out=outs[:2], gout=outs[2:])
    for x, y in zip((*got[0], *got[1]), (*want[0], *want[1])):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("Dk,Dv", [(16, 24), (64, 64), (64, 100), (100, 72), (128, 128)])
@pytest.mark.parametrize("bad", [False, True])
def test_delta_many_sequences_are_what_a_few_are(dtype, Dk, Dv, bad):
    """More tiles than compute units: workgroups of the gradients then go from tile to tile and from head to head."""
    c = Delta(43, dtype, 130, 70, 3, Dk, Dv)
    if bad:
        c.v[17, 33, 1, 2] = float("nan")
        c.q[18, 64, 2, 0] = float("inf")
        c.do[40, 0, 0, 1] = float("nan")
    want = c.run()
    whole = {n: getattr(c, n) for n in ("q", "k", "v", "f", "b", "do", "s0", "dlast", "reset")}
    for at in range(0, 130, 26):
        for n, x in whole.items():
            setattr(c, n, x[at:at + 26])
        got = c.run()
        for x, y in zip((got[0], got[1], *got[2]), (want[0], want[1], *want[2])):
            y = y[at:at + 26]
            assert torch.equal(x.nan_to_num(7.0, 8.0, 9.0), y.nan_to_num(7.0, 8.0, 9.0)) and torch.equal(x.isnan(), y.isnan())
    assert bad == bool(want[2][2].isnan().any())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,B,H,Dk,Dv,resets", [(3300, 1, 1, 64, 64, 0), (3300, 1, 2, 33, 20, 0.001), (4100, 2, 1, 20, 72, 0.002), (3109, 1, 1, 128, 128, 0.001), (8200, 1, 1, 16, 17, 0.0005)])
def test_delta_ranges_in_groups(dtype, T, B, H, Dk, Dv, resets):
    """So many ranges that they are joined in groups, the last one smaller; some with an episode's start."""
    c = Delta(T, dtype, B, T, H, Dk, Dv, resets=resets)
    c.check(*c.run())


def test_delta_groups_and_what_is_not_finite():
    """A state that is NaN and a value that is infinite end with their episodes, whatever is joined."""
    clean, c = (Delta(5, "bf16", 1, 4096, 2, 32, 32, resets=0) for _ in range(2))
    for x in (clean, c):
        x.reset = torch.zeros(1, 4096, dtype=torch.uint8, device=DEV)
        x.reset[0, [1000, 1700, 3000]] = 1
    want = clean.run()
    c.s0[:] = float("nan")
    c.dlast[0, 1] = float("nan")
    c.v[0, 2000, 0, 3] = float("inf")
    got = c.run()
    assert not torch.isfinite(got[0][0, :1000]).any() and not torch.isfinite(got[0][0, 2000:3000, 0, 3]).any() and torch.isfinite(got[1]).all()
    # A tile with such a number is formed step by step, the clean run's by its products, which take 16 bits of the state: with |q| < 1, columns of the
    # state below 8 and the scale 32^-1/2 those are 2^-17 * 8 / 5.7 < 2^-16 off, fp32 roundings of either far less.  Rounded by half a step each, the two
    # are one step of bf16 (2^-7) and 2^-16 apart at most.
    for part in (slice(1000, 2000), slice(3000, 4096)):
        assert torch.allclose(got[0][0, part].float(), want[0][0, part].float(), rtol=2.0 ** -7, atol=2.0 ** -16)
    for x, y in zip(got[2][:5], want[2][:5]):
        assert torch.isfinite(x[0, 1000:1700]).all() and torch.isfinite(x[0, 3000:, 0]).all()
        # another tile's way of forming it: a step of bf16
        assert torch.allclose(x[0, 1000:1700].float(), y[0, 1000:1700].float(), rtol=2.0 ** -7, atol=2.0 ** -8)
    assert not torch.isfinite(got[2][2][0, 3000:, 1]).all()
