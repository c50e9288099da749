"""Where the recurrent network's operators meet the ends of their types and of their launches, against their definitions in
64 bits (tests/seq_ref.py)."""
import numpy as np
import pytest
import torch

import seq_ref as ref
from test_gpu_seq import TYPES, close, host, rnd, scan_case, seq  # noqa: F401

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


# B, T, C: a thread per four channels and per channel; strips of pairs and of single channels; whole lines, ranges of lines, an odd
# last channel; a workgroup per sequence; a thread per channel and range, 8 and 32 steps at a time
FORMS = [(3, 5, 64), (2, 8, 3), (300, 20, 64), (260, 40, 65), (2100, 20, 64), (2, 700, 64), (1, 300, 67), (9, 300, 16), (3, 20000, 1), (700, 9001, 1)]
SMALLEST = 2.0 ** -126      # of a normal number; a gate below it may count as zero


def gates_case(B, T, C, dtype, values, seed):
    g = torch.Generator().manual_seed(seed)
    f = torch.tensor(values)[torch.randint(0, len(values), (B, T, C), generator=g)].to(TYPES[dtype]).cuda()
    return f, rnd(seed + 1, B, T, C, dtype=TYPES[dtype]), rnd(seed + 2, B, C), rnd(seed + 3, B, T, C, dtype=TYPES[dtype]), rnd(seed + 4, B, C)


def check_scan(seq, f, x, h0, reset, dh, dlast, bf):
    """Forward and backward within the bounds of seq_ref and what gates below SMALLEST, taken as zero, would have let through."""
    hf, hx, hh, hr = host(f), host(x), host(h0), None if reset is None else reset.cpu().numpy()
    h, last, carry = seq.scan(f, x, h0=h0, reset=reset, save=True)
    want, wl, _, eh, el, _ = ref.scan(hf, hx, hh, hr)
    size = max(np.nanmax(np.abs(want)), np.abs(hx).max(), np.abs(hh).max())
    lost = 2 * SMALLEST * f.shape[1] * size
    close(h, want, ref.stored(eh, want, bf) + lost, "h")
    close(last, wl, el + lost + 1e-37, "last")
    df, dx, dh0 = seq.scan_backward(dh, f, x, carry, reset=reset, dlast=dlast)
    wants, bounds = ref.scan_backward(host(dh), hf, hx, hh, hr, host(dlast))
    sent = np.abs(host(dh)).sum(1).max() + np.abs(host(dlast)).max()      # no more than this comes from later steps
    lost = 2 * SMALLEST * f.shape[1] * sent * (2 * size + 1)
    close(df, wants[0], ref.stored(bounds[0], wants[0], bf) + lost, "df")
    close(dx, wants[1], ref.stored(bounds[1], wants[1], bf) + lost, "dx")
    close(dh0, wants[2], bounds[2] + lost + 1e-37, "dh0")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,T,C", FORMS)
def test_scan_gates_whose_exponential_is_almost_infinite(seq, B, T, C, dtype):  # noqa: F811
    """exp(88.7) is the largest exponential that is finite; from exp(87.4) on the gate itself is below the smallest normal number,
    but the input still comes through whole."""
    print("case gates", B, T, C, dtype, flush=True)
    v = [87.0, 87.3, 87.4, 87.5, 88.0, 88.5, 88.7, 89.0, 103.0]
    args = gates_case(B, T, C, dtype, [-u for u in v] + v[::2] + [0.0, 1.0, -1.0, 16.0, -16.0, -17.0], 400)
    check_scan(seq, *args[:3], None, *args[3:], dtype == "bf16")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,T,C", FORMS)
def test_scan_a_gate_that_is_not_a_number(seq, B, T, C, dtype):  # noqa: F811
    """It spoils the state from its step to the next episode, and the gradients of its step and of those before it in its episode."""
    f, x, h0, dh, dlast = gates_case(B, T, C, dtype, [0.0, 1.0, -1.0, 2.0], 420)
    reset = (torch.rand(B, T, generator=torch.Generator().manual_seed(421)) < 4.0 / T).cuda()
    f[0, T // 2, 0] = f[-1, T - 1, C - 1] = f[B // 2, 0, C // 2] = NAN
    reset[0, T // 2] = False
    check_scan(seq, f, x, h0, reset, dh, dlast, dtype == "bf16")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,T,C", [(9, 512, 16), (30, 300, 3), (32, 333, 3), (300, 250, 16), (32, 300, 16), (40, 13, 16), (5, 9, 1), (300, 4000, 1), (9, 513, 16), (3, 20000, 1), (300, 20, 64), (260, 40, 65)])
def test_scan_state_in_place_of_every_form(seq, B, T, C, dtype):  # noqa: F811
    """The final state may take the initial one's place where several waves begin from that."""
    print("case in place", B, T, C, dtype, flush=True)
    f, x, h0, reset = scan_case(B, T, C, "half", True, 0.5 / T, dtype, 430)
    f = f - 2.0 + 4.0 * (T > 100)      # the initial state counts to the end
    h, last, carry = seq.scan(f, x, h0=h0, reset=reset, save=True)
    for _ in range(8):
        s = h0.clone()
        h1, last1, carry1 = seq.scan(f, x, h0=s, reset=reset, save=True, last=s)
        assert last1 is s and torch.equal(s, last) and torch.equal(h1, h) and torch.equal(carry1, carry)


# ------------------------------------------------------------------ 8-bit rows
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("K", [40, 64, 200, 1500])
def test_rows_of_small_numbers(seq, K, dtype):  # noqa: F811
    """Rows whose largest number is near the smallest of the type, with zeros among them: q scale is the number to half a step of
    e4m3 (2^-4 of it; 2^-10 scales below e4m3's normal numbers) and the rounding of the scale, and a zero is a zero."""
    tops = [1e-30, 1e-35, 5e-36, 1.4e-36, 1e-36, 1e-37, 2e-38, 1e-38, 1e-40]
    unit = rnd(440, len(tops), K).clamp(-3, 3)
    unit[:, 1::3] = 0
    unit[:, 0] = 3.0
    x = (unit.double() * torch.tensor(tops).double().cuda()[:, None] / 3).to(TYPES[dtype])
    for q, scale, name in ((*seq.rows(x), "rows"), (*seq.norm_rows(x, torch.ones(K, device="cuda"), eps=1.0)[:2], "norm")):
        hx = host(x)      # the norm's mean square is nothing beside 1
        hq, hs = host(q), host(scale)
        assert (hs > 0).all(), name
        assert (hq[hx == 0] == 0).all(), name
        bound = np.maximum(np.abs(hx) * 2.0 ** -4, hs[:, None] * 2.0 ** -10) * 1.01 + 2.0 ** -148
        off = np.abs(hq * hs[:, None] - hx)
        assert (off <= bound).all(), (name, float((off / bound).max()))
    zero = torch.zeros(2, K, dtype=TYPES[dtype], device="cuda")
    q, scale = seq.rows(zero)
    assert bool((q.float() == 0).all()) and bool((scale == 0).all())


# ------------------------------------------------------------------ AdamW
@pytest.mark.parametrize("size", [1e-12, 1e-16, 1e-17, 1e-18, 1e-20, 1e-37, 1e-39])
def test_adamw_moments_of_small_gradients(seq, size):  # noqa: F811
    """8-bit moments of gradients near the smallest numbers, with zeros among them: a zero stays zero, the others are within a step
    of their type of the moment in 64 bits (a step is 2^-3 / 2^-2 of the number, or the smallest number of the type), and
    a second moment that fp32 can hold does not become zero."""
    n = 1024
    unit = torch.exp(rnd(450, n).clamp(-2, 2)) * torch.where(rnd(451, n) > 0, 1.0, -1.0)
    unit[::3] = 0
    g = (unit.double() * size).float()
    p = torch.zeros(n, device="cuda")
    opt = seq.AdamW([p], [g], bits=8, lr=0.0)
    opt.step(1, seed=9)
    hg = host(g)
    for got, scale, want, step, least in ((opt.m, opt.m_scale, 0.1 * hg, 2.0 ** -3, 2.0 ** -9), (opt.v, opt.v_scale, 0.001 * hg * hg, 2.0 ** -2, 2.0 ** -16)):
        hs = np.repeat(host(scale), 256)
        off = np.abs(host(got) * hs - want)
        # squares and products below 2^-126 are multiples of 2^-149: two of them, rounded, and a scale's own rounding
        bound = np.maximum(np.abs(want) * step, hs * least) * 1.01 + 2.0 ** -147
        assert (host(got)[hg == 0] == 0).all()
        assert (off <= bound).all(), float((off / bound).max())
        assert (host(got)[np.abs(want) > 2.0 ** -126] != 0).all() or step == 2.0 ** -3


@pytest.mark.parametrize("lr", [1e-5, 1e-6])
def test_adamw_small_decay(seq, lr):  # noqa: F811
    """A decay far below a parameter's rounding is not lost beside the gradient's part, and is as large as it should be.  A step is
    5 roundings of the change's size and one of the parameter's off, which is at random over many parameters:
    a mean over 65,536 of them, 200 steps each, is 2^-25 sqrt(200 / 65536) off (standard deviation at most), six of which are allowed."""
    n, steps, decay = 65536, 200, 0.1
    p0 = 1.0 + torch.rand(n, generator=torch.Generator().manual_seed(460)).cuda() * 0.9
    p, g = p0.clone(), torch.zeros(n, device="cuda")
    opt = seq.AdamW([p], [g], lr=lr, weight_decay=decay)
    moved = seq.AdamW([q := p0.clone()], [g], lr=lr, weight_decay=0.0)
    want, m, v = p0.double(), torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    still = p0.double()
    for t in range(1, steps + 1):
        g.copy_(rnd(1000 + t, n))
        opt.step(t)
        moved.step(t)
        m, v = 0.9 * m + 0.1 * g.double(), 0.999 * v + 0.001 * g.double() ** 2
        change = lr / (1 - 0.9 ** t) * m / ((v / (1 - 0.999 ** t)).sqrt() + 1e-8)
        want, still = want * (1 - lr * decay) - change, still - change
    noise = 6 * 2.0 ** -24 * (steps / n) ** 0.5
    for got, exact in ((p, want), (q, still)):
        off = float((got.double() - exact).mean())
        assert abs(off) < noise + 1e-3 * lr * decay * steps, (off, noise)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_second_moment_below_the_normal_numbers(seq, bits):  # noqa: F811
    """With an eps that small the step is lr whatever the gradient's size, for a second moment below 2^-126 too.  There it is a
    multiple of 2^-149, which its root is 2^-150 / v off by, and the bound has four times that."""
    n = 512
    g = torch.logspace(-18.5, -16, n, device="cuda")
    p = torch.zeros(n, device="cuda")
    opt = seq.AdamW([p], [g], bits=bits, lr=1.0, eps=1e-25, weight_decay=0.0)
    opt.step(1, seed=1)
    hg = host(g)
    v = 0.001 * hg * hg
    root = np.sqrt(v / 0.001) + 1e-25
    want = -hg / root
    bound = np.abs(want) * (24 * ref.U + 2.0 ** -148 / v)
    assert (np.abs(host(p) - want) <= bound).all(), float((np.abs(host(p) - want) / bound).max())


# ------------------------------------------------------------------ views
def test_one_step_of_views_whose_steps_are_far_apart(seq):  # noqa: F811
    """With one step there is no next one: its stride is whatever the tensor it was cut from has."""
    B, C = 6, 40
    f, x, dh = (rnd(470 + k, B, 1, C) for k in range(3))
    far = [v.as_strided((B, 1, C), (C, 1 << 30, 1)) for v in (f, x, dh)]
    h, last, carry = seq.scan(f, x, save=True)
    h1, last1, carry1 = seq.scan(*far[:2], save=True, out=torch.empty_like(h).as_strided((B, 1, C), (C, 1 << 30, 1)))
    assert torch.equal(h, h1) and torch.equal(last, last1)
    for a, b in zip(seq.scan_backward(dh, f, x, carry), seq.scan_backward(far[2], *far[:2], carry1)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_windows_that_slide_over_a_signal(seq, dtype):  # noqa: F811
    """Inputs whose rows lie on top of each other, a step of one element apart, fewer than a row has elements."""
    bf = dtype == "bf16"
    signal, w = rnd(480, 200, dtype=TYPES[dtype]), rnd(481, 48, scale=0.2, at=1.0)
    x, res = signal.unfold(0, 48, 1)[:9], signal.unfold(0, 48, 1)[20:29]
    y, r, saved = seq.norm(x, w, residual=res)
    wr, wy, wrstd, er, ey, _ = ref.norm(host(x), host(w), host(res))
    close(r, wr, ref.stored(er, wr, bf), "r")
    close(y, wy, ref.stored(ey, wy, bf), "y")
    dx, dw = seq.norm_backward(x, r, saved, w, dr=res)
    (wdx, wdw), (edx, edw) = ref.norm_backward(host(x), wr, host(saved[0]), host(w), host(res))
    close(dx, wdx, ref.stored(edx, wdx, bf), "dx")
    close(dw, wdw, edw + 1e-37, "dw")
    y, r, saved = seq.norm(x, w)
    dx, dw = seq.norm_backward(res, x, saved, w)
    wr, wy, wrstd, er, ey, _ = ref.norm(host(x), host(w))
    (wdx, wdw), (edx, edw) = ref.norm_backward(host(res), wr, host(saved[0]), host(w))
    close(y, wy, ref.stored(ey, wy, bf), "y")
    close(dx, wdx, ref.stored(edx, wdx, bf), "dx")
    q, scale, r8 = seq.norm_rows(x, w, residual=res)
    assert q.shape == (9, 48) and r8.stride(1) == 1
    f, v = (signal[k:].as_strided((5, 12, 48), (1, 2, 1)) for k in (0, 30))
    h, last, carry = seq.scan(f, v, save=True)
    want, wl, _, eh, el, _ = ref.scan(host(f), host(v))
    close(h, want, ref.stored(eh, want, bf), "h")
    wants, bounds = ref.scan_backward(host(v), host(f), host(v))
    for got, a, b in zip(seq.scan_backward(v, f, v, carry), wants, bounds):
        close(got, a, ref.stored(b, a, bf and got.ndim == 3), "gradient")


def test_adamw_steps_without_a_seed_round_differently(seq):  # noqa: F811
    """A step's own number is its seed: with the same bits at every step a second moment that was once rounded to itself always is."""
    def run(seeds):
        g = rnd(490, 4096)
        opt = seq.AdamW([torch.zeros(4096, device="cuda")], [g], bits=8)
        for t in range(1, 6):
            opt.step(t, **({} if seeds is None else dict(seed=seeds[t - 1])))
        return opt.v.view(torch.uint8).clone()

    assert torch.equal(run(None), run([1, 2, 3, 4, 5]))
    assert not torch.equal(run(None), run([0, 0, 0, 0, 0]))


def test_adamw_steps_on_its_own_gpu_only(seq, monkeypatch):  # noqa: F811
    """As with every other call, tensors of another GPU than the current one are refused, before anything is launched."""
    p = torch.zeros(10, device="cuda")
    opt = seq.AdamW([p], [torch.ones(10, device="cuda")])
    monkeypatch.setattr(seq, "_current_device", lambda: p.get_device() + 1)
    monkeypatch.setattr(seq, "_raw_stream", lambda device: pytest.fail("a launch was prepared"))
    with pytest.raises(ValueError, match="current GPU"):
        opt.step(1)
    monkeypatch.undo()
    opt.step(1)
    assert bool((p != 0).all())


# ------------------------------------------------------------------ autograd
def test_a_gradient_that_nobody_records_is_not_lost_silently(seq):  # noqa: F811
    """Calls on tensors that require a gradient warn while autograd records; their results are what they always are."""
    import warnings
    x, f, w, b = rnd(500, 2, 4, 16), rnd(501, 2, 4, 16), rnd(502, 16), rnd(503, 5)
    w8 = seq.rows(rnd(504, 5, 16))
    calls = {"scan": lambda x, w, b: seq.scan(f, x), "norm": lambda x, w, b: seq.norm(x.view(8, 16), w), "norm_rows": lambda x, w, b: seq.norm_rows(x.view(8, 16), w),
             "rows": lambda x, w, b: seq.rows(x.view(8, 16)), "product": lambda x, w, b: (seq.product(seq.rows(f.view(8, 16)), w8, bias=b),)}
    for name, call in calls.items():
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            want = call(x, w, b)
            leaves = [t.clone().requires_grad_() for t in (x, w, b)]
            with torch.no_grad():
                call(*leaves)
        with pytest.warns(UserWarning, match=name + " records nothing"):
            got = call(*leaves)
        # (the second output of norm is x itself where there is no residual)
        assert torch.equal(got[0].view(torch.uint8), want[0].view(torch.uint8)) and not got[0].requires_grad, name
    p = torch.nn.Parameter(torch.zeros(10, device="cuda"))
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        seq.AdamW([p], [torch.ones(10, device="cuda")]).step(1)      # an optimizer's tensors require gradients by their nature
    assert bool((p != 0).all())


# ------------------------------------------------------------------ product
@pytest.mark.parametrize("big", [256.0, 288.0, 448.0])
@pytest.mark.parametrize("M,N,K,at", [(9, 21, 128, 1), (9, 21, 128, 127), (50, 70, 400, 200), (300, 300, 1024, 1023), (1100, 1111, 640, 129), (40, 50, 8000, 7999)])
def test_product_of_sums_that_cancel(seq, M, N, K, at, big):  # noqa: F811
    """Two large products that cancel, among many of one size, at any distance.  fp32 outputs: sums in fp32.  bf16 outputs:
    128 products at a time, each kept to 16 bits below the largest one's exponent, so a part is off by less than 128 2^-16 of its largest
    product; the parts are added up in fp32."""
    print("case cancel", M, N, K, at, big, flush=True)
    g = torch.Generator().manual_seed(510)
    size = lambda n: torch.exp2(torch.randint(-6, 8, (n, 1), generator=g).float()) * (1 + torch.randint(0, 8, (n, 1), generator=g) / 8)  # noqa: E731
    a, w = size(M).expand(M, K).clone(), size(N).expand(N, K).clone()
    a[:, 0], a[:, at], w[:, 0], w[:, at] = big, -big, big, big
    pad = torch.zeros(M + N, (K + 15) // 16 * 16, dtype=torch.uint8)
    pad[:, :K] = torch.cat([a, w]).to(torch.float8_e4m3fn).view(torch.uint8)
    q = pad.cuda().view(torch.float8_e4m3fn)[:, :K]
    one = torch.ones(M + N, device="cuda")
    ha, hw = host(q)[:M], host(q)[M:]
    assert np.array_equal(ha, a.numpy()) and np.array_equal(hw, w.numpy())      # numbers of e4m3
    want, most = ha @ hw.T, np.abs(ha) @ np.abs(hw).T
    parts = sum((np.abs(ha[:, None, k:k + 128]) * np.abs(hw[None, :, k:k + 128])).max(2) for k in range(0, K, 128))
    sums = ref.U * (K / 32 + 40) * most
    for dtype in (torch.float32, torch.bfloat16):
        bf = dtype == torch.bfloat16
        y = seq.product((q[:M], one[:M]), (q[M:], one[M:]), dtype=dtype)
        close(y, want, ref.stored(sums + (2.0 ** -9 * parts if bf else 0.0), want, bf), "bf16" if bf else "fp32")


def test_adamw_dropped_while_another_stream_steps(seq):  # noqa: F811
    """The table and the moments of an optimizer that is gone are not given to others before its last step has read them."""
    n = 300000
    p, g = rnd(520, n), rnd(521, n)
    want = p.clone()
    seq.AdamW([want], [g], bits=8).step(1)
    a = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    for _ in range(3):
        q = p.clone()
        opt = seq.AdamW([q], [g], bits=8)
        held = [(t.data_ptr(), t.numel()) for t in (opt._plan, opt.m, opt.v)]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(20):
                a @ a
            opt.step(1)
        del opt
        others = [torch.zeros(k, dtype=torch.uint8, device="cuda") for _, k in held for _ in range(4)]
        assert not {t.data_ptr() for t in others} & {at for at, _ in held}
        torch.cuda.synchronize()
        assert torch.equal(q, want)
