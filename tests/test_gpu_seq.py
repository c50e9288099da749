"""The recurrent network's operators against their definitions in 64 bits (tests/seq_ref.py, which derives the bounds)."""
import numpy as np
import pytest
import torch

import seq_ref as ref

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def seq():
    from paper_1804_05834_amd import seq
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return seq


def rnd(seed, *shape, scale=1.0, at=0.0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale + at).to(dtype).cuda()


def host(t):
    return None if t is None else t.double().cpu().numpy()


def close(got, want, bound, what):
    got = host(got)
    assert got.shape == want.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    off = np.abs(got - want)
    bad = ~(off <= bound) & ~np.isnan(want) & ~(got == want)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.nanmax(off / bound)))


# ------------------------------------------------------------------ gated linear recurrence
SCANS = [  # B, T, C, layout, initial state, chance of a reset
    (1, 1, 1, "plain", True, 0.0), (3, 1, 512, "half", True, 0.3), (2, 0, 8, "plain", True, 0.0), (5, 2, 3, "plain", False, 0.5),
    (2, 7, 64, "half", True, 0.1), (1, 8, 4, "plain", True, 0.0), (2, 9, 260, "plain", True, 0.1), (3, 16, 65, "half", False, 0.1), (2, 17, 64, "time", True, 0.1),
    (1, 63, 128, "half", True, 0.02), (2, 65, 130, "odd", True, 0.02), (4, 255, 68, "plain", True, 0.01), (2, 256, 64, "half", False, 0.01),
    (1, 257, 261, "plain", True, 0.01), (3, 300, 64, "broadcast", True, 0.01), (1, 1000, 512, "half", True, 0.003), (2, 777, 33, "odd", True, 0.0),
    (1, 5000, 64, "plain", True, 0.001), (1, 4097, 5, "plain", True, 0.0), (2, 2048, 72, "half", False, 1.0), (300, 3, 64, "half", True, 0.2),
    (70, 33, 192, "time", True, 0.05),
    # many sequences: strips of channels in one workgroup, and whole sequences per wave
    (300, 20, 64, "half", True, 0.05), (260, 150, 60, "plain", True, 0.02), (90, 300, 130, "odd", True, 0.01), (256, 129, 64, "time", False, 0.0), (64, 1030, 256, "half", True, 0.002),
    (1, 20000, 1, "plain", True, 0.0005), (5, 3001, 2, "odd", True, 0.001), (40, 700, 16, "time", False, 0.01), (3, 2500, 31, "half", True, 0.002),
    (3000, 1100, 2, "half", True, 0.003), (6500, 1001, 1, "time", False, 0.003),      # more than six million elements of few channels
    # few channels: more than six million elements in long sequences, whole sequences per thread, and either side of a workgroup each
    (700, 9001, 1, "half", True, 0.001), (780, 4111, 2, "time", True, 0.003), (8200, 515, 16, "plain", True, 0.003),
    (9, 512, 16, "odd", True, 0.01), (9, 513, 16, "half", True, 0.01), (30, 2730, 3, "time", True, 0.001), (4, 1025, 8, "broadcast", True, 0.5),
    # ranges whose lanes share waves, pairs of channels at any address, an odd last channel, rows far apart
    (7, 1030, 261, "plain", True, 0.004), (2, 999, 17, "odd", True, 0.01), (1, 777, 19, "time", True, 0.05), (3, 2100, 64, "half", False, 0.002), (2, 641, 127, "odd", False, 0.0),
    (1, 640, 129, "half", True, 0.3), (5, 333, 41, "broadcast", True, 0.02), (2, 40, 21, "far", True, 0.1), (1, 70, 100, "far", False, 0.0),
    # few channels in many ranges, of few sequences and of many
    (3, 5000, 2, "odd", True, 0.001), (2, 4500, 3, "half", True, 0.01), (5, 3000, 4, "time", True, 0.0), (64, 2100, 5, "plain", False, 0.002), (66, 4000, 5, "half", True, 0.002), (140, 2100, 3, "plain", True, 0.001),
    (1, 40000, 2, "half", True, 0.0002), (300, 1100, 20, "half", True, 0.003), (600, 1030, 17, "plain", True, 0.003), (2, 1003, 29, "odd", True, 0.5),
    (2100, 20, 12, "plain", True, 0.05), (2060, 17, 130, "half", True, 0.05), (2050, 24, 5, "odd", False, 0.1),
]


def scan_case(B, T, C, layout, state, chance, dtype, seed=0):
    """f, x, h0, reset as device tensors in the layout"""
    t = TYPES[dtype]
    f, x = rnd(seed, B, T, C, scale=1.5, at=2.0, dtype=t), rnd(seed + 1, B, T, C, dtype=t)
    if layout == "half":
        z = torch.cat([f, x], 2)
        f, x = z[..., :C], z[..., C:]
    elif layout == "time":      # [T][B][C] in memory
        f, x = (v.transpose(0, 1).contiguous().transpose(0, 1) for v in (f, x))
    elif layout == "odd":       # rows that begin anywhere
        z = torch.zeros(B, T, 2 * C + 3, dtype=t, device="cuda")
        z[..., 1:C + 1], z[..., C + 2:2 * C + 2] = f, x
        f, x = z[..., 1:C + 1], z[..., C + 2:2 * C + 2]
    elif layout == "far":       # a step every million and a half elements
        z = torch.empty(T * (1500001 + B) * 2, dtype=t, device="cuda")
        f, x = (z[k * T * (1500001 + B):].as_strided((B, T, C), (C, 1500001, 1)).copy_(v) for k, v in enumerate((f, x)))
    elif layout == "broadcast":     # one sequence of gates for all
        f = f[:1].expand(B, T, C)
    h0 = rnd(seed + 2, B, C) if state else None
    reset = (torch.rand(B, T, generator=torch.Generator().manual_seed(seed + 3)) < chance).cuda() if chance else None
    if layout == "time" and reset is not None:
        reset = reset.t().contiguous().t()
    return f, x, h0, reset


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("case", SCANS, ids=lambda c: "-".join(str(v) for v in c))
def test_scan(seq, case, dtype):
    print("case scan", case, dtype, flush=True)
    B, T, C, layout, state, chance = case
    f, x, h0, reset = scan_case(*case, dtype)
    bf = dtype == "bf16"
    hf, hx, hh, hr = host(f), host(x), host(h0), None if reset is None else reset.cpu().numpy()
    h, last, carry = seq.scan(f, x, h0=h0, reset=reset, save=True)
    want, wl, _, eh, el, _ = ref.scan(hf, hx, hh, hr)
    close(h, want, ref.stored(eh, want, bf), "h")
    close(last, wl, el + 1e-37, "last")
    h2, last2 = seq.scan(f, x, h0=h0, reset=reset)
    assert torch.equal(h, h2) and torch.equal(last, last2)
    dh, dlast = rnd(7, B, T, C, dtype=TYPES[dtype]), rnd(8, B, C) if state else None
    wide = torch.full((B, T, 2 * C), 77.0, dtype=TYPES[dtype], device="cuda")
    out = (wide[..., :C], wide[..., C:]) if layout in ("half", "odd") else None
    df, dx, dh0 = seq.scan_backward(dh, f, x, carry, reset=reset, dlast=dlast, out=out)
    wants, bounds = ref.scan_backward(host(dh), hf, hx, hh, hr, host(dlast))
    close(df, wants[0], ref.stored(bounds[0], wants[0], bf), "df")
    close(dx, wants[1], ref.stored(bounds[1], wants[1], bf), "dx")
    close(dh0, wants[2], bounds[2] + 1e-37, "dh0")


def test_scan_state_in_place_and_outputs_apart(seq):
    """The final state may take the initial one's place, and nothing is written beside the outputs."""
    for B, T, C in ((4, 1, 100), (1, 6000, 96), (3, 130, 64)):
        f, x, h0, reset = scan_case(B, T, C, "half", True, 0.01, "bf16", 20)
        h, last = seq.scan(f, x, h0=h0, reset=reset)
        wide = torch.full((B, T, C + 8), 5.0, dtype=torch.bfloat16, device="cuda")
        s = h0.clone()
        seq.scan(f, x, h0=s, reset=reset, out=wide[..., 4:C + 4], last=s)
        assert torch.equal(s, last) and torch.equal(wide[..., 4:C + 4], h)
        assert bool((wide[..., :4] == 5).all() and (wide[..., C + 4:] == 5).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,T,C", [(1, 6000, 97), (3, 130, 67), (2, 800, 21), (2100, 20, 33), (300, 40, 65)])
def test_scan_odd_channels_and_outputs_apart(seq, B, T, C, dtype):
    """Nothing is written beside rows of an odd number of channels, forward and backward, nor beside the states."""
    t = TYPES[dtype]
    f, x, h0, reset = scan_case(B, T, C, "half", True, 0.01, dtype, 20)
    h, last, carry = seq.scan(f, x, h0=h0, reset=reset, save=True)
    wide, s = torch.full((B, T, C + 4), 5.0, dtype=t, device="cuda"), h0.clone()
    seq.scan(f, x, h0=s, reset=reset, out=wide[..., 3:C + 3], last=s)
    assert torch.equal(s, last) and torch.equal(wide[..., 3:C + 3], h)
    assert bool((wide[..., :3] == 5).all() and (wide[..., C + 3:] == 5).all())
    dh = rnd(7, B, T, C, dtype=t)
    df, dx, dh0 = seq.scan_backward(dh, f, x, carry, reset=reset, dlast=h0)
    wide = torch.full((B, T, 2 * C + 3), 5.0, dtype=t, device="cuda")
    seq.scan_backward(dh, f, x, carry, reset=reset, dlast=h0, out=(wide[..., 1:C + 1], wide[..., C + 2:2 * C + 2]))
    assert torch.equal(wide[..., 1:C + 1], df) and torch.equal(wide[..., C + 2:2 * C + 2], dx)
    assert bool((wide[..., 0] == 5).all() and (wide[..., C + 1] == 5).all() and (wide[..., 2 * C + 2] == 5).all())


@pytest.mark.parametrize("B,T", [(2, 1), (2, 5), (2, 40), (2, 600), (2, 9000), (300, 20), (300, 300), (2100, 30)])
@pytest.mark.parametrize("C", [64, 3])
def test_scan_a_reset_forgets_anything(seq, B, T, C):
    """A state that is NaN or infinite does not reach past an episode's start, forward or backward."""
    f, x = rnd(1, B, T, C, at=1.0), rnd(2, B, T, C)
    cut = T // 2
    reset = torch.zeros(B, T, dtype=torch.uint8, device="cuda")
    reset[:, cut] = 1
    clean, cl, cc = seq.scan(f, x, reset=reset, save=True)
    h0 = torch.full((B, C), NAN, device="cuda")
    h0[1::2] = INF
    h, last, carry = seq.scan(f, x, h0=h0, reset=reset, save=True)
    assert torch.equal(h[:, cut:], clean[:, cut:]) and torch.equal(last, cl)
    assert bool(torch.isnan(h[::2, :cut]).all()) and not bool(torch.isfinite(h[1::2, :cut]).any())
    dh = rnd(3, B, T, C)
    ref_df, ref_dx, _ = seq.scan_backward(dh, f, x, cc, reset=reset)
    df, dx, dh0 = seq.scan_backward(dh, f, x, carry, reset=reset)
    assert torch.equal(df[:, cut:], ref_df[:, cut:]) and torch.equal(dx, ref_dx)
    bad = dh.clone()
    bad[:, cut:] = NAN
    df, dx, dh0 = seq.scan_backward(bad, f, x, cc, reset=reset)
    want = dh.clone()
    want[:, cut:] = 0
    rf, rx, r0 = seq.scan_backward(want, f, x, cc, reset=reset)
    assert torch.equal(df[:, :cut], rf[:, :cut]) and torch.equal(dx[:, :cut], rx[:, :cut]) and torch.equal(dh0, r0)


def test_scan_extreme_gates(seq):
    """Gates that are shut or open: f of +-infinity, of +-100, of the type's lowest value; a memory that lasts."""
    vals = [INF, -INF, 100.0, -100.0, float(torch.finfo(torch.float32).min), float(torch.finfo(torch.float32).max), 15.0, -15.0]
    for T in (1, 3, 50, 700):
        f = torch.tensor(vals).repeat(8).expand(1, T, 64).contiguous().cuda()
        x, h0 = rnd(4, 1, T, 64), rnd(5, 1, 64)
        h, last, carry = seq.scan(f, x, h0=h0, save=True)
        want, wl, _, eh, el, _ = ref.scan(host(f), host(x), host(h0))
        close(h, want, eh + 1e-37, "h")
        assert bool((h[0, :, 0] == h0[0, 0]).all()) and torch.equal(h[0, :, 1], x[0, :, 1])
        df, dx, dh0 = seq.scan_backward(x, f, x, carry)
        wants, bounds = ref.scan_backward(host(x), host(f), host(x), host(h0))
        for got, w, b in zip((df, dx, dh0), wants, bounds):
            close(got, w, b + 1e-37, "gradient")


def test_scan_gradients_against_differences(seq):
    """Derivatives along random directions by central differences of the kernel's own outputs, summed in 64 bits.  Step 2^-6:
    the third derivative of the sums is a few times the first, so the truncation is below 1e-3 of the gradient's norm."""
    B, T, C = 2, 37, 64
    f, x, h0, reset = scan_case(B, T, C, "plain", True, 0.05, "fp32", 30)
    dh, dlast = rnd(33, B, T, C), rnd(34, B, C)

    def loss(f, x, h0):
        h, last = seq.scan(f, x, h0=h0, reset=reset)
        return float((h.double() * dh.double()).sum() + (last.double() * dlast.double()).sum())

    _, _, carry = seq.scan(f, x, h0=h0, reset=reset, save=True)
    grads = seq.scan_backward(dh, f, x, carry, reset=reset, dlast=dlast)
    step = 2.0 ** -6
    for k in range(3):
        for seed in (1, 2):
            args, d = [f, x, h0], rnd(50 + seed, *(f, x, h0)[k].shape)
            up, down = list(args), list(args)
            up[k], down[k] = args[k] + step * d, args[k] - step * d
            slope = (loss(*up) - loss(*down)) / (2 * step)
            want = float((grads[k].double() * d.double()).sum())
            assert abs(slope - want) <= 2e-3 * float(grads[k].double().norm() * 1.0) * 8, (k, slope, want)


# ------------------------------------------------------------------ norm
NORMS = [(1, 1, False), (1, 4, True), (3, 7, True), (5, 64, True), (2, 250, False), (33, 512, True), (4, 1001, True), (3, 1024, False), (2, 2049, True),
         (7, 4096, True), (2, 8192, True), (1, 16384, True), (1000, 36, True), (2, 5000, False), (4099, 8, True), (130, 512, False)]


def norm_case(M, C, residual, dtype, layout="plain", seed=40):
    t = TYPES[dtype]
    x, res = rnd(seed, M, C, dtype=t), rnd(seed + 1, M, C, scale=2.0, dtype=t) if residual else None
    if layout == "odd":
        z = torch.zeros(M, 2 * C + 3, dtype=t, device="cuda")
        z[:, 1:C + 1] = x
        x = z[:, 1:C + 1]
    return x, res, rnd(seed + 2, C, scale=0.2, at=1.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["plain", "odd"])
@pytest.mark.parametrize("M,C,residual", NORMS)
def test_norm(seq, M, C, residual, layout, dtype):
    print("case norm", M, C, residual, layout, dtype, flush=True)
    bf = dtype == "bf16"
    x, res, w = norm_case(M, C, residual, dtype, layout)
    y, r, saved = seq.norm(x, w, residual=res)
    rstd = saved[0]
    wr, wy, wrstd, er, ey, erel = ref.norm(host(x), host(w), host(res))
    close(r, wr, ref.stored(er, wr, bf), "r")
    close(y, wy, ref.stored(ey, wy, bf), "y")
    close(rstd, wrstd, wrstd * erel, "rstd")
    # 8 bits: the scale is the largest value over 448, a number is off by half a step (and the value's own error)
    q, scale, r8 = seq.norm_rows(x, w, residual=res)
    assert torch.equal(r8, r)
    top = np.abs(wy).max(1)
    close(scale, top / 448, top / 448 * (erel + 8 * ref.U), "scale")
    exact = wy / (top / 448)[:, None]
    close(q, exact, np.maximum(np.abs(exact) * 2.0 ** -4, 2.0 ** -10) * 1.001 + np.abs(exact) * 2 * erel, "q")
    pad = (C + 15) // 16 * 16
    assert q.stride(0) == pad
    whole = q.as_strided((M, pad), (pad, 1)).view(torch.uint8)
    assert int(whole[:, C:].sum()) == 0
    # gradients, from the rstd that is handed over and the sum as it is before it is rounded
    dy, dr = rnd(50, M, C, dtype=TYPES[dtype]), rnd(51, M, C, dtype=TYPES[dtype]) if residual else None
    dx, dw = seq.norm_backward(dy, r, saved, w, dr=dr)
    (wdx, wdw), (edx, edw) = ref.norm_backward(host(dy), wr, host(rstd), host(w), host(dr))
    close(dx, wdx, ref.stored(edx, wdx, bf), "dx")
    close(dw, wdw, edw + 1e-37, "dw")
    dx2, dw2 = seq.norm_backward(dy, r, saved, w, dr=dr)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)      # no order that changes


def test_norm_rows_that_are_special(seq):
    """Rows of zeros, of the type's largest values, with a NaN or an infinity."""
    for dtype in TYPES.values():
        x = rnd(60, 6, 200, dtype=dtype)
        w = torch.ones(200, device="cuda")
        x[0] = 0
        x[1] = 1e-30
        x[2, 5], x[3, 7] = NAN, INF
        x[4] = 1e18
        y, _, rstd = seq.norm(x, w, eps=1e-6)
        q, scale, _ = seq.norm_rows(x, w, eps=1e-6)
        assert bool((y[0] == 0).all()) and bool((q[0].float() == 0).all()) and float(scale[0]) == 0
        assert bool(torch.isnan(y[2]).all()) and bool(torch.isnan(scale[2:4]).all()) and bool(torch.isnan(y[3, 7]))
        close(y[4:5], np.ones((1, 200)), np.full((1, 200), 0.01), "large")
        assert bool(torch.isfinite(y[[0, 1, 4, 5]]).all()) and bool(torch.isfinite(scale[[0, 1, 4, 5]]).all())
        assert float(scale[5]) > 0
    y, r, rstd = seq.norm(torch.zeros(0, 5, device="cuda"), torch.ones(5, device="cuda"))
    assert y.shape == (0, 5)
    dx, dw = seq.norm_backward(y, y, rstd, torch.ones(5, device="cuda"))
    assert dx.shape == (0, 5) and bool((dw == 0).all())


def test_norm_gradients_against_differences(seq):
    M, C = 6, 96
    x, res, w = norm_case(M, C, True, "fp32", seed=70)
    dy, dr = rnd(73, M, C), rnd(74, M, C)

    def loss(x, w):
        y, r, _ = seq.norm(x, w, residual=res)
        return float((y.double() * dy.double()).sum() + (r.double() * dr.double()).sum())

    _, r, rstd = seq.norm(x, w, residual=res)
    grads = seq.norm_backward(dy, r, rstd, w, dr=dr)
    step = 2.0 ** -6
    for k, d in ((0, rnd(75, M, C)), (1, rnd(76, C))):
        up, down = [x, w], [x, w]
        up[k], down[k] = up[k] + step * d, down[k] - step * d
        slope = (loss(*up) - loss(*down)) / (2 * step)
        want = float((grads[k].double() * d.double()).sum())
        assert abs(slope - want) <= 2e-3 * float(grads[k].double().norm()) * 8, (k, slope, want)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K", [(1, 1), (3, 16), (5, 17), (64, 512), (7, 1000), (2, 8192), (1, 16384)])
def test_rows(seq, M, K, dtype):
    x = rnd(80, M, K, dtype=TYPES[dtype])
    x[0, 0] = -9.0
    q, scale = seq.rows(x)
    hx = host(x)
    top = np.abs(hx).max(1)
    close(scale, top / 448, top / 448 * 2 * ref.U, "scale")
    exact = hx / (top / 448)[:, None]
    close(q, exact, np.maximum(np.abs(exact) * 2.0 ** -4, 2.0 ** -10) * 1.001, "q")
    assert float(q[0].float().abs().max()) == 448.0
    assert np.array_equal(host(q), ref.e4m3(q.view(torch.uint8).cpu().numpy()))


# ------------------------------------------------------------------ product
PRODUCTS = [(1, 1, 1), (1, 16, 32), (2, 3, 7), (16, 16, 16), (17, 33, 100), (32, 1024, 512), (31, 100, 129), (1, 2048, 2048), (64, 64, 64), (100, 36, 513), (128, 128, 128),
            (129, 257, 384), (200, 512, 1000), (256, 256, 2048), (300, 130, 4100), (3, 5, 8192), (1000, 18, 512), (513, 1100, 640),
            (1030, 1100, 640), (1024, 1024, 200), (1100, 1111, 16), (3333, 3700, 400), (4096, 3592, 256), (3600, 3601, 1025)]


def small_rows(seed, n, K, pad=0x7F, high=3):
    """Rows of small whole numbers as e4m3, with NaN codes in the places between K and the stride."""
    g = torch.Generator().manual_seed(seed)
    v = torch.randint(-high, high + 1, (n, K), generator=g)
    rs = (K + 15) // 16 * 16 + 16
    buf = torch.full((n, rs), pad, dtype=torch.uint8)
    buf[:, :K] = v.float().to(torch.float8_e4m3fn).view(torch.uint8)
    return buf.cuda().view(torch.float8_e4m3fn)[:, :K], v.numpy().astype(np.int64)


@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product_of_whole_numbers(seq, M, N, K):
    """Sums of small whole numbers are exact in any order: every output is the whole number it should be."""
    print("case product", M, N, K, flush=True)
    (a, ha), (w, hw) = small_rows(1, M, K), small_rows(2, N, K)
    one = lambda n: torch.ones(n, device="cuda")  # noqa: E731
    wide = torch.full((M, N + 3), 77.0, device="cuda")
    y = seq.product((a, one(M)), (w, one(N)), dtype=torch.float32, out=wide[:, 1:N + 1])
    assert np.array_equal(host(y), ha.astype(np.float64) @ hw.T.astype(np.float64))
    if N % 8 == 0:      # whole lines of y in bf16: whole numbers of up to 8 bits are exact in it too
        y = seq.product((a, one(M)), (w, one(N)), dtype=torch.bfloat16)
        assert torch.equal(y, torch.from_numpy(ha.astype(np.float64) @ hw.T.astype(np.float64)).to(torch.bfloat16).cuda())
    assert bool((wide[:, 0] == 77).all() and (wide[:, N + 1:] == 77).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product(seq, M, N, K, dtype):
    print("case product", M, N, K, dtype, flush=True)
    a, w = seq.rows(rnd(3, M, K)), seq.rows(rnd(4, N, K, scale=0.05))
    bias = rnd(5, N) if M % 2 else None
    y = seq.product(a, w, bias=bias, dtype=TYPES[dtype])
    fa, fw = host(a[0]) * host(a[1])[:, None], host(w[0]) * host(w[1])[:, None]
    want, most = fa @ fw.T, np.abs(fa) @ np.abs(fw).T
    if bias is not None:
        want = want + host(bias)
    # products of two 4-bit mantissas are exact; sums over K in pieces of 32 or more, joined one after the other; the
    # matrix instructions on 8-bit numbers, which bf16 outputs take, keep 13 bits at least of the sum of the absolute values
    bound = (ref.U * (K / 32 + 40) if dtype == "fp32" else 2.0 ** -13) * most + 4 * ref.U * np.abs(want)
    close(y, want, ref.stored(bound, want, dtype == "bf16"), "y")
    assert torch.equal(y, seq.product(a, w, bias=bias, dtype=TYPES[dtype]))


def test_product_of_nothing_and_of_nan(seq):
    empty = (torch.zeros(4, 16, device="cuda").to(torch.float8_e4m3fn)[:, :0], torch.ones(4, device="cuda"))
    bias = rnd(6, 4)
    y = seq.product(empty, empty, bias=bias, dtype=torch.float32)
    assert torch.equal(y, bias.expand(4, 4))
    a, w = seq.rows(rnd(7, 20, 40)), seq.rows(rnd(8, 30, 40))
    a[0].view(torch.uint8)[3, 39] = 0x7F
    w[1][7] = INF
    y = seq.product(a, w, dtype=torch.float32)
    assert bool(torch.isnan(y[3]).all()) and int(torch.isnan(y).sum()) == 30 and bool(torch.isinf(y[:3, 7]).all())


# ------------------------------------------------------------------ AdamW
LENGTHS = [1, 255, 256, 257, 2048, 2049, 10000, 3, 70001, 0, 512]


def adamw_case(seq, bits, gdtype, odd, seed=90):
    """Tensors (views at odd places where `odd`), gradients, copies, an optimizer with moments from earlier steps."""
    P = sum((n + 255) // 256 * 256 for n in LENGTHS)
    params, grads, copies = [], [], []
    for i, n in enumerate(LENGTHS):
        o = 1 if odd else 0
        params.append(rnd(seed + i, n + 2, scale=0.05)[o:o + n])
        grads.append((rnd(seed + 50 + i, n + 2, scale=10.0 ** -(i % 4)) * (rnd(seed + 99 + i, n + 2) > -1)).to(TYPES[gdtype])[o:o + n])
        copies.append(torch.zeros(n + 2, dtype=torch.bfloat16, device="cuda")[o:o + n])
    decays = [0.01 * (i % 3) for i in range(len(LENGTHS))]
    opt = seq.AdamW(params, grads, bits=bits, lr=1e-3, weight_decay=decays, copies=copies)
    assert opt.m.numel() == P
    return opt, params, grads, copies, decays


def adamw_want(opt, params, grads, decays, step, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8):
    """(old parameters, new ones, m and v as 32-bit arithmetic gives them one operation after the other, and the size of
    the update were its terms not to cancel), in 64 bits but for the moments"""
    P = opt.m.numel()
    g, p, d = np.zeros(P), np.zeros(P), np.zeros(P)
    at = 0
    for x, y, w in zip(params, grads, decays):
        n = x.numel()
        p[at:at + n], g[at:at + n], d[at:at + n] = host(x), host(y), w
        at += (n + 255) // 256 * 256
    m, v = host(opt.m.float()).astype(np.float32), host(opt.v.float()).astype(np.float32)
    if opt.bits == 8:
        m = (m.reshape(-1, 256) * opt.m_scale.cpu().numpy()[:, None]).reshape(-1)
        v = (v.reshape(-1, 256) * opt.v_scale.cpu().numpy()[:, None]).reshape(-1)
    g32, f = g.astype(np.float32), np.float32
    m32 = (m * f(b1)).astype(f) + (g32 * f(1 - b1)).astype(f)
    v32 = (v * f(b2)).astype(f) + ((g32 * g32).astype(f) * f(1 - b2)).astype(f)
    m64, v64 = m * b1 + g * (1 - b1), v * b2 + g * g * (1 - b2)
    root = np.sqrt(v64 / (1 - b2 ** step)) + eps
    new = p - lr * d * p - lr * (m64 / (1 - b1 ** step)) / root
    return p, new, m32, v32, lr * ((np.abs(m * b1) + np.abs(g * (1 - b1))) / (1 - b1 ** step)) / root


@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("gdtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(seq, bits, gdtype, odd):
    print("case adamw", bits, gdtype, odd, flush=True)
    opt, params, grads, copies, decays = adamw_case(seq, bits, gdtype, odd)
    for step in (1, 2, 3):
        old, new, m32, v32, size = adamw_want(opt, params, grads, decays, step)
        opt.step(step, seed=1000 + step)
        got, at = np.zeros(opt.m.numel()), 0
        for x, c in zip(params, copies):
            got[at:at + x.numel()] = host(x)
            assert torch.equal(c, x.to(torch.bfloat16))
            at += (x.numel() + 255) // 256 * 256
        # the update is a few roundings of its terms' size off, the parameter two of its own
        assert (np.abs(got - new) <= 2 * ref.U * np.abs(old) + 24 * ref.U * size + 1e-30).all()
        if bits == 32:
            assert np.array_equal(opt.m.cpu().numpy(), m32) and np.array_equal(opt.v.cpu().numpy(), v32)
        else:
            qm, sm, qv, sv = ref.moments8(m32, v32, 1000 + step)
            assert np.array_equal(opt.m_scale.cpu().numpy(), sm) and np.array_equal(opt.v_scale.cpu().numpy(), sv)
            assert np.array_equal(ref.e4m3(opt.m.view(torch.uint8).cpu().numpy()), qm.astype(np.float64))
            assert np.array_equal(ref.e5m2(opt.v.view(torch.uint8).cpu().numpy()), qv.astype(np.float64))
        for i, g in enumerate(grads):
            g.copy_(rnd(300 + 20 * step + i, g.numel(), scale=10.0 ** -(i % 4)).to(g.dtype))
    opt.close()


def test_adamw_writes_its_tensors_only(seq):
    buf = torch.full((5000,), 3.0, device="cuda")
    g = torch.ones(5000, device="cuda")
    opt = seq.AdamW([buf[1:700], buf[1001:3001]], [g[:699], g[:2000]], bits=8, lr=0.5)
    opt.step(1, seed=4)
    inside = torch.zeros(5000, dtype=torch.bool, device="cuda")
    inside[1:700] = True
    inside[1001:3001] = True
    assert bool((buf[~inside] == 3).all()) and bool((buf[inside] != 3).all())
    m = opt.m.float()
    assert bool((m[699:768] == 0).all()) and bool((m[768 + 2000:] == 0).all()) and bool((m[:699] != 0).all())


def test_adamw_units_that_are_off_and_gradients_that_are_not_finite(seq):
    for bits in (32, 8):
        p, g = torch.ones(1024, device="cuda"), torch.zeros(1024, device="cuda")
        opt = seq.AdamW([p], [g], bits=bits, weight_decay=0.0)
        for t in (1, 2):
            opt.step(t, seed=t)
        assert bool((p == 1).all()) and bool((opt.m.float() == 0).all()) and bool((opt.v.float() == 0).all())
        g[300] = NAN
        opt.step(3, seed=3)
        opt.step(4, seed=4)
        touched = torch.isnan(p)
        assert bool(touched[300]) and not bool(touched[:256].any()) and not bool(touched[512:].any())
        assert bits == 8 or int(touched.sum()) == 1


def test_adamw_eight_bits_keep_the_second_moment_on_average(seq):
    """Gradients of a fixed size per element, spread over two orders of magnitude within each 256: the 8-bit second moment
    stays what the 32-bit one is on average, at the start, after thousands of steps and after the gradients become a tenth.
    An element's rounding noise is a third of its value at most (a step of the type is a quarter, it is taken about once
    in 250 steps and forgotten after 1000), so the mean over 65,536 of them is within 0.2 % and 1 % is five times that."""
    n = 65536
    size = torch.exp(rnd(1, n, scale=0.8))
    p8, p32, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    o8, o32 = seq.AdamW([p8], [g], bits=8, lr=0.0), seq.AdamW([p32], [g], bits=32, lr=0.0)
    for t in range(1, 3001):
        g.copy_(size * (0.1 if t > 1500 else 1.0) * (1 if t % 2 else -1))
        o8.step(t, seed=t)
        o32.step(t, seed=t)
        if t in (10, 1500, 3000):
            v8 = (o8.v.float().view(-1, 256) * o8.v_scale[:, None]).view(-1)
            ratio = float((v8.double() / o32.v.double()).mean())
            assert abs(ratio - 1) < 0.01, (t, ratio)


# ------------------------------------------------------------------ streams, recordings
def test_recorded_and_on_another_stream(seq):
    """One block's forward and backward, its 8-bit form and the optimizer's step recorded into a graph: every replay gives
    what eager calls give on the same data, with eager work in between; and so do calls on a side stream."""
    B, T, C = 4, 600, 128
    z, dh = rnd(1, B, T, 2 * C, dtype=torch.bfloat16), rnd(2, B, T, C, dtype=torch.bfloat16)
    reset = (torch.rand(B, T, generator=torch.Generator().manual_seed(3)) < 0.02).cuda()
    w, w8 = rnd(4, C, scale=0.1, at=1.0), seq.rows(rnd(5, 3 * C, C))
    p, state = rnd(6, C), torch.zeros(B, C, device="cuda")

    def work(p, opt, grad, state):
        h, last, carry = seq.scan(z[..., :C], z[..., C:], h0=state, reset=reset, save=True)
        y, r, rstd = seq.norm(h.view(B * T, C), w, residual=dh.view(B * T, C))
        dx, dw = seq.norm_backward(dh.view(B * T, C), r, rstd, w)
        df, dz, dh0 = seq.scan_backward(dx.view(B, T, C), z[..., :C], z[..., C:], carry, reset=reset)
        q, scale, _ = seq.norm_rows(h.view(B * T, C), w)
        out = seq.product((q, scale), w8)
        grad.copy_(dw)
        opt.step(5, seed=11)
        state.copy_(last)
        return [h, last, y, dx, dw, df, dz, dh0, q, scale, out, p, opt.m, opt.v]

    def fresh():
        q, g = p.clone(), torch.zeros(C, device="cuda")
        return q, seq.AdamW([q], [g], bits=8), g, state.clone()

    a, b, c = fresh(), fresh(), fresh()
    work(*fresh())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = work(*b)
    side = torch.cuda.Stream()
    for i in range(4):
        z.copy_(rnd(100 + i, B, T, 2 * C, dtype=torch.bfloat16))
        eager = [t.clone() for t in work(*a)]
        graph.replay()
        torch.cuda.synchronize()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = work(*c)
        torch.cuda.synchronize()
        for k, (x, y, v) in enumerate(zip(eager, recorded, other)):
            x, y, v = (t.view(torch.uint8) if t.element_size() == 1 else t for t in (x, y, v))
            assert torch.equal(x, y) and torch.equal(x, v), (i, k)


# ------------------------------------------------------------------ refusals
def test_refusals(seq):
    f, x = rnd(1, 2, 4, 8), rnd(2, 2, 4, 8)
    from paper_1804_05834_amd.dqn import ERR_INVALID_ARG, DqnError
    for call in (lambda: seq.scan(f, x[:, :3]), lambda: seq.scan(f, x.to(torch.bfloat16)), lambda: seq.scan(f.half(), x.half()),
                 lambda: seq.scan(f, x.cpu()), lambda: seq.scan(f, x, h0=rnd(3, 2, 9)), lambda: seq.scan(f, x, reset=torch.zeros(2, 5, device="cuda")),
                 lambda: seq.scan(f.transpose(1, 2), x.transpose(1, 2)), lambda: seq.scan_backward(f, f, x, rnd(1, 3)),
                 lambda: seq.norm(f.view(8, 8), rnd(1, 7)), lambda: seq.norm(f, rnd(1, 8)), lambda: seq.norm_backward(rnd(1, 2, 4), rnd(1, 2, 4), (rnd(1, 3), rnd(1, 2, 4), None), rnd(1, 4)),
                 lambda: seq.product(seq.rows(rnd(1, 3, 16)), seq.rows(rnd(1, 3, 17))), lambda: seq.product(seq.rows(rnd(1, 3, 16)), seq.rows(rnd(1, 3, 16)), bias=rnd(1, 4)),
                 lambda: seq.AdamW([f], []), lambda: seq.AdamW([f], [x[0]]), lambda: seq.AdamW([f.to(torch.bfloat16)], [x])):
        with pytest.raises(ValueError):
            call()
    wide = torch.zeros(4, 40, device="cuda").to(torch.float8_e4m3fn)
    opt = seq.AdamW([f], [x])
    for call in (lambda: seq.scan(f, x, out=torch.zeros(1, 4, 8, device="cuda").expand(2, 4, 8)),       # rows on top of each other
                 lambda: seq.norm(rnd(1, 2, 20000), rnd(1, 20000)), lambda: seq.norm(f.view(8, 8), rnd(1, 8), eps=-1.0), lambda: seq.norm(f.view(8, 8), rnd(1, 8), eps=NAN),
                 lambda: seq.product((wide[:, 1:17], torch.ones(4, device="cuda")), (wide[:, :16], torch.ones(4, device="cuda"))),
                 lambda: seq.product((wide.view(-1)[:32].view(4, 8), torch.ones(4, device="cuda")), (wide[:, :8], torch.ones(4, device="cuda"))),
                 lambda: seq.AdamW([f], [x], bits=16), lambda: seq.AdamW([f], [x], weight_decay=-0.1), lambda: opt.step(0), lambda: opt.step(1, lr=NAN)):
        with pytest.raises(DqnError) as e:
            call()
        assert e.value.code == ERR_INVALID_ARG and len(str(e.value)) > 30
    assert torch.equal(seq.scan(f, x)[0], seq.scan(f, x)[0])      # and goes on working
