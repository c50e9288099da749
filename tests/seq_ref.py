"""The recurrent network's operators in 64 bits on the CPU (numpy), step by step from their definitions, with bounds
for what a computation in 32 bits may differ by: every bound follows the errors of single operations through the
formula (u: the distance of 1 to the next float32; a gate computed by exp and a division is off by a few u
and by |f| u, since a relative error of exp's argument is an absolute one of its exponent)."""
import numpy as np

U = 2.0 ** -23
BF16 = 2.0 ** -7        # the distance of 1 to the next bf16; a number and its bf16 differ by at most half of this, relatively


def stored(bound, value, bf16):
    """`bound` of an fp32 result once it is rounded to its type."""
    return bound + (0.5 * BF16 * (np.abs(value) + bound) if bf16 else 0.0) + 1e-37


def scan(f, x, h0=None, reset=None):
    """-> h, final state, state before each step (after the reset), their bounds (h, final, before)"""
    B, T, C = f.shape
    with np.errstate(over="ignore"):
        a, i = 1 / (1 + np.exp(-f)), 1 / (1 + np.exp(f))
    s = np.zeros((B, C)) if h0 is None else h0.astype(np.float64).copy()
    e = np.zeros((B, C))
    h, before, eh, eb = (np.zeros((B, T, C)) for _ in range(4))
    rel = U * (8 + 2 * np.minimum(np.abs(f), 1e3))
    for t in range(T):
        if reset is not None:
            cut = reset[:, t, None] != 0
            s, e = np.where(cut, 0.0, s), np.where(cut, 0.0, e)
        before[:, t], eb[:, t] = s, e
        e = a[:, t] * e + rel[:, t] * (a[:, t] * np.abs(s) + i[:, t] * np.abs(x[:, t]))
        s = a[:, t] * s + i[:, t] * x[:, t]
        h[:, t], eh[:, t] = s, e
    return h, s, before, eh, e, eb


def scan_backward(dh, f, x, h0=None, reset=None, dlast=None):
    """-> (df, dx, dh0), their bounds"""
    B, T, C = f.shape
    _, _, before, _, _, eb = scan(f, x, h0, reset)
    with np.errstate(over="ignore"):
        a, i = 1 / (1 + np.exp(-f)), 1 / (1 + np.exp(f))
    rel = U * (8 + 2 * np.minimum(np.abs(f), 1e3))
    mu = np.zeros((B, C)) if dlast is None else dlast.astype(np.float64).copy()
    em = np.zeros((B, C))
    df, dx, edf, edx = (np.zeros((B, T, C)) for _ in range(4))
    for t in range(T - 1, -1, -1):
        lam = dh[:, t] + mu
        el = em + U * (np.abs(dh[:, t]) + np.abs(mu))
        ai, gap = a[:, t] * i[:, t], before[:, t] - x[:, t]
        dx[:, t], edx[:, t] = i[:, t] * lam, i[:, t] * (el + rel[:, t] * np.abs(lam))
        df[:, t] = ai * lam * gap
        edf[:, t] = ai * (el * np.abs(gap) + np.abs(lam) * (eb[:, t] + U * (np.abs(before[:, t]) + np.abs(x[:, t]))) + 2 * rel[:, t] * np.abs(lam * gap))
        mu, em = a[:, t] * lam, a[:, t] * (el + rel[:, t] * np.abs(lam))
        if reset is not None:
            cut = reset[:, t, None] != 0
            mu, em = np.where(cut, 0.0, mu), np.where(cut, 0.0, em)
    return (df, dx, mu), (edf, edx, em)


def norm(x, weight, residual=None, eps=1e-6):
    """-> r, y, rstd, bounds of r and y and the relative one of rstd"""
    r = x + (0.0 if residual is None else residual)
    er = U * np.abs(r)
    ms = (r * r).mean(1, keepdims=True)
    # C squares added up, at least 64 sums at a time
    erel = U * (x.shape[1] / 64 + 24)
    rstd = 1 / np.sqrt(ms + eps)
    y = r * rstd * weight
    return r, y, rstd[:, 0], er, np.abs(y) * (erel + 4 * U), erel


def norm_backward(dy, r, rstd, weight, dr=None):     # r: the sum before it is rounded
    """-> (dx, dw), their bounds"""
    M, C = r.shape
    xh, g = r * rstd[:, None], dy * weight
    mean, most = (g * xh).mean(1, keepdims=True), np.abs(g * xh).mean(1, keepdims=True)
    dx = rstd[:, None] * (g - xh * mean)
    e = U * (C / 64 + 24) * rstd[:, None] * (np.abs(g) + np.abs(xh) * most)
    if dr is not None:
        dx = dx + dr
        e = e + U * np.abs(dx)
    dw = (dy * xh).sum(0)
    return (dx, dw), (e, U * (M / 2 + 64) * np.abs(dy * xh).sum(0))


# ------------------------------------------------------------------ 8-bit numbers
def e4m3(codes):
    """The numbers that bytes stand for (NaN: 0x7F, 0xFF)."""
    c = codes.astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * np.exp2(e - 10.0))
    return np.where((c & 127) == 127, np.nan, np.where(c & 128, -v, v))


def e5m2(codes):
    c = codes.astype(np.int64)
    e, m = (c >> 2) & 31, c & 3
    v = np.where(e == 0, m * 2.0 ** -16, (4 + m) * np.exp2(e - 17.0))
    v = np.where(e == 31, np.where(m == 0, np.inf, np.nan), v)
    return np.where(c & 128, -v, v)


def draws(seed, n):
    """32 bits for each of n elements: halves of the library's draws, lower half first."""
    with np.errstate(over="ignore"):
        z = np.uint64(seed) + np.arange(1, (n + 1) // 2 + 1, dtype=np.uint64) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
    return np.ascontiguousarray(z).view("<u4")[:n]


def moments8(m, v, seed):
    """New moments (fp32 arrays, a multiple of 256 long) -> numbers and scales of both, in 32-bit arithmetic."""
    bits = draws(seed, m.size)
    out = []
    for x, top, word, mantissa, lowest in ((m, 448.0, bits & 0xFFFF, 3, -6), (v, 57344.0, bits >> 16, 2, -14)):
        b = x.reshape(-1, 256)
        most = np.abs(b).max(1)
        inv = np.where(most > 0, np.float32(1) / np.where(most > 0, most, 1).astype(np.float32) * np.float32(top), np.float32(0)).astype(np.float32)
        q = np.abs((b * inv[:, None]).astype(np.float32)).reshape(-1)
        # above 2^lowest the lattice of 32-bit numbers themselves, their lower bits being the part that is rounded
        drop = 23 - mantissa
        up = ((q.view(np.uint32) + (word.astype(np.uint32) << np.uint32(drop - 16))) & np.uint32(~((1 << drop) - 1) & 0xFFFFFFFF)).view(np.float32)
        unit = np.float32(2.0 ** (lowest - mantissa))
        small = np.floor((q / unit + word.astype(np.float32) / np.float32(65536)).astype(np.float32)) * unit
        q = np.minimum(np.where(q < 2.0 ** lowest, small, up), np.float32(top))
        if mantissa == 2:
            q = np.where(x > 0, np.maximum(q, unit), q)
        out += [np.copysign(q, x), (most * (np.float32(1) / np.float32(top))).astype(np.float32)]
    return out
