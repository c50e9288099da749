"""The matrix memory's operators in 64 bits on the CPU (numpy), step by step from their definitions, with bounds for what a
computation in 32 bits may differ by (u: the distance of 1 to the next float32)."""
import numpy as np

U = 2.0 ** -23
BF16 = 2.0 ** -7        # the distance of 1 to the next bf16; a number and its bf16 differ by at most half of this, relatively
TILE = 64               # steps over which sums may be formed together


def stored(bound, value, bf16):
    """`bound` of an fp32 result once it is rounded to its type."""
    return bound + (0.5 * BF16 * (np.abs(value) + bound) if bf16 else 0.0) + 1e-37


def _sigmoid(x):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-x))


def _norm(x, axes):
    return np.sqrt((x * x).sum(axes))


def delta(q, k, v, f, b, s0=None, reset=None, scale=1.0):
    """-> o, final state, bounds of the 2-norm of the error of o per row and of the final state per head, and the states.

    The bound: a step is S <- a (I - beta k k^T) S + beta k v^T with |k| <= 1, so an error that is there does not grow, and
    what a step adds are rounded sums of up to Dk + TILE products of numbers of the size of the state and of the value:
    e <- a e + c u (|S| + |v|), c = Dk + TILE + 16, 2-norms throughout."""
    B, T, H, Dk = q.shape
    Dv = v.shape[3]
    c = (Dk + TILE + 16) * U
    a, beta = _sigmoid(f), _sigmoid(b)
    S = np.zeros((B, H, Dk, Dv)) if s0 is None else s0.astype(np.float64).copy()
    e = np.zeros((B, H))
    o, eo, states, errs = np.zeros((B, T, H, Dv)), np.zeros((B, T, H)), [S], [e]
    for t in range(T):
        if reset is not None:
            cut = reset[:, t] != 0
            S, e = np.where(cut[:, None, None, None], 0.0, S), np.where(cut[:, None], 0.0, e)
        held = a[:, t, :, None, None] * S
        gap = v[:, t] - np.einsum("bhkv,bhk->bhv", held, k[:, t])
        size = _norm(S, (2, 3)) + _norm(v[:, t], 2)
        S = held + (beta[:, t, :, None] * k[:, t])[..., None] * gap[:, :, None]
        e = a[:, t] * e + c * size
        o[:, t] = scale * np.einsum("bhkv,bhk->bhv", S, q[:, t])
        eo[:, t] = abs(scale) * _norm(q[:, t], 2) * (e + c * (_norm(S, (2, 3)) + size))
        states.append(S)
        errs.append(e)
    return o, S, eo, e, states, errs


def delta_backward(do, q, k, v, f, b, s0=None, reset=None, dlast=None, scale=1.0):
    """-> (dq, dk, dv, df, db, ds0), bounds: of the 2-norm per row for the first three, per number for df and db, of the 2-norm
    per head for ds0.  The gradient of the state passes the transposed steps: the same kind of bound.  df is a sum over the
    steps of a tile, whose errors it takes over."""
    B, T, H, Dk = q.shape
    c = (Dk + TILE + 16) * U
    o, last, eo, elast, states, errs = delta(q, k, v, f, b, s0, reset, scale)
    a, beta = _sigmoid(f), _sigmoid(b)
    D = np.zeros((B, H, Dk, v.shape[3])) if dlast is None else dlast.astype(np.float64).copy()
    e = np.zeros((B, H))
    out = [np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros_like(f), np.zeros_like(b)]
    err = [np.zeros((B, T, H)) for _ in range(5)]
    dla, part, end = np.zeros((B, T, H)), np.zeros((B, T, H)), np.zeros((B, H))
    for t in range(T - 1, -1, -1):
        if t == T - 1 or t % TILE == TILE - 1:       # what reaches beyond the tile
            n = _norm(D, (2, 3))
            end = e * _norm(states[t + 1], (2, 3)) + n * errs[t + 1] + c * n * (_norm(states[t + 1], (2, 3)) + _norm(states[t], (2, 3)))
            part_after = end.copy()
        S, before, eb = states[t + 1], states[t], errs[t]
        if reset is not None:
            cut = reset[:, t] != 0
            before, eb = np.where(cut[:, None, None, None], 0.0, before), np.where(cut[:, None], 0.0, eb)
        held = a[:, t, :, None, None] * before
        gap = v[:, t] - np.einsum("bhkv,bhk->bhv", held, k[:, t])
        nh, ng, nv, no, nq = _norm(held, (2, 3)), _norm(gap, 2), _norm(v[:, t], 2), _norm(do[:, t], 2), _norm(q[:, t], 2)
        egap = eb + c * (nh + nv)
        D = D + scale * q[:, t, :, :, None] * do[:, t, :, None]
        e = e + c * (_norm(D, (2, 3)) + abs(scale) * nq * no)
        nD = _norm(D, (2, 3))
        out[0][:, t] = scale * np.einsum("bhkv,bhv->bhk", S, do[:, t])
        err[0][:, t] = abs(scale) * no * (errs[t + 1] + c * (_norm(S, (2, 3)) + nh + nv))
        toward = np.einsum("bhkv,bhv->bhk", D, gap)
        etoward = e * ng + nD * egap + c * nD * (ng + nv + nh)
        dgap = beta[:, t, :, None] * np.einsum("bhkv,bhk->bhv", D, k[:, t])
        edgap = e + c * nD
        out[1][:, t] = beta[:, t, :, None] * toward - np.einsum("bhkv,bhv->bhk", held, dgap)
        err[1][:, t] = etoward + eb * nD + nh * edgap + c * nh * nD
        out[2][:, t], err[2][:, t] = dgap, edgap
        out[4][:, t] = (toward * k[:, t]).sum(2) * beta[:, t] * (1 - beta[:, t])
        err[4][:, t] = etoward + c * nD * ng
        D = D - k[:, t, :, :, None] * dgap[:, :, None]
        out[3][:, t] = (D * before).sum((2, 3)) * a[:, t] * (1 - a[:, t])
        no_o = _norm(o[:, t], 2)
        part[:, t] = no * eo[:, t] + nv * edgap + c * (no * (no_o + abs(scale) * nq * (nh + nv)) + nv * nD)
        part_after = part_after + part[:, t]
        err[3][:, t] = (1 - a[:, t]) * part_after * (1 + 2 * U) + 8 * U * np.abs(out[3][:, t]) * (1 + np.minimum(np.abs(f[:, t]), 100))
        e = a[:, t] * (e + c * nD)
        D = a[:, t, :, None, None] * D
        if reset is not None:
            D, e = np.where(cut[:, None, None, None], 0.0, D), np.where(cut[:, None], 0.0, e)
            out[3][:, t] = np.where(cut[:, None], 0.0, out[3][:, t])
    return (*out, D), (*err, e)


# ------------------------------------------------------------------ queries and keys per head
def _spin(position, turns):
    """Cosines and sines [M][R/2]; the product in 64 bits of mantissa, so that its fraction is known for far positions too."""
    t = np.asarray(position, np.longdouble)[:, None] * np.asarray(turns, np.longdouble)
    t = (2 * np.pi * (t - np.floor(t))).astype(np.float64)
    return np.cos(t)[:, None], np.sin(t)[:, None]


def _turn(x, cos, sin):
    h = cos.shape[-1]
    lo, hi = x[..., :h], x[..., h:2 * h]
    return np.concatenate([lo * cos - hi * sin, hi * cos + lo * sin, x[..., 2 * h:]], -1)


def _partners(x, h):
    """|x| + |what x is turned with|"""
    lo, hi = np.abs(x[..., :h]), np.abs(x[..., h:2 * h])
    return np.concatenate([lo + hi, lo + hi, np.abs(x[..., 2 * h:])], -1)


def heads(x, weight, position, turns, eps):
    """x [M][H][D] -> y, rstd, bounds of y and of rstd's relative error.  A sine or cosine is off by 2^-24 at most: by the angle's 2^-32 of a
    turn and the series' end and rounding; a sum of D squares by D / 8 + 24 u."""
    cos, sin = _spin(position, turns)
    rstd = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    z = x * rstd * weight
    erel = U * (x.shape[-1] / 8 + 24)
    return _turn(z, cos, sin), rstd[..., 0], _partners(z, len(turns)) * (erel + 8 * U), erel


def heads_backward(dy, x, weight, position, turns, eps):
    """-> (dx, dweight), their bounds"""
    cos, sin = _spin(position, turns)
    M, H, D = x.shape
    rstd = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    back, size = _turn(dy, cos, -sin), _partners(dy, len(turns))
    xh, g, gs = x * rstd, back * weight, size * np.abs(weight)
    mean, most = (g * xh).mean(-1, keepdims=True), (gs * np.abs(xh)).mean(-1, keepdims=True)
    dx = rstd * (g - xh * mean)
    return (dx, (back * xh).sum((0, 1))), (U * (D / 8 + 32) * rstd * (gs + np.abs(xh) * most), U * (M * H / 2 + 96 + D / 8) * (size * np.abs(xh)).sum((0, 1)))


# ------------------------------------------------------------------ steps for matrices
POLY = (3.4445, -4.7750, 2.0315)
PAIR = 2.0 ** -18       # a number and its pair of bf16 differ by at most this, relatively: half a step of each of two times 8 bits


def muon(p, g, m, lr, mu, nesterov=True, eps=1e-7, decay=0.0, rounds=5):
    """-> p, m, the bound of the 2-norm of the error of p - that of rounding p itself left out.

    Per round the errors of the products (each operand within PAIR, the product of both lower halves left out, another PAIR, sums of
    K terms in fp32), all in 2-norms; an error that is there grows by the derivative of X -> a X + b X X^T X + c (X X^T)^2 X, whose factors at
    singular values s, t are the quotients (f(s) - f(t)) / (s - t), (f(s) + f(t)) / (s + t) and f(s) / s."""
    if not p.size:
        return p, m, 0.0
    a, b, c = POLY
    m = mu * m + g
    u = g + mu * m if nesterov else m
    tall = u.shape[0] > u.shape[1]
    x = (u.T if tall else u) / (np.sqrt((u * u).sum()) + eps)
    r, k = x.shape
    f = lambda s: a * s + b * s ** 3 + c * s ** 5  # noqa: E731
    size = lambda y: np.sqrt((y * y).sum())  # noqa: E731
    e = (PAIR + 8 * U) * size(x)
    wide, square = 3 * PAIR + k * U / 2, 3 * PAIR + r * U / 2
    for _ in range(rounds):
        s = np.linalg.svd(x, compute_uv=False)
        gram = x @ x.T
        poly = b * gram + c * gram @ gram
        ga, pa, sa = size(gram), size(poly), s.max()
        ea = wide * size(x) * sa + PAIR * ga
        eb = abs(b) * (ea + PAIR * ga) + abs(c) * (2 * sa ** 2 * ea + square * ga * sa ** 2) + PAIR * pa + 4 * U * (abs(b) + abs(c) * sa ** 2) * ga
        new = a * x + poly @ x
        top = np.linalg.svd(poly, compute_uv=False).max()
        ex = eb * sa + square * min(pa * sa, top * size(x)) + PAIR * (size(new) + a * size(x)) + 4 * U * size(new)
        si, sj = s[:, None], s[None]
        with np.errstate(divide="ignore", invalid="ignore"):
            slope = np.where(np.abs(si - sj) > 1e-9, (f(si) - f(sj)) / (si - sj), a + 3 * b * si ** 2 + 5 * c * si ** 4)
            other = np.where(si + sj > 1e-9, (f(si) + f(sj)) / (si + sj), a)
        e = max(np.abs(slope).max(), np.abs(other).max(), a if s.min() < 1e-6 else 0.0) * e + ex
        x = new
    x = x.T if tall else x
    scale = np.sqrt(max(1.0, u.shape[0] / u.shape[1]))
    return p - lr * decay * p - lr * scale * x, m, lr * scale * (e + 4 * U * size(x))


def within(got, want, bound, axes, bf16, what):
    """2-norms of the error over `axes` against a bound of the fp32 result, the rounding to its type coming on top."""
    d = got.astype(np.float64) - want
    assert np.isfinite(got).all(), what
    off = np.sqrt((d * d).sum(axes)) if axes else np.abs(d)
    size = np.sqrt((want * want).sum(axes)) if axes else np.abs(want)
    most = stored(bound, size, bf16)
    worst = float((off / most).max()) if off.size else 0.0
    assert worst <= 1, "%s: %.3g times the bound" % (what, worst)
    return worst
