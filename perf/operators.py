"""The operators of a recurrent Q-network, as cases that can be timed and compared.

A network that sees more than four frames keeps a memory of its episode: blocks of a normalised
residual stream, a projection, a gated linear recurrence over time and a second projection, trained
over stored sequences and stepped once per environment step while acting.  Four operators:

  scan     h_t = a_t h_{t-1} + (1 - a_t) x_t with a_t = sigmoid(f_t) per channel, the state set to
           zero before a step whose `reset` flag is set (a new episode); f and x are the two halves of
           one projection.  mode "forward": a sequence or, with T = 1, the step of an acting agent;
           "train": forward and backward.
  norm     r = x + residual, y = weight r / sqrt(mean r^2 + eps) per row.  mode "rows8": y in 8 bits
           (e4m3, one scale per row: the largest value stands for 448); "train": y in the type of
           x, then the gradients of x (that of the residual is the same) and of the weight.
  product  y = (a w^T) a_scale w_scale + bias for 8-bit rows a [M][K] and weights w [N][K]
  adamw    one AdamW step over many tensors, moments in 32 bits or in 8 (e4m3 and e5m2 with a
           scale per 256 elements, rounded up or down at random so that small changes are kept on
           average).  The random bits are a function of the seed and the element's number.

Sizes: 512 channels and the batch of 32 are the network's and the paper's own, 2048 environments and
up to 8192 observations are this repository's acting configurations, the small sets of tensors are the
Q-network's; the rest are generic.  1 % of the steps start an episode, as in the configurations.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
EPS = 1e-6                        # of the norm
LR, BETA1, BETA2, ADAM_EPS, DECAY = 2.5e-4, 0.9, 0.999, 1e-8, 0.01
M_MAX, V_MAX = 448.0, 57344.0     # largest numbers of e4m3 and e5m2
BLOCK = 256                       # elements that share a scale
MOST_ELEMENTS, MOST_PRODUCT, MOST_PARAMETERS = 1 << 26, 1 << 36, 1 << 26


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # 32 environments ask for their next action: one step of the memory, nothing but latency
        dict(name="scan_step_32", kind="scan", mode="forward", dtype="bf16", B=32, T=1, C=512, state=True),
        # a minibatch of 32 stored sequences of 512 steps
        dict(name="scan_train_32x512", kind="scan", mode="train", dtype="bf16", B=32, T=512, C=512, state=True),
        # ragged in every direction, full precision, few channels and a longer sequence
        dict(name="scan_train_7x4099", kind="scan", mode="train", dtype="fp32", B=7, T=4099, C=261, state=False),
        # one long recorded stream is read through once
        dict(name="scan_read_131072", kind="scan", mode="forward", dtype="bf16", B=1, T=131072, C=512, state=True),
        # 32 acting environments: rows for an 8-bit product
        dict(name="norm_rows8_32", kind="norm", mode="rows8", dtype="bf16", M=32, C=512, residual=True),
        # the tokens of the minibatch of sequences, with gradients
        dict(name="norm_train_16384", kind="norm", mode="train", dtype="bf16", M=16384, C=512, residual=True),
        # many rows of an odd width in full precision
        dict(name="norm_train_30011", kind="norm", mode="train", dtype="fp32", M=30011, C=1001, residual=True),
        # acting of 32 environments: the projection to the two halves f and x
        dict(name="product_32", kind="product", dtype="bf16", M=32, N=1024, K=512, bias=True),
        # the largest acting batch through a wide projection
        dict(name="product_8192", kind="product", dtype="bf16", M=8192, N=4096, K=2048, bias=True),
        # the Q-network's twelve tensors
        dict(name="adamw_qnet_32bit", kind="adamw", bits=32, grad="fp32", tensors=0, total=0, shapes=0),
        # the same with 8-bit moments, gradients in bf16
        dict(name="adamw_qnet_8bit", kind="adamw", bits=8, grad="bf16", tensors=0, total=0, shapes=0),
        # a large network of many tensors, matrices and vectors
        dict(name="adamw_large_8bit", kind="adamw", bits=8, grad="bf16", tensors=150, total=100000000, shapes=7),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["scan", "scan", "norm", "norm", "product", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if kind == "scan":
        mode = rng.choice(["forward", "train", "train"])
        B, C = _log_int(rng, 1, 2048), _log_int(rng, 1, 1024)
        room = (MOST_ELEMENTS >> (mode == "train") >> (dtype == "fp32")) // (B * C)
        return dict(kind=kind, mode=mode, dtype=dtype, B=B, T=_log_int(rng, 1, max(1, min(131072, room))), C=C,
                    state=rng.random() < 0.5)
    if kind == "norm":
        mode, C = rng.choice(["rows8", "train"]), _log_int(rng, 4, 8192)
        return dict(kind=kind, mode=mode, dtype=dtype, M=_log_int(rng, 1, min(131072, (MOST_ELEMENTS >> 1) // C)), C=C,
                    residual=rng.random() < 0.7)
    if kind == "product":
        N, K = _log_int(rng, 1, 8192), _log_int(rng, 1, 8192)
        return dict(kind=kind, dtype=dtype, M=_log_int(rng, 1, min(8192, MOST_PRODUCT // (N * K))), N=N, K=K,
                    bias=rng.random() < 0.5)
    tensors = _log_int(rng, 1, 300)
    return dict(kind=kind, bits=rng.choice([8, 32]), grad=dtype, tensors=tensors,
                total=_log_int(rng, 1000, MOST_PARAMETERS), shapes=rng.randrange(1 << 20))


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case):
    """Elements of each tensor of an adamw case."""
    if not case["tensors"]:      # the Q-network with a dueling head of 18 actions: weights and biases layer by layer
        return [8192, 32, 32768, 64, 36864, 64, 512 * 3136, 512, 512, 1, 18 * 512, 18]
    r = random.Random(case["shapes"])
    part = [math.exp(r.uniform(0.0, 9.0)) for _ in range(case["tensors"])]
    return [max(1, int(case["total"] * p / sum(part))) for p in part]


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]

    def normal(*shape, scale=1.0, at=0.0):
        return torch.randn(*shape, generator=g, device=DEV) * scale + at

    if kind == "scan":
        B, T, C, t = case["B"], case["T"], case["C"], _type(case)
        z = torch.empty(B, T, 2 * C, dtype=t, device=DEV)
        z[..., :C] = normal(B, T, C, scale=1.5, at=2.0).to(t)
        z[..., C:] = normal(B, T, C).to(t)
        s = dict(z=z, reset=(torch.rand(B, T, generator=g, device=DEV) < 0.01).to(torch.uint8),
                 h0=normal(B, C, scale=0.5) if case["state"] else None)
        if case["mode"] == "train":
            s["dh"] = normal(B, T, C, scale=0.1).to(t)
            s["dlast"] = normal(B, C, scale=0.1) if case["state"] else None
    elif kind == "norm":
        M, C, t = case["M"], case["C"], _type(case)
        s = dict(x=normal(M, C).to(t), res=normal(M, C, scale=2.0).to(t) if case["residual"] else None,
                 weight=normal(C, scale=0.2, at=1.0))
        if case["mode"] == "train":
            s["dy"] = normal(M, C, scale=0.1).to(t)
            s["dr"] = normal(M, C, scale=0.1).to(t) if case["residual"] else None
    elif kind == "product":
        # rows as the framework keeps them: a stride that is a multiple of 16
        def rows(n, scale):
            v = normal(n, case["K"], scale=scale)
            top = v.abs().amax(1)
            buf = torch.zeros(n, (case["K"] + 15) // 16 * 16, device=DEV)
            buf[:, :case["K"]] = v * (M_MAX / top)[:, None]
            return buf.clamp(-M_MAX, M_MAX).to(torch.float8_e4m3fn)[:, :case["K"]], top / M_MAX

        a, w = rows(case["M"], 1.0), rows(case["N"], 1.0 / math.sqrt(case["K"]))
        s = dict(a=a, w=w, bias=normal(case["N"], scale=0.1) if case["bias"] else None)
    else:
        # one buffer per kind of data, in which a tensor begins at a multiple of 256 elements; a tenth of the gradients
        # are zero (units that are off), their sizes differ from tensor to tensor
        lengths = _lengths(case)
        at = [0]
        for n in lengths:
            at.append(at[-1] + (n + BLOCK - 1) // BLOCK * BLOCK)
        P = at[-1]
        real = torch.zeros(P, dtype=torch.bool, device=DEV)
        size, decay = torch.empty(P, device=DEV), torch.empty(P, device=DEV)
        r = random.Random(int(seed))
        decays = [DECAY if n > 1000 else 0.0 for n in lengths]      # vectors do not decay
        for n, a, b, d in zip(lengths, at, at[1:], decays):
            real[a:a + n] = True
            size[a:b] = math.exp(r.uniform(-9.0, -4.0))
            decay[a:b] = d
        live = real & (torch.rand(P, generator=g, device=DEV) < 0.9)
        p = normal(P, scale=0.05) * real
        grad = (normal(P) * size * live).to(torch.bfloat16 if case["grad"] == "bf16" else torch.float32)
        m, v = normal(P, scale=0.3) * size * real, (size * normal(P, scale=0.7)).square() * real
        del live, size, real
        s = dict(p=p, grad=grad, decay=decay, step=100 + int(seed) % 100, seed=int(seed) * 7919 + 5)
        if case["bits"] == 8:
            def codes(t, top, kind8):
                b = t.view(-1, BLOCK)
                most = b.abs().amax(1, keepdim=True)
                inv = torch.where(most > 0, top / most, torch.zeros_like(most))
                return (b * inv).clamp(-top, top).to(kind8).view(-1), (most / top).view(-1)

            s["m"], s["ms"] = codes(m, M_MAX, torch.float8_e4m3fn)
            s["v"], s["vs"] = codes(v, V_MAX, torch.float8_e5m2)
        else:
            s["m"], s["v"], s["ms"], s["vs"] = m, v, None, None
        if own:     # the optimizer that a training program keeps: its table of tensors
            from paper_1804_05834_amd import seq
            views = [(p[a:a + n], grad[a:a + n]) for n, a in zip(lengths, at)]
            s["opt"] = seq.AdamW([x for x, _ in views], [x for _, x in views], bits=case["bits"], lr=LR, betas=(BETA1, BETA2),
                                 eps=ADAM_EPS, weight_decay=decays, state=(s["m"], s["v"], s["ms"], s["vs"]))
    s["case"] = dict(case)
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    return (_own if own else _plain)[case["kind"]](state, case)


def _own_scan(s, case):
    from paper_1804_05834_amd import seq
    C = case["C"]
    f, x = s["z"][..., :C], s["z"][..., C:]
    if case["mode"] == "forward":
        h, last = seq.scan(f, x, h0=s["h0"], reset=s["reset"])
        return {"h": h, "last": last}
    h, last, carry = seq.scan(f, x, h0=s["h0"], reset=s["reset"], save=True)
    dz = torch.empty_like(s["z"])
    _, _, dh0 = seq.scan_backward(s["dh"], f, x, carry, reset=s["reset"], dlast=s["dlast"], out=(dz[..., :C], dz[..., C:]))
    return {"h": h, "last": last, "dz": dz, "dh0": dh0}


def _own_norm(s, case):
    from paper_1804_05834_amd import seq
    if case["mode"] == "rows8":
        q, scale, r = seq.norm_rows(s["x"], s["weight"], residual=s["res"], eps=EPS)
        return {"q": q, "scale": scale, "r": r if case["residual"] else None}
    y, r, rstd = seq.norm(s["x"], s["weight"], residual=s["res"], eps=EPS)
    dx, dw = seq.norm_backward(s["dy"], r, rstd, s["weight"], dr=s["dr"])
    return {"y": y, "r": r if case["residual"] else None, "dx": dx, "dw": dw}


def _own_product(s, case):
    from paper_1804_05834_amd import seq
    return {"y": seq.product(s["a"], s["w"], bias=s["bias"], dtype=_type(case))}


def _own_adamw(s, case):
    s["opt"].step(s["step"], seed=s["seed"])
    return {k: s[k] for k in ("p", "m", "v", "ms", "vs")}


def _inclusive(a, b):
    """All h_t = a_t h_{t-1} + b_t of h_{-1} = 0 along dimension 1, by doubling: log2 T steps over the whole sequence."""
    s = 1
    while s < a.shape[1]:
        b = torch.cat([b[:, :s], torch.addcmul(b[:, s:], a[:, s:], b[:, :-s])], 1)
        a = torch.cat([a[:, :s], a[:, s:] * a[:, :-s]], 1)
        s *= 2
    return b


def _plain_scan(s, case):
    C, t = case["C"], _type(case)
    f, x = s["z"][..., :C].float(), s["z"][..., C:].float()
    a, i = torch.sigmoid(f), torch.sigmoid(-f)
    keep = torch.where(s["reset"][..., None] != 0, torch.zeros_like(a), a)
    b = i * x
    if s["h0"] is not None:
        b[:, 0] += keep[:, 0] * s["h0"]
    h = _inclusive(keep, b)
    out = {"h": h.to(t), "last": h[:, -1].clone()}
    if case["mode"] == "forward":
        return out
    d = s["dh"].float()
    if s["dlast"] is not None:
        d[:, -1] += s["dlast"]
    after = torch.cat([keep[:, 1:], torch.zeros_like(keep[:, :1])], 1)      # what carries h_t on to the next step
    lam = _inclusive(after.flip(1), d.flip(1)).flip(1)
    before = torch.zeros_like(h)
    before[:, 1:] = h[:, :-1]
    if s["h0"] is not None:
        before[:, 0] = s["h0"]
    before = torch.where(s["reset"][..., None] != 0, torch.zeros_like(before), before)
    return {**out, "dz": torch.cat([lam * (before - x) * a * i, lam * i], 2).to(t), "dh0": keep[:, 0] * lam[:, 0]}


def _plain_norm(s, case):
    t = _type(case)
    r = s["x"].float()
    if s["res"] is not None:
        r = r + s["res"].float()
    rstd = torch.rsqrt(r.square().mean(1, keepdim=True) + EPS)
    xh = r * rstd
    y = xh * s["weight"]
    stored = r.to(t) if s["res"] is not None else None
    if case["mode"] == "rows8":
        top = y.abs().amax(1, keepdim=True)
        inv = torch.where(top > 0, M_MAX / top, torch.zeros_like(top))
        return {"q": (y * inv).clamp(-M_MAX, M_MAX).to(torch.float8_e4m3fn), "scale": (top / M_MAX)[:, 0], "r": stored}
    dy = s["dy"].float()
    g = dy * s["weight"]
    dx = rstd * (g - xh * (g * xh).mean(1, keepdim=True))
    if s["dr"] is not None:
        dx = dx + s["dr"].float()
    return {"y": y.to(t), "r": stored, "dx": dx.to(t), "dw": (dy * xh).sum(0)}


def _plain_product(s, case):
    (a, sa), (w, sw) = s["a"], s["w"]
    y = torch.matmul(a.float(), w.float().t()) * sa[:, None] * sw
    if s["bias"] is not None:
        y = y + s["bias"]
    return {"y": y.to(_type(case))}


def _bits(seed, n):
    """16 random bits for the first and 16 for the second moment of each of n elements: the output of the generator
    of this repository's draws number i // 2, its lower half for even i and its upper half for odd i."""
    z = torch.arange(1, (n + 1) // 2 + 1, dtype=torch.int64, device=DEV) * -7046029254386353131 + _signed(seed)
    z = (z ^ ((z >> 30) & 0x3FFFFFFFF)) * -4658895280553007687
    z = (z ^ ((z >> 27) & 0x1FFFFFFFFF)) * -7723592293110705685
    z = z ^ ((z >> 31) & 0x1FFFFFFFF)
    z = torch.stack([z & 0xFFFFFFFF, (z >> 32) & 0xFFFFFFFF], 1).view(-1)[:n].to(torch.int64)
    return z & 0xFFFF, z >> 16


def _signed(seed):
    seed &= (1 << 64) - 1
    return seed - (1 << 64) if seed >> 63 else seed


def _rounded(x, bits, mantissa, lowest):
    """x to `mantissa` bits (below the number 2^lowest: to multiples of 2^(lowest - mantissa)), up where the random bits
    are the larger and down where they are not."""
    drop = 23 - mantissa
    normal = ((x.abs().view(torch.int32) + (bits << (drop - 16)).to(torch.int32)) & -(1 << drop)).view(torch.float32)
    unit = 2.0 ** (lowest - mantissa)
    small = torch.floor(x.abs() / unit + bits.float() / 65536.0) * unit
    return torch.where(x.abs() < 2.0 ** lowest, small, normal) * torch.sign(x)


def _plain_adamw(s, case):
    grad, p, eight = s["grad"].float(), s["p"], case["bits"] == 8
    m, v = s["m"].float(), s["v"].float()
    if eight:
        m = (m.view(-1, BLOCK) * s["ms"][:, None]).view(-1)
        v = (v.view(-1, BLOCK) * s["vs"][:, None]).view(-1)
    m = m * BETA1 + grad * (1 - BETA1)
    v = v * BETA2 + grad * grad * (1 - BETA2)
    c1, c2 = 1 - BETA1 ** s["step"], 1 - BETA2 ** s["step"]
    p.copy_(p * (1 - LR * s["decay"]) - (LR / c1) * m / (torch.sqrt(v) * (1 / math.sqrt(c2)) + ADAM_EPS))
    if eight:
        mr, vr = _bits(s["seed"], p.numel())
        most = m.view(-1, BLOCK).abs().amax(1)
        inv = torch.where(most > 0, M_MAX / most, torch.zeros_like(most))
        q = _rounded((m.view(-1, BLOCK) * inv[:, None]).view(-1), mr, 3, -6).clamp(-M_MAX, M_MAX)
        s["m"].copy_(q.to(torch.float8_e4m3fn))
        s["ms"].copy_(most / M_MAX)
        most = v.view(-1, BLOCK).amax(1)
        inv = torch.where(most > 0, V_MAX / most, torch.zeros_like(most))
        q = _rounded((v.view(-1, BLOCK) * inv[:, None]).view(-1), vr, 2, -14).clamp(0, V_MAX)
        q = torch.where(v > 0, q.clamp(min=2.0 ** -16), q)      # a second moment that is not zero does not become zero
        s["v"].copy_(q.to(torch.float8_e5m2))
        s["vs"].copy_(most / V_MAX)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return {k: s[k] for k in ("p", "m", "v", "ms", "vs")}


_own = {"scan": _own_scan, "norm": _own_norm, "product": _own_product, "adamw": _own_adamw}
_plain = {"scan": _plain_scan, "norm": _plain_norm, "product": _plain_product, "adamw": _plain_adamw}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind == "adamw":
        n = float(sum(_lengths(case)))
        grad = 2 if case["grad"] == "bf16" else 4
        return {"bytes": n * (8 + grad + (16 if case["bits"] == 32 else 4 + 16 / BLOCK)), "flops": 14 * n}
    es = 2 if case["dtype"] == "bf16" else 4
    if kind == "scan":
        n, ends = float(case["B"]) * case["T"] * case["C"], 4.0 * case["B"] * case["C"]
        train = case["mode"] == "train"
        return {"bytes": n * es * (6 if train else 3) + case["B"] * case["T"] + ends * ((2 if case["state"] else 1) + (2 if train else 0)),
                "flops": n * (22 if train else 8)}
    if kind == "norm":
        M, C, train, res = float(case["M"]), case["C"], case["mode"] == "train", bool(case["residual"])
        inputs, outputs = (2 if res else 1) * (2 if train else 1), (2 if train else 0) + (1 if res else 0)
        return {"bytes": M * C * (es * (inputs + outputs) + (0 if train else 1)) + 4 * C * (2 if train else 1) + (0 if train else 4 * M),
                "flops": M * C * (16 if train else 6)}
    M, N, K = float(case["M"]), case["N"], case["K"]
    return {"bytes": M * K + N * K + M * N * es + 4 * (M + N) + (4 * N if case["bias"] else 0), "flops": 2 * M * N * K}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    host = {k: v.double().cpu().numpy() for k, v in s.items() if isinstance(v, torch.Tensor)}
    return {"scan": _exact_scan, "norm": _exact_norm, "product": _exact_product, "adamw": _exact_adamw}[case["kind"]](s, host, case)


def _exact_scan(s, n, case):
    B, T, C = case["B"], case["T"], case["C"]
    if B * T * C > MOST_ELEMENTS:
        return None
    f, x, cut = n["z"][..., :C], n["z"][..., C:], n["reset"] != 0
    h, before = np.empty((B, T, C)), np.empty((B, T, C))
    gate = 1.0 / (1.0 + np.exp(-f))
    other = 1.0 / (1.0 + np.exp(f))
    state = n["h0"].copy() if s["h0"] is not None else np.zeros((B, C))
    for t in range(T):
        state = np.where(cut[:, t, None], 0.0, state)
        before[:, t] = state
        state = gate[:, t] * state + other[:, t] * x[:, t]
        h[:, t] = state
    out = {"h": h, "last": state}
    if case["mode"] == "forward":
        return out
    lam = n["dlast"].copy() if s["dlast"] is not None else np.zeros((B, C))
    dz = np.empty((B, T, 2 * C))
    for t in range(T - 1, -1, -1):
        lam = lam + n["dh"][:, t]
        dz[:, t, :C] = lam * (before[:, t] - x[:, t]) * gate[:, t] * other[:, t]
        dz[:, t, C:] = lam * other[:, t]
        lam = np.where(cut[:, t, None], 0.0, gate[:, t] * lam)
    return {**out, "dz": dz, "dh0": lam}


def _nearest(x, mantissa, lowest):
    """To the nearest number of `mantissa` bits, ties to the even one."""
    e = np.maximum(np.floor(np.log2(np.maximum(np.abs(x), 1e-300))), lowest)
    unit = np.exp2(e - mantissa)
    return np.rint(x / unit) * unit


def _exact_norm(s, n, case):
    r = n["x"] + (n["res"] if s["res"] is not None else 0.0)
    back = 1.0 / np.sqrt((r * r).mean(1, keepdims=True) + EPS)
    y = r * back * n["weight"]
    stored = r if s["res"] is not None else None
    if case["mode"] == "rows8":
        scale = np.abs(y).max(1) / M_MAX
        q = np.divide(y, scale[:, None], out=np.zeros_like(y), where=scale[:, None] > 0)
        return {"q": _nearest(q, 3, -6), "scale": scale, "r": stored}
    # the derivative of y_j by r_k is back (weight_j [j = k] - weight_j r_j r_k back^2 / C)
    inner = (n["dy"] * n["weight"] * r).sum(1, keepdims=True)
    dx = back * n["dy"] * n["weight"] - back ** 3 / case["C"] * inner * r
    if s["dr"] is not None:
        dx = dx + n["dr"]
    return {"y": y, "r": stored, "dx": dx, "dw": (n["dy"] * r * back).sum(0)}


def _exact_product(s, n, case):
    (a, sa), (w, sw) = s["a"], s["w"]
    a = (a.float().double() * sa.double()[:, None]).cpu().numpy()
    w = (w.float().double() * sw.double()[:, None]).cpu().numpy()
    y = a @ w.T
    return {"y": y + n["bias"] if s["bias"] is not None else y}


def _exact_adamw(s, n, case):
    eight, step = case["bits"] == 8, s["step"]
    blocks = lambda t: t.reshape(-1, BLOCK)  # noqa: E731
    m = (blocks(n["m"]) * n["ms"][:, None]).reshape(-1) if eight else n["m"]
    v = (blocks(n["v"]) * n["vs"][:, None]).reshape(-1) if eight else n["v"]
    m = BETA1 * m + (1 - BETA1) * n["grad"]
    v = BETA2 * v + (1 - BETA2) * n["grad"] ** 2
    update = m / (1 - BETA1 ** step) / (np.sqrt(v / (1 - BETA2 ** step)) + ADAM_EPS)
    out = {"p": n["p"] - LR * (n["decay"] * n["p"] + update), "m": m, "v": v, "ms": None, "vs": None}
    if eight:
        with np.errstate(over="ignore"):
            z = np.uint64(s["seed"]) + np.arange(1, (m.size + 1) // 2 + 1, dtype=np.uint64) * np.uint64(0x9E3779B97F4A7C15)
            z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
            z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
            z = z ^ (z >> np.uint64(31))
        words = np.ascontiguousarray(z).view("<u4")[:m.size]
        for k, t, top, word, mantissa, lowest in (("m", m, M_MAX, words & np.uint32(0xFFFF), 3, -6), ("v", v, V_MAX, words >> np.uint32(16), 2, -14)):
            scale = np.abs(blocks(t)).max(1) / top
            q = np.divide(blocks(t), scale[:, None], out=np.zeros_like(blocks(t)), where=scale[:, None] > 0).reshape(-1)
            unit = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(q), 1e-300))), lowest) - mantissa)
            up = np.floor(np.abs(q) / unit + word / 65536.0) * unit
            up = np.where((t != 0) & (k == "v"), np.maximum(up, 2.0 ** (lowest - mantissa)), up)
            out[k], out[k + "s"] = np.minimum(up, top) * np.sign(q), scale
    return out
