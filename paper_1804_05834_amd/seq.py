"""The operators of a recurrent Q-network (the second half of include/dqn.h) on torch tensors.

  scan, scan_backward       gated linear recurrence over time, per channel
  norm, norm_backward       root-mean-square norm with the residual's addition
  norm_rows, rows           the same, or no norm, with the output in 8-bit rows
  product                   8-bit rows times 8-bit weights
  AdamW                     one step over many tensors, moments in 32 or 8 bits

Argument marshalling only, as in dqn.py: the arithmetic runs in the HIP kernels of the library, on the
current stream; torch allocates outputs.  Activations are float32 or bfloat16, states, weights of the norm
and scales float32.  The last dimension of a tensor has stride 1, the others any (a half of a wider tensor is fine).
Nothing is recorded for autograd: results are detached (a call that autograd would have recorded warns), and the
*_backward calls give the gradients.
A wrong shape, type or device raises ValueError; what the library refuses raises dqn.DqnError.
"""
import ctypes as C
import functools
import struct
import warnings

import torch

from .dqn import DqnError, _current_device, _raw_stream, lib

F32, BF16 = 0, 1
_TYPES = {torch.float32: F32, torch.bfloat16: BF16}
_vp, _i64, _f32 = C.c_void_p, C.c_int64, C.c_float

# The structs of arguments of include/dqn.h, as bytes: a call reads them and keeps nothing, and packing them costs a third of
# filling a ctypes.Structure.  i: int32, q: int64, f: float, P: pointer, in C's own layout.
SCAN_ARGS = struct.Struct("iiiqPPqqqqPPqqPqqPPP")
SCAN_GRAD_ARGS = struct.Struct("iiiqPPqqqqPPqqPqqPPPqqqqPP")
NORM_ARGS = struct.Struct("iiqPPqqPfPqPqPqPP")
NORM_GRAD_ARGS = struct.Struct("iiqPPPPqqqqPPPqPP")
PRODUCT_ARGS = struct.Struct("iiiqPPqqPPPPq")


class _AdamWTensor(C.Structure):
    _fields_ = [("param", _vp), ("grad", _vp), ("copy", _vp), ("n", _i64), ("decay", _f32)]


class _AdamWBytes(C.Structure):
    _fields_ = [("elements", _i64), ("m", C.c_size_t), ("v", C.c_size_t), ("m_scale", C.c_size_t), ("v_scale", C.c_size_t),
                ("plan", C.c_size_t)]


class _AdamWBuffers(C.Structure):
    _fields_ = [("m", _vp), ("v", _vp), ("m_scale", _vp), ("v_scale", _vp), ("plan", _vp)]


def _call(rc):
    if rc:
        raise DqnError(rc, (lib().dqn_last_error(None) or b"").decode())


def _refuse(t, name, dtype, shape, device, why):
    """Says what is wrong with a tensor that a look at it has found wanting."""
    if t.dtype is not dtype or t.shape != shape:
        why = "%s of shape %s expected, got %s of shape %s" % (dtype, tuple(shape), t.dtype, tuple(t.shape))
    elif t.get_device() != device:
        why = "not on the current GPU"
    raise ValueError("%s: %s" % (name, why))


def _rows(t, name, dtype, shape, device):
    """(address, strides) of a tensor whose last dimension lies in one piece."""
    st = t.stride()
    if t.dtype is dtype and t.shape == shape and t.get_device() == device and (st[-1] == 1 or shape[-1] <= 1):
        return t.data_ptr(), st
    _refuse(t, name, dtype, shape, device, "the last dimension must have stride 1")


def _flat(t, name, dtype, shape, device):
    """The address of a tensor that must lie in one piece."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    _refuse(t, name, dtype, shape, device, "must be contiguous")


def _kind(t, name):
    k = _TYPES.get(t.dtype)
    if k is None:
        raise ValueError("%s: float32 or bfloat16 expected, got %s" % (name, t.dtype))
    return k


def _detached(call, backward):
    """An input requires a gradient: says that the result will not, unless nobody expects it to."""
    if torch.is_grad_enabled():
        warnings.warn("%s records nothing for autograd: its results are detached from its inputs; %s, or call it under torch.no_grad()"
                      % (call, "%s gives the gradients" % backward if backward else "it has no gradient"), stacklevel=3)


def _scratch(n, device):
    """(a workspace of n bytes or None, its address or 0)"""
    if not n:
        return None, 0
    t = torch.empty(n, dtype=torch.uint8, device=device)
    return t, t.data_ptr()


def _like(t):
    """(an output of t's shape and type, its address, its strides): in t's order of dimensions, but for rows, which stay in one piece
    (where t's rows lie on top of each other, a signal's windows say, its order may have them in columns)."""
    o = torch.empty_like(t)
    st = o.stride()
    if st[-1] != 1:
        o = torch.empty(t.shape, dtype=t.dtype, device=t.device)
        st = o.stride()
    return o, o.data_ptr(), st


# ------------------------------------------------------------------ gated linear recurrence
@functools.lru_cache(maxsize=256)
def _scan_sizes(kind, B, T, Ch):
    carry, work = C.c_size_t(), C.c_size_t()
    _call(lib().dqn_scan_sizes(kind, B, T, Ch, C.byref(carry), C.byref(work)))
    return carry.value, work.value


def _reset(reset, B, T, device):
    """(address, stride of a sequence, stride of a step)"""
    if reset is None:
        return 0, 0, 0
    if reset.dtype not in (torch.uint8, torch.bool) or reset.shape != (B, T) or reset.get_device() != device:
        raise ValueError("reset: uint8 or bool of shape (%d, %d) on the current GPU expected" % (B, T))
    return (reset.data_ptr(), *reset.stride())


def scan(f, x, h0=None, reset=None, save=False, out=None, last=None):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t with a = sigmoid(f), the state zero before a step whose reset flag is set.

    f, x: [B][T][C]; h0: [B][C] float32 or None (zeros); reset: [B][T] uint8 / bool or None.  out: a tensor for h;
    last: one for the final state, which may be h0 itself.  -> (h, final state [B][C] float32), and with save=True a
    third value that scan_backward needs."""
    if f.requires_grad or x.requires_grad or (h0 is not None and h0.requires_grad):
        _detached("scan", "scan_backward")
    kind, dt, shape, dev = _kind(f, "f"), f.dtype, f.shape, _current_device()
    if len(shape) != 3:
        raise ValueError("f: [B][T][C] expected")
    B, T, Ch = shape
    fp, fs = _rows(f, "f", dt, shape, dev)
    xp, xs = _rows(x, "x", dt, shape, dev)
    carry_n, work_n = _scan_sizes(kind, B, T, Ch)
    if out is None:
        h, hp, hs = _like(f)
    else:
        h = out
        hp, hs = _rows(h, "out", dt, shape, dev)
    if last is None:
        last = torch.empty_strided((B, Ch), (Ch, 1), dtype=torch.float32, device=f.device)
        lp = last.data_ptr()
    else:
        lp = _flat(last, "last", torch.float32, (B, Ch), dev)
    carry = torch.empty(carry_n // 4, dtype=torch.float32, device=f.device) if save else None
    work, wp = _scratch(work_n, f.device)
    rp, rb, rt = _reset(reset, B, T, dev)
    args = SCAN_ARGS.pack(kind, B, Ch, T, fp, xp, fs[0], fs[1], xs[0], xs[1],
                          0 if h0 is None else _flat(h0, "h0", torch.float32, (B, Ch), dev), rp, rb, rt, hp, hs[0], hs[1],
                          lp, carry.data_ptr() if save else 0, wp)
    _call(lib().dqn_scan_forward(args, _raw_stream(dev)))
    return (h, last, carry) if save else (h, last)


def scan_backward(dh, f, x, carry, reset=None, dlast=None, out=None):
    """Gradients of scan: dh [B][T][C] of h, dlast [B][C] float32 of the final state (or None), f, x, reset as they were,
    carry from scan(save=True).  out: (df, dx) to write into.  -> (df, dx, dh0 [B][C] float32)"""
    kind, dt, shape, dev = _kind(f, "f"), f.dtype, f.shape, _current_device()
    if len(shape) != 3:
        raise ValueError("f: [B][T][C] expected")
    B, T, Ch = shape
    fp, fs = _rows(f, "f", dt, shape, dev)
    xp, xs = _rows(x, "x", dt, shape, dev)
    gp, gs = _rows(dh, "dh", dt, shape, dev)
    carry_n, work_n = _scan_sizes(kind, B, T, Ch)
    if out is None:
        (df, dfp, dfs), (dx, dxp, dxs) = _like(f), _like(x)
    else:
        df, dx = out
        dfp, dfs = _rows(df, "df", dt, shape, dev)
        dxp, dxs = _rows(dx, "dx", dt, shape, dev)
    dh0 = torch.empty_strided((B, Ch), (Ch, 1), dtype=torch.float32, device=f.device)
    work, wp = _scratch(work_n, f.device)
    rp, rb, rt = _reset(reset, B, T, dev)
    args = SCAN_GRAD_ARGS.pack(kind, B, Ch, T, fp, xp, fs[0], fs[1], xs[0], xs[1], _flat(carry, "carry", torch.float32, (carry_n // 4,), dev),
                               rp, rb, rt, gp, gs[0], gs[1], 0 if dlast is None else _flat(dlast, "dlast", torch.float32, (B, Ch), dev),
                               dfp, dxp, dfs[0], dfs[1], dxs[0], dxs[1], dh0.data_ptr(), wp)
    _call(lib().dqn_scan_backward(args, _raw_stream(dev)))
    return df, dx, dh0


# ------------------------------------------------------------------ norm
def _matrix(t, name):
    k, shape = _kind(t, name), t.shape
    if len(shape) != 2:
        raise ValueError("%s: [M][C] expected" % name)
    return k, shape


def _rows8(M, K, device):
    """8-bit rows as the library lays them out, their stride a multiple of 16: (the rows, that stride)"""
    st = (K + 15) & -16
    q = torch.empty_strided((M, st), (st, 1), dtype=torch.float8_e4m3fn, device=device)
    return (q if st == K else q[:, :K]), st


def _residual(x, residual, shape, dev):
    """(address, stride, r to write, its address and stride); nothing of it without a residual"""
    if residual is None:
        return 0, 0, x, 0, 0
    p, st = _rows(residual, "residual", x.dtype, shape, dev)
    r, rp, rs = _like(x)
    return p, st[0], r, rp, rs[0]


def norm(x, weight, residual=None, eps=1e-6):
    """Per row of x [M][C]: r = x + residual, y = weight r / sqrt(mean r^2 + eps).  -> (y, r, what norm_backward needs);
    without a residual r is x."""
    if x.requires_grad or weight.requires_grad or (residual is not None and residual.requires_grad):
        _detached("norm", "norm_backward")
    (kind, shape), dev = _matrix(x, "x"), _current_device()
    M, Ch = shape
    xp, xs = _rows(x, "x", x.dtype, shape, dev)
    sp, ss, r, rp, rs = _residual(x, residual, shape, dev)
    y, yp, ys = _like(x)
    rstd = torch.empty(M, dtype=torch.float32, device=x.device)
    args = NORM_ARGS.pack(kind, Ch, M, xp, sp, xs[0], ss, _flat(weight, "weight", torch.float32, (Ch,), dev), eps, rp, rs,
                          yp, ys[0], 0, 0, 0, rstd.data_ptr())
    _call(lib().dqn_norm_forward(args, _raw_stream(dev)))
    # in bf16 the backward pass forms the sum again from its two terms, since r is rounded
    return y, r, (rstd, x, residual) if kind == BF16 else (rstd, r, None)


def norm_rows(x, weight, residual=None, eps=1e-6):
    """The same with y in 8 bits: -> (q [M][C] e4m3, scale [M], r) with y ~ q scale[:, None]."""
    if x.requires_grad or weight.requires_grad or (residual is not None and residual.requires_grad):
        _detached("norm_rows", None)
    (kind, shape), dev = _matrix(x, "x"), _current_device()
    M, Ch = shape
    xp, xs = _rows(x, "x", x.dtype, shape, dev)
    sp, ss, r, rp, rs = _residual(x, residual, shape, dev)
    q, qs = _rows8(M, Ch, x.device)
    scale = torch.empty(M, dtype=torch.float32, device=x.device)
    args = NORM_ARGS.pack(kind, Ch, M, xp, sp, xs[0], ss, _flat(weight, "weight", torch.float32, (Ch,), dev), eps, rp, rs,
                          0, 0, q.data_ptr(), qs, scale.data_ptr(), 0)
    _call(lib().dqn_norm_forward(args, _raw_stream(dev)))
    return q, scale, r


@functools.lru_cache(maxsize=256)
def _norm_sizes(M, Ch):
    work = C.c_size_t()
    _call(lib().dqn_norm_sizes(M, Ch, C.byref(work)))
    return work.value


def norm_backward(dy, r, saved, weight, dr=None):
    """dy of y and dr of r (or None), r and saved from norm() -> (gradient of x and of the residual alike [M][C], of the
    weight [C])."""
    (kind, shape), dev = _matrix(r, "r"), _current_device()
    M, Ch = shape
    dt = r.dtype
    rstd, x, residual = saved
    gp, gs = _rows(dy, "dy", dt, shape, dev)
    xp, xs = _rows(x, "x", dt, shape, dev)
    sp, ss = (0, (0,)) if residual is None else _rows(residual, "residual", dt, shape, dev)
    rp, rs = (0, (0,)) if dr is None else _rows(dr, "dr", dt, shape, dev)
    dx, dxp, dxs = _like(r)
    dw = torch.empty(Ch, dtype=torch.float32, device=r.device)
    work, wp = _scratch(_norm_sizes(M, Ch), r.device)
    args = NORM_GRAD_ARGS.pack(kind, Ch, M, gp, xp, sp, rp, gs[0], xs[0], ss[0], rs[0], _flat(weight, "weight", torch.float32, (Ch,), dev),
                               _flat(rstd, "rstd", torch.float32, (M,), dev), dxp, dxs[0], dw.data_ptr(), wp)
    _call(lib().dqn_norm_backward(args, _raw_stream(dev)))
    return dx, dw


# ------------------------------------------------------------------ 8-bit rows and their product
def rows(x):
    """x [M][K] in 8 bits: -> (q [M][K] e4m3, scale [M]) with x ~ q scale[:, None]."""
    if x.requires_grad:
        _detached("rows", None)
    (kind, shape), dev = _matrix(x, "x"), _current_device()
    M, K = shape
    xp, xs = _rows(x, "x", x.dtype, shape, dev)
    q, qs = _rows8(M, K, x.device)
    scale = torch.empty(M, dtype=torch.float32, device=x.device)
    _call(lib().dqn_rows_quantize(kind, M, K, xp, xs[0], q.data_ptr(), qs, scale.data_ptr(), _raw_stream(dev)))
    return q, scale


def product(a, w, bias=None, dtype=torch.bfloat16, out=None):
    """a = (q [M][K], scale [M]) and w = (q [N][K], scale [N]) as rows() and norm_rows() give them, bias [N] float32 or None
    -> y [M][N] of `dtype`.  For float32 its sums are fp32; for bfloat16 a sum is off by up to 2^-9 of the largest of every 128
    products, well below what their rounding to 8 bits did to them."""
    if bias is not None and bias.requires_grad:
        _detached("product", None)
    (qa, sa), (qw, sw), dev = a, w, _current_device()
    kind, shape, N = _TYPES.get(dtype), qa.shape, sw.shape[0] if sw.shape else 0
    if kind is None or len(shape) != 2:
        raise ValueError("dtype: float32 or bfloat16 expected; rows: [M][K] and [N][K]")
    M, K = shape
    ap, as_ = _rows(qa, "a", torch.float8_e4m3fn, (M, K), dev)
    wp, ws = _rows(qw, "w", torch.float8_e4m3fn, (N, K), dev)
    if out is None:
        y = torch.empty_strided((M, N), (N, 1), dtype=dtype, device=qa.device)
        yp, ys = y.data_ptr(), N
    else:
        y = out
        yp, (ys, _) = _rows(y, "out", dtype, (M, N), dev)
    args = PRODUCT_ARGS.pack(kind, N, K, M, ap, wp, as_[0], ws[0], _flat(sa, "a's scale", torch.float32, (M,), dev),
                             _flat(sw, "w's scale", torch.float32, (N,), dev), 0 if bias is None else _flat(bias, "bias", torch.float32, (N,), dev),
                             yp, ys)
    _call(lib().dqn_rows_product(args, _raw_stream(dev)))
    return y


# ------------------------------------------------------------------ AdamW
class AdamW:
    """AdamW over `params` (contiguous float32 tensors, updated in place) with gradients in the buffers `grads`
    (float32 or bfloat16, one type for all), which the program fills before each step().  weight_decay: one number
    or one per tensor.  bits: 32, or 8 for moments in e4m3 / e5m2.  copies: bfloat16 tensors that receive the new
    parameters, or None.  state: (m, v, m_scale, v_scale) of an earlier optimizer of the same tensors; they become
    this one's.  Moments lie in one buffer each, tensor after tensor, every tensor at a multiple of 256 elements."""

    def __init__(self, params, grads, bits=32, lr=2.5e-4, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, copies=None, state=None):
        n = len(params)
        decays = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
        copies = list(copies) if copies is not None else [None] * n
        if not n or len(grads) != n or len(decays) != n or len(copies) != n:
            raise ValueError("one gradient, weight decay and copy per parameter expected")
        kind, gt, dev, device = _kind(grads[0], "grads"), grads[0].dtype, _current_device(), params[0].device
        table = (_AdamWTensor * n)()
        for i, (p, g, d, c) in enumerate(zip(params, grads, decays, copies)):
            table[i] = _AdamWTensor(_flat(p, "params", torch.float32, p.shape, dev), _flat(g, "grads", gt, p.shape, dev),
                                    None if c is None else _flat(c, "copies", torch.bfloat16, p.shape, dev), p.numel(), d)
        self._keep = (list(params), list(grads), copies)     # the table holds their addresses
        sz = _AdamWBytes()
        _call(lib().dqn_adamw_sizes(table, n, bits, C.byref(sz)))
        P, eight = sz.elements, bits == 8
        mt, vt = (torch.float8_e4m3fn, torch.float8_e5m2) if eight else (torch.float32, torch.float32)
        if state is None:
            state = (torch.zeros(P, device=device).to(mt), torch.zeros(P, device=device).to(vt),
                     torch.zeros(P // 256, device=device) if eight else None, torch.zeros(P // 256, device=device) if eight else None)
        self.m, self.v, self.m_scale, self.v_scale = state
        b = _AdamWBuffers(_flat(self.m, "m", mt, (P,), dev), _flat(self.v, "v", vt, (P,), dev),
                          _flat(self.m_scale, "m_scale", torch.float32, (P // 256,), dev) if eight else None,
                          _flat(self.v_scale, "v_scale", torch.float32, (P // 256,), dev) if eight else None)
        self._plan = torch.empty(sz.plan, dtype=torch.uint8, device=device)
        b.plan = self._plan.data_ptr()
        self.lr, self.betas, self.eps, self.bits = lr, betas, eps, bits
        h = C.c_void_p()
        stream = _raw_stream(dev)
        _call(lib().dqn_adamw_init(C.byref(h), table, n, bits, kind, C.byref(b), stream))
        self._h, self._device, self._stream = h, dev, stream

    def step(self, step, seed=None, lr=None):
        """Step number `step` (from 1).  seed: of the random rounding of 8-bit moments, another one for each step (None: the
        step's number).  A step recorded into a graph repeats its number, rate and seed with every replay."""
        dev = _current_device()
        if dev != self._device:
            raise ValueError("step: the optimizer's tensors are not on the current GPU")
        stream = _raw_stream(dev)
        if stream != self._stream:      # what the optimizer holds must outlast this step, also if it is dropped before
            for t in (self._plan, self.m, self.v, self.m_scale, self.v_scale):
                if t is not None:
                    t.record_stream(torch.cuda.current_stream())
        _call(lib().dqn_adamw_step(self._h, self.lr if lr is None else lr, self.betas[0], self.betas[1], self.eps, step,
                                   (step if seed is None else seed) & 0xFFFFFFFFFFFFFFFF, stream))

    def close(self):
        if getattr(self, "_h", None):
            lib().dqn_adamw_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
