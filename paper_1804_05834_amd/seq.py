"""The operators of a recurrent Q-network (the second half of include/dqn.h) on torch tensors.

  scan, scan_backward       gated linear recurrence over time, per channel
  norm, norm_backward       root-mean-square norm with the residual's addition
  norm_rows, rows           the same, or no norm, with the output in 8-bit rows
  product                   8-bit rows times 8-bit weights
  AdamW                     one step over many tensors, moments in 32 or 8 bits

Argument marshalling only, as in dqn.py: the arithmetic runs in the HIP kernels of the library, on the
current stream; torch allocates outputs.  Activations are float32 or bfloat16, states, weights of the norm
and scales float32.  The last dimension of a tensor has stride 1, the others any (a half of a wider tensor is fine).
A wrong shape, type or device raises ValueError; what the library refuses raises dqn.DqnError.
"""
import ctypes as C

import torch

from .dqn import DqnError, _current_device, _raw_stream, lib

F32, BF16 = 0, 1
_TYPES = {torch.float32: F32, torch.bfloat16: BF16}
_vp, _i32, _i64, _f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float


class _ScanArgs(C.Structure):
    _fields_ = [("dtype", _i32), ("B", _i32), ("C", _i32), ("T", _i64), ("f", _vp), ("x", _vp), ("f_bs", _i64), ("f_ts", _i64),
                ("x_bs", _i64), ("x_ts", _i64), ("h0", _vp), ("reset", _vp), ("reset_bs", _i64), ("reset_ts", _i64),
                ("h", _vp), ("h_bs", _i64), ("h_ts", _i64), ("h_last", _vp), ("carry", _vp), ("workspace", _vp)]


class _ScanGradArgs(C.Structure):
    _fields_ = [("dtype", _i32), ("B", _i32), ("C", _i32), ("T", _i64), ("f", _vp), ("x", _vp), ("f_bs", _i64), ("f_ts", _i64),
                ("x_bs", _i64), ("x_ts", _i64), ("carry", _vp), ("reset", _vp), ("reset_bs", _i64), ("reset_ts", _i64),
                ("dh", _vp), ("dh_bs", _i64), ("dh_ts", _i64), ("dlast", _vp), ("df", _vp), ("dx", _vp),
                ("df_bs", _i64), ("df_ts", _i64), ("dx_bs", _i64), ("dx_ts", _i64), ("dh0", _vp), ("workspace", _vp)]


class _NormArgs(C.Structure):
    _fields_ = [("dtype", _i32), ("C", _i32), ("M", _i64), ("x", _vp), ("residual", _vp), ("x_rs", _i64), ("residual_rs", _i64),
                ("weight", _vp), ("eps", _f32), ("r", _vp), ("r_rs", _i64), ("y", _vp), ("y_rs", _i64), ("q", _vp), ("q_rs", _i64),
                ("scale", _vp), ("rstd", _vp)]


class _NormGradArgs(C.Structure):
    _fields_ = [("dtype", _i32), ("C", _i32), ("M", _i64), ("dy", _vp), ("r", _vp), ("dr", _vp), ("dy_rs", _i64), ("r_rs", _i64),
                ("dr_rs", _i64), ("weight", _vp), ("rstd", _vp), ("dx", _vp), ("dx_rs", _i64), ("dw", _vp), ("workspace", _vp)]


class _ProductArgs(C.Structure):
    _fields_ = [("dtype", _i32), ("N", _i32), ("K", _i32), ("M", _i64), ("a", _vp), ("w", _vp), ("a_rs", _i64), ("w_rs", _i64),
                ("a_scale", _vp), ("w_scale", _vp), ("bias", _vp), ("y", _vp), ("y_rs", _i64)]


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


def _need(t, name, dtype, shape):
    """t's address, after a look at what it is."""
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError("%s: %s of shape %s expected, got %s of shape %s" % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    if t.get_device() != _current_device():
        raise ValueError("%s: not on the current GPU" % name)
    if t.ndim and t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError("%s: the last dimension must have stride 1" % name)
    return t.data_ptr()


def _flat(t, name, dtype, shape):
    """The same for a tensor that must lie in one piece, or None."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("%s: must be contiguous" % name)
    return _need(t, name, dtype, shape)


def _dtype(t, name):
    if t.dtype not in _TYPES:
        raise ValueError("%s: float32 or bfloat16 expected, got %s" % (name, t.dtype))
    return t.dtype


def _stream():
    return _raw_stream(_current_device())


def _scratch(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _at(t):
    return None if t is None else t.data_ptr()


# ------------------------------------------------------------------ gated linear recurrence
def _scan_sizes(kind, B, T, Ch):
    carry, work = C.c_size_t(), C.c_size_t()
    _call(lib().dqn_scan_sizes(kind, B, T, Ch, C.byref(carry), C.byref(work)))
    return carry.value, work.value


def _reset(reset, B, T):
    """(address, stride of a sequence, stride of a step)"""
    if reset is None:
        return None, 0, 0
    if reset.dtype not in (torch.uint8, torch.bool) or reset.shape != (B, T) or reset.get_device() != _current_device():
        raise ValueError("reset: uint8 or bool of shape (%d, %d) on the current GPU expected" % (B, T))
    return reset.data_ptr(), reset.stride(0), reset.stride(1)


def scan(f, x, h0=None, reset=None, save=False, out=None, last=None):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t with a = sigmoid(f), the state zero before a step whose reset flag is set.

    f, x: [B][T][C]; h0: [B][C] float32 or None (zeros); reset: [B][T] uint8 / bool or None.  out: a tensor for h;
    last: one for the final state, which may be h0 itself.  -> (h, final state [B][C] float32), and with save=True a
    third value that scan_backward needs."""
    dt = _dtype(f, "f")
    if f.ndim != 3:
        raise ValueError("f: [B][T][C] expected")
    shape = f.shape
    B, T, Ch = shape
    kind = _TYPES[dt]
    fp, xp = _need(f, "f", dt, shape), _need(x, "x", dt, shape)
    h0p = _flat(h0, "h0", torch.float32, (B, Ch))
    rp, rb, rt = _reset(reset, B, T)
    carry_n, work_n = _scan_sizes(kind, B, T, Ch)
    h = torch.empty(shape, dtype=dt, device=f.device) if out is None else out
    hp = _need(h, "out", dt, shape)
    if last is None:
        last = torch.empty(B, Ch, dtype=torch.float32, device=f.device)
    lp = _flat(last, "last", torch.float32, (B, Ch))
    carry = torch.empty(carry_n // 4, dtype=torch.float32, device=f.device) if save else None
    work = _scratch(work_n, f.device)
    fs, xs, hs = f.stride(), x.stride(), h.stride()
    a = _ScanArgs(kind, B, Ch, T, fp, xp, fs[0], fs[1], xs[0], xs[1], h0p, rp, rb, rt, hp, hs[0], hs[1], lp, _at(carry), _at(work))
    _call(lib().dqn_scan_forward(C.byref(a), _stream()))
    return (h, last, carry) if save else (h, last)


def scan_backward(dh, f, x, carry, reset=None, dlast=None, out=None):
    """Gradients of scan: dh [B][T][C] of h, dlast [B][C] float32 of the final state (or None), f, x, reset as they were,
    carry from scan(save=True).  out: (df, dx) to write into.  -> (df, dx, dh0 [B][C] float32)"""
    dt = _dtype(f, "f")
    if f.ndim != 3:
        raise ValueError("f: [B][T][C] expected")
    shape = f.shape
    B, T, Ch = shape
    kind = _TYPES[dt]
    fp, xp, gp = _need(f, "f", dt, shape), _need(x, "x", dt, shape), _need(dh, "dh", dt, shape)
    rp, rb, rt = _reset(reset, B, T)
    carry_n, work_n = _scan_sizes(kind, B, T, Ch)
    cp = _flat(carry, "carry", torch.float32, (carry_n // 4,))
    dlp = _flat(dlast, "dlast", torch.float32, (B, Ch))
    df, dx = (torch.empty(shape, dtype=dt, device=f.device), torch.empty(shape, dtype=dt, device=f.device)) if out is None else out
    dfp, dxp = _need(df, "df", dt, shape), _need(dx, "dx", dt, shape)
    dh0 = torch.empty(B, Ch, dtype=torch.float32, device=f.device)
    work = _scratch(work_n, f.device)
    fs, xs, gs, ds, es = f.stride(), x.stride(), dh.stride(), df.stride(), dx.stride()
    a = _ScanGradArgs(kind, B, Ch, T, fp, xp, fs[0], fs[1], xs[0], xs[1], cp, rp, rb, rt, gp, gs[0], gs[1], dlp, dfp, dxp,
                      ds[0], ds[1], es[0], es[1], dh0.data_ptr(), _at(work))
    _call(lib().dqn_scan_backward(C.byref(a), _stream()))
    return df, dx, dh0


# ------------------------------------------------------------------ norm
def _rows_of(x):
    if x.ndim != 2:
        raise ValueError("x: [M][C] expected")
    return _dtype(x, "x"), x.shape


def _new_rows8(M, K, device):
    """8-bit rows as the library lays them out: a stride that is a multiple of 16."""
    return torch.empty(M, (K + 15) // 16 * 16, dtype=torch.float8_e4m3fn, device=device)[:, :K]


def _norm(x, weight, residual, eps, eight):
    dt, shape = _rows_of(x)
    M, Ch = shape
    xp, wp = _need(x, "x", dt, shape), _flat(weight, "weight", torch.float32, (Ch,))
    r = y = q = scale = rstd = rp = None
    if residual is not None:
        rp = _need(residual, "residual", dt, shape)
        r = torch.empty(shape, dtype=dt, device=x.device)
    if eight:
        q, scale = _new_rows8(M, Ch, x.device), torch.empty(M, dtype=torch.float32, device=x.device)
    else:
        y, rstd = torch.empty(shape, dtype=dt, device=x.device), torch.empty(M, dtype=torch.float32, device=x.device)
    a = _NormArgs(_TYPES[dt], Ch, M, xp, rp, x.stride(0), residual.stride(0) if residual is not None else 0, wp, eps,
                  _at(r), Ch, _at(y), Ch, _at(q), q.stride(0) if eight else 0, _at(scale), _at(rstd))
    _call(lib().dqn_norm_forward(C.byref(a), _stream()))
    r = x if r is None else r
    return (q, scale, r) if eight else (y, r, rstd)


def norm(x, weight, residual=None, eps=1e-6):
    """Per row of x [M][C]: r = x + residual, y = weight r / sqrt(mean r^2 + eps).  -> (y, r, 1 / sqrt(...) [M]);
    without a residual r is x."""
    return _norm(x, weight, residual, eps, False)


def norm_rows(x, weight, residual=None, eps=1e-6):
    """The same with y in 8 bits: -> (q [M][C] e4m3, scale [M], r) with y ~ q scale[:, None]."""
    return _norm(x, weight, residual, eps, True)


def norm_backward(dy, r, rstd, weight, dr=None):
    """dy of y and dr of r (or None) -> (gradient of x and of the residual alike [M][C], of the weight [C])."""
    dt, shape = _rows_of(r)
    M, Ch = shape
    work_n = C.c_size_t()
    _call(lib().dqn_norm_sizes(M, Ch, C.byref(work_n)))
    dx, dw = torch.empty(shape, dtype=dt, device=r.device), torch.empty(Ch, dtype=torch.float32, device=r.device)
    work = _scratch(work_n.value, r.device)
    a = _NormGradArgs(_TYPES[dt], Ch, M, _need(dy, "dy", dt, shape), _need(r, "r", dt, shape),
                      None if dr is None else _need(dr, "dr", dt, shape), dy.stride(0), r.stride(0), 0 if dr is None else dr.stride(0),
                      _flat(weight, "weight", torch.float32, (Ch,)), _flat(rstd, "rstd", torch.float32, (M,)), dx.data_ptr(), Ch,
                      dw.data_ptr(), _at(work))
    _call(lib().dqn_norm_backward(C.byref(a), _stream()))
    return dx, dw


# ------------------------------------------------------------------ 8-bit rows and their product
def rows(x):
    """x [M][K] in 8 bits: -> (q [M][K] e4m3, scale [M]) with x ~ q scale[:, None]."""
    dt, (M, K) = _rows_of(x)
    xp = _need(x, "x", dt, (M, K))
    q, scale = _new_rows8(M, K, x.device), torch.empty(M, dtype=torch.float32, device=x.device)
    _call(lib().dqn_rows_quantize(_TYPES[dt], M, K, xp, x.stride(0), q.data_ptr(), q.stride(0), scale.data_ptr(), _stream()))
    return q, scale


def product(a, w, bias=None, dtype=torch.bfloat16, out=None):
    """a = (q [M][K], scale [M]) and w = (q [N][K], scale [N]) as rows() and norm_rows() give them, bias [N] float32 or None
    -> y [M][N] of `dtype`."""
    (qa, sa), (qw, sw) = a, w
    M, K = qa.shape
    N = qw.shape[0]
    if dtype not in _TYPES:
        raise ValueError("dtype: float32 or bfloat16 expected")
    y = torch.empty(M, N, dtype=dtype, device=qa.device) if out is None else out
    args = _ProductArgs(_TYPES[dtype], N, K, M, _need(qa, "a", torch.float8_e4m3fn, (M, K)), _need(qw, "w", torch.float8_e4m3fn, (N, K)),
                        qa.stride(0), qw.stride(0), _flat(sa, "a's scale", torch.float32, (M,)), _flat(sw, "w's scale", torch.float32, (N,)),
                        _flat(bias, "bias", torch.float32, (N,)), _need(y, "out", dtype, (M, N)), y.stride(0))
    _call(lib().dqn_rows_product(C.byref(args), _stream()))
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
        gt = _dtype(grads[0], "grads")
        table = (_AdamWTensor * n)()
        for i, (p, g, d, c) in enumerate(zip(params, grads, decays, copies)):
            table[i] = _AdamWTensor(_flat(p, "params", torch.float32, p.shape), _flat(g, "grads", gt, p.shape),
                                    _flat(c, "copies", torch.bfloat16, p.shape), p.numel(), d)
        self._keep = (list(params), list(grads), copies)     # the table holds their addresses
        dev = params[0].device
        sz = _AdamWBytes()
        _call(lib().dqn_adamw_sizes(table, n, bits, C.byref(sz)))
        P, eight = sz.elements, bits == 8
        mt, vt = (torch.float8_e4m3fn, torch.float8_e5m2) if eight else (torch.float32, torch.float32)
        if state is None:
            state = (torch.zeros(P, device=dev).to(mt), torch.zeros(P, device=dev).to(vt),
                     torch.zeros(P // 256, device=dev) if eight else None, torch.zeros(P // 256, device=dev) if eight else None)
        self.m, self.v, self.m_scale, self.v_scale = state
        b = _AdamWBuffers(_flat(self.m, "m", mt, (P,)), _flat(self.v, "v", vt, (P,)),
                          _flat(self.m_scale, "m_scale", torch.float32, (P // 256,)) if eight else None,
                          _flat(self.v_scale, "v_scale", torch.float32, (P // 256,)) if eight else None)
        self._plan = torch.empty(sz.plan, dtype=torch.uint8, device=dev)
        b.plan = self._plan.data_ptr()
        self.lr, self.betas, self.eps, self.bits = lr, betas, eps, bits
        h = C.c_void_p()
        _call(lib().dqn_adamw_init(C.byref(h), table, n, bits, _TYPES[gt], C.byref(b), _stream()))
        self._h = h

    def step(self, step, seed=0, lr=None):
        """Step number `step` (from 1).  seed: of the random rounding of 8-bit moments, another one for each step."""
        _call(lib().dqn_adamw_step(self._h, self.lr if lr is None else lr, self.betas[0], self.betas[1], self.eps, step,
                                   seed & 0xFFFFFFFFFFFFFFFF, _stream()))

    def close(self):
        if getattr(self, "_h", None):
            lib().dqn_adamw_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
