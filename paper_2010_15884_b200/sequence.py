"""Sequence operators on CUDA tensors: causal convolution with carried state, selective state space scan, group norm.

A thin layer over ``include/sysconv_sequence.h``: arguments are checked and marshalled here, every step of the
computation runs in ``libsysconv.so``; there is no CPU fallback.  Channels are last and contiguous everywhere (a token is
a row of channels), any batch and time strides are taken as they are.  Tokens are float32, bfloat16 or float16; sums,
states and statistics are float32.

Sequences are dense, ``(batch, length, channels)``, or packed, ``(tokens, channels)`` with ``offsets`` (an int32 or int64
CUDA tensor of sequences + 1 ascending numbers, the first 0 and the last ``tokens``); a packed sequence may be empty.
``longest`` tells the longest packed sequence where the caller knows it (it sizes the launch; without it ``tokens``
is assumed).

Every call takes ``stream``: results, workspaces and launches then belong to that stream (default: the current one).
Results of tensors with no tokens are empty (or zero) without a launch.
"""
import contextlib
import ctypes
import struct
from collections import namedtuple

import torch

from . import binding
from .binding import SysconvError

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_ACTS = {None: 0, "none": 0, "silu": 1}

_CAUSAL = struct.Struct("qqqPq" "qqqqq" + "Pqq" * 3 + "PPP" "P" "P" "PPP" "Pq")
_CAUSAL_STEP = struct.Struct("qqqqqqq" "Pq" "Pq" "Pq" "PPP")
_SCAN = struct.Struct("qqqPq" "qqqqq" + "Pqq" * 6 + "PPPP" "P" "P" + "Pqq" * 6 + "PPP" "P" "P" "Pq")
_SCAN_STEP = struct.Struct("qqqqqqq" + "Pq" * 6 + "PPP" "Pq" "P")
_NORM = struct.Struct("qqqqqq" "d" + "Pqq" * 4 + "PP" "PPPP" "Pq")

_NONE3 = (0, 0, 0)
_lib = None

ScanGrads = namedtuple("ScanGrads", "du ddelta dA dB dC dD dz ddelta_bias dstate")


def _library():
    global _lib
    if _lib is None:
        lib = binding.load_library()
        for name in ("sysconv1d_causal", "sysconv1d_causal_backward", "sysconv1d_causal_step", "sysscan",
                     "sysscan_backward", "sysscan_step", "sysgroupnorm", "sysgroupnorm_backward"):
            f = getattr(lib, name)
            f.restype, f.argtypes = ctypes.c_int, [ctypes.c_char_p, ctypes.c_void_p]
        for name in ("sysconv1d_causal_backward_workspace_bytes", "sysscan_saved_blocks", "sysscan_workspace_bytes",
                     "sysscan_backward_workspace_bytes", "sysgroupnorm_workspace_bytes",
                     "sysgroupnorm_backward_workspace_bytes"):
            f = getattr(lib, name)
            f.restype, f.argtypes = ctypes.c_longlong, [ctypes.c_char_p]
        _lib = lib
    return _lib


def _check(status, where):
    if status != 0:
        raise SysconvError(status, where)


def _bytes(size, where):
    if size < 0:
        raise SysconvError(1, where)
    return size


class _on:
    """The device of x and the stream of the call made current; costs nothing where they already are."""

    __slots__ = ("stack", "stream")

    def __init__(self, x, stream, where):
        if not x.is_cuda:
            raise SysconvError(-1, "%s (not a CUDA tensor; there is no CPU path)" % where)
        self.stack = None
        if stream is not None or x.device.index != torch.cuda.current_device():
            self.stack = contextlib.ExitStack()
            self.stack.enter_context(torch.cuda.device(x.device))
            if stream is not None:
                if isinstance(stream, int):
                    stream = torch.cuda.ExternalStream(stream, device=x.device)
                self.stack.enter_context(torch.cuda.stream(stream))
        self.stream = torch._C._cuda_getCurrentRawStream(x.device.index)

    def __enter__(self):
        return self.stream

    def __exit__(self, *exc):
        if self.stack is not None:
            self.stack.close()
        return False


def _type(x):
    t = _TYPES.get(x.dtype)
    if t is None:
        raise TypeError("tokens must be float32, bfloat16 or float16, got %s" % x.dtype)
    return t


def _act(activation):
    a = _ACTS.get(activation)
    if a is None:
        raise ValueError("activation must be None or 'silu', got %r" % (activation,))
    return a


def _tok(x, name, like, channels_like=True):
    """(pointer, batch stride, time stride) of a token tensor with the type, device and leading sizes of `like`."""
    if x.dtype != like.dtype or x.device != like.device:
        raise TypeError("%s: type and device must be those of the tokens (%s on %s), got %s on %s"
                        % (name, like.dtype, like.device, x.dtype, x.device))
    shape, want = x.shape, like.shape
    if (shape != want) if channels_like else (shape[: len(want) - 1] != want[:-1]):
        raise ValueError("%s: shape %s does not go with tokens %s" % (name, tuple(shape), tuple(want)))
    s = x.stride()
    if s[-1] != 1 and shape[-1] > 1 and x.numel() > 0:
        raise ValueError("%s: channels must be contiguous" % name)
    if len(want) == 3:
        return x.data_ptr(), s[0], s[1]
    return x.data_ptr(), 0, s[0]


def _par(x, name, shape, dtype, device, optional=True):
    """Pointer of a packed parameter; 0 for None."""
    if x is None:
        if optional:
            return 0
        raise ValueError("%s is needed" % name)
    if x.dtype != dtype or x.device != device:
        raise TypeError("%s must be %s on %s, got %s on %s" % (name, dtype, device, x.dtype, x.device))
    if tuple(x.shape) != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, shape, tuple(x.shape)))
    if not x.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return x.data_ptr()


def _sequences(x, offsets, longest=None):
    """((sequences, length, total, offsets pointer, 64-bit), sequences) of a token tensor."""
    if offsets is None:
        if x.dim() != 3:
            raise ValueError("dense tokens are (batch, length, channels); packed ones need offsets")
        b, n, _ = x.shape
        return (b, n, b * n, 0, 0), b
    if x.dim() != 2:
        raise ValueError("packed tokens are (tokens, channels)")
    if offsets.dim() != 1 or offsets.shape[0] < 1 or offsets.device != x.device or not offsets.is_contiguous():
        raise ValueError("offsets: a contiguous vector of sequences + 1 numbers on the tokens' device")
    if offsets.dtype not in (torch.int32, torch.int64):
        raise TypeError("offsets must be int32 or int64, got %s" % offsets.dtype)
    total, r = x.shape[0], offsets.shape[0] - 1
    most = total if longest is None else min(int(longest), total)
    return (r, max(most, 0), total, offsets.data_ptr(), 1 if offsets.dtype == torch.int64 else 0), r


def _slots(slots, rows, device):
    if slots is None:
        return 0
    if slots.dtype != torch.int32 or slots.device != device or slots.dim() != 1 or slots.shape[0] != rows or not slots.is_contiguous():
        raise ValueError("slots: a contiguous int32 vector with one slot per row, on the tokens' device")
    return slots.data_ptr()


def _room(size, device):
    """A workspace of `size` bytes."""
    return torch.empty(size, dtype=torch.uint8, device=device) if size else None


# ---------------------------------------------------------------------------------------------- causal convolution


def _causal_params(x, weight, bias):
    if weight.dim() != 2 or weight.shape[0] != x.shape[-1]:
        raise ValueError("weight must be (channels, taps), got %s for %d channels" % (tuple(weight.shape), x.shape[-1]))
    if weight.dtype != x.dtype and weight.dtype != torch.float32:
        raise TypeError("weight must be float32 or of the tokens' type")
    d, k = weight.shape
    if k < 1:
        raise ValueError("weight has no taps")
    w = _par(weight, "weight", (d, k), weight.dtype, x.device)
    b = _par(bias, "bias", (d,), weight.dtype, x.device)
    return d, k, w, b, _TYPES[weight.dtype]


def conv1d_causal(x, weight, bias=None, activation=None, state=None, offsets=None, return_state=False, out=None, stream=None):
    """Causal convolution per channel: y[t] = act(bias + sum_k weight[:, k] * line[t + k]), line = state ++ x.

    weight (channels, taps), taps <= 8; bias (channels); both float32 or of x's type.  state (sequences, taps-1, channels) of
    x's type: the inputs before the first token (zeros without it).  Returns y, or (y, final state) with return_state.
    """
    with _on(x, stream, "conv1d_causal") as s:
        t, act = _type(x), _act(activation)
        seq, r = _sequences(x, offsets)
        d, k, w, b, wt = _causal_params(x, weight, bias)
        st = _par(state, "state", (r, k - 1, d), x.dtype, x.device)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
        final = torch.empty((r, k - 1, d), dtype=x.dtype, device=x.device) if return_state else None
        if r > 0 and d > 0:
            args = _CAUSAL.pack(*seq, d, k, t, wt, act, *_tok(x, "x", x), *_tok(y, "out", x), *_NONE3, w, b, st,
                                final.data_ptr() if final is not None else 0, 0, 0, 0, 0, 0, 0)
            _check(_library().sysconv1d_causal(args, s), "sysconv1d_causal")
        return (y, final) if return_state else y


def conv1d_causal_backward(dy, x, weight, bias=None, activation=None, state=None, offsets=None, dfinal=None, stream=None):
    """Gradients of conv1d_causal: (dx, dweight, dbias, dstate), the last two None where bias or state is None.

    dfinal: gradient with respect to the final state, if that was used.
    """
    with _on(x, stream, "conv1d_causal_backward") as s:
        t, act = _type(x), _act(activation)
        seq, r = _sequences(x, offsets)
        d, k, w, b, wt = _causal_params(x, weight, bias)
        st = _par(state, "state", (r, k - 1, d), x.dtype, x.device)
        df = _par(dfinal, "dfinal", (r, k - 1, d), x.dtype, x.device)
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        dw = torch.empty_like(weight)
        db = torch.empty_like(bias) if bias is not None else None
        ds = torch.empty_like(state) if state is not None else None
        if r == 0 or d == 0:
            return dx, dw.zero_(), db.zero_() if db is not None else None, ds
        head = (*seq, d, k, t, wt, act, *_tok(x, "x", x), *_tok(dy, "dy", x), *_tok(dx, "dx", x), w, b, st, 0, df,
                ds.data_ptr() if ds is not None else 0, dw.data_ptr(), db.data_ptr() if db is not None else 0)
        lib = _library()
        size = _bytes(lib.sysconv1d_causal_backward_workspace_bytes(_CAUSAL.pack(*head, 0, 0)), "sysconv1d_causal_backward")
        room = _room(size, x.device)
        args = _CAUSAL.pack(*head, room.data_ptr() if room is not None else 0, size)
        _check(lib.sysconv1d_causal_backward(args, s), "sysconv1d_causal_backward")
        return dx, dw, db, ds


def conv1d_causal_step(x, state, weight, bias=None, activation=None, slots=None, out=None, stream=None):
    """One token of each row: x (rows, channels); state (slots, taps-1, channels) takes it in place.  Returns y.

    slots (int32, one per row): the slot of each row; a slot outside the cache (-1, say) gives zeros and touches no
    state.  Without it row r uses slot r.  No two rows may name the same slot.
    """
    with _on(x, stream, "conv1d_causal_step") as s:
        t, act = _type(x), _act(activation)
        if x.dim() != 2:
            raise ValueError("x must be (rows, channels)")
        rows = x.shape[0]
        d, k, w, b, wt = _causal_params(x, weight, bias)
        n = _cache(state, (k - 1, d), x.dtype, x.device)
        at = _slots(slots, rows, x.device)
        if slots is None and n < rows:
            raise ValueError("state has %d slots for %d rows" % (n, rows))
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
        xp, _, xs = _tok(x, "x", x)
        yp, _, ys = _tok(y, "out", x)
        if rows > 0 and d > 0:
            args = _CAUSAL_STEP.pack(rows, n, d, k, t, wt, act, xp, xs, yp, ys, state.data_ptr(), state.stride(0), w, b, at)
            _check(_library().sysconv1d_causal_step(args, s), "sysconv1d_causal_step")
        return y


def _cache(state, shape, dtype, device):
    """Slots of a cache of states: each slot packed, any stride between them."""
    if state.dtype != dtype or state.device != device:
        raise TypeError("state must be %s on %s, got %s on %s" % (dtype, device, state.dtype, state.device))
    if state.dim() != 3 or tuple(state.shape[1:]) != shape:
        raise ValueError("state must be (slots, %d, %d), got %s" % (shape[0], shape[1], tuple(state.shape)))
    s = state.stride()
    if state.numel() > 0 and ((shape[1] > 1 and s[2] != 1) or (shape[0] > 1 and s[1] != shape[1])):
        raise ValueError("each slot of state must be contiguous")
    return state.shape[0]


# ---------------------------------------------------------------------------------------------- state space scan


def _scan_shapes(u, A, B, C):
    d = u.shape[-1]
    if A.dim() != 2 or A.shape[0] != d:
        raise ValueError("A must be (channels, states), got %s for %d channels" % (tuple(A.shape), d))
    n, lead = A.shape[1], u.dim() - 1
    if B.dim() == lead + 1:
        g = 1
    elif B.dim() == lead + 2:
        g = B.shape[lead]
    else:
        raise ValueError("B and C must be (..., states) or (..., groups, states)")
    if B.shape != C.shape or B.shape[-1] != n or B.shape[:lead] != u.shape[:-1]:
        raise ValueError("B %s and C %s do not go with tokens %s and %d states"
                         % (tuple(B.shape), tuple(C.shape), tuple(u.shape), n))
    if g < 1 or d % g != 0:
        raise ValueError("%d channels do not divide into %d groups" % (d, g))
    return d, n, g


def _bc(x, name, u, n, g):
    """B or C: like tokens, the groups' states packed within a token."""
    if x.dim() == u.dim() + 1 and g > 1 and x.stride(-2) != n:
        raise ValueError("%s: the groups of a token must be contiguous" % name)
    return _tok(x, name, u, channels_like=False)


def _scan_head(u, delta, A, B, C, D, z, delta_bias, softplus, offsets, longest):
    t = _type(u)
    seq, r = _sequences(u, offsets, longest)
    d, n, g = _scan_shapes(u, A, B, C)
    f32, dev = torch.float32, u.device
    head = (*seq, d, n, g, t, 1 if softplus else 0, *_tok(u, "u", u), *_tok(delta, "delta", u),
            *(_tok(z, "z", u) if z is not None else _NONE3), *_bc(B, "B", u, n, g), *_bc(C, "C", u, n, g))
    params = (_par(A, "A", (d, n), f32, dev, False), _par(D, "D", (d,), f32, dev),
              _par(delta_bias, "delta_bias", (d,), f32, dev))
    return head, params, r, d, n, g


def state_scan(u, delta, A, B, C, D=None, z=None, delta_bias=None, softplus=False, state=None, offsets=None, longest=None,
               return_state=False, save=False, out=None, stream=None):
    """Selective state space scan: h[t] = exp(d[t] A) h[t-1] + d[t] u[t] B[t], y[t] = (C[t].h[t] + D u[t]) * silu(z[t]).

    u, delta, z: tokens; d = delta + delta_bias, through log(1 + exp(.)) with softplus.  B, C (..., states) or
    (..., groups, states), channels in equal groups.  A (channels, states), D, delta_bias (channels), state
    (sequences, channels, states): float32.  states <= 128.
    Returns y; with return_state also the final state, with save also what state_scan_backward needs, in this order.
    """
    with _on(u, stream, "state_scan") as s:
        head, params, r, d, n, g = _scan_head(u, delta, A, B, C, D, z, delta_bias, softplus, offsets, longest)
        dev, f32 = u.device, torch.float32
        st = _par(state, "state", (r, d, n), f32, dev)
        y = torch.empty(u.shape, dtype=u.dtype, device=dev) if out is None else out
        yt = _tok(y, "out", u)
        final = torch.empty((r, d, n), dtype=f32, device=dev) if return_state else None
        lib, saved = _library(), None
        fp = final.data_ptr() if final is not None else 0
        body, rest = (*head, *yt, *params, st, fp), _NONE3 * 6 + (0,) * 5     # rest: the backward call's members
        args = _SCAN.pack(*body, 0, *rest, 0, 0)
        if save:
            blocks = lib.sysscan_saved_blocks(args) if r > 0 else 0
            saved = torch.empty((max(blocks, 0), d, n), dtype=f32, device=dev)
        if r > 0 and d > 0:
            size = _bytes(lib.sysscan_workspace_bytes(args), "sysscan")
            if size or save:
                room = _room(size, dev)
                args = _SCAN.pack(*body, saved.data_ptr() if save else 0, *rest, room.data_ptr() if size else 0, size)
            _check(lib.sysscan(args, s), "sysscan")
        if not return_state and not save:
            return y
        return (y,) + ((final,) if return_state else ()) + ((saved,) if save else ())


def state_scan_backward(dy, u, delta, A, B, C, saved, D=None, z=None, delta_bias=None, softplus=False, offsets=None,
                        longest=None, dfinal=None, state_grad=False, stream=None):
    """Gradients of state_scan from dy and `saved` (state_scan(..., save=True) on the same inputs), as ScanGrads.

    dfinal: gradient with respect to the final state, if that was used.  dz, dD, ddelta_bias are None where z, D, delta_bias
    are; dstate (the gradient with respect to the initial state) is computed on state_grad.
    """
    with _on(u, stream, "state_scan_backward") as s:
        head, params, r, d, n, g = _scan_head(u, delta, A, B, C, D, z, delta_bias, softplus, offsets, longest)
        dev, f32 = u.device, torch.float32
        df = _par(dfinal, "dfinal", (r, d, n), f32, dev)
        du = torch.empty(u.shape, dtype=u.dtype, device=dev)
        dd = torch.empty(u.shape, dtype=u.dtype, device=dev)
        dz = torch.empty(u.shape, dtype=u.dtype, device=dev) if z is not None else None
        dB = torch.empty(B.shape, dtype=B.dtype, device=dev)
        dC = torch.empty(C.shape, dtype=C.dtype, device=dev)
        dA = torch.empty((d, n), dtype=f32, device=dev)
        dD = torch.empty(d, dtype=f32, device=dev) if D is not None else None
        dbias = torch.empty(d, dtype=f32, device=dev) if delta_bias is not None else None
        dstate = torch.empty((r, d, n), dtype=f32, device=dev) if state_grad else None
        if r == 0 or d == 0:
            dA.zero_()
            for v in (dD, dbias):
                if v is not None:
                    v.zero_()
            return ScanGrads(du, dd, dA, dB, dC, dD, dz, dbias, dstate)

        def ptr(v):
            return v.data_ptr() if v is not None else 0

        lib = _library()
        probe = _SCAN.pack(*head, *_NONE3, *params, 0, 0, 0, *_NONE3 * 6, 0, 0, 0, 0, 0, 0, 0)
        blocks = lib.sysscan_saved_blocks(probe)
        _par(saved, "saved", (blocks, d, n), f32, dev, False)
        body = (*head, *_NONE3, *params, 0, 0, ptr(saved), *_tok(dy, "dy", u), *_tok(du, "du", u), *_tok(dd, "ddelta", u),
                *(_tok(dz, "dz", u) if dz is not None else _NONE3), *_bc(dB, "dB", u, n, g), *_bc(dC, "dC", u, n, g),
                ptr(dA), ptr(dD), ptr(dbias), df, ptr(dstate))
        size = _bytes(lib.sysscan_backward_workspace_bytes(_SCAN.pack(*body, 0, 0)), "sysscan_backward")
        room = _room(size, dev)
        _check(lib.sysscan_backward(_SCAN.pack(*body, ptr(room), size), s), "sysscan_backward")
        return ScanGrads(du, dd, dA, dB, dC, dD, dz, dbias, dstate)


def state_scan_step(u, delta, A, B, C, state, D=None, z=None, delta_bias=None, softplus=False, slots=None, out=None, stream=None):
    """One token of each row: u, delta, z (rows, channels), B, C (rows[, groups], states); state (slots, channels, states),
    float32, is updated in place.  Slots as in conv1d_causal_step.  Returns y."""
    with _on(u, stream, "state_scan_step") as s:
        t = _type(u)
        if u.dim() != 2:
            raise ValueError("u must be (rows, channels)")
        d, n, g = _scan_shapes(u, A, B, C)
        rows, f32, dev = u.shape[0], torch.float32, u.device
        slots_n = _cache(state, (d, n), f32, dev)
        at = _slots(slots, rows, dev)
        if slots is None and slots_n < rows:
            raise ValueError("state has %d slots for %d rows" % (slots_n, rows))
        y = torch.empty(u.shape, dtype=u.dtype, device=dev) if out is None else out
        up, _, us = _tok(u, "u", u)
        dp, _, ds = _tok(delta, "delta", u)
        zp, _, zs = _tok(z, "z", u) if z is not None else _NONE3
        bp, _, bs = _bc(B, "B", u, n, g)
        cp, _, cs = _bc(C, "C", u, n, g)
        yp, _, ys = _tok(y, "out", u)
        if rows > 0 and d > 0:
            args = _SCAN_STEP.pack(rows, slots_n, d, n, g, t, 1 if softplus else 0, up, us, dp, ds, zp, zs, bp, bs, cp, cs,
                                   yp, ys, _par(A, "A", (d, n), f32, dev, False), _par(D, "D", (d,), f32, dev),
                                   _par(delta_bias, "delta_bias", (d,), f32, dev), state.data_ptr(), state.stride(0), at)
            _check(_library().sysscan_step(args, s), "sysscan_step")
        return y


# ---------------------------------------------------------------------------------------------- group norm


def _norm_view(x, name, like=None):
    """x as (batch, space, channels): the dimensions between the first and the last must have one common stride."""
    if like is not None and (x.shape != like.shape or x.dtype != like.dtype or x.device != like.device):
        raise ValueError("%s must have the shape, type and device of x" % name)
    if x.dim() < 2:
        raise ValueError("%s must be (batch, ..., channels)" % name)
    if x.dim() == 3:
        return x
    b, c = x.shape[0], x.shape[-1]
    n = 1
    for v in x.shape[1:-1]:
        n *= v
    return x.view(b, n, c)


def _norm_head(x, groups, weight, bias, eps, activation):
    t, act = _type(x), _act(activation)
    v = _norm_view(x, "x")
    b, n, c = v.shape
    groups = int(groups)
    if groups < 1 or c % groups != 0:
        raise ValueError("%d channels do not divide into %d groups" % (c, groups))
    f32 = torch.float32
    w = _par(weight, "weight", (c,), f32, x.device)
    bb = _par(bias, "bias", (c,), f32, x.device)
    return v, (b, n, c, groups, t, act, float(eps), *_tok(v, "x", v)), w, bb


def groupnorm(x, groups, weight=None, bias=None, eps=1e-5, activation=None, return_stats=False, out=None, stream=None):
    """Group norm, channels last: x (batch, ..., channels) is normalised over everything between batch and channels and
    over the channels of each group; y = act((x - mean) * rstd * weight + bias).  weight, bias (channels), float32.
    Returns y, or (y, mean, rstd) with return_stats, which groupnorm_backward needs."""
    with _on(x, stream, "groupnorm") as s:
        v, head, w, b = _norm_head(x, groups, weight, bias, eps, activation)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
        yv = _norm_view(y, "out", x)
        mean = rstd = None
        if return_stats:
            mean = torch.empty((v.shape[0], head[3]), dtype=torch.float32, device=x.device)
            rstd = torch.empty_like(mean)
        if x.numel() > 0:
            lib = _library()
            body = (*head, *_tok(yv, "out", v), *_NONE3, *_NONE3, w, b, mean.data_ptr() if return_stats else 0,
                    rstd.data_ptr() if return_stats else 0, 0, 0)
            args = _NORM.pack(*body, 0, 0)
            size = _bytes(lib.sysgroupnorm_workspace_bytes(args), "sysgroupnorm")
            if size:
                room = _room(size, x.device)
                args = _NORM.pack(*body, room.data_ptr(), size)
            _check(lib.sysgroupnorm(args, s), "sysgroupnorm")
        return (y, mean, rstd) if return_stats else y


def groupnorm_backward(dy, x, groups, mean, rstd, weight=None, bias=None, activation=None, stream=None):
    """Gradients of groupnorm: (dx, dweight, dbias), the last two None where weight or bias is None."""
    with _on(x, stream, "groupnorm_backward") as s:
        v, head, w, b = _norm_head(x, groups, weight, bias, 0.0, activation)
        dyv = _norm_view(dy, "dy", x)
        shape = (v.shape[0], head[3])
        mp = _par(mean, "mean", shape, torch.float32, x.device, False)
        rp = _par(rstd, "rstd", shape, torch.float32, x.device, False)
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        dw = torch.empty_like(weight) if weight is not None else None
        db = torch.empty_like(bias) if bias is not None else None
        if x.numel() == 0:
            return dx, dw.zero_() if dw is not None else None, db.zero_() if db is not None else None
        lib = _library()
        body = (*head, *_NONE3, *_tok(dyv, "dy", v), *_tok(_norm_view(dx, "dx"), "dx", v), w, b, mp, rp,
                dw.data_ptr() if dw is not None else 0, db.data_ptr() if db is not None else 0)
        size = _bytes(lib.sysgroupnorm_backward_workspace_bytes(_NORM.pack(*body, 0, 0)), "sysgroupnorm_backward")
        room = _room(size, x.device)
        _check(lib.sysgroupnorm_backward(_NORM.pack(*body, room.data_ptr() if size else 0, size), s), "sysgroupnorm_backward")
        return dx, dw, db
