"""Sequence operators from their definitions, one sequence at a time, in numpy float64: causal convolution with carried
state, selective state space scan, group norm, and their gradients.

Every function also returns, for each value, the MAGNITUDE of what was summed to get it (the same formula over absolute
values): rounding errors of any summation order are bounded by a small multiple of 2^-24 times it.
"""
import numpy as np


def sigmoid(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-v))


def silu(v):
    return v * sigmoid(v)


def silu_slope(v):
    s = sigmoid(v)
    return s * (1.0 + v * (1.0 - s))


def softplus(v):
    return np.maximum(v, 0.0) + np.log1p(np.exp(-np.abs(v)))


# ------------------------------------------------------------------------------------------ causal convolution


def conv_causal(x, w, b, state, act):
    """x (L, D), w (D, K), b (D), state (K-1, D) or None -> y (L, D), final state (K-1, D), magnitude of pre (L, D)."""
    n, d = x.shape
    k = w.shape[1]
    line = np.concatenate([np.zeros((k - 1, d)) if state is None else state, x])
    pre, mag = np.zeros((n, d)), np.zeros((n, d))
    for t in range(n):
        for c in range(d):
            pre[t, c] = b[c] + np.dot(w[c], line[t:t + k, c])
            mag[t, c] = abs(b[c]) + np.dot(np.abs(w[c]), np.abs(line[t:t + k, c]))
    return silu(pre) if act else pre, line[n:], mag


def conv_causal_backward(dy, x, w, b, state, act, dfinal):
    """-> dict of dx, dw, db, dstate, each with its magnitude under the name + '_mag'."""
    n, d = x.shape
    k = w.shape[1]
    line = np.concatenate([np.zeros((k - 1, d)) if state is None else state, x])
    pre, _, mag = conv_causal(x, w, b, state, False)
    # an error e of pre moves the slope by at most 0.5 e: it counts with the magnitude of pre
    dpre = dy * silu_slope(pre) if act else dy.copy()
    size = np.abs(dy) * (1.1 + mag) if act else np.abs(dy)
    dline, dline_m = np.zeros(line.shape), np.zeros(line.shape)
    dw, dw_m = np.zeros((d, k)), np.zeros((d, k))
    for t in range(n):
        for j in range(k):
            dline[t + j] += dpre[t] * w[:, j]
            dline_m[t + j] += size[t] * np.abs(w[:, j])
            dw[:, j] += dpre[t] * line[t + j]
            dw_m[:, j] += size[t] * np.abs(line[t + j])
    if dfinal is not None:
        dline[n:] += dfinal
        dline_m[n:] += np.abs(dfinal)
    return {"dx": dline[k - 1:], "dx_mag": dline_m[k - 1:], "dstate": dline[:k - 1], "dstate_mag": dline_m[:k - 1],
            "dw": dw, "dw_mag": dw_m, "db": dpre.sum(0), "db_mag": size.sum(0)}


# ------------------------------------------------------------------------------------------ state space scan


def _per_channel(v, d):
    """(G, N) -> (D, N): channel c takes group c / (D/G)."""
    return np.repeat(v, d // v.shape[0], axis=0)


def scan(u, delta, A, B, C, D, z, bias, plus, state):
    """u, delta, z (L, D); B, C (L, G, N); A (D, N); D, bias (D) or None; state (D, N) or None.

    -> dict: y, y_mag (L, D), final, final_mag (D, N), all states h and their magnitudes hm (L, D, N), d (L, D).
    A magnitude also counts what an error of the exponent does: x exp(x) <= 1/e for negative x."""
    n, d = u.shape
    raw = delta + (0.0 if bias is None else bias)
    dl = softplus(raw) if plus else raw
    h = np.zeros(A.shape) if state is None else state.astype(np.float64)
    hm = np.abs(h)
    hs, hms = np.zeros((n,) + A.shape), np.zeros((n,) + A.shape)
    y, ym = np.zeros((n, d)), np.zeros((n, d))
    for t in range(n):
        b, c = _per_channel(B[t], d), _per_channel(C[t], d)
        a = np.exp(dl[t][:, None] * A)
        x = np.abs(dl[t][:, None] * A)
        inp = (dl[t] * u[t])[:, None] * b
        h = a * h + inp
        hm = a * (1.0 + EXP_ERR * (1.0 + x)) * hm + np.abs(inp)
        hs[t], hms[t] = h, hm
        y[t] = (h * c).sum(1)
        ym[t] = (hm * np.abs(c)).sum(1)
        if D is not None:
            y[t] += D * u[t]
            ym[t] += np.abs(D * u[t])
    out = {"core": y, "core_mag": ym, "h": hs, "hm": hms, "d": dl, "raw": raw, "final": h, "final_mag": hm}
    out["y"], out["y_mag"] = (y * silu(z), ym * np.abs(silu(z))) if z is not None else (y, ym)
    return out


# The relative error of one factor exp(d A) in fp32 is about 2^-22 of the exponential itself and 2^-22 (d and its product
# rounded) times the exponent.  Magnitudes grow by 2^-6 (1 + |exponent|) per step, so that 2^-16 of a magnitude bounds what
# these errors add up to over any number of steps.
EXP_ERR = 2.0 ** -6


def scan_backward(dout, u, delta, A, B, C, D, z, bias, plus, state, dfinal):
    """Gradients by the reverse recurrence; dict of values and '_mag' magnitudes."""
    f = scan(u, delta, A, B, C, D, z, bias, plus, state)
    n, d = u.shape
    g = B.shape[1]
    h0 = np.zeros(A.shape) if state is None else state.astype(np.float64)
    dl, hs, hms = f["d"], f["h"], f["hm"]
    sz = silu(z) if z is not None else np.ones_like(u)
    dy, dym = dout * sz, np.abs(dout * sz)
    out = {k: np.zeros_like(u) for k in ("du", "du_mag", "dd", "dd_mag")}
    dA, dAm = np.zeros(A.shape), np.zeros(A.shape)
    dB, dBm, dC, dCm = (np.zeros(B.shape) for _ in range(4))
    carry = np.zeros(A.shape) if dfinal is None else dfinal.astype(np.float64)
    cm = np.abs(carry)
    for t in range(n - 1, -1, -1):
        b, c = _per_channel(B[t], d), _per_channel(C[t], d)
        x = dl[t][:, None] * A
        a = np.exp(x)
        prev, pm = (hs[t - 1], hms[t - 1]) if t > 0 else (h0, np.abs(h0))
        dh = carry + dy[t][:, None] * c
        dhm = cm + dym[t][:, None] * np.abs(c)
        am = a * (1.0 + EXP_ERR * (1.0 + np.abs(x)))
        dC[t] = (hs[t] * dy[t][:, None]).reshape(g, d // g, -1).sum(1)
        dCm[t] = (hms[t] * dym[t][:, None]).reshape(g, d // g, -1).sum(1)
        du_in = (dl[t] * u[t])[:, None]
        dB[t] = (dh * du_in).reshape(g, d // g, -1).sum(1)
        dBm[t] = (dhm * np.abs(du_in)).reshape(g, d // g, -1).sum(1)
        r1, r1m = (dh * b).sum(1), (dhm * np.abs(b)).sum(1)
        carry, cm = dh * a, dhm * am
        p, q = carry * prev, cm * pm
        r2, r2m = (p * A).sum(1), (q * np.abs(A)).sum(1)
        dA += p * dl[t][:, None]
        dAm += q * np.abs(dl[t][:, None])
        out["du"][t], out["du_mag"][t] = dl[t] * r1, np.abs(dl[t]) * r1m
        out["dd"][t], out["dd_mag"][t] = r2 + u[t] * r1, r2m + np.abs(u[t]) * r1m
        if D is not None:
            out["du"][t] += dy[t] * D
            out["du_mag"][t] += dym[t] * np.abs(D)
    if plus:
        out["dd"], out["dd_mag"] = out["dd"] * sigmoid(f["raw"]), out["dd_mag"] * sigmoid(f["raw"])
    out.update(dA=dA, dA_mag=dAm, dB=dB, dB_mag=dBm, dC=dC, dC_mag=dCm, dstate=carry, dstate_mag=cm,
               dD=(dy * u).sum(0), dD_mag=(dym * np.abs(u)).sum(0), dbias=out["dd"].sum(0), dbias_mag=out["dd_mag"].sum(0))
    if z is not None:
        out["dz"], out["dz_mag"] = dout * f["core"] * silu_slope(z), np.abs(dout) * f["core_mag"] * 1.1
    return out


# ------------------------------------------------------------------------------------------ group norm


def groupnorm(x, groups, w, b, eps, act):
    """x (B, S, C) -> y, mean, rstd (B, G), xhat, pre."""
    n, s, c = x.shape
    v = x.reshape(n, s, groups, c // groups)
    mean = v.mean(axis=(1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    rstd = 1.0 / np.sqrt(var + eps)
    xhat = ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(x.shape)
    pre = xhat * (1.0 if w is None else w) + (0.0 if b is None else b)
    return silu(pre) if act else pre, mean, rstd, xhat, pre


def groupnorm_backward(dy, x, groups, w, b, eps, act):
    n, s, c = x.shape
    _, _, rstd, xhat, pre = groupnorm(x, groups, w, b, eps, act)
    e = dy * silu_slope(pre) if act else dy
    p = (e * (1.0 if w is None else w)).reshape(n, s, groups, c // groups)
    q = xhat.reshape(p.shape)
    m1, m2 = p.mean(axis=(1, 3), keepdims=True), (p * q).mean(axis=(1, 3), keepdims=True)
    dx = rstd[:, None, :, None] * (p - m1 - q * m2)
    big = np.abs(dy) * (1.1 + np.abs(pre)) if act else np.abs(dy)
    size = rstd[:, None, :, None] * (np.abs(p) + np.abs(p).mean(axis=(1, 3), keepdims=True)
                                     + np.abs(q) * np.abs(p * q).mean(axis=(1, 3), keepdims=True))
    return {"dx": dx.reshape(x.shape), "dx_mag": size.reshape(x.shape), "dw": (e * xhat).sum((0, 1)),
            "dw_mag": (big * (1.0 + np.abs(xhat))).sum((0, 1)), "db": e.sum((0, 1)), "db_mag": big.sum((0, 1))}
