"""The sequence operators from their definitions, in 64 bits, one position after the other (numpy; shares nothing with the
kernels).  Sequences are [N, L, C]; parameters as the operators take them, without padding.

Each function takes ``mag``: with it every number that is multiplied or added counts with its absolute value, so that what comes out
bounds the sum of the magnitudes that a result was summed from.  The exponentials, sigmoids and lengths stay as they are.
"""
import numpy as np


def _abs(mag, *xs):
    return [None if x is None else np.abs(x) if mag else x for x in xs]


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-x))


def softplus(x):
    return np.logaddexp(x, 0)


def ends(lengths, N, L):
    return [L] * N if lengths is None else [min(max(int(n), 0), L) for n in lengths]


def conv(x, w, bias, silu=True, state=None, lengths=None, mag=False):
    """y, the state behind each sequence [N, W-1, C]."""
    N, L, C = x.shape
    W = w.shape[0]
    y, after = np.zeros((N, L, C)), np.zeros((N, W - 1, C))
    for n, end in enumerate(ends(lengths, N, L)):
        line = np.concatenate([np.zeros((W - 1, C)) if state is None else state[n], x[n, :end]])
        for l in range(end):
            s = np.zeros(C) if bias is None else bias.copy()
            for j in range(W):
                s = s + w[j] * line[l + j]
            if mag:
                m = np.abs(0 if bias is None else bias) + sum(np.abs(w[j] * line[l + j]) for j in range(W))
                # (a gate's slope is at most 1.1; the exponential of a sum is off by the sum's own error and |s| units)
                y[n, l] = m * (1.1 + np.abs(s)) if silu else m
            else:
                y[n, l] = s * sigmoid(s) if silu else s
        after[n] = line[len(line) - (W - 1):]
    return y, after


def conv_bwd(x, w, bias, dy, silu=True, lengths=None, mag=False):
    """dx, dw, dbias."""
    N, L, C = x.shape
    W = w.shape[0]
    dx, dw, db = np.zeros((N, L, C)), np.zeros((W, C)), np.zeros(C)
    for n, end in enumerate(ends(lengths, N, L)):
        for l in range(end):
            s = np.zeros(C) if bias is None else bias.copy()
            for j in range(W):
                if l - W + 1 + j >= 0:
                    s = s + w[j] * x[n, l - W + 1 + j]
            p = sigmoid(s)
            ds = dy[n, l] * (p * (1 + s * (1 - p)) if silu else 1)
            if mag:
                ds = np.abs(dy[n, l]) * (2 + np.abs(s)) ** 2
            db += ds
            for j in range(W):
                at = l - W + 1 + j
                if at >= 0:
                    dx[n, at] += np.abs(ds * w[j]) if mag else ds * w[j]
                    dw[j] += np.abs(ds * x[n, at]) if mag else ds * x[n, at]
    return dx, dw, db


def _scan_parts(x, dt, A, B, Cm, dt_bias, use_softplus, G):
    N, L, C = x.shape
    raw = dt + (0 if dt_bias is None else dt_bias)
    d = softplus(raw) if use_softplus else raw
    slope = sigmoid(raw) if use_softplus else np.ones_like(raw)
    group = np.arange(C) // (C // G)
    S = A.shape[0]
    Bg = B.reshape(N, L, G, S)[:, :, group].transpose(0, 1, 3, 2)  # [N, L, S, C]
    Cg = Cm.reshape(N, L, G, S)[:, :, group].transpose(0, 1, 3, 2)
    return d, slope, group, Bg, Cg


def scan(x, dt, A, B, Cm, D=None, z=None, dt_bias=None, G=1, use_softplus=True, state=None, lengths=None, mag=False):
    """y, the state behind each sequence [N, S, C].  A: [S, C]; B, Cm: [N, L, G * S]."""
    N, L, C = x.shape
    S = A.shape[0]
    d, _, _, Bg, Cg = _scan_parts(x, dt, A, B, Cm, dt_bias, use_softplus, G)
    x, Bg, Cg, D, state = _abs(mag, x, Bg, Cg, D, state)
    dm = np.abs(d) if mag else d
    y, after = np.zeros((N, L, C)), np.zeros((N, S, C))
    for n, end in enumerate(ends(lengths, N, L)):
        h = np.zeros((S, C)) if state is None else state[n].astype(np.float64)
        for l in range(end):
            h = np.exp(d[n, l] * A) * h + dm[n, l] * x[n, l] * Bg[n, l]
            o = (Cg[n, l] * h).sum(0) + (0 if D is None else D * x[n, l])
            if z is not None:
                g = z[n, l] * sigmoid(z[n, l])
                o = o * (np.abs(g) * (1 + np.abs(z[n, l])) if mag else g)
            y[n, l] = o
        after[n] = h
    return y, after


def scan_bwd(x, dt, A, B, Cm, dy, D=None, z=None, dt_bias=None, G=1, use_softplus=True, lengths=None, mag=False):
    """dict of dx, ddt, dA, dB, dC, dD, dz, ddt_bias."""
    N, L, C = x.shape
    S = A.shape[0]
    d, slope, group, Bg, Cg = _scan_parts(x, dt, A, B, Cm, dt_bias, use_softplus, G)
    E = A
    x, Bg, Cg, D, dy, A = _abs(mag, x, Bg, Cg, D, dy, A)
    dm = np.abs(d) if mag else d
    Dv = np.zeros(C) if D is None else D
    out = {"dx": np.zeros((N, L, C)), "ddt": np.zeros((N, L, C)), "dA": np.zeros((S, C)), "dB": np.zeros((N, L, G, S)), "dC": np.zeros((N, L, G, S)),
           "dD": np.zeros(C), "dz": np.zeros((N, L, C)), "ddt_bias": np.zeros(C)}
    for n, end in enumerate(ends(lengths, N, L)):
        h = np.zeros((end + 1, S, C))
        for l in range(end):
            h[l + 1] = np.exp(d[n, l] * E) * h[l] + dm[n, l] * x[n, l] * Bg[n, l]
        back = np.zeros((S, C))
        for l in reversed(range(end)):
            up = dy[n, l]
            if z is not None:
                p = sigmoid(z[n, l])
                o = (Cg[n, l] * h[l + 1]).sum(0) + Dv * x[n, l]
                out["dz"][n, l] = up * o * ((2 + np.abs(z[n, l])) ** 2 if mag else p * (1 + z[n, l] * (1 - p)))
                up = up * (np.abs(z[n, l] * p) * (1 + np.abs(z[n, l])) if mag else z[n, l] * p)
            g = back + up * Cg[n, l]
            dC, dB = up * h[l + 1], g * dm[n, l] * x[n, l]
            for k in range(G):
                out["dC"][n, l, k] = dC[:, group == k].sum(1)
                out["dB"][n, l, k] = dB[:, group == k].sum(1)
            back = g * np.exp(d[n, l] * E)
            gB, t = (g * Bg[n, l]).sum(0), back * h[l]
            out["dx"][n, l] = Dv * up + dm[n, l] * gB
            out["ddt"][n, l] = ((t * A).sum(0) + x[n, l] * gB) * slope[n, l]
            out["dA"] += t * dm[n, l]
            out["dD"] += up * x[n, l]
            out["ddt_bias"] += out["ddt"][n, l]
    out["dB"], out["dC"] = out["dB"].reshape(N, L, G * S), out["dC"].reshape(N, L, G * S)
    return out


def norm(r, w, eps):
    return r * w / np.sqrt((r * r).mean(-1, keepdims=True) + eps)


def norm_bwd(r, w, dy, dr, eps, mag=False):
    rstd = 1 / np.sqrt((r * r).mean(-1, keepdims=True) + eps)
    r, w, dy, dr = _abs(mag, r, w, dy, dr)
    wdy = w * dy
    dot = r * rstd * rstd * (wdy * r).mean(-1, keepdims=True)
    dx = rstd * (wdy + dot if mag else wdy - dot)
    return dx + (0 if dr is None else dr), (dy * r * rstd).reshape(-1, r.shape[-1]).sum(0)


def mv4(x, q, scale, group, xscale=None, bias=None, mag=False):
    """x: [M, C]; q: [K, C] whole numbers; scale: [ceil(C / group), K]."""
    x, q, scale, xscale, bias = _abs(mag, x, q, scale, xscale, bias)
    y = np.zeros((x.shape[0], q.shape[0]))
    for c in range(x.shape[1]):
        y += np.outer(x[:, c], q[:, c] * scale[c // group])
    if xscale is not None:
        y = y * xscale[:, None]
    return y + (0 if bias is None else bias)
