"""The gated linear recurrence, the layer norm and the AdamW step from their definitions, in 64 bits (numpy; shares nothing with the kernels), each
with bounds of what fp32 may make of a result: first-order sums of the roundings on the way to it, U = 2^-24 each.

The hardware's exponential, reciprocal and roots are good to one unit in the last place (2 U), the others to half of one (U).
"""
import numpy as np

from seq_oracle import ends, sigmoid

U = 2.0 ** -24


def _gate(x, bias):
    """sigmoid(x + bias) and its relative error: the exponent's is three roundings of its two parts, then an exponential, a sum and a reciprocal."""
    bias = np.zeros(x.shape[-1]) if bias is None else bias
    return sigmoid(x + bias), (3 * (np.abs(x) + np.abs(bias)) + 5) * U


def _parts(x, f, i, A, f_bias, i_bias):
    """Of every position: s, g, t, a, k and the relative errors of s, g, t, a, k."""
    A = np.minimum(A, 0)
    s, es = _gate(f, f_bias)
    g, eg = _gate(i, i_bias)
    with np.errstate(invalid="ignore"):
        t = np.where((s == 0) & np.isinf(A), 0.0, A * s)
    et = es + 3 * U  # (A times log2(e), and times s)
    a, k = np.exp(t), np.sqrt(-np.expm1(2 * t))
    with np.errstate(invalid="ignore"):
        ea = np.where(np.isinf(t), 0, np.abs(t) * et) + 2 * U
    # 1 - a^2: near zero as exact as t, but for a polynomial of 2 U and five roundings; else the difference loses a factor of 3.1 of a's at most, where
    # t's part of that is at most its own (2 t / (e^2t - 1) <= 1); the root halves it
    ek = (et + 14 * U) / 2 + 2 * U
    # fp32's normal numbers end at 2^-126: 1 - a^2 below that counts as zero, so that k, below 2^-63 then, is lost as a whole, and so is what comes of it
    ek = np.where(k * k < 2.0 ** -126 * (1 + 1e-4), 1.0, ek)
    return s, g, t, a, k, es, eg, et, ea, ek


def _scan(a, u, ea, eu, h0, live, back=False):
    """h[l] = a[l] h[l-1] + u[l] of [N, L, C] (back: from the last position, with a of the one behind), sums of magnitudes and errors.  A join of runs
    multiplies once more and adds once more for each position: 3 U."""
    N, L, C = a.shape
    h, m, e = (np.zeros((N, L + 1, C)) for _ in range(3))  # before each position (back: behind)
    order = range(L - 1, -1, -1) if back else range(L)
    ch, cm, ce = h0.copy(), np.abs(h0), np.zeros_like(h0)
    for l in order:
        on = live[:, l]
        if back:  # (what a position hands on: a times what has come, with its own)
            h[:, l], m[:, l], e[:, l] = ch, cm, ce
            nh, nm = ch + u[:, l], cm + np.abs(u[:, l])
            ne = ce + eu[:, l] + U * nm
            ch, cm, ce = np.where(on, a[:, l] * nh, ch), np.where(on, a[:, l] * nm, cm), np.where(on, a[:, l] * (ne + nm * (ea[:, l] + 3 * U)), ce)
        else:
            h[:, l], m[:, l], e[:, l] = ch, cm, ce
            nh, nm = a[:, l] * ch + u[:, l], a[:, l] * cm + np.abs(u[:, l])
            ne = a[:, l] * (ce + cm * (ea[:, l] + 3 * U)) + eu[:, l] + U * nm
            ch, cm, ce = np.where(on, nh, ch), np.where(on, nm, cm), np.where(on, ne, ce)
    h[:, L], m[:, L], e[:, L] = ch, cm, ce
    return h, m, e


def _live(lengths, N, L):
    live = np.zeros((N, L, 1), dtype=bool)
    for n, end in enumerate(ends(lengths, N, L)):
        live[n, :end] = True
    return live


def _silu(z):
    """z sigmoid(z), its slope, and the errors of both."""
    p = sigmoid(z)
    ep = (3 * np.abs(z) + 5) * U
    slope = p * (1 + z * (1 - p))
    return z * p, slope, np.abs(z * p) * (ep + U), p * (ep * (1 + np.abs(z)) + (1 + 2 * np.abs(z)) * 4 * U)


def rec(x, f, i, A, z=None, f_bias=None, i_bias=None, state=None, lengths=None):
    """(y, the state behind each sequence), and the errors of both."""
    N, L, C = x.shape
    s, g, t, a, k, es, eg, et, ea, ek = _parts(x, f, i, A, f_bias, i_bias)
    u = k * g * x
    h, m, e = _scan(a, u, ea, np.abs(u) * (ek + eg + 2 * U), np.zeros((N, C)) if state is None else state.astype(np.float64), _live(lengths, N, L))
    y, ey = h[:, 1:].copy(), e[:, 1:].copy()
    if z is not None:
        gate, _, egate, _ = _silu(z)
        y, ey = y * gate, ey * np.abs(gate) + m[:, 1:] * (egate + 2 * U * np.abs(gate))
    live = _live(lengths, N, L)
    return (y * live, h[:, L]), (ey * live, e[:, L])


def rec_bwd(x, f, i, A, dy, z=None, f_bias=None, i_bias=None, lengths=None):
    """Dicts of dx, df, di, dz, dA, df_bias, di_bias and of their errors."""
    N, L, C = x.shape
    live = _live(lengths, N, L)
    s, g, t, a, k, es, eg, et, ea, ek = _parts(x, f, i, A, f_bias, i_bias)
    u = k * g * x
    h, m, e = _scan(a, u, ea, np.abs(u) * (ek + eg + 2 * U), np.zeros((N, C)), live)
    out, err = {}, {}
    dy = dy * live
    up, eup = dy, np.zeros_like(dy)
    if z is not None:
        gate, slope, egate, eslope = _silu(z)
        out["dz"] = dy * h[:, 1:] * slope
        err["dz"] = np.abs(dy) * (e[:, 1:] * np.abs(slope) + m[:, 1:] * (eslope + 3 * U * np.abs(slope)))
        up, eup = dy * gate, np.abs(dy) * (egate + U * np.abs(gate))
    b, bm, be = _scan(a, up, ea, eup, np.zeros((N, C)), live, back=True)
    b, bm, be = b[:, :L], bm[:, :L], be[:, :L]
    dh, dm, de = (b + up) * live, (bm + np.abs(up)) * live, (be + eup + U * (bm + np.abs(up))) * live
    # (1 - g is off by g's own error and a rounding)
    out["dx"], err["dx"] = dh * k * g, (de + dm * (ek + eg + 2 * U)) * k * g
    out["di"] = dh * k * x * g * (1 - g)
    err["di"] = np.abs(k * x) * g * (de * (1 - g) + dm * ((1 - g) * (ek + eg + 4 * U) + g * eg + U))
    with np.errstate(divide="ignore", invalid="ignore"):
        pays = np.where(k > 0, g * x * a / k, 0)
    before, mb, eb = h[:, :L], m[:, :L], e[:, :L]
    dt = dh * a * (before - pays)
    mt = dm * a * (mb + np.abs(pays))
    et_ = a * (de * (np.abs(before) + np.abs(pays)) + dm * (eb + (mb + np.abs(pays)) * (2 * ea + ek + eg + 6 * U)))
    with np.errstate(invalid="ignore"):
        T = np.where(np.isinf(t), 0, np.abs(t))  # (a is zero there)
    out["df"] = dt * -T * (1 - s)
    err["df"] = T * (et_ * (1 - s) + mt * ((1 - s) * (et + 4 * U) + s * es + U))
    out["dA"] = (dt * s).sum((0, 1))
    err["dA"] = (et_ * s + mt * s * (es + U)).sum((0, 1)) + N * L * U * (mt * s).sum((0, 1))
    for to, of, mag in (("df_bias", "df", mt * T * (1 - s)), ("di_bias", "di", dm * np.abs(k * x) * g * (1 - g))):
        out[to], err[to] = out[of].sum((0, 1)), err[of].sum((0, 1)) + N * L * U * mag.sum((0, 1))
    return out, err


def _sum_units(C):
    # a sum over C numbers: some 8 joins of lanes and waves behind a thread's own, of which there are 64 at most before it goes over them again
    return (10 + min(C, 64) + C / 512) * U


def _lnorm_parts(r, eps):
    C = r.shape[-1]
    mean = r.mean(-1, keepdims=True)
    emean = _sum_units(C) * np.abs(r).mean(-1, keepdims=True)
    d = r - mean
    ed = emean + U * np.abs(d)
    var = (d * d).mean(-1, keepdims=True)
    # (an error of the mean that all differences share moves their squares' sum by its own square alone, and by the sum of what rounding left)
    evar = _sum_units(C) * var + 2 * U * var + emean * emean + 2 * emean * U * np.abs(d).mean(-1, keepdims=True) + C * 0
    with np.errstate(divide="ignore", invalid="ignore"):
        rstd = 1 / np.sqrt(var + eps)
        er = evar / (var + eps) / 2 + 4 * U  # relative
    return d, ed, rstd, er


def lnorm(r, w, b, eps):
    """y and its error."""
    d, ed, rstd, er = _lnorm_parts(r, eps)
    y = d * rstd * w
    ey = np.abs(w) * rstd * ed + np.abs(y) * (er + 3 * U)
    if b is not None:
        y = y + b
        ey = ey + U * np.abs(y)
    return y, ey


def lnorm_bwd(r, w, dy, dr, eps):
    """(dx, dw, db) and their errors."""
    C, rows = r.shape[-1], r[..., 0].size
    d, ed, rstd, er = _lnorm_parts(r, eps)
    u = d * rstd
    eu = ed * rstd + np.abs(u) * (er + U)
    g = dy * w
    n = _sum_units(C) + 3 * U
    through, along = g.mean(-1, keepdims=True), (g * u).mean(-1, keepdims=True)
    ethrough, ealong = n * np.abs(g).mean(-1, keepdims=True), n * np.abs(g * u).mean(-1, keepdims=True) + (np.abs(g) * eu).mean(-1, keepdims=True)
    dx = rstd * (g - through - u * along)
    mag = np.abs(g) + np.abs(through) + np.abs(u * along)
    edx = rstd * (ethrough + np.abs(u) * ealong + eu * np.abs(along) + mag * (er + 6 * U))
    if dr is not None:
        dx = dx + dr
        edx = edx + U * np.abs(dx)
    dw, db = (dy * u).reshape(rows, C).sum(0), dy.reshape(rows, C).sum(0)
    edw = (np.abs(dy) * (eu + 2 * U * np.abs(u))).reshape(rows, C).sum(0) + rows * U * np.abs(dy * u).reshape(rows, C).sum(0)
    return (dx, dw, db), (edx, edw, rows * U * np.abs(dy).reshape(rows, C).sum(0))


def adamw(p, g, m, v, rate, t, factor, beta1, beta2, eps, decay):
    """p, m, v after step t, and their errors."""
    s = factor * g
    m1 = beta1 * m + (1 - beta1) * s
    em = 4 * U * (np.abs(beta1 * m) + np.abs((1 - beta1) * s))
    v1 = beta2 * v + (1 - beta2) * s * s
    ev = 6 * U * v1
    root = np.sqrt(v1 / (1 - beta2 ** t))
    with np.errstate(invalid="ignore", divide="ignore"):
        move = rate * (m1 / (1 - beta1 ** t)) / (root + eps)
        # (m's error, v's halved, and roundings of the root, both corrections, the sum, the quotient and the products)
        emove = np.abs(move) * 16 * U + rate / (1 - beta1 ** t) * em / (root + eps)
    p1 = p - rate * decay * p - move
    return (p1, m1, v1), (3 * U * np.abs(p) + 4 * U * np.abs(rate * decay * p) + U * np.abs(p1) + emove, em, ev)
