"""Plain 64-bit forms of the recognition operators, row by row in numpy, and the
error that rounding allows each result, from the magnitudes that enter it.

u is the unit roundoff of the sums (2^-24 or 2^-53), u_out that of the result's
type (2^-8 for bfloat16).  The bounds count roundings along the longest chain of a
sum, so they hold for any order of the terms up to the stated lengths."""
import numpy as np

U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -24, "f64": 2.0 ** -53}
U_OUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f64": 2.0 ** -53}

# longest chain of roundings of a sum over a row (32 elements a thread, 64 lanes, 16 waves), plus
# the few operations around it
CHAIN = 64


def layer_norm(x, w, b, eps):
    D = x.shape[1]
    mean = x.sum(1) / D
    rstd = ((x - mean[:, None]) ** 2).sum(1) / D + eps
    rstd = rstd ** -0.5
    return (x - mean[:, None]) * rstd[:, None] * w + b, mean, rstd


def layer_norm_tol(x, w, b, eps, kind):
    u, u_out = U[kind], U_OUT[kind]
    y, mean, rstd = layer_norm(x, w, b, eps)
    big = np.abs(x).max(1)
    xh = np.abs((x - mean[:, None]) * rstd[:, None])
    # the mean is off by CHAIN u max|x|, so x - mean and, relatively, rstd are too
    rel = CHAIN * u * (1 + big * rstd)
    ty = rel[:, None] * (1 + xh) * np.abs(w) + 2 * u * np.abs(b) + (u_out + u) * np.abs(y)
    return ty, CHAIN * u * big, 2 * rel * rstd


def layer_norm_grads(x, w, mean, rstd, dy):
    D = x.shape[1]
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * w
    dx = rstd[:, None] * (g - g.sum(1, keepdims=True) / D - xh * (g * xh).sum(1, keepdims=True) / D)
    return dx, (dy * xh).sum(0), dy.sum(0)


def layer_norm_grads_tol(x, w, mean, rstd, dy, kind):
    u, u_out = U[kind], U_OUT[kind]
    D = x.shape[1]
    xh = np.abs((x - mean[:, None]) * rstd[:, None])
    # x - mean of the arrays as given: one rounding of the difference
    g = np.abs(dy * w)
    t = rstd[:, None] * (g + g.sum(1, keepdims=True) / D + xh * (g * xh).sum(1, keepdims=True) / D)
    dx = np.abs(layer_norm_grads(x, w, mean, rstd, dy)[0])
    return CHAIN * u * t + u_out * dx, CHAIN * u * (np.abs(dy) * xh).sum(0), CHAIN * u * np.abs(dy).sum(0)


def sigmoid(g):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))


def _order(lo, hi, reverse):
    return range(hi - 1, lo - 1, -1) if reverse else range(lo, hi)


# roundings of one row of the recurrence, those of the gate included, and of the two joins
ROW = 16


def recurrence(x, gate, offsets, h0, reverse, kind="f64"):
    """h, h_last and what rounding may add to each."""
    u, u_out = U[kind], U_OUT[kind]
    N, D = x.shape
    B = len(offsets) - 1
    a, b = sigmoid(gate)
    h, th = np.zeros((N, D)), np.zeros((N, D))
    last, tlast = np.zeros((B, D)), np.zeros((B, D))
    for q in range(B):
        s = h0[q].copy() if h0 is not None else np.zeros(D)
        big, err = np.abs(s), np.zeros(D)
        for t in _order(offsets[q], offsets[q + 1], reverse):
            s = a[t] * s + b[t] * x[t]
            big = a[t] * big + b[t] * np.abs(x[t])
            err = a[t] * err + ROW * u * big
            h[t], th[t] = s, err + u_out * np.abs(s)
        last[q], tlast[q] = s, err
    return h, last, th, tlast


def recurrence_grads(x, gate, h, dh, offsets, h0, dh_last, reverse, kind="f64"):
    """dx, dgate, dh0 and what rounding may add to each; h is the array as given."""
    u, u_out = U[kind], U_OUT[kind]
    N, D = x.shape
    B = len(offsets) - 1
    a, b = sigmoid(gate)
    dx, dg, tx, tg = (np.zeros((N, D)) for _ in range(4))
    d0, t0 = np.zeros((B, D)), np.zeros((B, D))
    for q in range(B):
        c = dh_last[q].copy() if dh_last is not None else np.zeros(D)
        big, err = np.abs(c), np.zeros(D)
        rows = list(_order(offsets[q], offsets[q + 1], reverse))
        for k in range(len(rows) - 1, -1, -1):
            t = rows[k]
            before = h[rows[k - 1]] if k else h0[q] if h0 is not None else np.zeros(D)
            G = dh[t] + c
            big = np.abs(dh[t]) + big
            err = err + ROW * u * big
            dx[t] = b[t] * G
            dg[t] = a[t] * b[t] * G * (before - x[t])
            tx[t] = b[t] * err + u_out * np.abs(dx[t])
            tg[t] = a[t] * b[t] * err * (np.abs(before) + np.abs(x[t])) + u_out * np.abs(dg[t])
            c, big, err = a[t] * G, a[t] * big, a[t] * err
        d0[q], t0[q] = c, err
    return dx, dg, d0, tx, tg, t0


def adamw(p, g, m, v, step, lr, b1, b2, eps, wd):
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    p = p * (1 - lr * wd) - lr / (1 - b1 ** step) * m / (np.sqrt(v / (1 - b2 ** step)) + eps)
    return p, m, v


def adamw_tol(p, g, m, v, step, lr, b1, b2, eps, wd, kind):
    u, u_out = U[kind], U_OUT[kind]
    pn, mn, vn = adamw(p, g, m, v, step, lr, b1, b2, eps, wd)
    tm = 4 * u * (b1 * np.abs(m) + (1 - b1) * np.abs(g))
    tv = 8 * u * vn
    # the step: m's error and the relative one of the root, the quotient and the factors
    denom = np.sqrt(vn / (1 - b2 ** step)) + eps
    scale = lr / (1 - b1 ** step)
    tp = scale * (tm + 12 * u * np.abs(mn)) / denom + 4 * u * np.abs(p) + u_out * np.abs(pn)
    return tp, tm, tv


# ------------------------------------------------------------------ 8-bit moments, in 32 bits

def values_m(codes, scale):
    """float32 values of int8 codes [blocks, 256], every operation rounded once."""
    r = np.abs(codes.astype(np.float32)) * np.float32(1 / 127)
    return scale[:, None] * (r * r) * np.sign(codes).astype(np.float32)


def values_v(codes, scale):
    r = codes.astype(np.float32) * np.float32(1 / 255)
    r2 = r * r
    return scale[:, None] * (r2 * r2)


def encode(m, v):
    """Codes and scales of float32 moments [blocks, 256]."""
    tiny = np.finfo(np.float32).tiny
    one = np.float32(1)
    sm, sv = np.abs(m).max(1), v.max(1)
    sm, sv = np.where(sm < tiny, np.float32(0), sm), np.where(sv < tiny, np.float32(0), sv)
    with np.errstate(divide="ignore"):
        im, iv = np.where(sm > 0, one / sm, np.float32(0)), np.where(sv > 0, one / sv, np.float32(0))
    cm = np.rint(np.sqrt(np.abs(m) * im[:, None]) * np.float32(127)) * np.sign(m)
    cv = np.rint(np.sqrt(np.sqrt(v * iv[:, None])) * np.float32(255))
    cv = np.where((v > 0) & (sv[:, None] > 0), np.maximum(cv, 1), cv)
    return cm.astype(np.int8), cv.astype(np.uint8), sm, sv
