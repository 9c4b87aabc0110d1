"""Float64 oracles of the gated linear recurrence and of the 4-bit gate product
(NumPy, one timestep after another, no code shared with the HIP path), and
bounds on what fp32 arithmetic may differ from them by.
"""

import numpy as np

U32 = 2.0 ** -24   # half a step of fp32, relative


def _sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0, e) / (1.0 + e)


def _gates(p, bias):
    H = p.shape[-1] // 4
    y = p.astype(np.float64) + (0.0 if bias is None else bias.astype(np.float64))
    return _sigmoid(y[..., :H]), _sigmoid(y[..., H:2 * H]), np.tanh(y[..., 2 * H:3 * H]), _sigmoid(y[..., 3 * H:])


def _live(T, B, lengths):
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    return np.arange(T)[:, None] < n


def linear_lstm(p, bias=None, lengths=None, c0=None):
    """h [T, B, H], c [T + 1, B, H] (c[0] the initial state) and, of the same
    shapes, elementwise bounds on their fp32 errors.

    One step's error: a sigmoid from the hardware's exponential and reciprocal
    is off by at most 4u (its argument's three roundings, 3u x s(1-s) <= 0.7u; the
    exponential, 2u s(1-s) <= 0.5u; the sum and the reciprocal, 3u), a tanh as
    1 - 2 sigmoid by 9u.  So f c + i g adds at most 4u |c| + 13u, and its own
    roundings 2u |c| + 2u; summing time in pieces, c = A c' + B with A = prod f,
    rounds A and B once more a step: 2u |c| + u.  |c| is taken as its envelope.
    """
    T, B, H4 = p.shape
    i, f, g, o = _gates(p, bias)
    live = _live(T, B, lengths)[..., None]
    c = np.zeros((T + 1, B, H4 // 4))
    if c0 is not None:
        c[0] = c0
    env, err = np.abs(c), np.zeros_like(c)
    for t in range(T):
        c[t + 1] = np.where(live[t], f[t] * c[t] + i[t] * g[t], c[t])
        env[t + 1] = np.where(live[t], f[t] * env[t] + np.abs(i[t] * g[t]), env[t])
        err[t + 1] = np.where(live[t], f[t] * err[t] + U32 * (8 * env[t] + 16), err[t])
    th = np.tanh(c[1:])
    h = np.where(live, o * th, 0.0)
    h_err = np.where(live, err[1:] + 14 * U32, 0.0)
    return h, c, h_err, err


def linear_lstm_grad(p, dh, dc_out=None, bias=None, lengths=None, c0=None):
    """Gradients dict(dp, dc0, dbias) of sum(dh h) + sum(dc_out c_T), and the same
    with bounds on their fp32 errors (dp before its own rounding).

    Along d_t = u_t + e_t, e_{t-1} = f_t d_t with u = dh o (1 - tanh(c)^2): tanh(c)
    is off by err(c) + 9u, so u by |dh| (2 (err(c) + 10u) + 6u); a step back
    adds at most 8u of |d|'s envelope, as forward.  The factors of d in dp are off
    by at most 16u (i and g), err(c)/4 + 8u |c| (f) and 24u (g's own).
    """
    T, B, H4 = p.shape
    H = H4 // 4
    i, f, g, o = _gates(p, bias)
    _, c, _, cerr = linear_lstm(p, bias, lengths, c0)
    live = _live(T, B, lengths)[..., None]
    dh = np.where(live, dh.astype(np.float64), 0.0)
    th = np.tanh(c[1:])
    e = np.zeros((B, H)) if dc_out is None else dc_out.astype(np.float64)
    env, err = np.abs(e), np.zeros((B, H))
    dp, bd = np.zeros((T, B, 4, H)), np.zeros((T, B, 4, H))
    for t in range(T - 1, -1, -1):
        d = dh[t] * o[t] * (1 - th[t] ** 2) + e
        de = np.abs(dh[t]) * o[t] * (1 - th[t] ** 2) + env
        derr = np.abs(dh[t]) * (2 * cerr[t + 1] + 26 * U32) + err
        ci, cf, cg = g[t] * i[t] * (1 - i[t]), c[t] * f[t] * (1 - f[t]), i[t] * (1 - g[t] ** 2)
        dp[t] = np.stack([d * ci, d * cf, d * cg, dh[t] * th[t] * o[t] * (1 - o[t])], 1)
        bd[t] = np.stack([derr * np.abs(ci) + de * 16 * U32,
                          derr * np.abs(cf) + de * (cerr[t] / 4 + (8 * np.abs(c[t]) + 1) * U32),
                          derr * np.abs(cg) + de * 24 * U32,
                          np.abs(dh[t]) * (cerr[t + 1] + 18 * U32)], 1)
        lv = live[t]
        dp[t] *= lv[:, None]
        bd[t] *= lv[:, None]
        e = np.where(lv, f[t] * d, e)
        err = np.where(lv, f[t] * derr + 8 * U32 * de, err)
        env = np.where(lv, f[t] * de, env)
    # sums of dp: no chain of additions is longer than T + B + 64
    db = dp.sum((0, 1)).reshape(H4)
    db_err = (bd.sum((0, 1)) + (T + B + 64) * U32 * np.abs(dp).sum((0, 1))).reshape(H4)
    return dict(dp=dp.reshape(T, B, H4), dc0=e, dbias=db), dict(dp=bd.reshape(T, B, H4), dc0=err, dbias=db_err)


def linear_lstm_small(p, dh, dc_out=None, bias=None, lengths=None, c0=None):
    """Bounds dict(h, c, dp, dc0) on fp32 errors that small values keep relative to
    themselves: nothing in them is a multiple of u alone.

    In units of u: y = p + bias is off by |y|, 2^(y log2 e) by 2.25 |y| (the sum, the
    product, the constant) and 2 (the exponential) of itself, so a sigmoid s by
    S = 3 + (1 - s)(2.25 |y| + 2) of itself (the sum 1, the reciprocal 2).  A tanh is off
    by 8 of itself (an odd series near 0, 1 - 2 / (1 + e^2y) elsewhere) and its argument's
    error.  f c adds S + 1, i g S + 10, and 3 of each for the roundings of a step and of
    the maps that join pieces of time.  The rest is the same a product at a time.
    """
    T, B, H4 = p.shape
    H = H4 // 4
    i, f, g, o = _gates(p, bias)
    y = np.abs(p.astype(np.float64) + (0.0 if bias is None else bias.astype(np.float64)))
    Si, Sf, So = (3 + (1 - s) * (2.25 * y[..., k * H:(k + 1) * H] + 2) for s, k in ((i, 0), (f, 1), (o, 3)))
    _, c, _, _ = linear_lstm(p, bias, lengths, c0)
    live = _live(T, B, lengths)[..., None]
    env, err = np.abs(c), np.zeros_like(c)
    for t in range(T):
        fc, ig = f[t] * env[t], np.abs(i[t] * g[t])
        env[t + 1] = np.where(live[t], fc + ig, env[t])
        err[t + 1] = np.where(live[t], f[t] * err[t] + U32 * (fc * (Sf[t] + 4) + ig * (Si[t] + 13)), err[t])
    th = np.abs(np.tanh(c[1:]))
    terr = err[1:] + 8 * U32 * th
    h = np.where(live, o * terr + U32 * o * th * (So + 1), 0.0)
    dh = np.where(live, np.abs(dh.astype(np.float64)), 0.0)
    env_e = np.zeros((B, H)) if dc_out is None else np.abs(dc_out.astype(np.float64))
    err_e, dp = np.zeros((B, H)), np.zeros((T, B, 4, H))
    a, up = np.abs(c), 1 - th ** 2
    for t in range(T - 1, -1, -1):
        de = dh[t] * o[t] * up[t] + env_e
        derr = dh[t] * o[t] * (up[t] * (So[t] + 3) * U32 + 2 * th[t] * terr[t]) + err_e + U32 * de
        i1, f1, g1, o1 = i[t] * (1 - i[t]), f[t] * (1 - f[t]), 1 - g[t] ** 2, o[t] * (1 - o[t])
        gi, gf = i[t] * np.abs(1 - 2 * i[t]) * Si[t], f[t] * np.abs(1 - 2 * f[t]) * Sf[t]
        ag = np.abs(g[t])
        dp[t] = np.stack([
            derr * ag * i1 + de * ag * U32 * (gi + 12 * i1),
            derr * a[t] * f1 + de * (a[t] * U32 * (gf + 3 * f1) + err[t] * f1),
            derr * i[t] * g1 + de * i[t] * U32 * (g1 * (Si[t] + 3) + 18 * g[t] ** 2),
            dh[t] * (o1 * (terr[t] + th[t] * (So[t] + 4) * U32) + th[t] * o[t] ** 2 * So[t] * U32)], 1)
        lv = live[t]
        dp[t] *= lv[:, None]
        err_e = np.where(lv, f[t] * derr + U32 * f[t] * de * (Sf[t] + 5), err_e)
        env_e = np.where(lv, f[t] * de, env_e)
    return dict(h=h, c=err, dp=dp.reshape(T, B, H4), dc0=err_e)


def q4_round(w, group):
    """Levels q [R, D], scale and zero [R, groups] of a float32 matrix."""
    R, D = w.shape
    n = -(-D // group)
    pad = np.zeros((R, n * group))
    pad[:, :D] = w
    pad = pad.reshape(R, n, group)
    lo, hi = np.minimum(pad.min(-1), 0.0), np.maximum(pad.max(-1), 0.0)
    s = ((hi - lo) / 15.0).astype(np.float32)
    sd = np.where(s > 0, s.astype(np.float64), 1.0)
    z = np.clip(np.rint(-lo / sd), 0, 15)
    q = np.clip(np.rint(pad / sd[..., None] + z[..., None]), 0, 15)
    return q.reshape(R, -1)[:, :D].astype(np.uint8), s, z.astype(np.uint8)


def q4_pack(q):
    """Two levels in a byte, even columns in the low half."""
    if q.shape[1] % 2:
        q = np.concatenate([q, np.zeros_like(q[:, :1])], 1)
    return (q[:, 0::2] | (q[:, 1::2] << 4)).astype(np.uint8)


def q4_product(q, s, z, group, x, bias=None):
    """y [N, R] and a bound on its fp32 error.

    Summed as sum_g s (sum q' x - z' sum x) with levels and zeros moved by the same
    amount, at most 31 each, no chain of additions longer than 3 D / 32 + 64.
    """
    R, D = q.shape
    of = np.arange(D) // group
    sd = s.astype(np.float64)[:, of]
    w = (q.astype(np.float64) - z.astype(np.float64)[:, of]) * sd
    x = x.astype(np.float64)
    b = np.zeros(R) if bias is None else bias.astype(np.float64)
    bound = U32 * (3 * D / 32 + 64) * (62 * (np.abs(x) @ np.abs(sd).T) + np.abs(b))
    return x @ w.T + b, bound
