"""Oracle of the serving operators (include/eora_serve.h): plain float64 numpy, one loop per token, head or sequence.

Beside each result stands a bound on what fp32 arithmetic with 16-bit operands may differ from it by, from the roundings of
the formula alone.  u is half a step of the 16-bit type (2^-11 fp16, 2^-8 bf16).
"""
import numpy as np

HALF_STEP = {"f16": 2.0**-11, "bf16": 2.0**-8, "f32": 2.0**-24}


def sum_error(n):
    """Relative to the sum of magnitudes: n exact products summed in fp32, eight or more per addition of the running sum, each addition off by
    at most a step (2^-23: the matrix instructions may cut instead of round), and the additions that join the parts."""
    return (n / 8 + 16) * 2.0**-23


def adapters(x, a, b, ids, ranks=None, scales=None, base=None, x_type="f16", y_type="f16"):
    """(y, bound): y[i] = base[i] + s_j (x[i] . A_j[:, :r_j]) . B_j[:r_j]; x [m][K], a [n][K][R], b [n][R][N] float64."""
    m, n, top = x.shape[0], a.shape[0], a.shape[2]
    y = np.zeros((m, b.shape[2])) if base is None else base.astype(np.float64).copy()
    off = np.zeros_like(y)
    for i, j in enumerate(ids):
        if not 0 <= j < n:
            continue
        r = top if ranks is None else min(max(int(ranks[j]), 0), top)
        s = 1.0 if scales is None else float(scales[j])
        if r == 0:
            continue
        A, B = a[j, :, :r], b[j, :r]
        t = x[i] @ A
        y[i] += s * (t @ B)
        # t: its sum, and what is left of it in a high and a low 16-bit part (the low part's own half step; relative to the token's largest, as
        # the parts share one power of two: fp16 ends 2^-24 below 1 and the largest is at least 2^9)
        dt = sum_error(x.shape[1]) * (np.abs(x[i]) @ np.abs(A)) + HALF_STEP[x_type] ** 2 * np.abs(t) + 2.0**-33 * np.abs(t).max()
        off[i] = abs(s) * (dt @ np.abs(B) + (sum_error(2 * r) + 2.0**-22) * (np.abs(t) @ np.abs(B)))
    return y, off + (HALF_STEP[y_type] + 2.0**-23) * (np.abs(y) + off) + 2.0**-25      # (half a step of fp16 below 2^-14)


def qk_norm_rope(x, weight, table, positions, heads, rot, pairs, eps, x_type="f16"):
    """(rows, bound) of q or k: x [m][heads * dim] float64; table [positions][rot]."""
    m = x.shape[0]
    u = x.reshape(m, heads, -1).copy()
    dim = u.shape[2]
    if weight is not None:
        u = u / np.sqrt((u * u).mean(-1, keepdims=True) + eps) * weight
    y, reach = u.copy(), np.abs(u)
    half = rot // 2
    for i in range(half):
        at, bt = (i, i + half) if pairs == "half" else (2 * i, 2 * i + 1)
        c, s = table[positions, i][:, None], table[positions, half + i][:, None]
        y[..., at] = u[..., at] * c - u[..., bt] * s
        y[..., bt] = u[..., bt] * c + u[..., at] * s
        reach[..., at] = reach[..., bt] = np.abs(u[..., at]) + np.abs(u[..., bt])
    # fp32: the mean of dim squares (dim / 8 additions in a lane and five across lanes at most), a reciprocal square root of two steps, four products, a sum
    off = (dim / 8 + 16) * 2.0**-23 * reach
    return y.reshape(m, -1), (off + HALF_STEP[x_type] * (np.abs(y) + off) + 2.0**-25).reshape(m, -1)


def attention(q, k, v, scale, x_type="f16", weight_step=None):
    """One sequence, one key head: q [g][d], k, v [t][d] float64.  (out, lse, bound of out, bound of lse).  weight_step: what a weight may be
    rounded by in the second product, relative to it (half a step of x_type unless given)."""
    if k.shape[0] == 0:
        return np.zeros_like(q), np.full(q.shape[0], -np.inf), np.zeros_like(q), np.zeros(q.shape[0])
    s = scale * (q @ k.T)
    top = s.max(1, keepdims=True)
    e = np.exp(s - top)
    total = e.sum(1, keepdims=True)
    w = e / total
    out = w @ v
    # scores: their sum, the scaling by scale / ln 2 and the difference to the maximum (one step of the value each); exp2 two steps.
    # A relative error d of every weight moves the output by d sum w |v|, once in the sum and once in the total.
    ds = (sum_error(q.shape[1]) * scale * (np.abs(q) @ np.abs(k).T) + 2.0**-22 * (np.abs(s) + np.abs(top))).max(1, keepdims=True) + 2.0**-21
    u, n = HALF_STEP[x_type], k.shape[0]
    mass = w @ np.abs(v)
    off = mass * (2 * ds + (u if weight_step is None else weight_step) + 2 * sum_error(n)) + n * 2.0**-40 / total * np.abs(v).max()      # fp16 has nothing below 2^-40 of the largest weight
    lse = (top + np.log(total))[:, 0]
    dl = ds[:, 0] + sum_error(n) + 2.0**-21 * (1 + np.abs(lse) + np.abs(top[:, 0]))
    return out, lse, off + u * (np.abs(out) + off) + 2.0**-25, dl
