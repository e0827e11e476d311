"""TEST INFRASTRUCTURE ONLY -- plain float64 statement of the calls between a block's products: norms of heads with rotation,
attention and its gradients, and how far binary32 arithmetic with rounded operands may be from them.  numpy; nothing in the product
path may import this module.
"""
import numpy as np

U = 2.0 ** -24                       # half a step of binary32, relative
LEAST = 2.0 ** -126                  # an exponential, an operand or a result of a matrix instruction below it may be zero


# ---- norms and rotation ---------------------------------------------------------------------------

def angles(positions, pair_axis, frequencies):
    """[rows, pairs] of positions [axes, rows]."""
    at = np.asarray(positions, np.int64)
    axis = np.zeros(len(frequencies), int) if pair_axis is None else np.minimum(np.asarray(pair_axis, int), len(at) - 1)
    return at[axis].T.astype(np.float64) * np.asarray(frequencies, np.float64)


def pairs_of(rope_dim, interleaved):
    """Indices of the first and second elements of the pairs."""
    j = np.arange(rope_dim // 2)
    return (2 * j, 2 * j + 1) if interleaved else (j, j + rope_dim // 2)


def turn(x, angle, interleaved, back=False):
    """Heads x [rows, heads, dim] rotated by angle [rows, pairs]."""
    a, b = pairs_of(2 * angle.shape[1], interleaved)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1 if back else 1)
    y = np.array(x, np.float64)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def mixed(x, angle, interleaved):
    """|a| + |b| of each element's pair, |x| of an element that is not rotated: what its rotation's error is relative to."""
    a, b = pairs_of(2 * angle.shape[1], interleaved)
    y = np.abs(np.array(x, np.float64))
    y[..., a] = y[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y


def norm_rope(x, weight, eps, angle, interleaved):
    """(result, what its error in binary32 is at most)."""
    x = np.asarray(x, np.float64)
    if eps > 0:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps))) * (1.0 if weight is None else weight)
    # a normed element: its factor and two products round; a cosine is off by pi / 2 half steps (its angle, rounded to binary32) and
    # two of the function itself, of 1; a product and the sum round
    return turn(x, angle, interleaved), 10 * U * mixed(x, angle, interleaved)


def norm_rope_grads(x, weight, eps, angle, interleaved, grad):
    """(grad_x, its bound, grad_weight, sum of the sizes of its terms)."""
    x, g = np.asarray(x, np.float64), turn(np.asarray(grad, np.float64), angle, interleaved, True)
    size = mixed(np.asarray(grad, np.float64), angle, interleaved)
    if eps == 0:
        return g, 8 * U * size, None, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps)))
    m, w = x * r, 1.0 if weight is None else weight
    u, usize = g * w, size * np.abs(w)
    gx = r * (u - m * (u * m).mean(-1, keepdims=True))
    # u: 8 of the rotation and a product; a sum of at most 256 products in 16 steps a lane and 4 over lanes, each term off by 8 + 3
    bound = U * r * (12 * usize + 48 * np.abs(m) * (usize * np.abs(m)).mean(-1, keepdims=True))
    return gx, bound, (g * m).sum((0, 1)), (size * np.abs(m)).sum((0, 1))


# ---- attention ------------------------------------------------------------------------------------

def attention(q, k, v, seen, scale, half, grad=None, tiny=0.0):
    """One head: q [n, d], k, v [m, d], seen [n, m].  A dict of the results and of their bounds ("out", "lse" and with grad "dq",
    "dk", "dv", each a pair), for arithmetic in binary32 whose operands p and ds are rounded by `half` relative and `tiny`."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    n, m, d = len(q), len(k), q.shape[1]
    if m == 0:
        z = np.zeros((n, d))
        return {"out": (z, z), "lse": (np.full(n, -np.inf), np.zeros(n)), "dq": (z, z), "dk": (z[:0], z[:0]), "dv": (z[:0], z[:0])}
    # what is not seen has no part in anything
    live = seen.any(0)
    k, v = np.where(live[:, None], k, 0), np.where(live[:, None], v, 0)
    s = np.where(seen, scale * (q @ k.T), -np.inf)
    top = np.where(seen.any(1), s.max(1, initial=-np.inf), 0.0)
    e = np.exp(s - top[:, None])
    total = e.sum(1)
    p = e / np.where(total > 0, total, 1)[:, None]
    out = p @ v
    with np.errstate(divide="ignore"):
        lse = np.where(total > 0, top + np.log(np.where(total > 0, total, 1)), -np.inf)
    # a score: d products and sums, each rounded (or cut) by at most 2 U; exponent: the scaled score, the factor and the difference round;
    # the exponential itself two
    ds = np.where(seen, scale * 2 * d * U * (np.abs(q) @ np.abs(k).T) + 4 * U * (np.abs(np.where(seen, s, 0)) + np.abs(top)[:, None] + 2), 0)
    of_p = ds.max(1, keepdims=True)
    rel = 2 * of_p + half + 4 * (m + 16) * U                      # of a probability in a normed sum
    tiny = tiny + LEAST
    ebound = rel * (p @ np.abs(v)) + tiny * (seen @ np.abs(v)) + 4 * U * np.abs(out) + m * LEAST
    r = {"out": (out, ebound), "lse": (lse, np.where(total > 0, of_p[:, 0] + 2 * (m + 16) * U + 4 * U * np.abs(lse) + 4 * U, 0))}
    if grad is not None:
        g = np.asarray(grad, np.float64)
        dp, delta = g @ v.T, (g * out).sum(1, keepdims=True)
        t = np.where(seen, p * (dp - delta), 0)
        prel = 3 * of_p + half + 4 * (m + 16) * U + 8 * U * np.abs(np.where(np.isfinite(lse), lse, 0))[:, None]
        # D is formed from the result as it was stored
        edelta = (np.abs(g) * (ebound + (half + 2 * d * U) * np.abs(out))).sum(1, keepdims=True)
        edp = 2 * d * U * (np.abs(g) @ np.abs(v).T)
        et = np.where(seen, p * (prel * np.abs(dp - delta) + edp + edelta + 4 * U * (np.abs(dp) + np.abs(delta))) + tiny + LEAST * np.abs(dp - delta), 0)
        sums = lambda c: 4 * (c + 16) * U
        r["dv"] = (p.T @ g, (p * prel + tiny * seen).T @ np.abs(g) + sums(n) * (p.T @ np.abs(g)) + n * LEAST)
        r["dq"] = (scale * (t @ k), scale * (et @ np.abs(k) + sums(m) * (np.abs(t) @ np.abs(k))) + m * LEAST)
        r["dk"] = (scale * (t.T @ q), scale * (et.T @ np.abs(q) + sums(n) * (np.abs(t).T @ np.abs(q))) + n * LEAST)
    return r


def causal(n, m):
    """[n, m]: row i sees keys up to i + m - n."""
    return np.arange(m)[None] <= np.arange(n)[:, None] + m - n


def tree_mask(n, m, words=None):
    """[n, m]: all keys before the last n, and of these the ones whose bit is set in words [n, w] (None: a chain)."""
    if words is None:
        return causal(n, m)
    bit = np.arange(m)[None] - (m - n)
    w = np.asarray(words).astype(np.uint64)
    at = np.clip(bit, 0, 64 * w.shape[1] - 1)
    set_ = (w[np.arange(n)[:, None], at // 64] >> (at % 64).astype(np.uint64)) & np.uint64(1)
    return (bit < 0) | ((set_ == 1) & (bit < 64 * w.shape[1]))
