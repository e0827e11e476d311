"""TEST INFRASTRUCTURE ONLY -- plain float64 statement of the language-model layers: RMS norm with residual,
rows in 8 bits, products with group-scaled 4-bit weights.  numpy; nothing in the product path may import this module.
"""
import numpy as np


def rms_norm(h, weight, eps):
    """(y, 1 / rms) of rows h [rows, dim] (the sum of input and residual, as it is stored)."""
    h = np.asarray(h, np.float64)
    r = 1.0 / np.sqrt((h * h).mean(axis=1) + float(np.float32(eps)))
    return h * r[:, None] * weight, r


def code_rows(h, weight, r):
    """(codes, scales) of the rows: 127 h w / max |h w| rounded, halves to even, decided in extended precision."""
    p = np.asarray(h, np.longdouble) * np.asarray(weight, np.longdouble)
    amax = np.abs(p).max(axis=1, keepdims=True)
    safe = np.where(amax > 0, amax, 1)
    return np.rint(127 * p / safe).astype(np.int64), (amax[:, 0].astype(np.float64) * r / 127.0)


def rms_norm_grads(h, weight, r, grad_y, grad_sum):
    """(grad_x, grad_weight) with 1 / rms given."""
    n = np.asarray(h, np.float64) * r[:, None]
    t = grad_y * weight
    gx = r[:, None] * (t - n * (t * n).mean(axis=1, keepdims=True))
    if grad_sum is not None:
        gx = gx + grad_sum
    return gx, (grad_y * n).sum(axis=0)


def cut_scale(s):
    """A float32 scale to the 20 significant bits that are kept, nearest."""
    bits = (np.asarray(s, np.float32).view(np.uint32).astype(np.uint64) + 8) & 0xFFFFFFF0
    return bits.astype(np.uint32).view(np.float32)


def quantize_w4(w, group, scale=None, zero=None):
    """(codes [N, K], scale, zero [N, G]) of float32 weights by the binary32 recipe."""
    w = np.asarray(w, np.float32)
    N, K = w.shape
    G = -(-K // group)
    f = np.float32
    codes = np.zeros((N, K), np.uint8)
    given = scale is not None
    s_all = np.asarray(scale, np.float32).copy() if given else np.zeros((N, G), np.float32)
    z_all = np.asarray(zero, np.uint8).copy() if given else np.zeros((N, G), np.uint8)
    for g in range(G):
        part = w[:, g * group:(g + 1) * group]
        if given:
            s, z = cut_scale(s_all[:, g]), np.minimum(z_all[:, g], 15).astype(f)
        else:
            lo = np.minimum(part.min(axis=1), f(0))
            hi = np.maximum(part.max(axis=1), f(0))
            s = cut_scale((hi - lo) / f(15))
            with np.errstate(divide="ignore", invalid="ignore"):
                z = np.where(s > 0, np.clip(np.rint(-lo / s), 0, 15), 0).astype(f)
        with np.errstate(divide="ignore", invalid="ignore"):
            c = np.clip(np.rint(part / s[:, None]) + z[:, None], 0, 15)
        codes[:, g * group:(g + 1) * group] = np.where(s[:, None] != 0, c, z[:, None]).astype(np.uint8)
        s_all[:, g], z_all[:, g] = s, z.astype(np.uint8)
    return codes, s_all, z_all


def unpack_w4(packed, scales, N, K, group):
    """(codes [N, K], scale, zero [N, G]) from the documented format."""
    up = lambda n: (n + 127) // 128 * 128
    Np, Kp = up(N), up(K)
    words = np.asarray(packed).view(np.uint32).reshape(Np // 16, Kp // 128, 4, 16, 4)       # [tile, block, q, r, t]
    codes = np.zeros((Np // 16, 16, Kp // 128, 4, 4, 8), np.uint8)                            # [tile, r, block, t, q, i]
    for i in range(8):
        c = (words >> np.uint32(8 * (i & 3) + 4 * (i >> 2))) & np.uint32(15)
        codes[..., i] = c.transpose(0, 3, 1, 4, 2)
    sc = np.asarray(scales).view(np.uint32).reshape(Np // 16, Kp // group, 16).transpose(0, 2, 1).reshape(Np, Kp // group)
    G = -(-K // group)
    return (codes.reshape(Np, Kp)[:N, :K], (sc & np.uint32(0xFFFFFFF0)).view(np.float32)[:N, :G],
            (sc & np.uint32(15)).astype(np.uint8)[:N, :G])


def levels(codes, scale, zero, group):
    """Real weights [N, K] of codes."""
    K = codes.shape[1]
    of_k = np.arange(K) // group
    return (codes.astype(np.float64) - zero.astype(np.float64)[:, of_k]) * scale.astype(np.float64)[:, of_k]


def linear(x, codes, scale, zero, group, bias=None):
    """(x W^T + bias, sum over groups of s (sum code |x| + z sum |x|)) in float64: the product and the size of its terms."""
    x = np.asarray(x, np.float64)
    K = codes.shape[1]
    of_k = np.arange(K) // group
    out = x @ levels(codes, scale, zero, group).T
    size = np.abs(x) @ ((codes.astype(np.float64) + zero.astype(np.float64)[:, of_k]) * np.abs(scale.astype(np.float64))[:, of_k]).T
    if bias is not None:
        out = out + np.asarray(bias, np.float64)
        size = size + np.abs(np.asarray(bias, np.float64))
    return out, size
