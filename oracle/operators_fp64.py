"""Plain fp64 definitions of the operators around a stage's op graph: values kept in 8 bits, the non-linear parts of a layer
from kept values, norms of queries and keys with the position rotation, the embedding.  Test infrastructure only."""
import numpy as np
from scipy.special import erfc

GPT, LLAMA = 0, 1
BLOCK = 32


def e4m3_values():
    """The non-negative e4m3 numbers in order: sign, 4 exponent bits (bias 7), 3 fraction bits; 0x7f is NaN, 448 the largest."""
    v = []
    for code in range(0x7F):
        e, m = code >> 3, code & 7
        v.append(m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(v)


E4M3 = e4m3_values()


def round_e4m3(y):
    """-> codes of the nearest values, ties to the even code, by looking the value up in the table of all of them."""
    a = np.abs(y)
    hi = np.clip(np.searchsorted(E4M3, a, side="left"), 1, len(E4M3) - 1)
    lo = hi - 1
    dl, dh = a - E4M3[lo], E4M3[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (code | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)


def pack8(x):
    """-> (codes [rows, cols], scales [rows, ceil(cols / 32)], values it stands for)"""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    codes, scales, values = np.zeros((rows, cols), np.uint8), np.zeros((rows, nb), np.uint8), np.zeros((rows, cols))
    powers = np.arange(-117, 120)
    for b in range(nb):
        v = x[:, b * BLOCK:(b + 1) * BLOCK]
        fine = np.isfinite(v)
        most = np.max(np.where(fine, np.abs(v), 0.0), axis=1)
        k = powers[np.minimum(np.searchsorted(448.0 * 2.0 ** powers, most, side="left"), len(powers) - 1)].astype(float)
        p = 2.0 ** k[:, None]
        c = round_e4m3(np.clip(np.where(fine, v, 0.0) / p, -448.0, 448.0))
        c = np.where(fine, c, 0x7F | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)
        codes[:, b * BLOCK:(b + 1) * BLOCK] = c
        scales[:, b] = (k + 127).astype(np.uint8)
        values[:, b * BLOCK:(b + 1) * BLOCK] = np.where(fine, np.where(c & 0x80, -1.0, 1.0) * E4M3[np.minimum(c & 0x7F, 0x7E)] * p, np.nan)
    return codes, scales, values


def activation(family, gu):
    if family == LLAMA:
        g, u = np.split(gu, 2, axis=1)
        return g / (1 + np.exp(-g)) * u
    return gu * 0.5 * erfc(-gu / np.sqrt(2))


def activation_bwd(family, gu, da):
    if family == LLAMA:
        g, u = np.split(gu, 2, axis=1)
        s = 1 / (1 + np.exp(-g))
        return np.concatenate([da * u * s * (1 + g / (1 + np.exp(g))), da * g * s], axis=1)
    return da * (0.5 * erfc(-gu / np.sqrt(2)) + gu * np.exp(-gu * gu / 2) / np.sqrt(2 * np.pi))


def norm_stats(family, x, eps):
    mean = x.mean(1, keepdims=True) if family == GPT else np.zeros((x.shape[0], 1))
    return mean, 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)


def norm(family, x, gamma, beta, mean, r):
    return (x - mean) * r * gamma + (beta if family == GPT else 0.0)


def norm_bwd(family, dn, x, mean, r, gamma, dres):
    """-> dx, dgamma, dbeta with the statistics as given"""
    xh, g = (x - mean) * r, dn * gamma
    dx = g - xh * (g * xh).mean(1, keepdims=True) - (g.mean(1, keepdims=True) if family == GPT else 0.0)
    return r * dx + (0.0 if dres is None else dres), (dn * xh).sum(0), dn.sum(0)


def rope_table(seq, d, base):
    ang = np.arange(seq)[:, None] * base ** (-2.0 * np.arange(d // 2) / d)
    return np.stack([np.cos(ang), np.sin(ang)], -1)


def rotate(x, table, seq, sign=1):
    """x [rows, heads, d]; element k of a head with k + d / 2, position = row % seq"""
    d = x.shape[-1]
    c, s = (table[np.arange(x.shape[0]) % seq][:, None, :, i] for i in (0, 1))
    lo, hi = x[..., :d // 2], x[..., d // 2:]
    return np.concatenate([lo * c - sign * hi * s, hi * c + sign * lo * s], -1)


def gains(gq, gk, n_q, n_kv):
    return np.concatenate([np.broadcast_to(gq, (n_q, len(gq))), np.broadcast_to(gk, (n_kv, len(gk)))])


def qknorm_stats(x, n_rot, d, eps):
    h = x.reshape(len(x), -1, d)[:, :n_rot]
    return 1 / np.sqrt((h * h).mean(2) + eps)


def qknorm(x, r, gq, gk, table, seq, n_q, n_kv, d):
    h = x.reshape(len(x), -1, d)
    n = rotate(h[:, :n_q + n_kv] * r[:, :, None] * gains(gq, gk, n_q, n_kv), table, seq)
    return np.concatenate([n, h[:, n_q + n_kv:]], 1).reshape(len(x), -1)


def qknorm_bwd(dy, x, r, gq, gk, table, seq, n_q, n_kv, d):
    """-> dx, dgamma_q, dgamma_k"""
    n_rot = n_q + n_kv
    h, dh = x.reshape(len(x), -1, d), dy.reshape(len(x), -1, d)
    dn, xh = rotate(dh[:, :n_rot], table, seq, -1), h[:, :n_rot] * r[:, :, None]
    g = dn * gains(gq, gk, n_q, n_kv)
    dx = r[:, :, None] * (g - xh * (g * xh).mean(2, keepdims=True))
    dgain = (dn * xh).sum(0)
    return np.concatenate([dx, dh[:, n_rot:]], 1).reshape(len(x), -1), dgain[:n_q].sum(0), dgain[n_q:].sum(0)


def embed(ids, weight, scale):
    ok = (ids >= 0) & (ids < len(weight))
    return np.where(ok[:, None], weight[np.where(ok, ids, 0)] * scale, 0.0)


def embed_bwd(ids, dy, vocab, scale):
    grad = np.zeros((vocab, dy.shape[1]))
    for r, t in enumerate(ids):
        if 0 <= t < vocab:
            grad[t] += scale * dy[r]
    return grad
