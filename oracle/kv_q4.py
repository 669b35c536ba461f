"""A KV cache in 4 bits in plain 64-bit arithmetic: what codes and scales stand for, how a row is rounded to them, attention over them and sequences
moved between places.  Shares no code with the library."""
import numpy as np

from oracle.forward import bf16_round

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _e4m3(code):
    e, m = code >> 3 & 15, code & 7
    v = np.nan if code & 127 == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    return -v if code & 128 else v


E4M3 = np.array([_e4m3(c) for c in range(256)])


def nearest_even(x, levels):
    """Index of the nearest of ascending levels for x >= 0, the even index of two equally near ones, the last one beyond them."""
    above = np.clip(np.searchsorted(levels, x), 1, len(levels) - 1)
    up, down = levels[above] - x, x - levels[above - 1]
    return np.where((up < down) | ((up == down) & (above % 2 == 0)), above, above - 1)


def quantise(x, exp):
    """Rows x [..., Dh], already rounded to bf16, as codes [..., Dh / 2] and scales [..., Dh / 16], both uint8."""
    g = (np.asarray(x, np.float64) * 2.0 ** -exp).reshape(*x.shape[:-1], -1, 16)
    top = np.abs(g).max(-1)
    bad = ~np.isfinite(np.asarray(x, np.float64).reshape(g.shape)).all(-1)
    scale = np.where(bad, 127, nearest_even(np.where(bad, 0.0, top) / 6, E4M3[:127])).astype(np.uint8)
    s = np.where(bad, 0.0, E4M3[scale])[..., None]
    q = np.where(s > 0, np.where(bad[..., None], 0.0, g) / np.where(s > 0, s, 1.0), 0.0)
    code = nearest_even(np.abs(q), LEVELS) + np.where(np.signbit(q), 8, 0)
    code = code.reshape(*x.shape[:-1], -1, 2)
    return (code[..., 0] + 16 * code[..., 1]).astype(np.uint8), scale


def pages(codes, scales):
    """Codes [..., TK, Dh / 2] and scales [..., TK, Dh / 16] as pages [..., bytes]."""
    flat = lambda a: a.reshape(*a.shape[:-2], -1)                        # noqa: E731
    return np.concatenate((flat(codes), flat(scales)), -1)


def split(pages_, TK, Dh):
    n = TK * Dh // 2
    return pages_[..., :n].reshape(*pages_.shape[:-1], TK, Dh // 2), pages_[..., n:].reshape(*pages_.shape[:-1], TK, Dh // 16)


def values(codes, scales, exp):
    nib = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)
    v = np.where(nib >= 8, -1.0, 1.0) * LEVELS[nib & 7]
    return v * np.repeat(E4M3[scales], 16, -1) * 2.0 ** exp


def rotate(x, cos, sin):
    """x [..., Dh] fp32 by cos, sin [..., Dh / 2] fp32: each result rounded to fp32 and then to bf16, from sums of exact products."""
    x, c, s = (np.asarray(a, np.float64) for a in (x, cos, sin))
    h = x.shape[-1] // 2
    lo, hi = x[..., :h], x[..., h:]
    with np.errstate(invalid="ignore"):
        return bf16_round(np.concatenate((lo * c - hi * s, hi * c + lo * s), -1).astype(np.float32))


def attention(q, K, V, first):
    """q [S, Hq, Dh] at positions first ... first + S - 1 over K, V [Hkv, n, Dh]: the result, and for every element the weighted mean of |V|, for every row
    the largest sum of |q k| / sqrt(Dh), and for every element the sum of |V|, which errors are bounded by."""
    S, Hq, Dh = q.shape
    G, n = Hq // K.shape[0], first + S
    out, mean, sums = np.zeros((3, S, Hq, Dh))
    most = np.zeros((S, Hq))
    for h in range(Hq):
        k, v = K[h // G, :n], V[h // G, :n]
        for t in range(S):
            m = first + t + 1
            s = k[:m] @ q[t, h] / np.sqrt(Dh)
            p = np.exp(s - s.max())
            out[t, h], mean[t, h] = p @ v[:m] / p.sum(), p @ np.abs(v[:m]) / p.sum()
            most[t, h] = (np.abs(k[:m]) @ np.abs(q[t, h])).max() / np.sqrt(Dh)
            sums[t, h] = np.abs(v[:m]).sum(0)
    return out, mean, most, sums


def moved(tiles, pairs, TK, length, widths):
    """tiles [n_tiles, B, Hkv, bytes] with the pairs (from, to; from -1: zeros) carried out on the first `length` positions; widths: bytes of a position in each
    of the page's parts."""
    out = tiles.copy()
    for j in range(len(tiles)):
        used = max(0, min(TK, length - j * TK))
        at = 0
        for w in widths:
            for a, b in pairs:
                out[j, b, :, at:at + used * w] = 0 if a < 0 else tiles[j, a, :, at:at + used * w]
            at += TK * w
    return out
