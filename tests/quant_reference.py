"""The 8-bit KV cache's operations in float64, written from their definitions:
e4m3 by its table of values, stores block by block, attention row by row."""

import numpy as np


def e4m3_table():
    """The value of each of the 256 codes (1 sign, 4 exponent, 3 significand
    bits, bias 7, subnormals; exponent and significand all ones: NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


TABLE = e4m3_table()
_POS = TABLE[:127]                       # ascending, 0 .. 448
_MID = (_POS[1:] + _POS[:-1]) / 2        # exact in float64


def encode(y):
    """Codes of float64 y, |y| <= 448 or NaN: nearest, the even code at ties."""
    a = np.abs(y)
    i = np.searchsorted(_MID, a, side="left")      # a in (mid[i-1], mid[i]]
    tie = (i < _MID.size) & (a == _MID[np.minimum(i, _MID.size - 1)])
    i = np.where(tie & (i % 2 == 1), i + 1, i)
    i = np.where(np.isnan(y), 127, i)
    return (i | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def exponent(amax):
    """The smallest e with amax <= 448 * 2^e, within [-117, 119]."""
    e = -117
    while e < 119 and amax > 448.0 * 2.0 ** e:
        e += 1
    return e


class Cache:
    """codes [n_slots, heads, d] and scales [blocks, heads] of K or V."""

    def __init__(self, codes, scales, block):
        self.codes, self.scales, self.block = codes.copy(), scales.astype(np.float64).copy(), block

    def store(self, x, slots):
        """x [n, heads, d] float64 (infinities and NaN allowed)."""
        n_slots, heads = self.codes.shape[:2]
        row = {}
        for i, s in enumerate(slots):
            if 0 <= s < n_slots:
                row[int(s)] = i  # the last of equal slots
        blocks = {}
        for s in row:
            blocks.setdefault(s // self.block, []).append(s)
        for b, named in blocks.items():
            everything = range(b * self.block, min((b + 1) * self.block, n_slots))
            rest = [s for s in everything if s not in row]
            rows = x[[row[s] for s in named]]
            for g in range(heads):
                v = rows[:, g]
                e = exponent(np.max(np.abs(np.where(np.isfinite(v), v, 0.0))))
                old = self.scales[b, g]
                if rest and old > 0:
                    e = max(e, int(np.log2(old)))
                y = np.clip(v * 2.0 ** -e, -448.0, 448.0)
                self.codes[named, g] = encode(np.where(np.isfinite(v), y, np.nan))
                if rest:
                    left = np.zeros((len(rest), v.shape[1])) if old == 0 else TABLE[self.codes[rest, g]] * (old / 2.0 ** e)
                    if old != 2.0 ** e:
                        self.codes[rest, g] = encode(left)
                self.scales[b, g] = 2.0 ** e

    def values(self, slots):
        """[n, heads, d]; zeros outside the cache and in empty blocks."""
        n_slots = self.codes.shape[0]
        slots = np.asarray(slots, dtype=np.int64)
        ok = (slots >= 0) & (slots < n_slots)
        at = np.where(ok, slots, 0)
        sc = self.scales[at // self.block][..., None]
        v = np.where(sc > 0, np.where(sc > 0, sc, 0.0) * np.where(sc > 0, TABLE[self.codes[at]], 0.0), 0.0)
        return np.where(ok[:, None, None], v, 0.0)


def attention(q, k, v, heads_per_kv):
    """One request: q [R, H, d], k and v [S, H_kv, d].  Returns out and lse,
    and for the error bounds sum_j p_j |v_j| and the largest sum_i |q_i k_i|
    (scaled) of each row and head."""
    R, H, d = q.shape
    out, weight = np.empty((R, H, d)), np.empty((R, H, d))
    lse, big = np.empty((R, H)), np.empty((R, H))
    for h in range(H):
        kk, vv = k[:, h // heads_per_kv], v[:, h // heads_per_kv]
        x = q[:, h] @ kk.T / np.sqrt(d)
        m = x.max(1, keepdims=True)
        p = np.exp(x - m)
        t = p.sum(1, keepdims=True)
        lse[:, h] = (m + np.log(t))[:, 0]
        out[:, h] = p @ vv / t
        weight[:, h] = p @ np.abs(vv) / t
        big[:, h] = (np.abs(q[:, h]) @ np.abs(kk).T / np.sqrt(d)).max(1)
    return out, lse, weight, big
