"""A cache in blocks, appended to and attended over, and the sampled commit, in plain
float64 from their definitions, with the error bounds the kernels' roundings allow."""

import math

import numpy as np
import torch

# half a step, relative to the value
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def slot(tables, n_blocks, block, b, p):
    """Slot of position p of request b, None if it has none."""
    if p < 0 or p // block >= tables.shape[1]:
        return None
    i = int(tables[b, p // block])
    return i * block + p % block if 0 <= i < n_blocks else None


def rotate(x, pos, base):
    """x [heads, d] float64 turned at pos."""
    d = x.shape[-1]
    a = pos * base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
    lo, hi = x[:, :d // 2], x[:, d // 2:]
    return torch.cat([lo * torch.cos(a) - hi * torch.sin(a), hi * torch.cos(a) + lo * torch.sin(a)], -1)


def rotate_bound(x, ref, half):
    """Angles' sine and cosine are within 2e-7 (a fp32 reduced angle and polynomial), the products and their sum
    round to fp32: 5e-7 of the pair's magnitudes, then the result rounds to its type."""
    d = x.shape[-1]
    pair = x.abs() + x.abs().roll(d // 2, -1)
    return half * ref.abs() + 5e-7 * pair * (1 + half)


def attention(q, key_len, k_pool, v_pool, block, tables, H, G, d, per):
    """(out, lse, bound of out, bound of lse) in float64; q [rows, H d], pools on the CPU."""
    n_blocks = k_pool.shape[0] // block
    half = HALF[q.dtype]
    rows = q.shape[0]
    out, bound = torch.zeros(rows, H, d, dtype=torch.float64), torch.zeros(rows, H, d, dtype=torch.float64)
    lse, lse_bound = torch.full((rows, H), -math.inf, dtype=torch.float64), torch.zeros(rows, H, dtype=torch.float64)
    qd = q.double().view(rows, H, d)
    cap = tables.shape[1] * block
    for b in range(rows // per if per else 0):
        top = min(max(int(key_len[b * per:(b + 1) * per].max()), 0), cap)
        at = [slot(tables, n_blocks, block, b, p) for p in range(top)]
        keep = torch.tensor([a is not None for a in at], dtype=torch.bool)
        idx = torch.tensor([a or 0 for a in at], dtype=torch.int64)
        k = torch.where(keep[:, None], k_pool[idx, :G * d].double(), 0.0).view(top, G, d)
        v = torch.where(keep[:, None], v_pool[idx, :G * d].double(), 0.0).view(top, G, d)
        for r in range(b * per, (b + 1) * per):
            n = min(max(int(key_len[r]), 0), cap)
            if n == 0:
                continue
            for h in range(H):
                kk, vv = k[:n, h // (H // G)], v[:n, h // (H // G)]
                s = kk @ qd[r, h] / math.sqrt(d)
                if bool((s == -math.inf).all()):
                    continue
                lse[r, h] = torch.logsumexp(s, 0)
                p = torch.softmax(s, 0)
                there = s != -math.inf  # a logit of -inf weighs nothing, whatever its value
                w, vv = p[there], vv[there]
                o = (w[:, None] * vv).sum(0)
                a = (w[:, None] * vv.abs()).sum(0)
                # a logit: d products summed in fp32, scaled, and as the exponent of 2 rounded again
                e = ((d + 4) * 2.0 ** -23 * (kk.abs() @ qd[r, h].abs()) / math.sqrt(d)).max()
                e = float(e) + 2.0 ** -21
                # weights and their sum off by e each, sums over n keys in fp32, bf16 weights for the product
                rel = 2 * e + (n + 64) * 2.0 ** -23 + (half if q.dtype == torch.bfloat16 else 0.0)
                out[r, h], bound[r, h] = o, a * rel + half * (o.abs() + a * rel)
                lse_bound[r, h] = e + (n + 64) * 2.0 ** -23 + 2.0 ** -22 * (1 + lse[r, h].abs())
    return out.view(rows, H * d), lse, bound.view(rows, H * d), lse_bound


def sample(x, u, temperature=None, top_k=None, top_p=None, min_p=None, got=None):
    """(token, conf, prob) of each row of x (float64 arrays of the settings, None: off).  A token of `got` is taken
    in place of the drawn one where rounding allows it: a weight is held to 2^-45 of the largest, so n of them and
    u times the kept ones are off by n 2^-45 each, and the token's share of the order has to come within 2 (n + 1)
    2^-45 of u times the kept weight."""
    x = np.asarray(x, dtype=np.float64)
    rows, n = x.shape
    out, conf, prob = np.zeros(rows, np.int64), np.zeros(rows), np.zeros(rows)
    slack = 2 * (n + 1) * 2.0 ** -45
    for i in range(rows):
        v = np.where(np.isnan(x[i]), -np.inf, x[i]) + 0.0
        m = v.max()
        if m == -np.inf:
            low = np.flatnonzero(x[i] == -np.inf)
            out[i] = low[0] if low.size else 0
            continue
        with np.errstate(invalid="ignore"):
            d = np.where(v == m, 0.0, v - m)
        t = 1.0 if temperature is None else temperature[i]
        order = np.argsort(-v, kind="stable")
        with np.errstate(over="ignore", under="ignore"):
            soft = np.exp(d)
            if not t > 0:
                pick, share = order[0], 1.0
            else:
                w = np.where(d == 0, 1.0, np.exp(d / min(t, 3.4028234663852886e38)))[order]
                k = n if top_k is None or top_k[i] <= 0 else min(int(top_k[i]), n)
                c = np.cumsum(w[:k])
                keep = k
                if top_p is not None and top_p[i] < 1:
                    keep = max(1, int((c - w[:k] < max(top_p[i], 0.0) * c[-1]).sum()))
                if min_p is not None and min_p[i] > 0:
                    keep = min(keep, int((w[:keep] >= min(min_p[i], 1.0)).sum()))
                uu = 0.0 if not u[i] > 0 else min(u[i], 1.0)
                at = min(int(np.searchsorted(c[:keep], uu * c[keep - 1], side="right")), keep - 1)
                while w[at] == 0:
                    at -= 1
                if got is not None and order[at] != got[i]:
                    r = int(np.flatnonzero(order == got[i])[0])
                    if r < keep and c[r] - w[r] - slack <= uu * c[keep - 1] <= c[r] + slack:
                        at = r
                pick, share = order[at], w[at] / c[keep - 1]
        out[i], conf[i], prob[i] = pick, soft[pick] / soft.sum(), share
    return out, conf, prob
