"""CPU oracle for the operators of an MoE block beside the DTS gate: gate logits, top-k gate, residual + RMS norm, 8-bit values
and the expert FFNs on them.  TEST INFRASTRUCTURE ONLY, as evomoe_oracle.py: float64 numpy, plain and slow.

Beside each value that is compared with a float32 computation a function returns, where the tests need it, the sum of
the magnitudes that went into it: what a bound of the rounding error is a multiple of.
"""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np

from oracle import evomoe_oracle as orc

F64 = np.float64


# ---- top-k gate --------------------------------------------------------------------------------------

@dataclass
class TopK:
    k: int
    score: str = "softmax"
    groups: int = 1
    top_groups: int = 1
    group_keys: int = 1
    renormalise: bool = True
    scale: float = 1.0


def scores(z, score):
    z = np.asarray(z, F64)
    with np.errstate(all="ignore"):
        if score == "sigmoid":
            return np.where(z >= 0, 1 / (1 + np.exp(-z)), np.where(np.isnan(z), z, np.exp(np.minimum(z, 0)) / (1 + np.exp(np.minimum(z, 0)))))
        m = np.max(z, axis=-1, keepdims=True)
        e = np.exp(z - np.where(np.isneginf(m), 0, m))
        s = e.sum(-1, keepdims=True)
        return np.where(s == 0, 0, e / np.where(s == 0, 1, s))


def _descending(key):
    """Indices by falling key, ties by index."""
    return sorted(range(len(key)), key=lambda i: (-key[i], i))


def topk_select(z, bias, o: TopK):
    """mask [T,E]: token by token, as the definition reads."""
    z = np.asarray(z, F64)
    T, E = z.shape
    s = scores(z, o.score)
    mask = np.zeros((T, E), bool)
    for t in range(T):
        key = z[t].copy() if bias is None and o.groups == 1 else s[t] + (0 if bias is None else np.asarray(bias, F64))
        key[np.isnan(key)] = np.inf
        key[np.isneginf(z[t])] = -np.inf
        if bias is not None:
            key[np.isneginf(bias)] = -np.inf
        if o.groups > 1:
            size, worth = E // o.groups, []
            for n in range(o.groups):
                best = [v for v in sorted(key[n * size:(n + 1) * size], reverse=True)[:o.group_keys] if v > -np.inf]
                worth.append(sum(best) if best else -np.inf)
            kept = set(_descending(worth)[:o.top_groups])
            for e in range(E):
                if e // size not in kept:
                    key[e] = -np.inf
        for e in _descending(key)[:o.k]:
            mask[t, e] = key[e] > -np.inf
    return mask


def _shares(z, mask, o: TopK):
    """w^: scores of the selected, renormalised or not; a ratio is taken between logarithms of scores."""
    s = scores(z, o.score)
    if not o.renormalise:
        return np.where(mask, s, 0)
    with np.errstate(all="ignore"):
        log = z if o.score == "softmax" else -np.logaddexp(0, -z)
        log = np.where(mask, log, -np.inf)
        top = log.max(1, keepdims=True)
        e = np.where(mask, np.exp(log - np.where(np.isneginf(top), 0, top)), 0)
        return np.where(mask, e / np.where(mask.any(1, keepdims=True), e.sum(1, keepdims=True), 1), 0)


def topk_weights(z, mask, o: TopK):
    return o.scale * _shares(np.asarray(z, F64), mask, o)


def topk_bwd(z, mask, dG, o: TopK, coef=None):
    """dlogits from dG [T,E] (read where selected), and the magnitudes that went into it."""
    z, s = np.asarray(z, F64), scores(z, o.score)
    w, dG = _shares(z, mask, o), np.where(mask, np.asarray(dG, F64), 0)
    c = 0 if coef is None else np.asarray(coef, F64)[None, :]
    if o.renormalise:
        u, mu = o.scale * w * (dG - (w * dG).sum(1, keepdims=True)), o.scale * w * (abs(dG) + (w * abs(dG)).sum(1, keepdims=True))
    else:
        u, mu = o.scale * w * dG, o.scale * w * abs(dG)
    u, mu = np.where(mask, u, 0), np.where(mask, mu, 0)          # (a NaN weight of the token's others is not theirs)
    v, mv = u + s * c, mu + s * abs(c)
    if o.score == "softmax":
        return v - s * v.sum(1, keepdims=True), mv + s * mv.sum(1, keepdims=True)
    with np.errstate(all="ignore"):
        rest = scores(-z, "sigmoid")
    return v * rest, mv * rest


# ---- gate logits ---------------------------------------------------------------------------------------

def logits(x, Wg, bg):
    """Values and magnitudes."""
    x, Wg = np.asarray(x, F64), np.asarray(Wg, F64)
    b = 0 if bg is None else np.asarray(bg, F64)[None, :]
    return x @ Wg + b, abs(x) @ abs(Wg) + abs(b)


def logits_bwd(dz, x, Wg, dx_in):
    """(dWg, dbg, dx) and their magnitudes."""
    dz, x, Wg = (np.asarray(a, F64) for a in (dz, x, Wg))
    d = 0 if dx_in is None else np.asarray(dx_in, F64)
    return ((x.T @ dz, dz.sum(0), d + dz @ Wg.T), (abs(x).T @ abs(dz), abs(dz).sum(0), abs(d) + abs(dz) @ abs(Wg).T))


# ---- norm ------------------------------------------------------------------------------------------------

def rmsnorm(h, gamma, eps):
    """(y, rstd) of rows that are already summed and rounded."""
    h = np.asarray(h, F64)
    rstd = 1 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return h * rstd * np.asarray(gamma, F64), rstd


def rmsnorm_bwd(dy, dh, h, gamma, eps):
    """(dx, dgamma) and their magnitudes."""
    dy, h, gamma = (np.asarray(a, F64) for a in (dy, h, gamma))
    d = 0 if dh is None else np.asarray(dh, F64)
    _, rstd = rmsnorm(h, gamma, eps)
    n = h * rstd
    g = gamma * dy
    dx = d + rstd * (g - n * (g * n).mean(1, keepdims=True))
    mag = abs(d) + rstd * (abs(g) + abs(n) * abs(g * n).mean(1, keepdims=True))
    return (dx, (dy * n).sum(0)), (mag, abs(dy * n).sum(0))


# ---- 8-bit values ------------------------------------------------------------------------------------------

def e4m3(v):
    """v rounded to nearest even among the e4m3 numbers (magnitudes up to 448)."""
    v = np.asarray(v, F64)
    step = np.exp2(np.floor(np.log2(np.maximum(abs(v), 2.0 ** -6))) - 3)
    return np.round(v / step) * step


def mx8_scale(amax):
    """The smallest power of two, 2^-127 at least, with amax / scale <= 448."""
    m, e = np.frexp(np.asarray(amax, F64))               # amax = m 2^e, 448 = 0.875 2^9
    return np.exp2(np.where(amax > 0, np.maximum(e - 9 + (m > 0.875), -127), -127).astype(F64))


def mx8(v):
    """(elements [.., n], scales [.., n/32]); what is not finite becomes NaN and has no part in the scale."""
    v = np.asarray(v, F64)
    g = v.reshape(*v.shape[:-1], -1, 32)
    ok = np.isfinite(g)
    scale = mx8_scale(np.where(ok, abs(g), 0).max(-1))
    q = np.where(ok, e4m3(np.where(ok, g, 0) / scale[..., None]), np.nan)
    return q.reshape(v.shape), scale


def mx8_value(q, scale):
    return np.asarray(q, F64) * np.repeat(np.asarray(scale, F64), 32, axis=-1)


def experts_mx8(x, pair_token, offsets, W1, b1, W2, b2, act, eps_sum, eps_act):
    """O from x, W1, W2 that are 8-bit values already, and a bound of what a computation with sums of relative error eps_sum
    (of the sum of magnitudes) and an activation of error eps_act max(|h|, 4.2) may differ by: act(H) may round to another
    8-bit value, or its group to another scale, where such an error takes it across a border."""
    x, W1, W2 = (np.asarray(a, F64) for a in (x, W1, W2))
    P, d = int(offsets[-1]), W2.shape[1]
    O, bound = np.zeros((P, d)), np.zeros((P, d))
    for e in range(len(offsets) - 1):
        r = slice(int(offsets[e]), int(offsets[e + 1]))
        if r.start == r.stop:
            continue
        rows = x if pair_token is None else x[pair_token[r]]
        rows = rows[r] if pair_token is None else rows
        c1, c2 = (0 if b is None else np.asarray(b, F64)[e][None, :] for b in (b1, b2))
        H = rows @ W1[e].T + c1
        off = 1.13 * eps_sum * (abs(rows) @ abs(W1[e]).T + abs(c1)) + eps_act * np.maximum(abs(H), 4.2)      # |act'| <= 1.13
        A = orc.activation(H, act)
        a = mx8_value(*mx8(A))
        delta = np.zeros_like(a)
        size = abs(A).reshape(A.shape[0], -1, 32)
        o = off.reshape(size.shape)
        for amax in ((size - o).max(-1), (size + o).max(-1)):
            scale = np.repeat(mx8_scale(np.maximum(amax, 0)), 32, axis=-1)
            for end in (A - off, A, A + off):
                delta = np.maximum(delta, abs(e4m3(np.clip(end / scale, -448, 448)) * scale - a))
        O[r] = a @ W2[e].T + c2
        bound[r] = delta @ abs(W2[e]).T + eps_sum * (abs(a) @ abs(W2[e]).T + abs(c2))
    return O, bound


def eights(xq, xs, wq, ws):
    """sum over k of x_rk w_nk of 8-bit values (elements [R,K], [N,K], scales [R,K/32], [N,K/32]) as the matrix instructions for 8-bit
    values bring them to their float32 sums: of eight neighbouring products each is cut off, towards zero, 13 bits below 2^(largest sum of
    the two factors' exponents); a subnormal element's exponent is -6.  Exact but for that; and the magnitudes."""
    exponent = lambda v: np.floor(np.log2(np.maximum(abs(v), 2.0 ** -6)))
    ex, ew = exponent(xq), exponent(wq)
    total, size = (np.zeros((xq.shape[0], wq.shape[0])) for _ in range(2))
    for k in range(0, xq.shape[1], 8):
        p = xq[:, None, k:k + 8] * wq[None, :, k:k + 8]
        e = np.where(p != 0, ex[:, None, k:k + 8] + ew[None, :, k:k + 8], -99).max(-1, keepdims=True)
        step = np.exp2(e - 13)
        s = xs[:, None, k // 32] * ws[None, :, k // 32]
        total += (np.trunc(p / step) * step).sum(-1) * s
        size += abs(p).sum(-1) * s
    return total, size
