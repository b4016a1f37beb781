"""Plain 64-bit forms of the router with scores and of the 8-bit path, for the GPU tests: definitions written out with torch and numpy,
and how far a result in 32 bits may be off."""
from __future__ import annotations

import numpy as np
import torch

BLOCK, TOP = 128, 448.0


# ---- gating ---------------------------------------------------------------------------------------
def route(z, bias, layer_of_token, K, sigmoid, n_group, topk_group, group_top, renorm, scale):
    """idx [T, K] (-1: empty), w [T, K]; z float64 [T, E]."""
    z = np.asarray(z, np.longdouble)
    T, E = z.shape
    z = np.where(np.isnan(z), -np.inf, np.minimum(z, float(np.finfo(np.float32).max)))
    dead = np.isneginf(z)
    if sigmoid:
        with np.errstate(over="ignore"):
            s = 1 / (1 + np.exp(-z))
    else:
        top = np.where(dead.all(1), 0, z.max(1))
        p = np.exp(z - top[:, None])
        s = p / np.maximum(p.sum(1, keepdims=True), 1e-300)
    # without a bias scores order like the logits, however near to 0 or 1 they lie
    c = z.copy() if bias is None and (n_group == 1 or group_top == 1) else s + (0 if bias is None else np.asarray(bias, np.longdouble)[layer_of_token])
    with np.errstate(invalid="ignore"):
        c = np.where(dead | np.isnan(c), -np.inf, c)
    idx, w = np.full((T, K), -1), np.zeros((T, K))
    size = E // n_group
    for t in range(T):
        value = []
        for g in range(n_group):
            best = sorted([v for v in c[t, g * size:(g + 1) * size] if v > -np.inf], reverse=True)[:group_top]
            value.append(sum(best) if best else -np.inf)
        kept = sorted(range(n_group), key=lambda g: (-value[g], g))[:topk_group]
        open_ = [e for g in kept for e in range(g * size, (g + 1) * size) if c[t, e] > -np.inf]
        chosen = sorted(open_, key=lambda e: (-c[t, e], e))[:K]
        idx[t, :len(chosen)] = chosen
        if not chosen:
            continue
        if renorm:   # ratios of scores, which have a value where the scores themselves vanish
            zc = z[t, chosen]
            shift = zc.max()
            r = np.exp(zc - shift) / (1 + np.exp(zc)) if sigmoid and shift < 0 else (s[t, chosen] if sigmoid else np.exp(zc - shift))
            w[t, :len(chosen)] = scale * r / r.sum()
        else:
            w[t, :len(chosen)] = scale * s[t, chosen]
    return idx, w


# ---- e4m3 -----------------------------------------------------------------------------------------
def nearest_e4m3(v):
    """float64 values to the nearest e4m3 value, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def spread(t, dim):
    """Scales to elements along `dim`."""
    return t.repeat_interleave(BLOCK, dim)


def quantise_rows(x):
    """float64 [R, n] -> (e4m3 values as float64, scales [R, blocks]).  The product with 448 comes first: the quotient is then exact where
    it lies halfway between two e4m3 values, for bf16 elements."""
    R, n = x.shape
    b = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(R, -1, BLOCK)
    m = b.abs().amax(2)
    q = nearest_e4m3(torch.where(m[..., None] > 0, b * TOP / m[..., None], 0.0))
    return q.view(R, -1)[:, :n], m / TOP


def quantise_weights(w):
    N, K = w.shape
    b = torch.nn.functional.pad(w, (0, -K % BLOCK, 0, -N % BLOCK)).view(-(-N // BLOCK), BLOCK, -(-K // BLOCK), BLOCK)
    m = b.abs().amax((1, 3), keepdim=True)
    q = nearest_e4m3(torch.where(m > 0, b * TOP / m, 0.0))
    return q.reshape(-(-N // BLOCK) * BLOCK, -1)[:N, :K], (m / TOP).view(-(-N // BLOCK), -1)


def values(q, s):
    """float64 values of an e4m3 matrix with a scale per 128 x 128 block."""
    return q.double() * spread(spread(s.double(), 0), 1)[:q.shape[0], :q.shape[1]]


def ffn(xq, xs, gate, up, down):
    """One expert on rows.  xq e4m3 [R, H], xs f32 [R, blocks]; gate, up, down: (q, scales).  Returns y in 64 bits and a bound on how far a
    result may be off that sums in 32 bits (below) and rounds to bf16.

    The error of a sum of n terms in 32 bits is at most n 2^-24 times the sum of their magnitudes (first order), twice that if each addition
    truncates.  gate and up are sums over H in blocks: dg = 2 (H + 8) 2^-24 |x| |Wg|, du alike.  h = silu(g) u is off by at most
    1.1 |u| dg + |silu(g)| du + |h| 2^-20 (exponential, quotient and product: |g| below 16 here), which for the value that is
    rounded to e4m3 adds to the relative error of the block's maximum.  Where such an interval holds a rounding border its two
    ends round to different values: their distance, times |Wd|, is what the row's sum may be off."""
    H, I = xq.shape[1], gate[0].shape[0]
    x = xq.double() * spread(xs.double(), 1)[:, :H]
    wg, wu, wd = values(*gate), values(*up), values(*down)
    g, u = x @ wg.T, x @ wu.T
    eps = 2.0 ** -24
    dg, du = 2 * (H + 8) * eps * (x.abs() @ wg.abs().T), 2 * (H + 8) * eps * (x.abs() @ wu.abs().T)
    sg = g * torch.sigmoid(g)
    h = sg * u
    dh = 1.1 * u.abs() * dg + sg.abs() * du + 1.1 * dg * du + h.abs() * 2.0 ** -20
    pad = lambda t: torch.nn.functional.pad(t, (0, -I % BLOCK)).view(len(t), -1, BLOCK)  # noqa: E731
    hb, db = pad(h), pad(dh)
    m, at = hb.abs().max(2, keepdim=True)
    unit = torch.where(m > 0, TOP / m, 0.0)
    dm = db.amax(2, keepdim=True)            # no maximum moves further than its largest element may
    off = db + hb.abs() * dm / m.clamp_min(1e-300)
    q = nearest_e4m3(hb * unit)
    lo, hi = nearest_e4m3(((hb - off) * unit).clamp(-TOP, TOP)), nearest_e4m3(((hb + off) * unit).clamp(-TOP, TOP))
    flat = lambda t: t.reshape(len(t), -1)[:, :I]  # noqa: E731
    a = flat(q / unit.clamp_min(1e-300))
    da = flat((hi - lo) / unit.clamp_min(1e-300)) + a.abs() * flat((dm / m.clamp_min(1e-300)).expand_as(hb))
    y = a @ wd.T
    tol = da @ wd.abs().T + 2 * (I + 8) * eps * (a.abs() @ wd.abs().T)
    return y, tol + 2.0 ** -8 * (y.abs() + tol) + 1e-30
