"""Plain 64-bit forms of routing from logits, its gradient, blocks of 8-bit floating point and the experts' products
(test infrastructure only; numpy, written from the definitions in include/pgmoe.h)."""
from __future__ import annotations

import numpy as np

LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
BLOCK = 128


# ------------------------------------------------------------------------------------ routing
def scores(z, kind):
    """z [T, E] -> scores; unavailable experts (NaN or -inf) score 0."""
    z = np.asarray(z, np.float64)
    live = z > -np.inf
    out = np.zeros_like(z)
    for t in range(z.shape[0]):
        if not live[t].any():
            continue
        v = z[t, live[t]]
        if kind == "sigmoid":
            with np.errstate(over="ignore"):
                out[t, live[t]] = 1.0 / (1.0 + np.exp(-v))
        else:
            m = v.max()
            with np.errstate(invalid="ignore"):
                e = np.where(v == m, 1.0, np.exp(v - m))
            out[t, live[t]] = e / e.sum()
    return out


def selected_shares(z, kind):
    """Shares of the selected experts' scores in their sum, from their available logits."""
    with np.errstate(over="ignore", invalid="ignore"):
        ls = z if kind == "softmax" else np.minimum(z, 0) - np.log1p(np.exp(-np.abs(z)))
        m = ls.max()
        e = np.where(ls == m, 1.0, np.exp(ls - m))
    return e / e.sum()


def route(z, kind, k, bias=None, n_groups=1, topk_groups=1, renormalize=False, scale=1.0):
    """-> (idx [T, k], weight [T, k], scores [T, E])."""
    z = np.asarray(z, np.float64)
    T, E = z.shape
    s = scores(z, kind)
    live = z > -np.inf
    if bias is None:
        v, b = z.copy(), np.zeros(E)
    else:
        b = np.where(np.isnan(bias), -np.inf, np.asarray(bias, np.float64))
        v = s + b
    idx = np.zeros((T, k), np.int64)
    for t in range(T):
        tier = np.where(live[t], 1, 0)                       # available before unavailable
        if n_groups > 1:
            size = E // n_groups
            worth = []
            for g in range(n_groups):
                sl = slice(g * size, (g + 1) * size)
                w = np.sort((s[t, sl] + b[sl])[live[t, sl] & (b[sl] > -np.inf)])[::-1][:2]
                worth.append((1, w.sum()) if len(w) else (0, 0.0))
            order = sorted(range(n_groups), key=lambda g: (-worth[g][0], -worth[g][1], g))[:topk_groups]
            kept = np.zeros(n_groups, bool)
            kept[order] = True
            tier = np.where(np.repeat(kept, size), tier, -1)
        key = np.where(tier == 1, v[t], -np.inf)
        idx[t] = sorted(range(E), key=lambda e: (-tier[e], -key[e], e))[:k]
    rows = np.arange(T)[:, None]
    weight = s[rows, idx]
    if renormalize:
        weight = np.zeros((T, k))
        for t in range(T):
            zt = z[t, idx[t]]
            on = zt > -np.inf
            if on.any():
                weight[t, on] = selected_shares(zt[on], kind)
    return idx, scale * weight, s


def route_loss_gradient(z, idx, kind, d_weight, d_scores=None, renormalize=False, scale=1.0):
    """-> (gradient of the logits, the sum of the magnitudes of the terms it is made of)."""
    z = np.asarray(z, np.float64)
    s = scores(z, kind)
    T, E = z.shape
    ds, mag = np.zeros((T, E)), np.zeros((T, E))
    if d_scores is not None:
        ds, mag = np.where(s > 0, np.asarray(d_scores, np.float64), 0.0), np.where(s > 0, np.abs(d_scores), 0.0).astype(np.float64)
    through, mthrough = np.zeros((T, E)), np.zeros((T, E))  # s * d_s of the selected, renormalised: finite where the s are not told from 0
    for t in range(T):
        on = [j for j, e in enumerate(idx[t]) if 0 <= e < E and z[t, e] > -np.inf]
        if not on:
            continue
        at, dw = idx[t, on], np.asarray(d_weight, np.float64)[t, on]
        if renormalize:
            r = selected_shares(z[t, at], kind)
            np.add.at(through[t], at, scale * r * (dw - (dw * r).sum()))
            np.add.at(mthrough[t], at, abs(scale) * r * (np.abs(dw) + (np.abs(dw) * r).sum()))
        else:
            np.add.at(ds[t], at, scale * dw)
            np.add.at(mag[t], at, np.abs(scale * dw))
    if kind == "softmax":
        return s * (ds - (s * ds).sum(1, keepdims=True)) + through, s * (mag + (s * mag).sum(1, keepdims=True)) + mthrough
    return (1 - s) * (s * ds + through), (1 - s) * (s * mag + mthrough)


# ------------------------------------------------------------------------------------ 8 bits
def round_to(v, kind):
    """Float64 -> the nearest value of the type, ties to even; NaN stays, infinities become NaN (e4m3) or stay (e5m2)."""
    v = np.asarray(v, np.float64)
    digits, least = (4, -6) if kind == "e4m3" else (3, -14)
    fine = np.isfinite(v)
    step = np.exp2(np.maximum(np.frexp(np.where(fine, v, 0.0))[1] - 1, least) - (digits - 1.0))
    out = np.where(fine, np.rint(np.where(fine, v, 0.0) / step) * step, v)
    return np.where(np.isinf(v), np.nan, out) if kind == "e4m3" else out


def block_codes(x, kind):
    """x [.., block]: float32 values of one block each -> (codes' values float64, scales float32 [..])."""
    x = np.asarray(x, np.float32)
    mag = np.where(np.isfinite(x), np.abs(x), np.float32(0)).max(axis=-1).astype(np.float32)
    scale = np.maximum(mag / np.float32(LARGEST[kind]), np.float32(2.0 ** -126))
    with np.errstate(invalid="ignore"):
        return round_to(np.float64(x / scale[..., None]), kind), scale


def pad_to(a, n, axis):
    widths = [(0, 0)] * a.ndim
    widths[axis] = (0, n - a.shape[axis])
    return np.pad(a, widths)


def quantize_rows(x, kind):
    """x [T, d] float32 -> (codes' values [T, 128 * blocks], scales [blocks, T])."""
    T, d = x.shape
    blocks = -(-d // BLOCK)
    q, s = block_codes(pad_to(np.asarray(x, np.float32), blocks * BLOCK, 1).reshape(T, blocks, BLOCK), kind)
    return q.reshape(T, -1), s.T


def tile_positions(n_in, n_out):
    """[n_in, n_out] -> byte of that code inside one expert's operand tiles."""
    kb = -(-n_in // BLOCK)
    i, o = np.arange(n_in)[:, None], np.arange(n_out)[None, :]
    return ((o // 16) * kb + i // 128) * 2048 + (i % 128 // 64) * 1024 + (i % 64 // 16) * 256 + (o % 16) * 16 + i % 16


def quantize_weights(w):
    """w [E, n_in, n_out] float32 -> (codes' values [E, n_in, n_out], scales [E, out blocks, in blocks])."""
    E, n_in, n_out = w.shape
    kb, nb = -(-n_in // BLOCK), -(-n_out // BLOCK)
    p = pad_to(pad_to(np.asarray(w, np.float32), kb * BLOCK, 1), nb * BLOCK, 2).reshape(E, kb, BLOCK, nb, BLOCK).transpose(0, 1, 3, 2, 4)
    q, s = block_codes(p.reshape(E, kb, nb, BLOCK * BLOCK), "e4m3")
    q = q.reshape(E, kb, nb, BLOCK, BLOCK).transpose(0, 1, 3, 2, 4).reshape(E, kb * BLOCK, nb * BLOCK)
    return q[:, :n_in, :n_out], s.transpose(0, 2, 1)


def expert_matmul(x, x_scale, w, w_scale, offsets, relu=False):
    """x [R, n_in] codes' values, x_scale [blocks, R], w [E, n_in, n_out] codes' values, w_scale [E, out blocks, in blocks]
    -> (y [R, n_out] float64, the sum of the magnitudes of the products; rows of no expert are NaN)."""
    R, n_in = x.shape
    n_out = w.shape[2]
    y, mag = np.full((R, n_out), np.nan), np.zeros((R, n_out))
    xs = x * np.repeat(np.asarray(x_scale, np.float64).T, BLOCK, axis=1)[:, :n_in]
    for e in range(w.shape[0]):
        lo, hi = offsets[e], offsets[e + 1]
        ws = w[e] * np.repeat(np.repeat(np.asarray(w_scale[e], np.float64).T, BLOCK, 0)[:n_in], BLOCK, 1)[:, :n_out]
        y[lo:hi] = xs[lo:hi] @ ws
        mag[lo:hi] = np.abs(xs[lo:hi]) @ np.abs(ws)
    return (np.where(y < 0, 0.0, y) if relu else y), mag
