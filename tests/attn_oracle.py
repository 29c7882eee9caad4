"""Plain attention and cache append in 64 bits on the CPU, sequence by
sequence and row by row of the definition, and error bounds of the 16-bit
kernels that follow from their arithmetic."""

import numpy as np
import torch

# Rounding to nearest with a significand of 8 or 11 bits: relative error at most 2^-8 or 2^-11 in the normal range, and
# half of the smallest step below it (float16: 2^-25; bfloat16's is under every bound here).
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = 2.0 ** -25


def attend(q, keys, values, seen, scale):
    """One sequence: q [n, hq, d], keys and values [L, hkv, d] float64, seen[i] keys for row i.
    Returns out, lse and the bound of the kernel's absolute error of both."""
    n, hq, d = q.shape
    G = hq // keys.shape[1] if keys.shape[1] else 1
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    tol, tol_lse = np.zeros((n, hq, d)), np.zeros((n, hq))
    for h in range(hq):
        k, v = keys[:, h // G], values[:, h // G]
        for i in range(n):
            m = int(seen[i])
            if m <= 0:
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                s = scale * (k[:m] @ q[i, h])
                top = s.max()
                p = np.exp(s - top)
                lse[i, h] = top + np.log(p.sum())
                p /= p.sum()
                out[i, h] = p @ v[:m]
                # float32 sums of d products, the exponent's rounding, exp2 and the sum over the keys
                ds = scale * (d + 2) * 2.0 ** -24 * (np.abs(k[:m]) @ np.abs(q[i, h])).max() + 2.0 ** -22 * (1 + np.abs(s).max())
                tol_lse[i, h] = 2 * ds + (m + 64) * 2.0 ** -24
                tol[i, h] = (2 * ds + (m + 64) * 2.0 ** -24) * (p @ np.abs(v[:m]))
                # weights below the type's normal range keep an absolute error
                tol[i, h] += 2.0 ** -25 * np.abs(v[:m]).sum(0)
                tol[i, h] += 1e-30
    return out, lse, tol, tol_lse


def bound(tol, out, weighted, unit):
    """Adds the roundings to the operands' type: the weights' (on sum p |v|) and the result's."""
    return tol + unit * (np.abs(out) + weighted) + np.where(tol > 0, TINY, 0)


def paged(q, k_cache, v_cache, off, kv_len, pages, scale):
    """(out, lse, bound of out, bound of lse) of fate_attn_paged, all float64 numpy; inputs CPU tensors."""
    unit, P = UNIT[q.dtype], k_cache.shape[2]
    qd, kc, vc = q.double().numpy(), k_cache.double().numpy(), v_cache.double().numpy()
    T, hq, d = q.shape
    out, lse = np.zeros((T, hq, d)), np.full((T, hq), -np.inf)
    tol, tol_lse = np.zeros((T, hq, d)), np.zeros((T, hq))
    for b in range(len(kv_len)):
        lo, hi, L = off[b], off[b + 1], kv_len[b]
        at = [(pages[b][j // P], j % P) for j in range(L)]
        keys = np.stack([kc[p, :, s] for p, s in at]) if L else np.zeros((0, kc.shape[1], d))
        vals = np.stack([vc[p, :, s] for p, s in at]) if L else np.zeros((0, kc.shape[1], d))
        seen = L - (hi - lo) + 1 + np.arange(hi - lo)
        o, s, t, tl = attend(qd[lo:hi], keys, vals, seen, scale)
        w = attend(qd[lo:hi], keys, np.abs(vals), seen, scale)[0]
        out[lo:hi], lse[lo:hi], tol[lo:hi], tol_lse[lo:hi] = o, s, bound(t, o, w, unit), tl
    return out, lse, tol, tol_lse


def prompt(q, k, v, off, scale):
    unit = UNIT[q.dtype]
    qd, kd, vd = q.double().numpy(), k.double().numpy(), v.double().numpy()
    T, hq, d = q.shape
    out, lse = np.zeros((T, hq, d)), np.full((T, hq), -np.inf)
    tol, tol_lse = np.zeros((T, hq, d)), np.zeros((T, hq))
    for lo, hi in zip(off[:-1], off[1:]):
        seen = 1 + np.arange(hi - lo)
        o, s, t, tl = attend(qd[lo:hi], kd[lo:hi], vd[lo:hi], seen, scale)
        w = attend(qd[lo:hi], kd[lo:hi], np.abs(vd[lo:hi]), seen, scale)[0]
        out[lo:hi], lse[lo:hi], tol[lo:hi], tol_lse[lo:hi] = o, s, bound(t, o, w, unit), tl
    return out, lse, tol, tol_lse


def rotate(x, pos, table, interleaved):
    """x [n, h, d] float64 rotated to positions pos: (rotated, bound of the float32 error before the rounding)."""
    rot = table.shape[1]
    half = rot // 2
    y, err = x.copy(), np.zeros_like(x)
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        c, s = table[pos, j][:, None], table[pos, half + j][:, None]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        err[..., a] = err[..., b] = 2.0 ** -22 * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, err
