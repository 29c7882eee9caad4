"""Plain forms of the calls around a wave's attention, on the CPU: page tables, sequence by sequence."""

import numpy as np

EINVAL, ESIZE = -1, -5


def reserve(new, kv, pages, free, n_free, P, T):
    """off, kv, n_free, taken, slots, positions, pages, status of fate_kv_reserve from lists and arrays."""
    pages, kv = pages.copy(), list(kv)
    B, width, n_pages = len(new), pages.shape[1], len(free)
    usable = n_free if 0 <= n_free <= n_pages else 0
    off, taken, slots, positions, status = [0], [0], [], [], [0] * B
    asked = rows = given = 0
    for b in range(B):
        if new[b] < 0 or kv[b] < 0 or kv[b] + new[b] > width * P:
            status[b] = EINVAL
        else:
            more = -(-(kv[b] + new[b]) // P) - -(-kv[b] // P)
            asked, rows = asked + more, rows + new[b]
            if (more and asked > usable) or rows > T:
                status[b] = ESIZE
            else:
                for x in range(more):
                    pages[b, -(-kv[b] // P) + x] = free[usable - 1 - given - x]
                given += more
                for at in range(kv[b], kv[b] + new[b]):
                    page = int(pages[b, at // P])
                    positions.append(at)
                    slots.append(page * P + at % P if 0 <= page < n_pages else -1)
                    if not 0 <= page < n_pages:
                        status[b] = EINVAL
                kv[b] += new[b]
        off.append(len(positions))
        taken.append(given)
    rest = [-1] * (T - len(slots))
    return (np.array(off), np.array(kv, np.int64).reshape(-1), np.array([n_free - given]), np.array(taken),
            np.array(slots + rest, np.int64), np.array(positions + rest, np.int64), pages, np.array(status, np.int64))


def trim(keep, kv, pages, free, n_free, P):
    """kv, n_free, given, free, status of fate_kv_trim."""
    free, kv = np.array(free), list(kv)
    B, width, n_pages = len(keep), pages.shape[1], len(free)
    given, status, total, asked = [0], [0] * B, 0, 0
    for b in range(B):
        stay = min(keep[b], kv[b])
        ok = keep[b] >= 0 and 0 <= kv[b] <= width * P
        mine = pages[b, -(-stay // P):-(-kv[b] // P)] if ok else []
        ok = ok and all(0 <= p < n_pages for p in mine)
        if ok and len(mine):
            asked += len(mine)
            ok = 0 <= n_free <= n_pages and n_free + asked <= n_pages
        if ok:
            free[n_free + total:n_free + total + len(mine)] = mine
            total += len(mine)
            kv[b] = stay
        else:
            status[b] = EINVAL
        given.append(total)
    return np.array(kv, np.int64).reshape(-1), np.array([n_free + total]), np.array(given), free, np.array(status, np.int64)


def attend_shaped(q, keys, values, pos, prefix, first, scale, cap=0.0, slopes=None):
    """One sequence: q [n, hq, d] at positions pos, keys and values [L, hkv, d], float64.  Returns out, lse, the bounds of the
    kernel's error of both before the roundings to the operands' type, and sum p |v|."""
    n, hq, d = q.shape
    L, hkv = keys.shape[:2]
    j = np.arange(L)
    seen = ((j < prefix) | ((j >= first[:, None]) & (j <= pos[:, None]))) & (pos[:, None] >= 0)
    some = seen.any(1)
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    tol, tol_lse, weighted = np.zeros((n, hq, d)), np.zeros((n, hq)), np.zeros((n, hq, d))
    for h in range(hq):
        if not some.any():
            break
        k, v = keys[:, h // (hq // hkv)], values[:, h // (hq // hkv)]
        k, v = (np.where(seen.any(0)[:, None], x, 0.0) for x in (k, v))  # what no row sees may be anything
        s = scale * (q[:, h] @ k.T)
        # a float32 sum of d products, and the scale
        e = scale * (d + 2) * 2.0 ** -24 * (np.abs(q[:, h]) @ np.abs(k.T)) + 2.0 ** -23 * np.abs(s)
        if cap:
            # argument, exp2, sum and reciprocal are each off by 2^-23 or less of theirs: three steps of 2^-22 of the cap;
            # caps over 100 / log2(e) by the series where the quotient is below 1/4, some roundings of the score itself
            series = (np.abs(s) < 0.25 * cap) & (cap * 1.4426950408889634 > 100)
            s = cap * np.tanh(s / cap)
            e = e + np.where(series, 2.0 ** -21 * np.abs(s), 3 * 2.0 ** -22 * cap)
        if slopes is not None:
            far = slopes[h] * np.abs(pos[:, None] - j)
            s = s - far
            e = e + 2.0 ** -22 * np.abs(far) + 2.0 ** -24 * np.abs(s)
        s = np.where(seen, s, -np.inf)[some]
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        total = p.sum(1, keepdims=True)
        lse[some, h] = (top + np.log(total))[:, 0]
        p /= total
        # the difference to the running maximum, exp2, the sum of the weights
        e = e[some] + 2.0 ** -22 + 2.0 ** -23 * (np.where(seen[some], np.abs(s), 0) + np.abs(top)) + (L + 64) * 2.0 ** -24
        out[some, h], weighted[some, h] = p @ v, p @ np.abs(v)
        mean = (p * e).sum(1, keepdims=True)
        tol[some, h] = 2 * ((p * e) @ np.abs(v) + mean * weighted[some, h]) + 2.0 ** -25 * (seen[some] @ np.abs(v)) + 1e-30
        tol_lse[some, h] = 2 * mean[:, 0] + 2.0 ** -22 * (1 + np.abs(lse[some, h]))
    return out, lse, tol, tol_lse, weighted


def sample(row, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """The token of one row and the logarithm of its share; sums in extended precision."""
    logits = np.where(np.isnan(row), -np.inf, np.asarray(row, np.float64))
    top = logits.max()
    if top == -np.inf:
        return -1, -np.inf
    if temperature == 0:
        return int(np.argmax(logits)), 0.0
    with np.errstate(invalid="ignore"):
        w = np.where(logits == top, 0.0, (logits - top) / np.float64(temperature))
    w = np.exp(w.astype(np.longdouble))
    order = np.argsort(-logits, kind="stable")
    order = order[logits[order] > -np.inf]
    if top_k:
        order = order[:top_k]
    ranked = w[order]
    keep = ranked >= min_p
    if top_p < 1:
        keep &= ranked.cumsum() - ranked < np.longdouble(top_p) * ranked.sum()
    keep[0] = True
    kept = np.sort(order[keep])
    upto = w[kept].cumsum()
    token = int(kept[min(np.searchsorted(upto, np.longdouble(u) * upto[-1], side="right"), len(kept) - 1)])
    return token, float(np.log(w[token] / upto[-1]))
